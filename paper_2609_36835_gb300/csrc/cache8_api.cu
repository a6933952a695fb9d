// C entry points of the 8-bit cache: argument checks and launches.  Contracts
// are in include/arckv.h.
#include "cache8.cuh"

using namespace arckv;

namespace {

inline bool misaligned(const void* p, size_t to = 16) { return ((uintptr_t)p % to) != 0; }

bool sizes_ok(int32_t S, int32_t H, int32_t cap) {
  // S and 2 H ride in grid dimensions; token counts are 32-bit, offsets 64-bit
  return S >= 1 && S <= 4096 && H >= 1 && H <= 32767 && cap >= kCB && cap % kCB == 0 && cap <= (1 << 26) &&
         (long long)S * H * (cap / kCB) < (1LL << 31);
}
bool rows_ok(int32_t S, int32_t H, int32_t n_pos, int32_t G) {
  return n_pos >= 1 && n_pos <= (1 << 24) && G >= 1 && G <= (1 << 16) &&
         (long long)S * H * n_pos < (1LL << 31) / G;
}

arckv_status check_cache(const arckv_cache8* c) {
  if (!c) return ARCKV_ERR_INVALID_ARG;
  if (c->d != 128) return ARCKV_ERR_UNSUPPORTED;
  if (!sizes_ok(c->S, c->H, c->cap)) return ARCKV_ERR_SHAPE;
  const void* all[] = {c->K, c->V, c->k_scale, c->v_scale, c->bounds, c->tail, c->tail_amax, c->len, c->state};
  for (const void* p : all)
    if (!p || misaligned(p)) return ARCKV_ERR_INVALID_ARG;
  if (misaligned(c->bias)) return ARCKV_ERR_INVALID_ARG;
  return ARCKV_OK;
}

// Row strides in elements of `size` bytes; false when a base or stride is off the 16-byte grid.
bool row_strides(const void* base, const int64_t* given, int64_t H, int64_t n, int64_t row, int size, RowStrides* out) {
  const int64_t dense[3] = {H * n * row, n * row, row};
  const int64_t* s = given ? given : dense;
  if (misaligned(base)) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] * size % 16 != 0) return false;
  *out = RowStrides{s[0], s[1], s[2]};
  return true;
}

// The end of a call: with NONBLOCKING at once, else the status word, read and cleared.
arckv_status finish(void* status, uint32_t flags, void* stream) {
  if (cudaGetLastError() != cudaSuccess) return ARCKV_ERR_CUDA;
  if (flags & ARCKV_FLAG_NONBLOCKING) return ARCKV_OK;
  return arckv_query_status(status, stream);
}

arckv_status check_query(const arckv_cache8* c, int32_t n_pos, int32_t G, const void* Q, const int64_t* q_strides,
                         void* ws, size_t ws_bytes, size_t scratch(int, int, int, int, int), uint32_t flags,
                         CacheQuery* q) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_CAUSAL)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_cache(c);
  if (e != ARCKV_OK) return e;
  if (!rows_ok(c->S, c->H, n_pos, G)) return ARCKV_ERR_SHAPE;
  if (!Q || !row_strides(Q, q_strides, c->H, n_pos, (int64_t)G * 128, 2, &q->qs)) return ARCKV_ERR_INVALID_ARG;
  if (!ws || misaligned(ws, 256) || ws_bytes < ARCKV_CACHE_WS_HEADER + scratch(c->S, c->H, c->cap, n_pos, G))
    return ARCKV_ERR_WORKSPACE;
  q->n_pos = n_pos;
  q->G = G;
  q->causal = (flags & ARCKV_FLAG_CAUSAL) != 0;
  q->Q = (const bf16*)Q;
  return ARCKV_OK;
}

}  // namespace

extern "C" {

size_t arckv_cache_attend_workspace_bytes(int32_t S, int32_t H, int32_t cap, int32_t d, int32_t n_pos, int32_t G) {
  if (d != 128 || !sizes_ok(S, H, cap) || !rows_ok(S, H, n_pos, G)) return 0;
  return ARCKV_CACHE_WS_HEADER + cache_attend_scratch(S, H, cap, n_pos, G);
}

size_t arckv_cache_select_workspace_bytes(int32_t S, int32_t H, int32_t cap, int32_t d, int32_t n_pos, int32_t G) {
  if (d != 128 || !sizes_ok(S, H, cap) || !rows_ok(S, H, n_pos, G)) return 0;
  return ARCKV_CACHE_WS_HEADER + cache_select_scratch(S, H, cap, n_pos, G);
}

size_t arckv_cache_workspace_bytes(int32_t S, int32_t H, int32_t cap, int32_t d, int32_t n_pos, int32_t G) {
  return std::max(arckv_cache_attend_workspace_bytes(S, H, cap, d, n_pos, G),
                  arckv_cache_select_workspace_bytes(S, H, cap, d, n_pos, G));
}

arckv_status arckv_cache_append(const arckv_cache8* c, int32_t n, const void* K, const int64_t* k_strides,
                                const void* V, const int64_t* v_strides, const float* bias, const int32_t* at,
                                const int32_t* counts, uint32_t flags, void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_F32)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_cache(c);
  if (e != ARCKV_OK) return e;
  if (n < 1 || n > c->cap) return ARCKV_ERR_SHAPE;
  const bool f32 = (flags & ARCKV_FLAG_F32) != 0;
  RowStrides ks, vs;
  if (!K || !V || (bias && !c->bias) || misaligned(bias, 4) || misaligned(at, 4) || misaligned(counts, 4) ||
      !row_strides(K, k_strides, c->H, n, 128, f32 ? 4 : 2, &ks) ||
      !row_strides(V, v_strides, c->H, n, 128, f32 ? 4 : 2, &vs))
    return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_cache_append(*c, n, f32, K, ks, V, vs, bias, at, counts, (cudaStream_t)stream) < 0)
    return ARCKV_ERR_CUDA;
  return finish(c->state, flags, stream);
}

arckv_status arckv_cache_read(const arckv_cache8* c, int32_t start, int32_t count, void* K_out, void* V_out,
                              uint32_t flags, void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_F32)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_cache(c);
  if (e != ARCKV_OK) return e;
  if (count < 1 || count > (1 << 26) || start < -(1 << 26) || start > (1 << 26)) return ARCKV_ERR_SHAPE;
  if ((!K_out && !V_out) || misaligned(K_out) || misaligned(V_out)) return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_cache_read(*c, start, count, (flags & ARCKV_FLAG_F32) != 0, K_out, V_out, (cudaStream_t)stream) < 0)
    return ARCKV_ERR_CUDA;
  return finish(c->state, flags, stream);
}

arckv_status arckv_cache_attend(const arckv_cache8* c, int32_t n_pos, int32_t G, float logit_scale, const void* Q,
                                const int64_t* q_strides, const int32_t* blocks, int32_t m, float* O,
                                const int64_t* o_strides, void* ws, size_t ws_bytes, uint32_t flags, void* stream) {
  CacheQuery q;
  const arckv_status e = check_query(c, n_pos, G, Q, q_strides, ws, ws_bytes, cache_attend_scratch, flags, &q);
  if (e != ARCKV_OK) return e;
  RowStrides os;
  if (!O || misaligned(blocks, 4) || !row_strides(O, o_strides, c->H, n_pos, (int64_t)G * 128, 4, &os))
    return ARCKV_ERR_INVALID_ARG;
  // blocks read in all are counted in 32 bits
  if (blocks && (m < 1 || m > c->cap / kCB + 8192 || (long long)c->S * c->H * n_pos * ((G + 3) / 4) * m >= (1LL << 31)))
    return ARCKV_ERR_SHAPE;
  if (!(logit_scale >= 0.f) || !isfinite(logit_scale)) return ARCKV_ERR_INVALID_ARG;
  const float scale = logit_scale > 0.f ? logit_scale : 1.0f / sqrtf((float)c->d);
  cudaGetLastError();
  if (launch_cache_attend(*c, q, scale, blocks, m, O, os, ws, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(ws, flags, stream);
}

arckv_status arckv_cache_select(const arckv_cache8* c, int32_t n_pos, int32_t G, int32_t m, int32_t keep_first,
                                int32_t keep_last, const void* Q, const int64_t* q_strides, int32_t* blocks, void* ws,
                                size_t ws_bytes, uint32_t flags, void* stream) {
  CacheQuery q;
  const arckv_status e = check_query(c, n_pos, G, Q, q_strides, ws, ws_bytes, cache_select_scratch, flags, &q);
  if (e != ARCKV_OK) return e;
  if (m < 1 || m > 8192 || keep_first < 0 || keep_last < 0 || (long long)keep_first + keep_last > m)
    return ARCKV_ERR_SHAPE;
  if (!blocks || misaligned(blocks, 4)) return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_cache_select(*c, q, m, keep_first, keep_last, blocks, ws, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(ws, flags, stream);
}

}  // extern "C"
