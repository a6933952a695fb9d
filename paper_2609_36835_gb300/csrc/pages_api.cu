// C entry points of the paged 4-bit cache and of rotary positions: argument
// checks and launches.  Contracts are in include/arckv.h.
#include "pages.cuh"

using namespace arckv;

namespace {

inline bool misaligned(const void* p, size_t to = 16) { return ((uintptr_t)p % to) != 0; }

bool sizes_ok(int32_t S, int32_t H, int32_t M) {
  // tokens of a request and rows of a table are 32-bit, offsets 64-bit; the requests' sums lie in shared memory
  return S >= 1 && S <= 4096 && H >= 1 && H <= 32767 && M >= 1 && M <= (1 << 20) && (long long)S * H * M < (1LL << 31);
}

arckv_status check_pages(const arckv_pages4* p) {
  if (!p) return ARCKV_ERR_INVALID_ARG;
  if (p->d != 128) return ARCKV_ERR_UNSUPPORTED;
  if (!sizes_ok(p->S, p->H, p->M) || p->P < 1 || p->P > (1 << 24)) return ARCKV_ERR_SHAPE;
  const void* words[] = {p->table, p->len, p->free, p->n_free};
  for (const void* w : words)
    if (!w || misaligned(w, 4)) return ARCKV_ERR_INVALID_ARG;
  if (!p->data || misaligned(p->data) || misaligned(p->bias) || !p->state || misaligned(p->state, 256))
    return ARCKV_ERR_INVALID_ARG;
  return ARCKV_OK;
}

// Row strides in elements of `size` bytes; false when a base or stride is off the 16-byte grid.
bool packed_strides(const void* base, const int64_t* given, int64_t row_i, int64_t row_h, int size, PackedStrides* out) {
  const int64_t dense[2] = {row_i, row_h};
  const int64_t* s = given ? given : dense;
  if (misaligned(base)) return false;
  for (int i = 0; i < 2; ++i)
    if (s[i] * size % 16 != 0) return false;
  *out = PackedStrides{s[0], s[1]};
  return true;
}

// The end of a call: with NONBLOCKING at once, else the status word, read and cleared.
arckv_status finish(void* status, uint32_t flags, void* stream) {
  if (cudaGetLastError() != cudaSuccess) return ARCKV_ERR_CUDA;
  if (flags & ARCKV_FLAG_NONBLOCKING) return ARCKV_OK;
  return arckv_query_status(status, stream);
}

bool attend_ok(int32_t S, int32_t H, int32_t M, int32_t max_count, int32_t G) {
  return sizes_ok(S, H, M) && max_count >= 1 && max_count <= (1 << 24) && G >= 1 && G <= (1 << 12) &&
         (long long)max_count * G < (1LL << 28);
}
// A CTA counts the pages of its share in 31 bits; the many-row kernel has one CTA on each of 128 SMs at least.  (A share that
// long is a call of half an hour.)
bool shares_ok(const arckv_pages4& p, int32_t N, int32_t G, int32_t max_count) {
  const double rows = pages_tile_rows((long long)max_count * G);
  return (double)p.H * p.M * ((double)N * G / rows + p.S) < 128.0 * 2147483648.0;
}

}  // namespace

extern "C" {

arckv_status arckv_pages_extend(const arckv_pages4* p, const int32_t* counts, int32_t N, int32_t* starts, int32_t* slots,
                                int32_t* positions, uint32_t flags, void* stream) {
  if (flags & ~ARCKV_FLAG_NONBLOCKING) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_pages(p);
  if (e != ARCKV_OK) return e;
  if (N < 0 || N >= (1 << 30)) return ARCKV_ERR_SHAPE;
  if (!counts || !starts || misaligned(counts, 4) || misaligned(starts, 4) || misaligned(slots, 4) || misaligned(positions, 4) ||
      (N > 0 && (!slots || !positions)))
    return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_pages_extend(*p, counts, N, starts, slots, positions, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(p->state, flags, stream);
}

arckv_status arckv_pages_truncate(const arckv_pages4* p, const int32_t* lens, uint32_t flags, void* stream) {
  if (flags & ~ARCKV_FLAG_NONBLOCKING) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_pages(p);
  if (e != ARCKV_OK) return e;
  if (!lens || misaligned(lens, 4)) return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_pages_truncate(*p, lens, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(p->state, flags, stream);
}

arckv_status arckv_pages_append(const arckv_pages4* p, int32_t N, const void* K, const int64_t* k_strides, const void* V,
                                const int64_t* v_strides, const int32_t* slots, const float* bias, uint32_t flags,
                                void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_F32)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_pages(p);
  if (e != ARCKV_OK) return e;
  if (N < 1 || N >= (1 << 30)) return ARCKV_ERR_SHAPE;
  const int size = flags & ARCKV_FLAG_F32 ? 4 : 2;
  PackedStrides ks, vs;
  if (!K || !V || !slots || misaligned(slots, 4) || (bias && !p->bias) || misaligned(bias, 4) ||
      !packed_strides(K, k_strides, (int64_t)p->H * 128, 128, size, &ks) ||
      !packed_strides(V, v_strides, (int64_t)p->H * 128, 128, size, &vs))
    return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_pages_append(*p, N, size == 4, K, ks, V, vs, slots, bias, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(p->state, flags, stream);
}

arckv_status arckv_pages_read(const arckv_pages4* p, int32_t N, const int32_t* slots, void* K_out, void* V_out,
                              uint32_t flags, void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_F32)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_pages(p);
  if (e != ARCKV_OK) return e;
  if (N < 1 || N >= (1 << 30)) return ARCKV_ERR_SHAPE;
  if (!slots || misaligned(slots, 4) || (!K_out && !V_out) || misaligned(K_out) || misaligned(V_out)) return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_pages_read(*p, N, (flags & ARCKV_FLAG_F32) != 0, slots, K_out, V_out, (cudaStream_t)stream) < 0)
    return ARCKV_ERR_CUDA;
  return finish(p->state, flags, stream);
}

size_t arckv_pages_attend_workspace_bytes(int32_t S, int32_t H, int32_t M, int32_t d, int32_t max_count, int32_t G) {
  if (d != 128 || !attend_ok(S, H, M, max_count, G)) return 0;
  return ARCKV_CACHE_WS_HEADER + pages_attend_scratch(S, H, M, max_count, G);
}

arckv_status arckv_pages_attend(const arckv_pages4* p, int32_t N, int32_t G, int32_t max_count, float logit_scale,
                                const void* Q, const int64_t* q_strides, const int32_t* starts, void* O,
                                const int64_t* o_strides, void* ws, size_t ws_bytes, uint32_t flags, void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_CAUSAL)) return ARCKV_ERR_INVALID_ARG;
  const arckv_status e = check_pages(p);
  if (e != ARCKV_OK) return e;
  if (N < 1 || N >= (1 << 30) || !attend_ok(p->S, p->H, p->M, max_count, G) || !shares_ok(*p, N, G, max_count))
    return ARCKV_ERR_SHAPE;
  PagesQuery q;
  if (!Q || !O || !starts || misaligned(starts, 4) ||
      !packed_strides(Q, q_strides, (int64_t)p->H * G * 128, (int64_t)G * 128, 2, &q.qs) ||
      !packed_strides(O, o_strides, (int64_t)p->H * G * 128, (int64_t)G * 128, 2, &q.os))
    return ARCKV_ERR_INVALID_ARG;
  if (!(logit_scale >= 0.f) || !isfinite(logit_scale)) return ARCKV_ERR_INVALID_ARG;
  if (!ws || misaligned(ws, 256) ||
      ws_bytes < ARCKV_CACHE_WS_HEADER + pages_attend_scratch(p->S, p->H, p->M, max_count, G))
    return ARCKV_ERR_WORKSPACE;
  q.N = N;
  q.G = G;
  q.max_count = max_count;
  q.causal = (flags & ARCKV_FLAG_CAUSAL) != 0;
  q.Q = (const bf16*)Q;
  q.starts = starts;
  q.O = (bf16*)O;
  const float scale = logit_scale > 0.f ? logit_scale : 1.0f / sqrtf((float)p->d);
  cudaGetLastError();
  if (launch_pages_attend(*p, q, scale, ws, (cudaStream_t)stream) < 0) return ARCKV_ERR_CUDA;
  return finish(ws, flags, stream);
}

arckv_status arckv_rotate(int32_t N, int32_t d, int32_t r, float f, const uint64_t* turns, const int32_t* positions,
                          const void* X, const int64_t* x_strides, void* Y, const int64_t* y_strides, int32_t heads,
                          const void* X2, const int64_t* x2_strides, void* Y2, const int64_t* y2_strides, int32_t heads2,
                          uint32_t flags, void* stream) {
  if (flags & ~(ARCKV_FLAG_NONBLOCKING | ARCKV_FLAG_F32 | ARCKV_FLAG_INTERLEAVED | ARCKV_FLAG_TRANSPOSE))
    return ARCKV_ERR_INVALID_ARG;
  if (d < 16 || d > 512 || d % 16 || r < 16 || r > d || r % 16) return ARCKV_ERR_UNSUPPORTED;
  if (N < 1 || N >= (1 << 30)) return ARCKV_ERR_SHAPE;
  if (!turns || misaligned(turns, 8) || !positions || misaligned(positions, 4) || !X || !Y || (!X2 && Y2) || (X2 && !Y2) ||
      !isfinite(f))
    return ARCKV_ERR_INVALID_ARG;
  if (heads < 1 || heads > 65535 || (X2 && (heads2 < 1 || heads2 > 65535))) return ARCKV_ERR_SHAPE;
  const int size = flags & ARCKV_FLAG_F32 ? 4 : 2;
  RotateTensor t[2] = {};
  auto take = [&](RotateTensor& to, const void* x, const int64_t* xs, void* y, const int64_t* ys, int32_t n) {
    to.x = x;
    to.y = y;
    to.heads = n;
    return packed_strides(x, xs, (int64_t)n * d, d, size, &to.xs) && packed_strides(y, ys, (int64_t)n * d, d, size, &to.ys) &&
           !(x == y && (to.xs.i != to.ys.i || to.xs.h != to.ys.h));
  };
  if (!take(t[0], X, x_strides, Y, y_strides, heads) || (X2 && !take(t[1], X2, x2_strides, Y2, y2_strides, heads2)))
    return ARCKV_ERR_INVALID_ARG;
  cudaGetLastError();
  if (launch_rotate(N, d, r, f, (const unsigned long long*)turns, positions, t, size == 4,
                    (flags & ARCKV_FLAG_INTERLEAVED) != 0, (flags & ARCKV_FLAG_TRANSPOSE) != 0, (cudaStream_t)stream) < 0)
    return ARCKV_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ARCKV_OK : ARCKV_ERR_CUDA;
}

}  // extern "C"
