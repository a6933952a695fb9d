// Block selection for sparse attention over an 8-bit cache.
//
// The logits of block b's keys are at most scale_b sum_e max(q_e lo_be, q_e hi_be)
// with lo, hi the least and largest key codes of dimension e.  With the query
// quantised to 8 bits too, the sum is an exact integer below 2^21, so scores
// are the same in whatever order they are added up.
#include "cache8.cuh"

namespace arckv {
namespace {

// score[item][b] of every candidate block; one thread per (item, block).
__global__ void __launch_bounds__(128) cache_score_kernel(const arckv_cache8 c, CacheQuery q, float* score) {
  const long long item = blockIdx.x;
  const int p = (int)(item % q.n_pos), nblk = c.cap / kCB;
  const long long sh = item / q.n_pos;
  const int h = (int)(sh % c.H), s = (int)(sh / c.H);
  const int see = visible_tokens(cache_len(c, s), q.n_pos, p, q.causal), cand = (see + kCB - 1) / kCB;
  __shared__ int s_q[2][32];   // the row's codes, positive and negative parts, packed
  __shared__ float s_scale;
  for (int g = 0; g < q.G; ++g) {
    __syncthreads();
    if (threadIdx.x < 32) {
      const bf16* qr = q.Q + s * q.qs.s + h * q.qs.h + p * q.qs.i + g * 128 + threadIdx.x * 4;
      float x[4], a = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = __bfloat162float(qr[e]);
        a = fmaxf(a, fabsf(x[e]));
      }
      a = fmaxf(warp_max(a), kCacheFloor);
      const float inv = __fdiv_rn(127.f, a);
      unsigned int pos = 0, neg = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = min(max(__float2int_rn(x[e] * inv), -127), 127);
        pos |= (unsigned int)(max(v, 0) & 0xff) << (8 * e);
        neg |= (unsigned int)(min(v, 0) & 0xff) << (8 * e);
      }
      s_q[0][threadIdx.x] = (int)pos;
      s_q[1][threadIdx.x] = (int)neg;
      if (threadIdx.x == 0) s_scale = a * kInv127;
    }
    __syncthreads();
    for (int b = blockIdx.y * 128 + threadIdx.x; b < cand; b += gridDim.y * 128) {
      const long long blk = sh * nblk + b;
      const int* lo = (const int*)(c.bounds + blk * 256);
      int dot = 0;
      for (int e = 0; e < 32; ++e) dot = __dp4a(s_q[0][e], lo[32 + e], __dp4a(s_q[1][e], lo[e], dot));
      const float v = __fmul_rn(__fmul_rn(s_scale, (float)dot), c.k_scale[blk]);
      float* at = score + item * nblk + b;
      *at = g == 0 ? v : fmaxf(*at, v);
    }
  }
}

// One CTA per item: block b is taken when fewer than m candidates come before
// it, by (forced, score, lower index).
__global__ void __launch_bounds__(256) cache_pick_kernel(const arckv_cache8 c, CacheQuery q, const float* score, int m,
                                                         int keep_first, int keep_last, int* blocks) {
  const long long item = blockIdx.x;
  const int p = (int)(item % q.n_pos), nblk = c.cap / kCB, s = (int)(item / q.n_pos / c.H);
  const int see = visible_tokens(cache_len(c, s), q.n_pos, p, q.causal), cand = (see + kCB - 1) / kCB;
  const float* sc = score + item * nblk;
  __shared__ int s_warp[8], s_base;
  auto key = [&](int b) {
    return (b < keep_first || b >= cand - keep_last) ? 0xffffffffu : f32_ordered(sc[b] + 0.f);
  };
  if (threadIdx.x == 0) s_base = 0;
  for (int b0 = 0; b0 < cand; b0 += 256) {
    const int b = b0 + threadIdx.x;
    bool take = false;
    if (b < cand) {
      const unsigned int mine = key(b);
      int before = 0;
      if (cand > m)
        for (int j = 0; j < cand; ++j) {
          const unsigned int o = key(j);
          before += o > mine || (o == mine && j < b);
        }
      take = before < m;
    }
    const unsigned int mask = __ballot_sync(0xffffffffu, take);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = __popc(mask);
    __syncthreads();
    int at = s_base + __popc(mask & ((1u << (threadIdx.x & 31)) - 1));
    for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) at += s_warp[w];
    if (take) blocks[item * m + at] = b;
    __syncthreads();
    if (threadIdx.x == 0)
      for (int w = 0; w < 8; ++w) s_base += s_warp[w];
    __syncthreads();
  }
  __syncthreads();
  for (int i = s_base + threadIdx.x; i < m; i += 256) blocks[item * m + i] = -1;
}

}  // namespace

size_t cache_select_scratch(int S, int H, int cap, int n_pos) {
  return (size_t)S * H * n_pos * (cap / kCB) * sizeof(float);
}

int launch_cache_select(const arckv_cache8& c, const CacheQuery& q, int m, int keep_first, int keep_last, int* blocks,
                        void* ws, cudaStream_t st) {
  const long long items = (long long)c.S * c.H * q.n_pos;
  float* score = (float*)((char*)ws + ARCKV_CACHE_WS_HEADER);
  cache_score_kernel<<<dim3((unsigned)items, std::min(16, cdiv(c.cap / kCB, 128))), 128, 0, st>>>(c, q, score);
  cache_pick_kernel<<<(unsigned)items, 256, 0, st>>>(c, q, score, m, keep_first, keep_last, blocks);
  return 2;
}

}  // namespace arckv
