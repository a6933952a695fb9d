// Attention over an 8-bit cache: O = softmax_j(scale q . k_j + bias_j) v_j over
// all visible tokens of a row, or over the blocks listed for its position.
#include "cache8.cuh"

namespace arckv {
namespace {

// One warp per query row, lane l dims 4l .. 4l+3, one key a step.
__global__ void __launch_bounds__(128) cache_attend_rows_kernel(const arckv_cache8 c, CacheQuery q, float scale,
                                                                const int* blocks, int m, float* O, RowStrides os,
                                                                long long rows, DevStatus* stt) {
  const long long row = blockIdx.x * 4ll + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= rows) return;
  const int g = (int)(row % q.G);
  const long long item = row / q.G;
  const int p = (int)(item % q.n_pos);
  const long long sh = item / q.n_pos;
  const int h = (int)(sh % c.H), s = (int)(sh / c.H);
  const int see = visible_tokens(cache_len(c, s), q.n_pos, p, q.causal), nblk = c.cap / kCB;
  float x[4];
  const bf16* qr = q.Q + s * q.qs.s + h * q.qs.h + p * q.qs.i + g * 128 + lane * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = scale * __bfloat162float(qr[e]);
  float top = -INFINITY, z = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  const int nb = blocks ? m : (see + kCB - 1) / kCB;
  for (int i = 0; i < nb; ++i) {
    const int b = blocks ? blocks[item * m + i] : i;
    if (b < 0) continue;
    if (b >= nblk) {
      if (lane == 0) set_status(stt, ARCKV_ERR_INVALID_ARG);
      continue;
    }
    if (b * kCB >= see) continue;
    const float ks = c.k_scale[sh * nblk + b], vs = c.v_scale[sh * nblk + b];
    for (int j = b * kCB; j < min(see, (b + 1) * kCB); ++j) {
      const long long tok = sh * c.cap + j;
      const unsigned int kw = *(const unsigned int*)(c.K + tok * 128 + lane * 4);
      float a = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) a = fmaf(x[e], (float)((int)((kw >> (8 * e)) & 0xffu) - 128), a);
      a = warp_sum(a) * ks;
      if (c.bias) a += c.bias[tok];
      if (a == -INFINITY) continue;
      const float up = fmaxf(top, a), f = expf(top - up), pr = expf(a - up);
      z = z * f + pr;
      top = up;
      const unsigned int vw = *(const unsigned int*)(c.V + tok * 128 + lane * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[e] = fmaf(pr * vs, (float)((int)((vw >> (8 * e)) & 0xffu) - 128), acc[e] * f);
    }
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;   // NaN stays NaN
  const float4 o = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  if (!(fabsf(o.x) <= 3.402823466e38f) || !(fabsf(o.y) <= 3.402823466e38f) || !(fabsf(o.z) <= 3.402823466e38f) ||
      !(fabsf(o.w) <= 3.402823466e38f))
    set_status(stt, ARCKV_ERR_NONFINITE);
  *(float4*)(O + s * os.s + h * os.h + p * os.i + g * 128 + lane * 4) = o;
}

}  // namespace

size_t cache_attend_scratch(int, int, int, int, int) { return 0; }

int launch_cache_attend(const arckv_cache8& c, const CacheQuery& q, float scale, const int* blocks, int m, float* O,
                        RowStrides os, void* ws, cudaStream_t st) {
  const long long rows = (long long)c.S * c.H * q.n_pos * q.G;
  cache_attend_rows_kernel<<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(c, q, scale, blocks, m, O, os, rows,
                                                                       (DevStatus*)ws);
  return 1;
}

}  // namespace arckv
