// Attention of packed queries over paged 4-bit caches:
//
//   O_r = sum_j e^{x_rj} v_j / sum_j e^{x_rj},  x_rj = scale q_r . k_j + bias_j
//
// A warp takes one query row of one head and goes over the request's pages: a
// lane has two tokens of a page for the logits, four dims for the output.
#include "pages.cuh"

namespace arckv {
namespace {

constexpr int kAW = 4;   // warps of a CTA

template <bool kBias>
__global__ void __launch_bounds__(32 * kAW) pages_attend_kernel(const arckv_pages4 p, PagesQuery a, float scale,
                                                                DevStatus* stt) {
  __shared__ float sq[kAW][128];
  __shared__ float sp[kAW][kPT];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_trigger();
  pdl_wait();
  const int total = min(max(a.starts[p.S], 0), a.N);
  const long long rows = (long long)a.N * p.H * a.G, step = (long long)gridDim.x * kAW;
  for (long long row = (long long)blockIdx.x * kAW + warp; row < rows; row += step) {
    const int g = (int)(row % a.G), h = (int)(row / a.G % p.H), i = (int)(row / a.G / p.H);
    if (i >= total) continue;
    int s = 0, hi = p.S;   // last request that begins at i or before it
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if (a.starts[mid] <= i) s = mid;
      else hi = mid;
    }
    const int end = a.starts[s + 1], len = pages_len(p, s);
    if (i < a.starts[s] || i >= end) continue;
    if (end - a.starts[s] > a.max_count) {
      set_status(stt, ARCKV_ERR_SHAPE);
      continue;
    }
    const int sees = a.causal ? max(0, min(len, len - (end - i) + 1)) : len;
    const bf16* q = a.Q + i * a.qs.i + h * a.qs.h + g * 128;
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 4; ++e) sq[warp][4 * lane + e] = __bfloat162float(q[4 * lane + e]);
    __syncwarp();
    float mx = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int b = 0; b * kPT < sees; ++b) {
      const int page = p.table[(long long)s * p.M + b];
      if (page < 0 || page >= p.P) {
        if (page >= p.P) set_status(stt, ARCKV_ERR_INVALID_ARG);
        continue;
      }
      const unsigned char* at = page_at(p, page, h);
      float x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int tok = lane + 32 * e;
        x[e] = -INFINITY;
        if (b * kPT + tok >= sees) continue;
        float sum = 0.f;
        for (int w = 0; w < 4; ++w) {
          const uint32_t par = *(const uint32_t*)(at + kPageKp + tok * 16 + w * 4);
          const float ks = bf16_lo(par), km = bf16_hi(par);
          for (int t = 0; t < 4; ++t) {
            const uint32_t c = *(const uint32_t*)(at + tok * 64 + t * 16 + w * 4);
            for (int f = 0; f < 8; ++f)
              sum = fmaf(sq[warp][32 * w + 8 * t + f], fmaf((float)((c >> (4 * (f >> 1) + 16 * (f & 1))) & 15u), ks, km), sum);
          }
        }
        x[e] = sum * scale;
        if (kBias) x[e] += p.bias[((long long)page * p.H + h) * kPT + tok];
      }
      const float top = warp_max(fmaxf(x[0], x[1])), ref = fmaxf(mx, top);
      if (ref == -INFINITY) continue;
      const float shrink = expf(mx - ref);
      mx = ref;
      __syncwarp();
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float w = expf(x[e] - ref);
        sp[warp][lane + 32 * e] = w;
        sum += w;
      }
      l = l * shrink + warp_sum(sum);
      __syncwarp();
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= shrink;
      const int n = min(kPT, sees - b * kPT);
      for (int tok = 0; tok < n; ++tok) {
        const float w = sp[warp][tok];
        const uint32_t par = *(const uint32_t*)(at + kPageVp + tok * 4);
        const float vs = bf16_lo(par), vm = bf16_hi(par);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int dim = 4 * lane + e, gg = dim & 7, xx = dim >> 3;
          const uint32_t c = (*(const unsigned short*)(at + page_v_word(tok >> 1, gg, xx >> 2) + (tok & 1) * 2) >> (4 * (xx & 3))) & 15u;
          o[e] = fmaf(w, fmaf((float)c, vs, vm), o[e]);
        }
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16* out = a.O + i * a.os.i + h * a.os.h + g * 128 + 4 * lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = o[e] * inv;
      if (!(fabsf(y) <= 3.3895e38f)) set_status(stt, ARCKV_ERR_NONFINITE);
      out[e] = __float2bfloat16_rn(y);
    }
  }
}

}  // namespace

size_t pages_attend_scratch(int, int, int, int, int) { return 0; }

int launch_pages_attend(const arckv_pages4& p, const PagesQuery& q, float scale, void* ws, cudaStream_t st) {
  const int ctas = stride_grid((long long)q.N * p.H * q.G, kAW, 16);
  const cudaError_t e = p.bias ? launch_pdl(pages_attend_kernel<true>, dim3(ctas), 32 * kAW, 0, st, p, q, scale, (DevStatus*)ws)
                               : launch_pdl(pages_attend_kernel<false>, dim3(ctas), 32 * kAW, 0, st, p, q, scale, (DevStatus*)ws);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
