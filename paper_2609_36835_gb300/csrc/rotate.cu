// Rotary positions of one or two tensors in one launch.
//
//   y1 = f (x1 cos a - x2 sin a),  y2 = f (x2 cos a + x1 sin a),  a = 2 pi pos turns_i / 2^64
//
// The angle is a whole number of 2^-64 turns: pos * turns_i mod 2^64 is exact, and what is left is within half a turn
// whatever the position, so cos and sin take no reduction and lose nothing far out.  A CTA takes a few tokens: it finds
// their cosines and sines once, in shared memory, and turns all heads with them.  A thread's unit is twice 16 bytes (of the
// layout in halves, two places of the head): bound by HBM for prompts, by latency for a decode step.  Measured (CUDA
// graph): 8191 tokens of 32 + 8 heads in fp32 52 us, 6.5 TB/s of reads and writes; in bf16 32 us; 64 tokens 2.3 us.
#include "pages.cuh"

namespace arckv {
namespace {

constexpr int kRT = 256;

struct RotateArgs {
  RotateTensor t[2];
  const unsigned long long* turns;
  const int* positions;
  float f;
  int N, d, r, tokens, split;   // tokens of a CTA, CTAs that share a token's heads
};

// Sixteen bytes as fp32.
__device__ __forceinline__ void load16(const bf16* p, float (&x)[8]) {
  const uint4 v = *(const uint4*)p;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = bf16_lo(w[e]);
    x[2 * e + 1] = bf16_hi(w[e]);
  }
}
__device__ __forceinline__ void load16(const float* p, float (&x)[4]) {
  const float4 a = *(const float4*)p;
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
}
__device__ __forceinline__ void store16(bf16* p, const float (&x)[8]) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
  *(uint4*)p = *(const uint4*)&h[0];
}
__device__ __forceinline__ void store16(float* p, const float (&x)[4]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
}

template <typename T, bool kInter>
__global__ void __launch_bounds__(kRT) pages_rotate_kernel(const RotateArgs a, bool transpose) {
  constexpr int kE = 16 / sizeof(T);   // elements of 16 bytes: a thread's unit is two of them, kE pairs
  extern __shared__ float2 cs[];       // [token][pair] f cos, f sin
  const int tid = threadIdx.x, half = a.r >> 1, n0 = blockIdx.x * a.tokens, tokens = min(a.tokens, a.N - n0);
  pdl_trigger();
  pdl_wait();
  for (int x = tid; x < tokens * half; x += kRT) {
    const int n = x / half, i = x - n * half, pos = a.positions[n0 + n];
    const unsigned long long turn = (unsigned long long)max(pos, 0) * a.turns[i];
    const float z = (float)(int)(turn >> 32) * 0x1p-31f;   // half turns, in [-1, 1]
    float s, c;
    sincospif(z, &s, &c);
    cs[x] = make_float2(a.f * c, transpose ? -a.f * s : a.f * s);
  }
  __syncthreads();
  const int units = a.d / (2 * kE), turned = a.r / (2 * kE), heads = a.t[0].heads + a.t[1].heads;
  const int h0 = (int)((long long)heads * blockIdx.y / a.split), hn = (int)((long long)heads * (blockIdx.y + 1) / a.split) - h0;
  const int u = tid % units, rows = kRT / units;   // rows of heads at a time
  for (int x = tid / units; x < tokens * hn; x += rows) {
    if (tid >= rows * units) break;
    const int n = tokens > 1 ? x / hn : 0;
    int h = h0 + x - n * hn;
    const bool second = h >= a.t[0].heads;
    const RotateTensor& t = a.t[second];
    if (second) h -= a.t[0].heads;
    const T* src = (const T*)t.x + (n0 + n) * t.xs.i + h * t.xs.h;
    T* dst = (T*)t.y + (n0 + n) * t.ys.i + h * t.ys.h;
    const bool turns = u < turned && a.positions[n0 + n] >= 0;
    if (!turns && (const void*)src == (const void*)dst) continue;
    const bool apart = !kInter && u < turned;
    const int at1 = apart ? kE * u : 2 * kE * u, at2 = apart ? half + kE * u : 2 * kE * u + kE;
    float p[kE], q[kE];
    load16(src + at1, p);
    load16(src + at2, q);
    if (turns) {
      const float2* w = cs + n * half + kE * u;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float2 z = w[e];
        constexpr int kH = kE / 2;
        float& x1 = kInter ? (e < kH ? p[2 * (e % kH)] : q[2 * (e % kH)]) : p[e];
        float& x2 = kInter ? (e < kH ? p[2 * (e % kH) + 1] : q[2 * (e % kH) + 1]) : q[e];
        const float y1 = x1 * z.x - x2 * z.y, y2 = x2 * z.x + x1 * z.y;
        x1 = y1;
        x2 = y2;
      }
    }
    store16(dst + at1, p);
    store16(dst + at2, q);
  }
}

}  // namespace

int launch_rotate(int N, int d, int r, float f, const unsigned long long* turns, const int* positions,
                  const RotateTensor (&t)[2], bool f32, bool interleaved, bool transpose, cudaStream_t st) {
  RotateArgs a;
  a.t[0] = t[0];
  a.t[1] = t[1];
  a.turns = turns;
  a.positions = positions;
  a.f = f;
  a.N = N;
  a.d = d;
  a.r = r;
  const int heads = t[0].heads + t[1].heads, sms = tc_gemm_sm_count();
  // Five rounds of a CTA's threads or so, while there are CTAs for every SM (8191 tokens of 40 heads: 52 us in fp32, 32 in bf16;
  // half as many rounds 51 and 35, twice as many 55 and 35); few tokens are shared by several CTAs
  const int units = heads * (f32 ? d >> 3 : d >> 4);
  a.tokens = std::max(1, std::min({16, 5 * kRT / units, N / (4 * sms)}));
  const int ctas = cdiv(N, a.tokens);
  a.split = std::max(1, std::min(cdiv((long long)a.tokens * units, kRT), 4 * sms / ctas));
  auto kern = f32 ? (interleaved ? pages_rotate_kernel<float, true> : pages_rotate_kernel<float, false>)
                  : (interleaved ? pages_rotate_kernel<bf16, true> : pages_rotate_kernel<bf16, false>);
  const int smem = a.tokens * (r / 2) * (int)sizeof(float2);
  return launch_pdl(kern, dim3(ctas, a.split), kRT, smem, st, a, transpose) == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
