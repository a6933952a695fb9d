// Writing rows into the pages of a 4-bit cache and reading them back.
//
//   m = bf16(min), s = max(bf16((max - m) / 15), 2^-100), c = clamp(rint((x - m) / s), 0, 15)
//
// A warp takes two rows of a head, 16 lanes each: a lane has 8 dims of the key and of
// the value.  Groups of K are four lanes, the value's group all 16, so both
// extremes are a few shuffles; nothing of a row depends on another, so rows are
// written once.  A value's codes lie four dims to a 16-bit unit, two tokens to a word:
// a quad of lanes transposes its nibbles, and where the rows are a pair of tokens
// their words are written whole, 128 bytes a warp.  Both calls are one pass over
// memory; prompts are bound by issue (74 % and 69 % of its slots), a decode step's
// rows by latency.  Measured (CUDA graph): 8191 tokens of 8 heads in bf16 appended
// and read back 20 us, 4.3 TB/s of what both have to move (a row a warp: 41 us);
// 64 tokens 3.5 us.
#include "pages.cuh"

namespace arckv {
namespace {

constexpr int kPW = 256;   // threads of a CTA: eight pairs of rows of one head

__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const uint4 v = *(const uint4*)p;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = bf16_lo(w[e]);
    x[2 * e + 1] = bf16_hi(w[e]);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *(const float4*)p, b = *((const float4*)p + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ float as_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

__device__ __forceinline__ float min_nan(float a, float b, float c) {   // NaN where one is
  float d;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Eight elements of a group that kLanes lanes share, quantised: (scale, least value) as a word, and the codes, code e at bit
// 16 (e % 2) + 4 (e / 2).
template <int kLanes>
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], uint32_t& codes, DevStatus* stt) {
  float lo = min_nan(min_nan(x[0], x[1], x[2]), min_nan(x[3], x[4], x[5]), min_nan(x[6], x[7], x[7]));
  float hi = max_nan(max_nan(x[0], x[1], x[2]), max_nan(x[3], x[4], x[5]), max_nan(x[6], x[7], x[7]));
  if (!(lo >= -kPagesMost && hi <= kPagesMost)) {   // (rare)
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!(fabsf(x[e]) <= 3.402823466e38f)) {
        bad = true;
        x[e] = 0.f;
      }
      x[e] = fminf(fmaxf(x[e], -kPagesMost), kPagesMost);
    }
    if (bad) set_status(stt, ARCKV_ERR_NONFINITE);
    lo = hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
    }
  }
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const float m = as_bf16(lo), s = fmaxf(as_bf16(__fmul_rn(__fsub_rn(hi, m), kInv15)), kScaleFloor);
  // In sixteenths: saturating at zero is free then (m may have been rounded up).  At the other end a quotient is 15 (1 + 2^-8)
  // at most, as s is off by half a step of a bf16, and rounds to 15.
  const float inv = __frcp_rn(s) * 0.0625f;
  // sixteenths plus 1.5 * 2^19 leave no fraction of a code: its bits are those of 1.5 * 2^19 with the code added
  constexpr uint32_t kBits = 0x49400000u;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = __saturatef(__fmul_rn(__fsub_rn(x[e], m), inv));
    w += __float_as_uint(__fadd_rn(y, 786432.f)) << (16 * (e & 1) + 4 * (e >> 1));
  }
  constexpr uint32_t kAdded = kBits * 0x11111111u;   // sum of 2^(16 (e % 2) + 4 (e / 2)) over e
  codes = w - kAdded;
  return (__float_as_uint(m) & 0xffff0000u) | (__float_as_uint(s) >> 16);
}

template <typename T>
__global__ void __launch_bounds__(kPW) pages_append_kernel(const arckv_pages4 p, int N, const T* K, PackedStrides ks,
                                                           const T* V, PackedStrides vs, const int* slots,
                                                           const float* bias) {
  const int lane = threadIdx.x & 31, x8 = lane & 15, h = blockIdx.y;
  DevStatus* stt = (DevStatus*)p.state;
  pdl_trigger();
  pdl_wait();
  const int i = 2 * (blockIdx.x * (kPW / 32) + (threadIdx.x >> 5)) + (lane >> 4);
  int slot = -1;
  float k[8], v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) k[e] = v[e] = 0.f;
  if (i < N) {
    slot = slots[i];
    load8(K + i * ks.i + h * ks.h + 8 * x8, k);
    load8(V + i * vs.i + h * vs.h + 8 * x8, v);
  }
  if (slot >= p.P * (long long)kPT) {
    if (x8 == 0) set_status(stt, ARCKV_ERR_INVALID_ARG);
    slot = -1;
  }
  if (slot < 0) {   // (not looked at: nothing of it is recorded)
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = v[e] = 0.f;
  }
  uint32_t kc, vc;
  const uint32_t kp = quantise8<4>(k, kc, stt), vp = quantise8<16>(v, vc, stt);
  // V: the quad's codes of dims 8 x + g go into units of four x: unit g in half g & 1 of register g / 2, nibble x % 4.  Code g is
  // now nibble g / 2 of half g & 1.
  const int q = x8 & 3;
  uint32_t r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = ((vc >> (4 * e)) & 0x000f000fu) << (4 * q);
  // lane q ends with register q: its own and the three others' parts of it
  uint32_t k0 = q & 1 ? r[1] : r[0], k1 = q & 1 ? r[3] : r[2];   // registers (q & 1), 2 + (q & 1)
  k0 |= __shfl_xor_sync(0xffffffffu, q & 1 ? r[0] : r[1], 1);
  k1 |= __shfl_xor_sync(0xffffffffu, q & 1 ? r[2] : r[3], 1);
  const uint32_t mine = (q & 2 ? k1 : k0) | __shfl_xor_sync(0xffffffffu, q & 2 ? k0 : k1, 2);
  // two tokens of a pair: one lane of each two takes the units of g = 2 q, the other those of 2 q + 1
  const int other = __shfl_xor_sync(0xffffffffu, slot, 16);
  const uint32_t theirs = __shfl_xor_sync(0xffffffffu, mine, 16);
  if (slot < 0) return;
  const int tok = slot % kPT, second = lane >> 4;
  unsigned char* at = p.data + ((long long)(slot / kPT) * p.H + h) * ARCKV_PAGE_BYTES;
  *(uint32_t*)(at + tok * 64 + q * 16 + (x8 >> 2) * 4) = kc;
  if (q == 0) *(uint32_t*)(at + kPageKp + tok * 16 + (x8 >> 2) * 4) = kp;
  if (x8 == 0) {
    *(uint32_t*)(at + kPageVp + tok * 4) = vp;
    if (p.bias) p.bias[((long long)(slot / kPT) * p.H + h) * kPT + tok] = bias ? bias[(long long)i * p.H + h] : 0.f;
  }
  if (second ? other == slot - 1 && (slot & 1) : other == slot + 1 && !(slot & 1)) {
    const uint32_t even = second ? theirs : mine, odd = second ? mine : theirs;
    *(uint32_t*)(at + page_v_word(tok >> 1, 2 * q + second, x8 >> 2)) = __byte_perm(even, odd, second ? 0x7632 : 0x5410);
  } else {
    const int half = (tok & 1) * 2;
    *(unsigned short*)(at + page_v_word(tok >> 1, 2 * q, x8 >> 2) + half) = (unsigned short)mine;
    *(unsigned short*)(at + page_v_word(tok >> 1, 2 * q + 1, x8 >> 2) + half) = (unsigned short)(mine >> 16);
  }
}

__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
  *(uint4*)p = *(const uint4*)&h[0];
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  *((float4*)p + 1) = make_float4(x[4], x[5], x[6], x[7]);
}

// Codes c of eight dims, code e in nibble e / 2 of half e % 2 of w, as values.
__device__ __forceinline__ void values8(uint32_t w, uint32_t par, float (&x)[8]) {
  const float s = bf16_lo(par), m = bf16_hi(par);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = __uint_as_float(((w >> (16 * (e & 1) + 4 * (e >> 1))) & 15u) | 0x4b000000u) - 8388608.f;
    x[e] = fmaf(c, s, m);   // (a code times a scale is exact)
  }
}

template <typename T>
__global__ void __launch_bounds__(kPW) pages_read_kernel(const arckv_pages4 p, int N, const int* slots, T* K, T* V) {
  const int lane = threadIdx.x & 31, x8 = lane & 15, q = x8 & 3, h = blockIdx.y;
  pdl_trigger();
  pdl_wait();
  const int i = 2 * (blockIdx.x * (kPW / 32) + (threadIdx.x >> 5)) + (lane >> 4);
  int slot = i < N ? slots[i] : -1;
  if (slot >= p.P * (long long)kPT) {
    if (x8 == 0) set_status((DevStatus*)p.state, ARCKV_ERR_INVALID_ARG);
    slot = -1;
  }
  uint32_t kw = 0, kp = 0, vp = 0, mine = 0;
  if (slot >= 0) {
    const int tok = slot % kPT, half = (tok & 1) * 2;
    const unsigned char* at = page_at(p, slot / kPT, h);
    kw = *(const uint32_t*)(at + tok * 64 + q * 16 + (x8 >> 2) * 4);
    kp = *(const uint32_t*)(at + kPageKp + tok * 16 + (x8 >> 2) * 4);
    vp = *(const uint32_t*)(at + kPageVp + tok * 4);
    mine = *(const unsigned short*)(at + page_v_word(tok >> 1, 2 * q, x8 >> 2) + half) |
           (uint32_t) * (const unsigned short*)(at + page_v_word(tok >> 1, 2 * q + 1, x8 >> 2) + half) << 16;
  }
  // lane q of a quad has the units of g = 2 q, 2 q + 1; nibble q of each is its own dim 8 x + g
  uint32_t vw = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) vw |= ((__shfl_sync(0xffffffffu, mine, (lane & ~3) | e) >> (4 * q)) & 0x000f000fu) << (4 * e);
  if (i >= N) return;
  const long long row = ((long long)i * p.H + h) * 128 + 8 * x8;
  float x[8];
  if (K) {
    values8(kw, kp, x);
    store8(K + row, x);
  }
  if (V) {
    values8(vw, vp, x);
    store8(V + row, x);
  }
}

}  // namespace

int launch_pages_append(const arckv_pages4& p, int N, bool f32, const void* K, PackedStrides ks, const void* V,
                        PackedStrides vs, const int* slots, const float* bias, cudaStream_t st) {
  const dim3 ctas(cdiv(N, 2 * (kPW / 32)), p.H);
  const cudaError_t e =
      f32 ? launch_pdl(pages_append_kernel<float>, ctas, kPW, 0, st, p, N, (const float*)K, ks, (const float*)V, vs, slots, bias)
          : launch_pdl(pages_append_kernel<bf16>, ctas, kPW, 0, st, p, N, (const bf16*)K, ks, (const bf16*)V, vs, slots, bias);
  return e == cudaSuccess ? 1 : -1;
}

int launch_pages_read(const arckv_pages4& p, int N, bool f32, const int* slots, void* K, void* V, cudaStream_t st) {
  const dim3 ctas(cdiv(N, 2 * (kPW / 32)), p.H);
  const cudaError_t e = f32 ? launch_pdl(pages_read_kernel<float>, ctas, kPW, 0, st, p, N, slots, (float*)K, (float*)V)
                            : launch_pdl(pages_read_kernel<bf16>, ctas, kPW, 0, st, p, N, slots, (bf16*)K, (bf16*)V);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
