// Writing rows into the pages of a 4-bit cache and reading them back.
//
//   m = bf16(min), s = max(bf16((max - m) / 15), 2^-100), c = clamp(rint((x - m) / s), 0, 15)
//
// A warp takes a token and head: 16 lanes its key, 16 its value, 8 dims each.
// Groups of K are four lanes, the value's group all 16, so both extremes are a few
// shuffles; nothing of a row depends on another, so rows are written once.
#include "pages.cuh"

namespace arckv {
namespace {

constexpr int kPW = 256;   // threads of a CTA: eight rows at a time

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

template <typename T>
__global__ void __launch_bounds__(kPW) pages_append_kernel(const arckv_pages4 p, int N, const T* K, PackedStrides ks,
                                                           const T* V, PackedStrides vs, const int* slots,
                                                           const float* bias) {
  const int lane = threadIdx.x & 31, x8 = lane & 15;
  const bool value = lane >= 16;
  DevStatus* stt = (DevStatus*)p.state;
  pdl_trigger();
  pdl_wait();
  const long long rows = (long long)N * p.H, step = (long long)gridDim.x * (kPW / 32);
  for (long long row = (long long)blockIdx.x * (kPW / 32) + (threadIdx.x >> 5); row < rows; row += step) {
    const int i = (int)quotient(row, p.H), h = (int)(row - (long long)i * p.H);
    const int slot = slots[i];
    float x[8];
    load8(value ? V + i * vs.i + h * vs.h + 8 * x8 : K + i * ks.i + h * ks.h + 8 * x8, x);
    if (slot < 0) continue;
    const int page = slot / kPT, tok = slot % kPT;
    if (page >= p.P) {
      if (lane == 0) set_status(stt, ARCKV_ERR_INVALID_ARG);
      continue;
    }
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!(fabsf(x[e]) <= kPagesMost)) {
        if (fabsf(x[e]) <= 3.402823466e38f) {
          x[e] = copysignf(kPagesMost, x[e]);
        } else {
          bad = true;
          x[e] = 0.f;
        }
      }
    }
    if (bad) set_status(stt, ARCKV_ERR_NONFINITE);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {   // a group of K is four lanes
      const float a = __shfl_xor_sync(0xffffffffu, lo, o), b = __shfl_xor_sync(0xffffffffu, hi, o);
      if (o < 4 || value) {
        lo = fminf(lo, a);
        hi = fmaxf(hi, b);
      }
    }
    const float m = as_bf16(lo), s = fmaxf(as_bf16(__fmul_rn(__fsub_rn(hi, m), kInv15)), kScaleFloor), inv = __frcp_rn(s);
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = fminf(fmaxf(__fmul_rn(__fsub_rn(x[e], m), inv), 0.f), 15.f);
      c[e] = __float_as_uint(__fadd_rn(y, 12582912.f)) & 15u;   // 1.5 * 2^23 leaves no fraction bits
    }
    unsigned char* at = p.data + ((long long)page * p.H + h) * ARCKV_PAGE_BYTES;
    const uint32_t par = (__float_as_uint(m) & 0xffff0000u) | (__float_as_uint(s) >> 16);
    // V: the quad's codes of dims 8 x + g go into units of four x: unit g in half g & 1 of register g / 2
    const int q = x8 & 3;
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (c[2 * e] | c[2 * e + 1] << 16) << (4 * q);
    // lane q ends with register q: its own and the three others' parts of it
    const uint32_t s0 = q & 1 ? r[0] : r[1], s1 = q & 1 ? r[2] : r[3];
    uint32_t k0 = q & 1 ? r[1] : r[0], k1 = q & 1 ? r[3] : r[2];   // registers (q & 1), 2 + (q & 1)
    k0 |= __shfl_xor_sync(0xffffffffu, s0, 1);
    k1 |= __shfl_xor_sync(0xffffffffu, s1, 1);
    const uint32_t other = __shfl_xor_sync(0xffffffffu, q & 2 ? k0 : k1, 2), mine = (q & 2 ? k1 : k0) | other;
    if (value) {
      const int pair = tok >> 1, half = (tok & 1) * 2, i4 = x8 >> 2;
      *(unsigned short*)(at + page_v_word(pair, 2 * q, i4) + half) = (unsigned short)mine;
      *(unsigned short*)(at + page_v_word(pair, 2 * q + 1, i4) + half) = (unsigned short)(mine >> 16);
      if (x8 == 0) *(uint32_t*)(at + kPageVp + tok * 4) = par;
    } else {
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w |= c[2 * e] << (4 * e) | c[2 * e + 1] << (4 * e + 16);
      *(uint32_t*)(at + tok * 64 + q * 16 + (x8 >> 2) * 4) = w;
      if (q == 0) *(uint32_t*)(at + kPageKp + tok * 16 + (x8 >> 2) * 4) = par;
      if (lane == 0 && p.bias) p.bias[((long long)page * p.H + h) * kPT + tok] = bias ? bias[row] : 0.f;
    }
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

template <typename T>
__global__ void __launch_bounds__(kPW) pages_read_kernel(const arckv_pages4 p, int N, const int* slots, T* K, T* V) {
  const int lane = threadIdx.x & 31, x8 = lane & 15;
  const bool value = lane >= 16;
  DevStatus* stt = (DevStatus*)p.state;
  pdl_trigger();
  pdl_wait();
  const long long rows = (long long)N * p.H, step = (long long)gridDim.x * (kPW / 32);
  T* out = value ? V : K;
  for (long long row = (long long)blockIdx.x * (kPW / 32) + (threadIdx.x >> 5); row < rows; row += step) {
    const int i = (int)quotient(row, p.H), h = (int)(row - (long long)i * p.H), slot = slots[i];
    const int page = slot / kPT, tok = slot % kPT;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && page >= p.P) {
      if (lane == 0) set_status(stt, ARCKV_ERR_INVALID_ARG);
    } else if (slot >= 0) {
      const unsigned char* at = page_at(p, page, h);
      const uint32_t par = *(const uint32_t*)(value ? at + kPageVp + tok * 4 : at + kPageKp + tok * 16 + (x8 >> 2) * 4);
      const float s = bf16_lo(par), m = bf16_hi(par);
      uint32_t w = 0;
      if (!value) w = *(const uint32_t*)(at + tok * 64 + (x8 & 3) * 16 + (x8 >> 2) * 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t c = (w >> (4 * (e >> 1) + 16 * (e & 1))) & 15u;
        if (value)
          c = (*(const unsigned short*)(at + page_v_word(tok >> 1, e, x8 >> 2) + (tok & 1) * 2) >> (4 * (x8 & 3))) & 15u;
        x[e] = fmaf((float)c, s, m);   // (a code times a scale is exact)
      }
    }
    if (out) store8(out + row * 128 + 8 * x8, x);
  }
}

}  // namespace

int launch_pages_append(const arckv_pages4& p, int N, bool f32, const void* K, PackedStrides ks, const void* V,
                        PackedStrides vs, const int* slots, const float* bias, cudaStream_t st) {
  const int ctas = stride_grid((long long)N * p.H, kPW / 32, 8);
  const cudaError_t e =
      f32 ? launch_pdl(pages_append_kernel<float>, dim3(ctas), kPW, 0, st, p, N, (const float*)K, ks, (const float*)V, vs, slots, bias)
          : launch_pdl(pages_append_kernel<bf16>, dim3(ctas), kPW, 0, st, p, N, (const bf16*)K, ks, (const bf16*)V, vs, slots, bias);
  return e == cudaSuccess ? 1 : -1;
}

int launch_pages_read(const arckv_pages4& p, int N, bool f32, const int* slots, void* K, void* V, cudaStream_t st) {
  const int ctas = stride_grid((long long)N * p.H, kPW / 32, 8);
  const cudaError_t e = f32 ? launch_pdl(pages_read_kernel<float>, dim3(ctas), kPW, 0, st, p, N, slots, (float*)K, (float*)V)
                            : launch_pdl(pages_read_kernel<bf16>, dim3(ctas), kPW, 0, st, p, N, slots, (bf16*)K, (bf16*)V);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
