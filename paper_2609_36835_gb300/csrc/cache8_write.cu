// Writing an 8-bit cache and reading it back.
//
//   a = max(max |x|, 2^-100) over the rows of a 64-token block, scale = a fl(1/127),
//   c = rint(x fl(127 / a)), stored as c + 128
//
// Both are one pass over memory, bound by HBM for prompts and by latency for a
// decode step's token.  Prompts: a CTA has one block's rows in registers; their
// least and largest elements by dimension give the magnitude and, as rounding
// keeps order, the bounds of the codes.  Few rows: a warp a head, which reads the
// staged rows again only when the magnitude has changed.
// Measured: 32 x 8 heads of 1638 fp32 rows written in 91 us (5.9 TB/s of sources and
// codes) and read back as bf16 in 55 (5.9 TB/s); 8 heads of 8191 bf16 rows in 15 us,
// bound by issue (75 %), and 9; one row of 64 x 8 heads in 6 to 8.5 us.
#include "cache8.cuh"

namespace arckv {
namespace {

constexpr int kWT = 256;    // threads of a block's CTA: 16 a row (8 dims each), 16 rows a round, 4 rounds
// Appends of up to so many rows take a warp for K or V of each head, and one launch (64 x 8 heads, one row: 5.9 us, eight:
// 6.7; by a CTA a block and the lengths behind it 9.3 and 11.5.  A single sequence: 5.4 and 4.4, but a launch more).
constexpr int kFewRows = 8;

// x * inv rounded to an integer, + 128, in the low byte: adding 1.5 * 2^23 leaves no fraction bits.  (The product is
// rounded first, as the definition says.)
__device__ __forceinline__ unsigned int code_bits(float x, float inv) {
  return __float_as_uint(__fadd_rn(__fmul_rn(x, inv), 12582912.f + 128.f));
}
__device__ __forceinline__ unsigned int pack4(unsigned int a, unsigned int b, unsigned int c, unsigned int d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ unsigned int codes4(float4 x, float inv) {
  return pack4(code_bits(x.x, inv), code_bits(x.y, inv), code_bits(x.z, inv), code_bits(x.w, inv));
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// Eight consecutive elements as they are held in memory.
struct Eight16 {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const bf16* p) { v = *(const uint4*)p; }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const unsigned int w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
struct Eight32 {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = *(const float4*)p;
    b = *((const float4*)p + 1);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
template <typename T> struct EightOf { using type = Eight32; };
template <> struct EightOf<bf16> { using type = Eight16; };

// Least and largest elements of a thread's 8 dims, NaN if there was one.
struct Range32 {
  float lo[8], hi[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = INFINITY;
      hi[e] = -INFINITY;
    }
  }
  __device__ __forceinline__ void add(const Eight32& q) {
    float x[8];
    q.get(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      asm("min.NaN.f32 %0, %0, %1;" : "+f"(lo[e]) : "f"(x[e]));
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(hi[e]) : "f"(x[e]));
    }
  }
  __device__ __forceinline__ void get(float (&l)[8], float (&h)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      l[e] = lo[e];
      h[e] = hi[e];
    }
  }
};
struct Range16 {   // two dims to a register
  __nv_bfloat162 lo[4], hi[4];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = __nv_bfloat162{__nv_bfloat16_raw{0x7f80}, __nv_bfloat16_raw{0x7f80}};
      hi[e] = __nv_bfloat162{__nv_bfloat16_raw{0xff80}, __nv_bfloat16_raw{0xff80}};
    }
  }
  __device__ __forceinline__ void add(const Eight16& q) {
    const unsigned int w[4] = {q.v.x, q.v.y, q.v.z, q.v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 x = *(const __nv_bfloat162*)&w[e];
      lo[e] = __hmin2_nan(lo[e], x);
      hi[e] = __hmax2_nan(hi[e], x);
    }
  }
  __device__ __forceinline__ void get(float (&l)[8], float (&h)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 a = __bfloat1622float2(lo[e]), b = __bfloat1622float2(hi[e]);
      l[2 * e] = a.x; l[2 * e + 1] = a.y;
      h[2 * e] = b.x; h[2 * e + 1] = b.y;
    }
  }
};
template <typename T> struct RangeOf { using type = Range32; };
template <> struct RangeOf<bf16> { using type = Range16; };

// Rows r0 .. r1 of a block are new, rows before r0 were written earlier and are
// staged in `tail`.  `stage`: the block becomes the newest one, its rows are staged.
template <typename T>
__device__ void write_block(const T* src, long long row_stride, int r0, int r1, bool stage, uint8_t* codes,
                            float* scale_at, int8_t* bounds, float* tail, float* tail_amax, DevStatus* stt) {
  __shared__ __align__(16) float s_lo[kWT / 32][128], s_hi[kWT / 32][128];
  __shared__ float s_amax[kWT / 32];
  const int tid = threadIdx.x, c8 = (tid & 15) * 8, rr = tid >> 4, lane = tid & 31, w = tid >> 5;
  typename EightOf<T>::type x[4];
  typename RangeOf<T>::type range;
  range.clear();
  if (r1 - r0 == kCB) {   // all loads before anything waits for them
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u].load(src + (long long)(rr + 16 * u) * row_stride + c8);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      x[u].zero();
      const int r = rr + 16 * u;
      if (r >= r0 && r < r1) x[u].load(src + (long long)(r - r0) * row_stride + c8);
    }
  }
  const float held = r0 > 0 ? *scale_at : 0.f;
  bool any = false;   // this thread has a new row
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = rr + 16 * u;
    if (r >= r0 && r < r1) {
      range.add(x[u]);
      any = true;
    }
  }
  float lo[8], hi[8], amax = 0.f;
  range.get(lo, hi);
  bool good = true;
  if (any) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      good = good && finite(lo[e]) && finite(hi[e]);
      amax = fmaxf(amax, fmaxf(-lo[e], hi[e]));
    }
  }
  if (__syncthreads_or(!good)) {   // elements that are not finite count, and are written, as zeros
    if (tid == 0) set_status(stt, ARCKV_ERR_NONFINITE);
    amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = INFINITY;
      hi[e] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float y[8];
      x[u].get(y);
      const bool here = rr + 16 * u >= r0 && rr + 16 * u < r1;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (here) {
          const float z = finite(y[e]) ? y[e] : 0.f;
          lo[e] = fminf(lo[e], z);
          hi[e] = fmaxf(hi[e], z);
          amax = fmaxf(amax, fabsf(z));
        }
    }
    good = false;
  }
  if (stage) {   // uniform over the block's threads
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = rr + 16 * u;
      float y[8], rm = 0.f;
      x[u].get(y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!finite(y[e])) y[e] = 0.f;
        rm = fmaxf(rm, fabsf(y[e]));
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) rm = fmaxf(rm, __shfl_xor_sync(0xffffffffu, rm, o));
      if (r >= r0 && r < r1) {
        *(float4*)(tail + r * 128 + c8) = make_float4(y[0], y[1], y[2], y[3]);
        *(float4*)(tail + r * 128 + c8 + 4) = make_float4(y[4], y[5], y[6], y[7]);
        if ((tid & 15) == 0) tail_amax[r] = rm;
      }
    }
  }
  if (r0 > 0) {   // earlier rows count for the bounds and the magnitude
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = rr + 16 * u;
      if (r < r0) {
        Eight32 q;
        q.a = *(const float4*)(tail + r * 128 + c8);
        q.b = *(const float4*)(tail + r * 128 + c8 + 4);
        float y[8];
        q.get(y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lo[e] = fminf(lo[e], y[e]);
          hi[e] = fmaxf(hi[e], y[e]);
          amax = fmaxf(amax, fabsf(y[e]));
        }
      }
    }
  }
  amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(amax))));   // (none is negative)
  if (lane == 0) s_amax[w] = amax;
  if (bounds) {   // of the warp's two rows of threads, then of its CTA
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = fminf(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], 16));
      hi[e] = fmaxf(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], 16));
    }
    if (lane < 16) {
      *(float4*)&s_lo[w][c8] = make_float4(lo[0], lo[1], lo[2], lo[3]);
      *(float4*)&s_lo[w][c8 + 4] = make_float4(lo[4], lo[5], lo[6], lo[7]);
      *(float4*)&s_hi[w][c8] = make_float4(hi[0], hi[1], hi[2], hi[3]);
      *(float4*)&s_hi[w][c8 + 4] = make_float4(hi[4], hi[5], hi[6], hi[7]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWT / 32; ++i) amax = fmaxf(amax, s_amax[i]);
  amax = fmaxf(amax, kCacheFloor);
  const float scale = amax * kInv127, inv = __fdiv_rn(127.f, amax);
  const bool again = r0 > 0 && held != scale;   // the earlier rows' codes change with the scale
  if (tid == 0) *scale_at = scale;
  if (bounds && tid < 64) {   // codes of the extremes: thread (low or high, four dims)
    const float(*src4)[128] = tid < 32 ? s_lo : s_hi;
    float4 m = *(const float4*)&src4[0][lane * 4];
#pragma unroll
    for (int i = 1; i < kWT / 32; ++i) {
      const float4 y = *(const float4*)&src4[i][lane * 4];
      if (tid < 32) m = make_float4(fminf(m.x, y.x), fminf(m.y, y.y), fminf(m.z, y.z), fminf(m.w, y.w));
      else m = make_float4(fmaxf(m.x, y.x), fmaxf(m.y, y.y), fmaxf(m.z, y.z), fmaxf(m.w, y.w));
    }
    *(unsigned int*)(bounds + (tid >> 5) * 128 + lane * 4) = codes4(m, inv) ^ 0x80808080u;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = rr + 16 * u;
    if (r < r1 && (r >= r0 || again)) {
      float y[8];
      x[u].get(y);
      if (r < r0) {
        Eight32 q;
        q.a = *(const float4*)(tail + r * 128 + c8);
        q.b = *(const float4*)(tail + r * 128 + c8 + 4);
        q.get(y);
      }
      if (!good)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = finite(y[e]) ? y[e] : 0.f;
      *(uint2*)(codes + r * 128 + c8) = make_uint2(codes4(make_float4(y[0], y[1], y[2], y[3]), inv),
                                                   codes4(make_float4(y[4], y[5], y[6], y[7]), inv));
    }
  }
  __syncthreads();   // shared arrays and the staged rows are free for the next block
}

// What an append does to one sequence.
struct Span {
  int a0, cnt;
  bool fits;
};
__device__ __forceinline__ Span span_of(const arckv_cache8& c, int s, int n, const int* at, const int* counts, int* len) {
  Span p;
  *len = c.len[s];
  p.cnt = counts ? counts[s] : n;
  p.a0 = at ? at[s] : *len;
  p.fits = *len >= 0 && *len <= c.cap && p.cnt >= 0 && p.cnt <= n && p.a0 >= 0 && p.a0 <= *len && p.cnt <= c.cap - p.a0 &&
           ((p.a0 & (kCB - 1)) == 0 || p.a0 / kCB == (*len - 1) / kCB);
  return p;
}

// The lengths after an append, from one CTA.
__device__ __forceinline__ void set_lengths(const arckv_cache8& c, int n, const int* at, const int* counts) {
  for (int i = threadIdx.x; i < c.S; i += blockDim.x) {
    int len;
    const Span p = span_of(c, i, n, at, counts, &len);
    if (p.fits && p.cnt > 0) c.len[i] = p.a0 + p.cnt;
  }
}

// The last CTA of a grid to get here advances the lengths (all threads of a CTA call it).
__device__ __forceinline__ void advance(const arckv_cache8& c, int n, const int* at, const int* counts) {
  __shared__ bool done;
  DevStatus* stt = (DevStatus*)c.state;
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned int all = gridDim.x * gridDim.y * gridDim.z;
    __threadfence();
    done = atomicAdd(state_ticket(stt), 1u) == all - 1;
    if (done) *state_ticket(stt) = 0;
  }
  __syncthreads();
  if (done) set_lengths(c, n, at, counts);
}

// The same as a kernel of its own, behind a prompt's many CTAs: a ticket would keep each of them for the 1.5 us that
// its counter takes to answer (32 x 8 heads of 1638 fp32 rows: 106 instead of 91 us).
__global__ void __launch_bounds__(256) cache_lengths_kernel(const arckv_cache8 c, int n, const int* at, const int* counts) {
  pdl_trigger();
  pdl_wait();
  set_lengths(c, n, at, counts);
}

// CTA (x, (head, K or V), sequence) writes the x-th touched block.  Where the
// first one holds earlier rows, which it reads where they are staged, its CTA
// writes the last one too, whose rows are then staged there.
template <typename T>
__global__ void __launch_bounds__(kWT, 4) cache_append_kernel(const arckv_cache8 c, int n, const T* K, RowStrides ks,
                                                           const T* V, RowStrides vs, const float* bias, const int* at,
                                                           const int* counts) {
  pdl_trigger();
  pdl_wait();
  const int s = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1;
  DevStatus* stt = (DevStatus*)c.state;
  int len;
  const Span p = span_of(c, s, n, at, counts, &len);
  if (!p.fits && threadIdx.x == 0) set_status(stt, ARCKV_ERR_SHAPE);
  if (p.fits && p.cnt > 0) {
    const int end = p.a0 + p.cnt, first = p.a0 / kCB, last = (end - 1) / kCB;
    const T* src = which ? V + s * vs.s + h * vs.h : K + s * ks.s + h * ks.h;
    const long long stride = which ? vs.i : ks.i, sh = (long long)s * c.H + h;
    const int nblk = c.cap / kCB;
    const bool both = (p.a0 & (kCB - 1)) != 0 && last != first;
    for (int pass = 0; pass < 2; ++pass) {
      const int b = pass == 0 ? first + (int)blockIdx.x : last;
      if (pass == 0 ? (b > last || (both && blockIdx.x > 0 && b == last)) : (blockIdx.x > 0 || !both)) continue;
      const int r0 = max(p.a0 - b * kCB, 0), r1 = min(end - b * kCB, kCB);
      const long long blk = sh * nblk + b;
      write_block(src + (long long)(b * kCB + r0 - p.a0) * stride, stride, r0, r1, b == last,
                  (which ? c.V : c.K) + blk * (kCB * 128), (which ? c.v_scale : c.k_scale) + blk,
                  which ? nullptr : c.bounds + blk * 256, c.tail + (sh * 2 + which) * (kCB * 128),
                  c.tail_amax + (sh * 2 + which) * kCB, stt);
      if (!which && c.bias && (int)threadIdx.x >= r0 && (int)threadIdx.x < r1) {
        const int j = b * kCB + threadIdx.x;
        c.bias[sh * c.cap + j] = bias ? bias[sh * n + j - p.a0] : 0.f;
      }
    }
  }
}

__device__ __forceinline__ float4 load4(const float* p) { return *(const float4*)p; }
__device__ __forceinline__ float4 load4(const bf16* p) {
  const uint2 v = *(const uint2*)p;
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xffff0000u));
}

// Up to kFewRows new rows: one warp for K or V of a head, lane l dims 4l .. 4l + 3.
template <typename T>
__global__ void __launch_bounds__(128) cache_append_few_kernel(const arckv_cache8 c, int n, const T* K, RowStrides ks,
                                                               const T* V, RowStrides vs, const float* bias,
                                                               const int* at, const int* counts) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, d4 = lane * 4, nblk = c.cap / kCB;
  const long long item = blockIdx.x * 4ll + (threadIdx.x >> 5);
  if (item < 2ll * c.S * c.H) {
    const long long sh = item >> 1;
    const int which = (int)(item & 1), s = (int)(sh / c.H), h = (int)(sh - (long long)s * c.H);
    DevStatus* stt = (DevStatus*)c.state;
    int len;
    const Span p = span_of(c, s, n, at, counts, &len);
    if (!p.fits && lane == 0) set_status(stt, ARCKV_ERR_SHAPE);
    const T* src = which ? V + s * vs.s + h * vs.h : K + s * ks.s + h * ks.h;
    const long long stride = which ? vs.i : ks.i;
    float* tail = c.tail + item * (kCB * 128);
    float* tail_amax = c.tail_amax + item * kCB;
    const int end = p.fits ? p.a0 + p.cnt : p.a0;   // (none of a span that does not fit)
    for (int j = p.a0; j < end;) {   // a block at a time
      const int b = j / kCB, r0 = j - b * kCB, r1 = min(kCB, end - b * kCB);
      const long long blk = sh * nblk + b;
      uint8_t* codes = (which ? c.V : c.K) + blk * (kCB * 128);
      float* scale_at = (which ? c.v_scale : c.k_scale) + blk;
      const float held = r0 > 0 ? *scale_at : 0.f;
      float amax = 0.f;
      if (lane < r0) amax = tail_amax[lane];
      if (lane + 32 < r0) amax = fmaxf(amax, tail_amax[lane + 32]);
      float4 x[kFewRows];
      float4 lo = make_float4(INFINITY, INFINITY, INFINITY, INFINITY), hi = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      auto widen = [&](float4 y) {
        lo = make_float4(fminf(lo.x, y.x), fminf(lo.y, y.y), fminf(lo.z, y.z), fminf(lo.w, y.w));
        hi = make_float4(fmaxf(hi.x, y.x), fmaxf(hi.y, y.y), fmaxf(hi.z, y.z), fmaxf(hi.w, y.w));
      };
#pragma unroll
      for (int i = 0; i < kFewRows; ++i)
        if (i < r1 - r0) x[i] = load4(src + (long long)(j - p.a0 + i) * stride + d4);
      // earlier rows whose bounds are not those held (others are to be written over), 16 loads at a time
      auto earlier = [&](auto use) {
        for (int r = 0; r < r0; r += 16) {
          float4 y[16];
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (r + i < r0) y[i] = *(const float4*)(tail + (r + i) * 128 + d4);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (r + i < r0) use(r + i, y[i]);
        }
      };
      const bool over = r0 > 0 && p.a0 != len;
      if (over && !which) earlier([&](int, float4 y) { widen(y); });
      bool good = true;
#pragma unroll
      for (int i = 0; i < kFewRows; ++i)
        if (i < r1 - r0) {
          float* y = &x[i].x;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!finite(y[e])) {
              y[e] = 0.f;
              good = false;
            }
          float m = fmaxf(fmaxf(fabsf(x[i].x), fabsf(x[i].y)), fmaxf(fabsf(x[i].z), fabsf(x[i].w)));
          m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
          amax = fmaxf(amax, m);
          widen(x[i]);
          if (lane == 0 && b == (end - 1) / kCB) tail_amax[r0 + i] = m;   // (rows before r0 are other elements)
        }
      if (!good) set_status(stt, ARCKV_ERR_NONFINITE);
      amax = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax))), kCacheFloor);
      const float scale = amax * kInv127, inv = __fdiv_rn(127.f, amax);
      const bool again = r0 > 0 && held != scale;   // the earlier rows' codes change with the scale
      if (lane == 0) *scale_at = scale;
#pragma unroll
      for (int i = 0; i < kFewRows; ++i)
        if (i < r1 - r0) *(unsigned int*)(codes + (r0 + i) * 128 + d4) = codes4(x[i], inv);
      if (again)
        earlier([&](int r, float4 y) {
          *(unsigned int*)(codes + r * 128 + d4) = codes4(y, inv);
          widen(y);
        });
      if (!which) {
        unsigned int l = codes4(lo, inv), g = codes4(hi, inv);
        unsigned int* bounds = (unsigned int*)(c.bounds + blk * 256) + lane;
        if (r0 > 0 && !again && !over) {
          l = __vminu4(l, bounds[0] ^ 0x80808080u);
          g = __vmaxu4(g, bounds[32] ^ 0x80808080u);
        }
        bounds[0] = l ^ 0x80808080u;
        bounds[32] = g ^ 0x80808080u;
        if (c.bias && lane < r1 - r0)
          c.bias[sh * c.cap + j + lane] = bias ? bias[sh * n + j - p.a0 + lane] : 0.f;
      }
      if (b == (end - 1) / kCB) {   // the newest block's rows stay staged (over those of a block that is now full)
#pragma unroll
        for (int i = 0; i < kFewRows; ++i)
          if (i < r1 - r0) *(float4*)(tail + (r0 + i) * 128 + d4) = x[i];
      }
      __syncwarp();
      j += r1 - r0;
    }
  }
  advance(c, n, at, counts);
}

__device__ __forceinline__ float code_value(unsigned int word, int byte, float scale) {
  return (float)((int)((word >> (8 * byte)) & 0xffu) - 128) * scale;
}

// Eight threads a row, 16 codes each.
template <bool kF32>
__global__ void __launch_bounds__(256) cache_read_kernel(const arckv_cache8 c, int start, int count, void* Ko,
                                                         void* Vo, long long rows) {
  pdl_trigger();
  pdl_wait();
  const bool v = blockIdx.y != 0;
  void* out = v ? Vo : Ko;
  if (!out) return;
  const uint8_t* codes = v ? c.V : c.K;
  const float* scales = v ? c.v_scale : c.k_scale;
  for (long long t = blockIdx.x * 256ll + threadIdx.x; t < rows * 8; t += gridDim.x * 256ll) {
    const long long row = t >> 3, sh = row / count;
    const int i = (int)(row - sh * count), ch = (int)(t & 7), len = cache_len(c, (int)(sh / c.H));
    const long long tok = (start < 0 ? (long long)len : 0) + start + i;
    uint4 q = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
    float sc = 0.f;
    if (tok >= 0 && tok < len) {
      q = *(const uint4*)(codes + (sh * c.cap + tok) * 128 + ch * 16);
      sc = scales[sh * (c.cap / kCB) + tok / kCB];
    }
    const unsigned int w[4] = {q.x, q.y, q.z, q.w};
    if (kF32) {
      float4* d = (float4*)((float*)out + row * 128 + ch * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        d[e] = make_float4(code_value(w[e], 0, sc), code_value(w[e], 1, sc), code_value(w[e], 2, sc),
                           code_value(w[e], 3, sc));
    } else {
      __nv_bfloat162 p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        p[e] = __floats2bfloat162_rn(code_value(w[e >> 1], 2 * (e & 1), sc), code_value(w[e >> 1], 2 * (e & 1) + 1, sc));
      uint4* d = (uint4*)((bf16*)out + row * 128 + ch * 16);
      d[0] = *(const uint4*)&p[0];
      d[1] = *(const uint4*)&p[4];
    }
  }
}

}  // namespace

int launch_cache_append(const arckv_cache8& c, int n, bool f32, const void* K, RowStrides ks, const void* V,
                        RowStrides vs, const float* bias, const int* at, const int* counts, cudaStream_t st) {
  if (n <= kFewRows) {
    const dim3 grid((unsigned)((2ll * c.S * c.H + 3) / 4));
    const cudaError_t e = f32 ? launch_pdl(cache_append_few_kernel<float>, grid, 128, 0, st, c, n, (const float*)K, ks,
                                           (const float*)V, vs, bias, at, counts)
                              : launch_pdl(cache_append_few_kernel<bf16>, grid, 128, 0, st, c, n, (const bf16*)K, ks,
                                           (const bf16*)V, vs, bias, at, counts);
    return e == cudaSuccess ? 1 : -1;
  }
  const dim3 grid((n + kCB - 2) / kCB + 1, c.H * 2, c.S);   // blocks that n rows can touch
  const cudaError_t e = f32 ? launch_pdl(cache_append_kernel<float>, grid, kWT, 0, st, c, n, (const float*)K, ks,
                                         (const float*)V, vs, bias, at, counts)
                            : launch_pdl(cache_append_kernel<bf16>, grid, kWT, 0, st, c, n, (const bf16*)K, ks,
                                         (const bf16*)V, vs, bias, at, counts);
  if (e != cudaSuccess || launch_pdl(cache_lengths_kernel, dim3(1), 256, 0, st, c, n, at, counts) != cudaSuccess) return -1;
  return 2;
}

int launch_cache_read(const arckv_cache8& c, int start, int count, bool f32, void* K, void* V, cudaStream_t st) {
  const long long rows = (long long)c.S * c.H * count;
  const dim3 grid(stride_grid(rows * 8, 256, 8), 2);
  const cudaError_t e = launch_pdl(f32 ? cache_read_kernel<true> : cache_read_kernel<false>, grid, 256, 0, st, c, start,
                                   count, K, V, rows);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
