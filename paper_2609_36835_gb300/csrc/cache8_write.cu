// Writing an 8-bit cache and reading it back.
//
//   a = max(max |x|, 2^-100) over the rows of a 64-token block, scale = a fl(1/127),
//   c = rint(x fl(127 / a)), stored as c + 128
//
// Both are one pass over memory.  A prompt moves 2 (bf16) bytes in and 1 out an
// element; a decode step's single token touches a few rows of one block.
#include "cache8.cuh"

namespace arckv {
namespace {

constexpr int kWT = 256;   // threads: 16 per row (8 dims each), 16 rows a round, 4 rounds

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = __ldg((const float4*)p), b = __ldg((const float4*)p + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const uint4 v = __ldg((const uint4*)p);
  const __nv_bfloat162* h = (const __nv_bfloat162*)&v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __bfloat1622float2(h[e]);
    x[2 * e] = f.x;
    x[2 * e + 1] = f.y;
  }
}

// Rows r0 .. r1 of a block are new, rows before r0 were written earlier and are
// staged in `tail`.  `stage`: the block becomes the newest one, its rows are staged.
template <typename T>
__device__ void write_block(const T* src, long long row_stride, int r0, int r1, bool stage, uint8_t* codes,
                            float* scale_at, int8_t* bounds, float* tail, float* tail_amax, DevStatus* stt) {
  __shared__ float s_amax[kWT / 32];
  __shared__ uint2 s_lo[kWT / 32][16], s_hi[kWT / 32][16];
  const int tid = threadIdx.x, c8 = (tid & 15) * 8, rr = tid >> 4, lane = tid & 31, w = tid >> 5;
  float x[4][8], amax = 0.f;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = rr + 16 * u;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
    if (r >= r0 && r < r1) {
      load8(src + (long long)(r - r0) * row_stride + c8, x[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!(fabsf(x[u][e]) <= 3.402823466e38f)) {
          x[u][e] = 0.f;
          bad = true;
        }
        m = fmaxf(m, fabsf(x[u][e]));
      }
    }
    if (stage) {   // uniform over the block's threads
      float rm = m;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) rm = fmaxf(rm, __shfl_xor_sync(0xffffffffu, rm, o));
      if (r >= r0 && r < r1) {
        *(float4*)(tail + r * 128 + c8) = make_float4(x[u][0], x[u][1], x[u][2], x[u][3]);
        *(float4*)(tail + r * 128 + c8 + 4) = make_float4(x[u][4], x[u][5], x[u][6], x[u][7]);
        if ((tid & 15) == 0) tail_amax[r] = rm;
      }
    }
    amax = fmaxf(amax, m);
  }
  if (bad) set_status(stt, ARCKV_ERR_NONFINITE);
  if (tid < r0) amax = fmaxf(amax, tail_amax[tid]);
  amax = warp_max(amax);
  if (lane == 0) s_amax[w] = amax;
  const float held = r0 > 0 ? *scale_at : 0.f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWT / 32; ++i) amax = fmaxf(amax, s_amax[i]);
  amax = fmaxf(amax, kCacheFloor);
  const float scale = amax * kInv127, inv = __fdiv_rn(127.f, amax);
  const bool again = r0 > 0 && held != scale;   // the earlier rows' codes change with the scale
  if (tid == 0) *scale_at = scale;
  unsigned int lo[2] = {0x7f7f7f7fu, 0x7f7f7f7fu}, hi[2] = {0x80808080u, 0x80808080u};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = rr + 16 * u;
    if (r >= r1) continue;
    uint2 q;
    if (r >= r0 || again) {
      if (r < r0) load8(tail + r * 128 + c8, x[u]);
      unsigned int b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = (unsigned int)__float2int_rn(x[u][e] * inv) & 0xffu;
      q.x = (b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24) ^ 0x80808080u;
      q.y = (b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24) ^ 0x80808080u;
      *(uint2*)(codes + r * 128 + c8) = q;
    } else if (bounds) {
      q = *(const uint2*)(codes + r * 128 + c8);
    }
    if (bounds) {
      lo[0] = __vmins4(lo[0], q.x ^ 0x80808080u);
      lo[1] = __vmins4(lo[1], q.y ^ 0x80808080u);
      hi[0] = __vmaxs4(hi[0], q.x ^ 0x80808080u);
      hi[1] = __vmaxs4(hi[1], q.y ^ 0x80808080u);
    }
  }
  if (bounds) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lo[i] = __vmins4(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], 16));
      hi[i] = __vmaxs4(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], 16));
    }
    if (lane < 16) {
      s_lo[w][lane] = make_uint2(lo[0], lo[1]);
      s_hi[w][lane] = make_uint2(hi[0], hi[1]);
    }
    __syncthreads();
    if (tid < 16) {
      uint2 l = s_lo[0][tid], g = s_hi[0][tid];
      for (int i = 1; i < kWT / 32; ++i) {
        l.x = __vmins4(l.x, s_lo[i][tid].x);
        l.y = __vmins4(l.y, s_lo[i][tid].y);
        g.x = __vmaxs4(g.x, s_hi[i][tid].x);
        g.y = __vmaxs4(g.y, s_hi[i][tid].y);
      }
      *(uint2*)(bounds + tid * 8) = l;
      *(uint2*)(bounds + 128 + tid * 8) = g;
    }
  }
  __syncthreads();   // shared arrays and the staged rows are free for the next block
}

// CTA (x, (head, K or V), sequence): x = 0 writes the first touched block, then
// the last one (whose staged rows replace those the first reads); x > 0 the
// x-th block between them.  The last CTA to finish advances the lengths.
template <typename T>
__global__ void __launch_bounds__(kWT) cache_append_kernel(const arckv_cache8 c, int n, const T* K, RowStrides ks,
                                                           const T* V, RowStrides vs, const float* bias, const int* at,
                                                           const int* counts) {
  const int s = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1;
  DevStatus* stt = (DevStatus*)c.state;
  const int len = c.len[s], cnt = counts ? counts[s] : n, a0 = at ? at[s] : len;
  const bool fits = len >= 0 && len <= c.cap && cnt >= 0 && cnt <= n && a0 >= 0 && a0 <= len && cnt <= c.cap - a0 &&
                    ((a0 & (kCB - 1)) == 0 || a0 / kCB == (len - 1) / kCB);
  if (!fits && threadIdx.x == 0) set_status(stt, ARCKV_ERR_SHAPE);
  if (fits && cnt > 0) {
    const int end = a0 + cnt, first = a0 / kCB, last = (end - 1) / kCB;
    const T* src = which ? V + s * vs.s + h * vs.h : K + s * ks.s + h * ks.h;
    const long long stride = which ? vs.i : ks.i, sh = (long long)s * c.H + h;
    const int nblk = c.cap / kCB;
    for (int pass = 0; pass < 2; ++pass) {
      const int b = pass == 0 ? first + (int)blockIdx.x : last;
      if (pass == 0 ? (b > last || (blockIdx.x > 0 && b == last)) : (blockIdx.x > 0 || last == first)) continue;
      const int r0 = max(a0 - b * kCB, 0), r1 = min(end - b * kCB, kCB);
      const long long blk = sh * nblk + b;
      write_block(src + (long long)(b * kCB + r0 - a0) * stride, stride, r0, r1, b == last,
                  (which ? c.V : c.K) + blk * (kCB * 128), (which ? c.v_scale : c.k_scale) + blk,
                  which ? nullptr : c.bounds + blk * 256, c.tail + (sh * 2 + which) * (kCB * 128),
                  c.tail_amax + (sh * 2 + which) * kCB, stt);
      if (!which && c.bias && threadIdx.x >= r0 && threadIdx.x < r1) {
        const int j = b * kCB + threadIdx.x;
        c.bias[sh * c.cap + j] = bias ? bias[sh * n + j - a0] : 0.f;
      }
    }
  }
  __shared__ bool done;
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned int all = gridDim.x * gridDim.y * gridDim.z;
    __threadfence();
    done = atomicAdd(state_ticket(stt), 1u) == all - 1;
    if (done) *state_ticket(stt) = 0;
  }
  __syncthreads();
  if (done)
    for (int i = threadIdx.x; i < c.S; i += kWT) {
      const int l = c.len[i], k = counts ? counts[i] : n, a = at ? at[i] : l;
      if (l >= 0 && l <= c.cap && k > 0 && k <= n && a >= 0 && a <= l && k <= c.cap - a &&
          ((a & (kCB - 1)) == 0 || a / kCB == (l - 1) / kCB))
        c.len[i] = a + k;
    }
}

__device__ __forceinline__ float code_value(unsigned int word, int byte, float scale) {
  return (float)((int)((word >> (8 * byte)) & 0xffu) - 128) * scale;
}

// Eight threads a row, 16 codes each.
template <bool kF32>
__global__ void __launch_bounds__(256) cache_read_kernel(const arckv_cache8 c, int start, int count, void* Ko,
                                                         void* Vo, long long rows) {
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
  // blocks between the first and the last that n rows can touch, and the CTA of those two
  const dim3 grid(std::max(1, (n + kCB - 2) / kCB), c.H * 2, c.S);
  if (f32)
    cache_append_kernel<float><<<grid, kWT, 0, st>>>(c, n, (const float*)K, ks, (const float*)V, vs, bias, at, counts);
  else
    cache_append_kernel<bf16><<<grid, kWT, 0, st>>>(c, n, (const bf16*)K, ks, (const bf16*)V, vs, bias, at, counts);
  return 1;
}

int launch_cache_read(const arckv_cache8& c, int start, int count, bool f32, void* K, void* V, cudaStream_t st) {
  const long long rows = (long long)c.S * c.H * count;
  const dim3 grid(stride_grid(rows * 8, 256, 4), 2);
  if (f32)
    cache_read_kernel<true><<<grid, 256, 0, st>>>(c, start, count, K, V, rows);
  else
    cache_read_kernel<false><<<grid, 256, 0, st>>>(c, start, count, K, V, rows);
  return 1;
}

}  // namespace arckv
