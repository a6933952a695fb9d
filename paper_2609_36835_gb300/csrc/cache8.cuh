// Shared definitions of the 8-bit cache kernels (arckv_cache8 in arckv.h).
#pragma once
#include <algorithm>

#include <cuda_fp16.h>

#include "kernels.h"

namespace arckv {

constexpr int kCB = ARCKV_CACHE_BLOCK;   // tokens of a block
constexpr int kTileBytes = kCB * 128;    // codes of one block, K or V
constexpr float kCacheFloor = 7.888609052210118e-31f;   // 2^-100: least block magnitude, so that 127 / a stays finite
constexpr float kInv127 = 0.007874015718698502f;        // fl(1 / 127)

// Rows addressed by (sequence, head, position), in elements from the base.
struct RowStrides {
  long long s, h, i;
};

// First counter of a cache's `state` after the status word.
__device__ __forceinline__ unsigned int* state_ticket(DevStatus* st) { return &st->pad[0]; }

// Tokens that position p of n_pos sees in a sequence of len tokens.
__device__ __forceinline__ int visible_tokens(int len, int n_pos, int p, bool causal) {
  return causal ? max(0, len - n_pos + 1 + p) : len;
}
__device__ __forceinline__ int cache_len(const arckv_cache8& c, int s) { return min(max(c.len[s], 0), c.cap); }

// Workspace of cache_attend: the header (status word, then one ticket for each
// CTA of the split kernels), then partial results.
constexpr int kCacheMaxCtas = 160;   // CTAs of the persistent kernels, at most one for each SM
__host__ __device__ inline int* ws_tickets(void* ws) { return (int*)((char*)ws + sizeof(DevStatus)); }
static_assert(sizeof(DevStatus) + kCacheMaxCtas * sizeof(int) <= ARCKV_CACHE_WS_HEADER, "tickets fit the header");

// a / b for a >= 0, b > 0, in 32 bits where both fit.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return (long long)((unsigned int)a / (unsigned int)b);
  return a / b;
}
// Equal shares of `total` units: CTA c has [start(c), start(c + 1)), one unit more for the first r.
struct CacheShares {
  long long total, q;
  int ctas, r;
  __device__ CacheShares(long long units, int grid) : total(units), ctas((int)min((long long)grid, units)) {
    q = quotient(total, ctas);
    r = (int)(total - q * ctas);
  }
  __device__ long long start(int c) const { return q * c + min(c, r); }
  __device__ int owner(long long u) const {   // the CTA that has unit u
    const long long big = r * (q + 1);
    return u < big ? (int)quotient(u, q + 1) : r + (int)quotient(u - big, q);
  }
};

// ---- codes as f16 operands ----------------------------------------------------
// Two bytes of w, codes + 128, as f16 codes: 1024 + u is 0x6400 | u.
template <unsigned kPick>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {
  const uint32_t y = __byte_perm(w, 0x64646464u, kPick);
  const __half2 z = __hsub2(*(const __half2*)&y, __half2{__half_raw{0x6480}, __half_raw{0x6480}});
  return *(const uint32_t*)&z;
}
// Four 8 x 8 matrices of 16-bit units, transposed; lane 8i + r gives the address of row r of matrix i.
__device__ __forceinline__ void load_transposed(uint32_t (&w)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "r"(addr));
}

// ---- softmax weights ------------------------------------------------------------
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// x - h, exactly, in one mixed-precision operation each.
__device__ __forceinline__ float2 minus_f16(float2 x, __half2 h) {
  float2 d;
  asm("{\n\t.reg .b16 p, q, m;\n\tmov.b32 {p, q}, %2;\n\tmov.b16 m, 0xBC00;\n\t"   // -1
      "fma.rn.f32.f16 %0, p, m, %3;\n\tfma.rn.f32.f16 %1, q, m, %4;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "r"(*(const uint32_t*)&h), "f"(x.x), "f"(x.y));
  return d;
}

// ---- launches that overlap their predecessor's end ---------------------------
// The kernels of this file's callers start while the kernel before them on the
// stream is still ending: pdl_wait() comes before their first access to memory
// that another kernel may write or read, and pdl_trigger() lets the next one in
// as soon as all CTAs have started.  What the kernel before may still write is not
// read-only for this one's whole life: loads are plain ones, never those of the
// read-only path, which the compiler may also move above the wait.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_pdl(void (*kern)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

// ---- launchers (each returns the kernels it enqueued, or -1) ---------------
int launch_cache_append(const arckv_cache8& c, int n, bool f32, const void* K, RowStrides ks, const void* V,
                        RowStrides vs, const float* bias, const int* at, const int* counts, cudaStream_t st);
int launch_cache_read(const arckv_cache8& c, int start, int count, bool f32, void* K, void* V, cudaStream_t st);

struct CacheQuery {
  int n_pos, G;
  bool causal;
  const bf16* Q;
  RowStrides qs;
};
size_t cache_attend_scratch(int S, int H, int cap, int n_pos, int G);
int launch_cache_attend(const arckv_cache8& c, const CacheQuery& q, float scale, const int* blocks, int m, float* O,
                        RowStrides os, void* ws, cudaStream_t st);
// the same for more than 16 rows of a head over all tokens
size_t cache_tiles_scratch(long long rows);
int launch_cache_tiles(const arckv_cache8& c, const CacheQuery& q, float scale, float* O, RowStrides os, void* ws,
                       cudaStream_t st);
size_t cache_select_scratch(int S, int H, int cap, int n_pos, int G);
int launch_cache_select(const arckv_cache8& c, const CacheQuery& q, int m, int keep_first, int keep_last, int* blocks,
                        void* ws, cudaStream_t st);

}  // namespace arckv
