// Shared definitions of the paged 4-bit cache kernels (arckv_pages4 in arckv.h).
#pragma once
#include "cache8.cuh"

namespace arckv {

// ---- a page of one head, 9472 bytes -------------------------------------------
// 64 rows of K codes, 64 bytes each: bytes 16 t + 4 w of a row hold the word of dims 32 w + 8 t .. + 7, so that 16 bytes
//   have eight dims of every group, what a lane (row, t) of a matrix product takes.  In a word, nibble j is dim 2 j and
//   nibble j + 4 dim 2 j + 1: one mask leaves a pair of neighbours in the halves.
// 32 pairs of tokens of V codes, 128 bytes each: chunk g ^ 2 (pair % 4) of 16 bytes holds dims g + 8 x, x = 0 .. 15, four to
//   a word; a word's low half is the even token's, its high half the odd one's: one mask leaves two tokens of one dim.
//   (The exclusive or spreads four pairs over the banks.)
// (s, m) of K, bf16 each, for 4 groups of 64 tokens; then of V for 64 tokens.
constexpr int kPT = ARCKV_PAGE_TOKENS;
constexpr int kPageV = 4096, kPageKp = 8192, kPageVp = 9216;
constexpr float kScaleFloor = 7.888609052210118e-31f;   // 2^-100: least scale, so that 1 / s stays finite
constexpr float kInv15 = 0.06666667014360428f;          // fl(1 / 15)
constexpr float kPagesMost = 1.8446744073709552e19f;     // 2^64: largest magnitude held, so that sums of 2^41 values times weights stay finite
constexpr float kLogitMost = 8388608.f;                  // 2^23: largest logit times log2 e that a reference of the softmax may take
static_assert(kPageVp + kPT * 4 == ARCKV_PAGE_BYTES && ARCKV_PAGE_BYTES % 16 == 0, "a page is copied in one piece");

__host__ __device__ inline int page_v_word(int pair, int g, int i) {   // byte offset of word i of chunk g
  return kPageV + pair * 128 + ((g ^ ((pair & 3) << 1)) << 4) + (i << 2);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ int pages_len(const arckv_pages4& p, int s) { return min(max(p.len[s], 0), p.M * kPT); }
__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPT - 1) / kPT; }
__device__ __forceinline__ const unsigned char* page_at(const arckv_pages4& p, int page, int h) {
  return p.data + ((long long)page * p.H + h) * ARCKV_PAGE_BYTES;
}

// Rows addressed by (row, head), in elements from the base.
struct PackedStrides {
  long long i, h;
};

struct PagesQuery {
  int N, G, max_count;
  bool causal;
  const bf16* Q;
  PackedStrides qs;
  const int* starts;
  bf16* O;
  PackedStrides os;
};

// Rows of a row tile of the many-row kernel where a request has up to `rows` rows of a head.
inline int pages_tile_rows(long long rows) { return rows <= 128 ? 128 : 256; }

// ---- launchers (each returns the kernels it enqueued, or -1) ---------------
int launch_pages_extend(const arckv_pages4& p, const int* counts, int N, int* starts, int* slots, int* positions,
                        cudaStream_t st);
int launch_pages_truncate(const arckv_pages4& p, const int* lens, cudaStream_t st);
int launch_pages_append(const arckv_pages4& p, int N, bool f32, const void* K, PackedStrides ks, const void* V,
                        PackedStrides vs, const int* slots, const float* bias, cudaStream_t st);
int launch_pages_read(const arckv_pages4& p, int N, bool f32, const int* slots, void* K, void* V, cudaStream_t st);
size_t pages_attend_scratch(int S, int H, int M, int max_count, int G);
int launch_pages_attend(const arckv_pages4& p, const PagesQuery& q, float scale, void* ws, cudaStream_t st);
// the same for requests of more than `above` rows of a head
size_t pages_tiles_scratch(long long rows);
int launch_pages_tiles(const arckv_pages4& p, const PagesQuery& q, float scale, int above, void* ws, cudaStream_t st);

struct RotateTensor {
  const void* x;
  void* y;
  PackedStrides xs, ys;
  int heads;
};
int launch_rotate(int N, int d, int r, float f, const unsigned long long* turns, const int* positions,
                  const RotateTensor (&t)[2], bool f32, bool interleaved, bool transpose, cudaStream_t st);

}  // namespace arckv
