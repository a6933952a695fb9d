// Attention of many query rows over an 8-bit cache (prompt chunks, reference
// queries): the products of cache8_attend.cu on tcgen05.
//
// With n rows a head every code is used n times, so the call is bound by the
// tensor pipe.  A CTA takes 128 or 256 rows of one head (one or two M = 128
// tiles) and goes over the keys a block of 64 at a time:
//   codes (1 warp)        TMA of a block's codes (64 x 128 of K and of V) into a ring
//   converters (4 warps)  codes to f16 operands in shared memory, V transposed by
//                         matrix loads and stores, three blocks ahead; a code costs
//                         about one instruction for 256 rows
//   MMA warp              S = Q K^T (exact products, fp32 sums in TMEM), O += P V
//   softmax (8 warps a tile, 16 rows each, four lanes a row)  turn S into weights
//                         in place: the f16 pair hi + lo of 32 keys takes the 32
//                         columns that their logits had; P is the MMA's operand
//                         from TMEM
//   scales, cuts (1 warp each)  the blocks' scales; which item other CTAs go on with
// P V runs once for hi and once for lo, which keeps 22 bits of a weight: three
// units of MMA work where f16 weights would do with two, so 2/3 of the pipe's
// peak is the most that the fp32 output allows.  A tile has two buffers of S in
// TMEM: the softmax of one block runs beside the products of its neighbours.  (With
// one buffer and Q in TMEM too, S takes 256 instead of 392 cycles a block and tile,
// but softmax and products wait for each other: 374 us instead of 338 then.)
//
// Work is dealt out in equal shares of blocks; an item (head and row tile) that
// several CTAs share is added up by cache_join_kernel behind this one.
// Measured (8 heads): 512 positions of 4 rows over 32K 294 us, 0.93 PFLOP/s of the
// 1.28 that two passes over V leave of the pipe's 1.91; softmax issue (61 %) and
// tensor pipe (77 % busy) bound it.  128 rows over 16 x 8K 130 us, 32 rows 109: one
// tile's chain of S, softmax and P V, 1700 cycles a block; 32 rows over 1K 13 us.
//
// The weight of key j of block b carries the block's scale of V:
//   w_j = 2^{x_j + log2 vs_b - ref + 7},  O = sum_j w_j c_j / sum_b (sum_{j in b} w_j) / vs_b
// so codes go into the product as they are and no partial sum depends on how
// far apart the blocks' scales lie.  ref follows the running maximum of x_j +
// log2 vs_b only when that has grown by more than 8 (weights then stay below
// 2^15, in the range of f16): O is read, scaled and written back on few steps.
//
// The pipe's fp32 sums round towards zero, and O would shrink by 7e-8 a block:
// after 32 blocks it is added to sums in the workspace (L2) and starts again.
#include "cache8.cuh"
#include "tc.cuh"

namespace arckv {
namespace {

constexpr int kHalf = 128 * 128;              // bytes of a 128 x 64 f16 operand tile
constexpr int kKTile = 64 * 128;              // of a 64 x 64 one
constexpr int kStages = 3, kStageBytes = 2 * kKTile + kHalf;   // blocks of (K, V) as operands
constexpr int kRawBytes = 2 * kTileBytes;                      // of a block as codes
constexpr int kFlush = 32;                    // blocks that O is summed up over in TMEM
constexpr float kFar = 60.f;                  // growth of ref (log2) past which the flushed sums are scaled down
constexpr float kGrow = 8.f, kLift = 7.f;     // see above
// Sums of weights are in units of kVsUnit / vs, for scales vs of V between 2^-107 (a block of zeros) and 2^121.  The weight
// of a row's reference is 2^7 to 2^15, so its sum is at least 2^-128 (22 bits), and that of 2^20 zeros of 2^7 is 2^120.
constexpr float kVsUnit = 0x1p-14f;

struct TileShape {
  int H, n_pos, G, nblk, tiles;   // tiles: row tiles of a head
  bool causal;
};

template <int kT>
struct TileCfg {
  static constexpr int kRows = 128 * kT;
  static constexpr int kSoft = 8 * kT;                   // softmax warps 0 .. kSoft - 1, then 4 converters, then MMA
  static constexpr int kSoftThreads = 32 * kSoft;
  static constexpr int kThreads = 32 * (kSoft + 8);      // whole warpgroups: MMA, scales, codes, cuts
  // registers at launch, and how the warpgroups share them: softmax (2 kT groups), converters, MMA
  static constexpr int kRegs = kT == 2 ? 80 : 128;
  static constexpr int kRegsSoft = kT == 2 ? 96 : 176, kRegsConv = kT == 2 ? 64 : 96, kRegsMma = kT == 2 ? 32 : 64;
  static_assert(2 * kT * kRegsSoft + kRegsConv + kRegsMma == (2 * kT + 2) * kRegs && kRegs * kThreads <= 65536,
                "the shares add up to what the block was launched with");
  static constexpr int kRaw = kT == 2 ? 2 : 4;           // blocks on their way as codes
  static constexpr int kSmem = kT * 2 * kHalf + kStages * kStageBytes + kRaw * kRawBytes + 1024;
  // floats of a partial result: 64 outputs and twice (ref, log2 vs of ref, sum, unused) of each softmax thread
  static constexpr int kSlot = 72 * kSoftThreads;
};

// The products of one block and row tile, issued by one elected lane of a converged warp with warp-uniform operands
// (from one lane of a divergent branch each MMA took 90 to 125 cycles to issue, twice what it runs).  A descriptor's
// low bits are the address in units of 16 bytes, so K steps are added to the tile's descriptor.
//
// S = Q K^T: Q 128 x 128 and K 64 x 128 in halves of 64 dims (16 KB and 8 KB apart).
__device__ __forceinline__ void mma_qk(uint32_t s, uint64_t q, uint64_t k, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred e, z, c;\n\t.reg .b64 a, b;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 z, 0, 0;\n\tsetp.eq.b32 c, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, z;\n\t"
      "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 1024;\n\tadd.s64 b, %2, 512;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 1026;\n\tadd.s64 b, %2, 514;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 1028;\n\tadd.s64 b, %2, 516;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t"
      "add.s64 a, %1, 1030;\n\tadd.s64 b, %2, 518;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, c;\n\t}\n" ::"r"(s),
      "l"(q), "l"(k), "r"(idesc)
      : "memory");
}
// O (+)= P V: P in TMEM, 16 keys in 8 columns, hi and then lo 16 columns on, 32 keys in 32 columns; V^T 128 x 64.
__device__ __forceinline__ void mma_pv(uint32_t o, uint32_t p, uint64_t v, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, c, y;\n\t.reg .b64 b;\n\t.reg .b32 a;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 c, %4, 0;\n\tsetp.eq.b32 y, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, c;\n\t"
      "add.u32 a, %1, 16;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], %2, %3, y;\n\t"
      "add.u32 a, %1, 8;\n\tadd.s64 b, %2, 2;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 24;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 32;\n\tadd.s64 b, %2, 4;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 48;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 40;\n\tadd.s64 b, %2, 6;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 56;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t}\n" ::"r"(o),
      "r"(p), "l"(v), "r"(idesc), "r"(accumulate)
      : "memory");
}
// tc::mma_commit by one elected lane of a converged warp.
__device__ __forceinline__ void commit_elected(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(tc::smem_u32(bar))
      : "memory");
}
// 16 lanes of TMEM spread over a warp: lane l has rows l / 4 and l / 4 + 8.
//   loads and stores of fp32 columns: v[4 j + 2 i + e] is row l / 4 + 8 i, column 8 j + 2 (l % 4) + e
//   stores of 16 columns of f16 pairs: r[2 j + i] is row l / 4 + 8 i, column 4 j + l % 4
__device__ __forceinline__ void tmem_ld_rows64(uint32_t taddr, float (&v)[32]) {   // not waited for
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_rows32(uint32_t taddr, float (&v)[16]) {   // not waited for
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_rows32(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
      "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_pairs16(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Nothing that uses v moves above this point (behind a wait).
template <int kN>
__device__ __forceinline__ void settle(float (&v)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; i += 16)
    asm volatile(""
                 : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                   "+f"(v[i + 6]), "+f"(v[i + 7]), "+f"(v[i + 8]), "+f"(v[i + 9]), "+f"(v[i + 10]), "+f"(v[i + 11]),
                   "+f"(v[i + 12]), "+f"(v[i + 13]), "+f"(v[i + 14]), "+f"(v[i + 15]));
}
// Two fp32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// x 2^by, where the factor alone may be out of range (a sum of weights beside values 2^126 as large).
__device__ __forceinline__ float scaled(float x, float by) {
  const float h = ex2_approx(0.5f * by);
  return x * h * h;
}
template <int kN>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kN)); }
template <int kN>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kN)); }

// kind::f16 with A = B = f16, D = fp32, both K-major, M = 128, N = n.
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

__device__ __forceinline__ void store_matrices(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}

// Blocks of a row tile: as far as its last row sees (one at least).
__device__ __forceinline__ int tile_steps(const TileShape& d, int len, int tile, int rows) {
  const int last = min((tile + 1) * rows, d.n_pos * d.G) - 1;
  return max(1, (visible_tokens(len, d.n_pos, last / d.G, d.causal) + kCB - 1) / kCB);
}

struct Segment {
  long long first;         // unit at which the item begins
  long long sh;
  int s, tile, step, count;   // from step `step` of `count`
};

// The item of unit u: units run over sequences (pre[s] of a head of the earlier ones), heads, row tiles, steps.
__device__ __forceinline__ Segment segment_of(long long u, const TileShape& d, const arckv_cache8& c, const long long* pre,
                                              int rows) {
  Segment g;
  int lo = 0, hi = c.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] * d.H <= u) lo = mid;
    else hi = mid;
  }
  g.s = lo;
  const long long per = pre[lo + 1] - pre[lo], rest = u - pre[lo] * d.H, h = quotient(rest, per);
  g.sh = (long long)lo * d.H + h;
  const int len = cache_len(c, lo), lane = threadIdx.x & 31;
  int at = (int)(rest - h * per);
  for (int t0 = 0;; t0 += 32) {   // the tile, 32 at a time
    const int mine = t0 + lane < d.tiles ? tile_steps(d, len, t0 + lane, rows) : 0;
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned int past = __ballot_sync(0xffffffffu, x > at);
    if (past) {
      const int w = __ffs(past) - 1;
      g.count = __shfl_sync(0xffffffffu, mine, w);
      g.step = at - (__shfl_sync(0xffffffffu, x, w) - g.count);
      g.tile = t0 + w;
      break;
    }
    at -= __shfl_sync(0xffffffffu, x, 31);
    if (t0 + 32 >= d.tiles) {   // not reached: `at` lies within the head's steps
      g.count = 1;
      g.step = 0;
      g.tile = d.tiles - 1;
      break;
    }
  }
  g.first = u - g.step;
  return g;
}

// Two columns of two rows of the output, at o + at0 and o + at1.
__device__ __forceinline__ void store_rows(float* o, long long at0, long long at1, bool row0, bool row1, float4 x,
                                           DevStatus* stt) {
  const float big = 3.402823466e38f;
  if (row0) *(float2*)(o + at0) = make_float2(x.x, x.y);
  if (row1) *(float2*)(o + at1) = make_float2(x.z, x.w);
  if ((row0 && !(fabsf(x.x) <= big && fabsf(x.y) <= big)) || (row1 && !(fabsf(x.z) <= big && fabsf(x.w) <= big)))
    set_status(stt, ARCKV_ERR_NONFINITE);
}

// Of a block: the scale of K, log2 of V's, and what the sum of weights is multiplied by, kVsUnit / vs.  Where that leaves
// the normal range, or the weights may, the sum is taken of weights 2^lift as large (see lift_of).
struct __align__(16) Meta {
  float ks, lv, iv, lift;
};
// Beside large values the weights of a block of tiny ones may all be below fp32's range, and their sum with them: they are
// lifted, by as much as keeps both sums of 2^15 and iv in range.  A row's reference lies at most `top`, the largest lv
// so far, above a logit, so weights of equal logits are otherwise 2^-93 at least.
__device__ __forceinline__ float lift_of(float lv, float top) {
  if (lv < top - 100.f) return lv < -30.f ? 106.f : 60.f;
  return lv >= 100.f ? -40.f : 0.f;
}

template <int kT, bool kBias>
__global__ void __launch_bounds__(TileCfg<kT>::kThreads, 1)
    cache_tiles_kernel(const __grid_constant__ CUtensorMap mK, const __grid_constant__ CUtensorMap mV, const arckv_cache8 c, TileShape d, const bf16* Q, RowStrides qs, float scale, float* O,
                       RowStrides os, float* parts, int4* cuts, DevStatus* stt) {
  using Cfg = TileCfg<kT>;
  constexpr int kSoft = Cfg::kSoft, kRows = Cfg::kRows, kRaw = Cfg::kRaw;
  extern __shared__ unsigned char smraw[];
  unsigned char* sQ = smraw + ((1024u - (tc::smem_u32(smraw) & 1023u)) & 1023u);   // [tile][half][128][128 B]
  unsigned char* sKV = sQ + kT * 2 * kHalf;                                        // [stage][K halves, V]
  unsigned char* sRaw = sKV + kStages * kStageBytes;                               // [raw stage][K, V]
  long long* pre = (long long*)(sRaw + kRaw * kRawBytes);                          // [S + 1] blocks of a head's tiles
  // of buffer (parity of the block) 0 and 1: S written, P written, P V done
  __shared__ __align__(8) uint64_t qfull, full[kStages], empty[kStages], sfull[kT][2], pfull[kT][2], odone[kT][2], drain;
  __shared__ __align__(8) uint64_t raw_full[kRaw], raw_empty[kRaw];
  __shared__ Meta meta[2 * kStages];
  __shared__ uint32_t tmem_slot;
  __shared__ long long s_share[2];
  __shared__ Segment s_first;
  __shared__ int abort_flag, stop_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abortp = &abort_flag;

  if (tid == 0) {
    tc::mbar_init(&qfull, kSoft);
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(&full[i], 5);   // four converters and the scales
      tc::mbar_init(&empty[i], 1);
    }
    for (int t = 0; t < kT; ++t)
      for (int i = 0; i < 2; ++i) {
        tc::mbar_init(&sfull[t][i], 1);
        tc::mbar_init(&pfull[t][i], 8);
        tc::mbar_init(&odone[t][i], 1);
      }
    for (int i = 0; i < kRaw; ++i) {
      tc::mbar_init(&raw_full[i], 1);
      tc::mbar_init(&raw_empty[i], 4);
    }
    tc::mbar_init(&drain, 1);
    abort_flag = 0;
    tc::mbar_fence_init();
  }
  if (warp == kSoft + 4) tc::tmem_alloc(&tmem_slot, 256 * kT);
  pdl_trigger();
  pdl_wait();
  for (int s = tid; s < c.S; s += Cfg::kThreads) {   // blocks of one head's tiles of each sequence
    const int len = cache_len(c, s);
    long long n = 0;
    if (d.causal)
      for (int t = 0; t < d.tiles; ++t) n += tile_steps(d, len, t, kRows);
    else
      n = (long long)d.tiles * tile_steps(d, len, 0, kRows);
    pre[s + 1] = n;
  }
  __syncthreads();
  if (warp == 0) {   // their prefix sums
    long long run = 0;
    for (int s0 = 0; s0 < c.S; s0 += 32) {
      long long x = s0 + lane < c.S ? pre[s0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (s0 + lane < c.S) pre[s0 + lane + 1] = run + x;
      run += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) pre[0] = 0;
    __syncwarp();
    // the CTA's share and its first item, found once: short calls take their code from memory, every copy of it
    const CacheShares sh(run * d.H, gridDim.x);
    const long long u0 = sh.start(min((int)blockIdx.x, sh.ctas)), u1 = sh.start(min((int)blockIdx.x + 1, sh.ctas));
    Segment g = {};
    if (u0 < u1) g = segment_of(u0, d, c, pre, kRows);
    if (lane == 0) {
      s_share[0] = u0;
      s_share[1] = u1;
      s_first = g;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;   // tile t: two buffers of S / P at columns 256 t, O at 256 t + 128
  const long long u0 = s_share[0], u1 = s_share[1];

  if (warp == kSoft + 7) {
    // ------------------------ the item that begins here and goes on in other CTAs
    regs_dec<Cfg::kRegsMma>();
    int4 cut = make_int4(0, 0, -1, 0);
    if (u0 < u1) {
      const CacheShares sh(pre[c.S] * d.H, gridDim.x);
      Segment g = s_first;
      if (g.first + g.count < u1) g = segment_of(u1 - 1, d, c, pre, kRows);
      const long long end = g.first + g.count;
      if (end > u1 && g.first >= u0) cut = make_int4((int)g.sh, g.tile, sh.owner(end - 1), 0);
    }
    if (lane == 0) cuts[blockIdx.x] = cut;
  } else if (warp == kSoft + 6) {
    // ---------------------------------------------------------------- codes
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int q = 0;   // blocks issued
    Segment g = s_first;
    for (long long u = u0; u < u1 && ok;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      for (int i = 0; i < n; ++i, ++q) {   // (blocks lie within the capacity: `count` does)
        const int st = q % kRaw;
        if (q >= kRaw) ok = __all_sync(0xffffffffu, tc::mbar_wait(&raw_empty[st], ((q / kRaw) - 1) & 1, abortp, stt));
        if (!ok) break;
        if (lane == 0) {
          tc::mbar_arrive_expect_tx(&raw_full[st], kRawBytes);
          tc::tma_load_3d(sRaw + st * kRawBytes, &mK, 0, (g.step + i) * kCB, (int)g.sh, &raw_full[st]);
          tc::tma_load_3d(sRaw + st * kRawBytes + kTileBytes, &mV, 0, (g.step + i) * kCB, (int)g.sh, &raw_full[st]);
        }
      }
      u += n;
      if (u < u1) g = segment_of(u, d, c, pre, kRows);
    }
    if (!ok) {   // let the copies in flight land before the CTA's memory goes
      volatile int never = 0;
      for (int p = max(0, q - kRaw); p < q; ++p) tc::mbar_wait(&raw_full[p % kRaw], (p / kRaw) & 1, &never, stt);
    }
  } else if (warp == kSoft + 5) {
    // ---------------------------------------------------------------- scales
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int it = 0;
    Segment g = s_first;
    for (long long u = u0; u < u1 && ok;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u), len = cache_len(c, g.s);
      float top = -INFINITY;   // largest log2 of V's scales so far
      Meta m;
      for (int i = 0; i < n && ok; ++i) {
        const int q = it + i, st = q % kStages;
        if ((i & 31) == 0) {   // of the next 32 blocks, a lane each
          const int b = g.step + i + lane;
          float ks = 1.f, vs = 1.f;   // of a block that holds nothing: its keys are masked
          if (i + lane < n && b * kCB < len) {
            ks = c.k_scale[g.sh * d.nblk + b];
            vs = c.v_scale[g.sh * d.nblk + b];
          }
          const float lv = log2f(vs);
          float upto = lv;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const float y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto = fmaxf(upto, y);
          }
          upto = fmaxf(upto, top);
          top = __shfl_sync(0xffffffffu, upto, 31);
          const float lift = lift_of(lv, upto);
          m = Meta{ks, lv, kVsUnit * __uint_as_float((unsigned)(127 - (int)lift) << 23) / vs, lift};
        }
        if (q >= kStages) ok = tc::mbar_wait(&empty[st], ((q / kStages) - 1) & 1, abortp, stt);
        ok = __all_sync(0xffffffffu, ok);
        if (ok && lane == (i & 31)) {
          meta[q % (2 * kStages)] = m;
          tc::mbar_arrive(&full[st]);
        }
      }
      it += n;
      u += n;
      if (u < u1) g = segment_of(u, d, c, pre, kRows);
    }
  } else if (warp == kSoft + 4) {
    // ------------------------------------------------------------ MMA issuer
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int q = 0, st = 0, sp = 0, phase = 0;   // blocks so far; stages of this block and of the one before
    // warp-wide reductions leave their result in uniform registers
    const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem);
    const uint64_t q_desc = tc::sdesc_k128(tc::smem_u32(sQ)), kv_desc = tc::sdesc_k128(tc::smem_u32(sKV));
    int steps = s_first.count - s_first.step;   // of this item
    int seg = 0, left = __reduce_max_sync(0xffffffffu, (int)(u1 - u0));   // blocks to come
    for (long long u = u0; left > 0 && ok; ++seg) {
      const int n = __reduce_max_sync(0xffffffffu, min(steps, left));
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&qfull, seg & 1, abortp, stt));
      // S of block i, then P V of block i - 1
      for (int i = 0; i <= n && ok; ++i) {
        if (i < n) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[st], phase, abortp, stt));
          if (!ok) break;
          tc::fence_after_sync();
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            mma_qk(tm + 256 * t + (q & 1) * 64, q_desc + t * (2 * kHalf >> 4), kv_desc + (st * kStageBytes >> 4),
                   idesc_f16(64));
            commit_elected(&sfull[t][q & 1]);
          }
        }
        if (i > 0) {
          const int p = q - 1;
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            ok = __all_sync(0xffffffffu, ok && tc::mbar_wait(&pfull[t][p & 1], (p >> 1) & 1, abortp, stt));
            if (!ok) break;
            tc::fence_after_sync();
            mma_pv(tm + 256 * t + 128, tm + 256 * t + (p & 1) * 64, kv_desc + ((sp * kStageBytes + 2 * kKTile) >> 4),
                   idesc_f16(128), (i - 1) % kFlush != 0);
            commit_elected(&odone[t][p & 1]);
          }
          if (!ok) break;
          commit_elected(&empty[sp]);
        }
        if (i < n) {
          sp = st;
          if (++st == kStages) {
            st = 0;
            phase ^= 1;
          }
          ++q;
        }
      }
      left -= n;
      u += n;
      if (left > 0) {
        const Segment next = segment_of(u, d, c, pre, kRows);
        steps = next.count - next.step;
      }
    }
    __syncwarp();
    {   // every MMA done before TMEM and shared memory go
      commit_elected(&drain);
      volatile int never = 0;
      tc::mbar_wait(&drain, 0, &never, stt);
    }
    __syncwarp();
  } else if (warp >= kSoft) {
    // ------------------------------------------------------------ converters
    regs_dec<Cfg::kRegsConv>();
    const int cw = warp - kSoft, total = (int)(u1 - u0);
    // K: 16 dims of a row (chunk kc) at a time.  Eight lanes have four chunks of rows r and r ^ 5, which neither as
    // codes nor as operands meet in a bank.
    const int kc = (lane & 3) + 4 * (lane >> 4), kr = cw * 16 + (((lane >> 2) & 1) * 5 ^ ((lane >> 3) & 1) * 2);
    // V: dims 32 cw .. 32 cw + 31 of 16 keys at a time.  Transposed loads leave dims 2 i, 2 i + 1 of two keys in a word;
    // the even and odd ones are stored as matrices of 8 dims x 8 keys.
    const int v_row = (lane & 15) * 128, v_chunk = ((2 * cw + (lane >> 4)) ^ (lane & 7)) << 4;
    const int m = lane >> 3, dim = 32 * cw + 2 * (lane & 7) + (m & 1);
    const int o_row = dim * 128, o_chunk = ((m >> 1) ^ (dim & 7)) << 4;
    const uint32_t raw0 = tc::smem_u32(sRaw), kv0 = tc::smem_u32(sKV);
    for (int q = 0; q < total; ++q) {
      const int st = q % kStages, rs = q % kRaw;
      bool ok = tc::mbar_wait(&raw_full[rs], (q / kRaw) & 1, abortp, stt);
      if (ok && q >= kStages) ok = tc::mbar_wait(&empty[st], ((q / kStages) - 1) & 1, abortp, stt);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const unsigned char* raw = sRaw + rs * kRawBytes;
      unsigned char* Ks = sKV + st * kStageBytes;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = kr ^ (j & 1) ^ (j & 2) << 2;
        const uint4 x = *(const uint4*)(raw + r * 128 + ((kc ^ (r & 7)) << 4));
        unsigned char* row = Ks + (kc >> 2) * kKTile + r * 128;
        *(uint4*)(row + ((((kc & 3) * 2) ^ (r & 7)) << 4)) =
            make_uint4(codes_f16<0x4140>(x.x), codes_f16<0x4342>(x.x), codes_f16<0x4140>(x.y), codes_f16<0x4342>(x.y));
        *(uint4*)(row + ((((kc & 3) * 2 + 1) ^ (r & 7)) << 4)) =
            make_uint4(codes_f16<0x4140>(x.z), codes_f16<0x4342>(x.z), codes_f16<0x4140>(x.w), codes_f16<0x4342>(x.w));
      }
      const uint32_t vs = raw0 + rs * kRawBytes + kTileBytes + v_row + v_chunk;
      const uint32_t vd = kv0 + st * kStageBytes + 2 * kKTile + o_row;
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
        uint32_t w[4];
        load_transposed(w, vs + mt * (16 * 128));
#pragma unroll
        for (int z = 0; z < 2; ++z)
          store_matrices(vd + z * (16 * 128) + ((mt << 5) ^ o_chunk), codes_f16<0x4240>(w[2 * z]),
                         codes_f16<0x4341>(w[2 * z]), codes_f16<0x4240>(w[2 * z + 1]), codes_f16<0x4341>(w[2 * z + 1]));
      }
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        tc::mbar_arrive(&raw_empty[rs]);
        tc::mbar_arrive(&full[st]);
      }
    }
  } else {
    // --------------------------------------------------------------- softmax
    // a warp has 16 rows of its tile: lane l rows l / 4 and l / 4 + 8 of them, two columns of eight.  Warp w has the
    // tile's rows 16 (w % 8) .. in the TMEM lanes that it can reach, so that few rows are spread over the SM's quarters;
    // warps that are left without rows only keep the count of the barriers.
    regs_inc<Cfg::kRegsSoft>();
    const int t = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3;   // (a warp reaches the lanes of its quarter)
    const int r_warp = 16 * (warp & 7), cl = 2 * (lane & 3);
    const uint32_t Sb = tmem + 256 * t + ((uint32_t)(quarter * 32 + half * 16) << 16), Ot = Sb + 128;
    const int nrows = d.n_pos * d.G;
    bool ok = true;
    // P V of block q is in O.  (The one before it, whose phase this could be taken for, is known to be: S of block
    // q + 1 was issued after it and has come in.)
    auto product_done = [&](int q) {
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&odone[t][q & 1], (q >> 1) & 1, abortp, stt));
      tc::fence_after_sync();
      return ok;
    };
    auto tile_sync = [&] { asm volatile("bar.sync %0, 256;" ::"r"(2 + t) : "memory"); };
    int it = 0;
    Segment g = s_first;
    for (long long u = u0; u < u1;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      const int row0 = g.tile * kRows + t * 128, h = (int)(g.sh - (long long)g.s * d.H), len = cache_len(c, g.s);
      float row_fac;
      {   // the queries as f16, each row scaled by a power of two: here a lane is a row, and has 64 dims
        const int r = quarter * 32 + lane, row = row0 + 64 * (lane >> 4) + 16 * quarter + (lane & 15);   // (r: TMEM lane)
        const int pos = row / d.G, gq = row - pos * d.G;
        uint4 x[8];
        float amax = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = make_uint4(0u, 0u, 0u, 0u);
          if (row < nrows)
            x[e] = *((const uint4*)(Q + g.s * qs.s + h * qs.h + pos * qs.i + gq * 128 + half * 64) + e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const __nv_bfloat162* y = (const __nv_bfloat162*)&x[e];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 z = __bfloat1622float2(y[k]);
            amax = fmaxf(amax, fmaxf(fabsf(z.x), fabsf(z.y)));
          }
        }
        float* half_max = (float*)(sQ + t * 2 * kHalf);   // (the products of the item before have been waited for)
        half_max[half * 128 + r] = amax;
        tile_sync();
        amax = fmaxf(amax, half_max[(half ^ 1) * 128 + r]);
        tile_sync();
        const int ex = max((int)((__float_as_uint(amax) >> 23) & 0xff) - 127, -100);
        const float up = __uint_as_float((unsigned)(14 - ex + 127) << 23);
        row_fac = __uint_as_float((unsigned)(ex - 14 + 127) << 23) * scale * (kBias ? 1.f : kLog2e);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const __nv_bfloat162* y = (const __nv_bfloat162*)&x[e];
          __half2 z[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 a = __bfloat1622float2(y[k]);
            z[k] = __floats2half2_rn(a.x * up, a.y * up);
          }
          *(uint4*)(sQ + (t * 2 + half) * kHalf + r * 128 + ((e ^ (r & 7)) << 4)) = *(const uint4*)&z[0];
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&qfull);
      }
      // products' factors (powers of two without biases, of e with them) and sight of this thread's two rows
      float fac[2];
      int see[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = r_warp + (lane >> 2) + 8 * i, row = row0 + r;
        fac[i] = __shfl_sync(0xffffffffu, row_fac, half * 16 + (lane >> 2) + 8 * i);   // (r is a row of this warp's lanes)
        see[i] = row < nrows ? visible_tokens(len, d.n_pos, row / d.G, d.causal) : 0;
      }
      const int see_min = __reduce_min_sync(0xffffffffu, min(see[0], see[1]));
      // this thread's sums in memory, 16 bytes of all threads together
      float* sums = parts + 2ll * kCacheMaxCtas * Cfg::kSlot + (long long)blockIdx.x * 64 * Cfg::kSoftThreads + tid * 4;
      // references of the flushed sums and of O (with biases the logit, and the log2 vs that came with it), sums of weights
      float bref[2] = {-INFINITY, -INFINITY}, brefv[2] = {0.f, 0.f}, ref[2] = {-INFINITY, -INFINITY};
      float refv[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};
      const float* bias = kBias ? c.bias + g.sh * c.cap : nullptr;
      const bool any_row = row0 + r_warp < nrows;
      for (int i = 0; i < n; ++i) {
        const int q = it + i, j0 = (g.step + i) * kCB + cl;
        const uint32_t S = Sb + (q & 1) * 64;
        // S is in, and with it the block's scales (written before `full`, which the MMA warp waited for)
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&sfull[t][q & 1], (q >> 1) & 1, abortp, stt));
        if (!ok) break;
        if (kT == 1 && !any_row) {
          if (lane == 0) tc::mbar_arrive(&pfull[t][q & 1]);
          continue;
        }
        tc::fence_after_sync();
        if (i > 0 && i % kFlush == 0) {
          if (!product_done(q - 1)) break;
          // O goes to the sums in memory and starts again at zero (see above)
          float up[2], down[2];
          bool redo = false;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float dd = kBias ? fmaf(ref[k] - bref[k], kLog2e, refv[k] - brefv[k]) : ref[k] - bref[k];
            const bool none = bref[k] == -INFINITY, far = !none && dd > kFar;
            up[k] = none || far ? 1.f : ex2_approx(dd);
            down[k] = none ? 0.f : far ? ex2_approx(-dd) : 1.f;
            if (none || far) {
              redo = true;
              bref[k] = ref[k];
              brefv[k] = refv[k];
            }
          }
          redo = __any_sync(0xffffffffu, redo);
#pragma unroll 1
          for (int ch = 0; ch < 4; ++ch) {
            float o[16];
            tmem_ld_rows32(Ot + ch * 32, o);
            tmem_wait_ld();
            settle(o);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float* b = sums + (long long)(ch * 4 + e) * Cfg::kSoftThreads * 4;
              float4 x = make_float4(o[4 * e] * up[0], o[4 * e + 1] * up[0], o[4 * e + 2] * up[1], o[4 * e + 3] * up[1]);
              if (redo) {
                if (i > kFlush) {
                  const float4 old = __ldcg((const float4*)b);
                  x = make_float4(fmaf(old.x, down[0], x.x), fmaf(old.y, down[0], x.y), fmaf(old.z, down[1], x.z),
                                  fmaf(old.w, down[1], x.w));
                }
                __stcg((float4*)b, x);
              } else {
                asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(b), "f"(x.x), "f"(x.y),
                             "f"(x.z), "f"(x.w)
                             : "memory");
              }
            }
          }
        }
        float v[32];
        tmem_ld_rows64(S, v);
        const Meta m = meta[q % (2 * kStages)];
        // (never zero: a masked product is -inf; a row of zeros over a block of zeros would come to 2^-220)
        const float f[2] = {fmaxf(fac[0] * m.ks, 0x1p-126f), fmaxf(fac[1] * m.ks, 0x1p-126f)};
        tmem_wait_ld();
        settle(v);
        const bool edge = j0 - cl + kCB > see_min;
        if (kBias) {   // logits; biases are read in pairs where a row sees something, within the capacity
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float2 x = make_float2(0.f, 0.f);
            if (j0 + 8 * j < max(see[0], see[1])) x = *(const float2*)(bias + j0 + 8 * j);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              v[4 * j + 2 * k] = fmaf(v[4 * j + 2 * k], f[k], x.x);
              v[4 * j + 2 * k + 1] = fmaf(v[4 * j + 2 * k + 1], f[k], x.y);
            }
          }
        }
        if (edge) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (j0 + 8 * j + (k & 1) >= see[k >> 1]) v[4 * j + k] = -INFINITY;
        }
        // Each lane looks whether one of its own logits is past what the reference allows; the rows' maxima are taken
        // where one is.  (f > 0: the largest product is the largest logit.)
        float top[2];
        bool grows = false;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float b = max3(v[4 + 2 * k], v[5 + 2 * k], v[8 + 2 * k]);
          top[k] = max3(v[2 * k], v[2 * k + 1], v[9 + 2 * k]);
#pragma unroll
          for (int j = 3; j < 8; j += 2) {
            top[k] = max3(top[k], v[4 * j + 2 * k], v[4 * j + 2 * k + 1]);
            if (j < 7) b = max3(b, v[4 * j + 4 + 2 * k], v[4 * j + 5 + 2 * k]);
          }
          top[k] = fmaxf(top[k], b);
          // in units of log2; with biases (x - ref) log2 e + lv - refv, differences of logits first, so that the type's
          // lowest value cancels against itself.  (A reference of -inf is past by any logit but -inf.)
          grows |= kBias ? fmaf(top[k] - ref[k], kLog2e, m.lv - refv[k]) > kGrow : fmaf(top[k], f[k], m.lv) > ref[k] + kGrow;
        }
        if (__any_sync(0xffffffffu, grows)) {
          float alpha[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
            const float to = kBias ? top[k] : fmaf(top[k], f[k], m.lv), tov = kBias ? m.lv : 0.f;
            // what the sums shrink by, as a power of two
            const float by = ref[k] == -INFINITY ? -INFINITY
                             : kBias             ? fmaf(ref[k] - to, kLog2e, refv[k] - tov)
                                                 : ref[k] - to;
            const bool up = to != -INFINITY && -by > kGrow;
            alpha[k] = up ? ex2_approx(by) : 1.f;
            if (up) {
              l[k] = scaled(l[k], by);
              ref[k] = to;
              refv[k] = tov;
            }
          }
          if (i % kFlush != 0) {   // scale O
            if (!product_done(q - 1)) break;
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              float o[16];
              tmem_ld_rows32(Ot + ch * 32, o);
              tmem_wait_ld();
              settle(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] *= alpha[(e >> 1) & 1];
              tmem_st_rows32(Ot + ch * 32, o);
            }
          }
        }
        float2 base[2], add[2], sum[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float b = ref[k] == -INFINITY ? 0.f : ref[k], a = (kBias ? m.lv - refv[k] : m.lv - b) + kLift;
          base[k] = make_float2(-b, -b);
          add[k] = make_float2(a, a);
          sum[k] = make_float2(0.f, 0.f);
        }
        float lifted[2] = {0.f, 0.f};
        if (m.lift != 0.f) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const int k = (e >> 1) & 1;
            const float x = kBias ? fmaf(v[e] + base[k].x, kLog2e, add[k].x) : fmaf(v[e], f[k], add[k].x);
            lifted[k] += ex2_approx(x + m.lift);
          }
        }
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {   // 32 keys: 16 columns of hi, 16 of lo
          uint32_t hr[8], lr[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = e & 1, j = ch * 4 + (e >> 1);
            float2 x = make_float2(v[4 * j + 2 * k], v[4 * j + 2 * k + 1]);
            if (kBias)
              x = fma2(add2(x, base[k]), make_float2(kLog2e, kLog2e), add[k]);
            else
              x = fma2(x, make_float2(f[k], f[k]), add[k]);
            x.x = ex2_approx(x.x);
            x.y = ex2_approx(x.y);
            sum[k] = add2(sum[k], x);
            // hi: x rounded to 11 bits; lo: the rest, at most 2^-11 of x, rounded to 11 bits
            const __half2 h2 = __floats2half2_rn(x.x, x.y);
            const float2 lo = minus_f16(x, h2);
            const __half2 l2 = __floats2half2_rn(lo.x, lo.y);
            hr[e] = *(const uint32_t*)&h2;
            lr[e] = *(const uint32_t*)&l2;
          }
          tmem_st_pairs16(S + ch * 32, hr);
          tmem_st_pairs16(S + ch * 32 + 16, lr);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) l[k] = fmaf(m.lift != 0.f ? lifted[k] : sum[k].x + sum[k].y, m.iv, l[k]);
        tmem_wait_st();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&pfull[t][q & 1]);
      }
      it += n;
      if (ok) product_done(it - 1);
      if (tid == 0) stop_flag = *abortp;   // one reading for all
      asm volatile("bar.sync 1, %0;" ::"r"(Cfg::kSoftThreads) : "memory");
      if (stop_flag) break;
      const bool whole = g.step == 0 && n == g.count, flushed = n > kFlush;
      float bw[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
        bw[k] = bref[k] == -INFINITY ? 0.f
                                     : ex2_approx(kBias ? fmaf(bref[k] - ref[k], kLog2e, brefv[k] - refv[k]) : bref[k] - ref[k]);
      }
      int q0 = row0 + r_warp + (lane >> 2);   // (not kept in registers through the loop)
      asm volatile("" : "+r"(q0));
      const int q1 = q0 + 8;
      const long long at0 = (q0 / d.G) * os.i + (q0 % d.G) * 128, at1 = (q1 / d.G) * os.i + (q1 % d.G) * 128;
      auto store = [&](int j, float4 x, float inv0, float inv1) {
        store_rows(O + g.s * os.s + h * os.h + 8 * j + cl, at0, at1, q0 < nrows, q1 < nrows,
                   make_float4(x.x * inv0, x.y * inv0, x.z * inv1, x.w * inv1), stt);
      };
      const float inv0 = l[0] == 0.f ? 0.f : kVsUnit / l[0], inv1 = l[1] == 0.f ? 0.f : kVsUnit / l[1];
      float* slot = parts + (2ll * blockIdx.x + (g.step == 0 ? 1 : 0)) * Cfg::kSlot + tid * 4;
#pragma unroll 1
      for (int ch = 0; ch < 4; ++ch) {
        float v[16];
        tmem_ld_rows32(Ot + ch * 32, v);
        float4 y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (flushed) y[e] = __ldcg((const float4*)(sums + (long long)(ch * 4 + e) * Cfg::kSoftThreads * 4));
        }
        tmem_wait_ld();
        settle(v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 x = make_float4(fmaf(y[e].x, bw[0], v[4 * e]), fmaf(y[e].y, bw[0], v[4 * e + 1]),
                                       fmaf(y[e].z, bw[1], v[4 * e + 2]), fmaf(y[e].w, bw[1], v[4 * e + 3]));
          if (whole) store(ch * 4 + e, x, inv0, inv1);
          else if (any_row) __stcg((float4*)(slot + (long long)(ch * 4 + e) * Cfg::kSoftThreads * 4), x);
        }
      }
      tc::fence_before_sync();
      if (!whole && any_row) {   // joined by the kernel behind this one
#pragma unroll
        for (int k = 0; k < 2; ++k)
          __stcg((float4*)(slot + (long long)(16 + k) * Cfg::kSoftThreads * 4), make_float4(ref[k], refv[k], l[k], 0.f));
      }
      u += n;
      if (u < u1) g = segment_of(u, d, c, pre, kRows);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kSoft + 4) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, 256 * kT);
  }
}

// Adds up the parts of the items that several CTAs of cache_tiles_kernel shared: cuts[c] is {sequence x head, tile, last
// CTA} of the item that begins in CTA c and goes on, or has a last CTA of -1.  (Left to the CTA that came last, an item's
// 16 parts of 128 rows took it 30 us, most of them waits for its loads.)  One work unit is the 16 rows that one
// softmax warp had.
constexpr int kJoinThreads = 256;
template <int kT, bool kBias>
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(int H, int n_pos, int G, float* O, RowStrides os,
                                                                  const float* parts, const int4* cuts, int n_cuts,
                                                                  DevStatus* stt) {
  using Cfg = TileCfg<kT>;
  __shared__ int4 s_cut[kCacheMaxCtas];   // of the items, in order; w: the CTA in which it begins
  __shared__ int s_items;
  __shared__ float s_w[kCacheMaxCtas][16], s_inv[16];
  const int tid = threadIdx.x, lane = tid & 31, nrows = n_pos * G;
  pdl_trigger();
  pdl_wait();
  if (tid < 32) {
    int4 cut[kCacheMaxCtas / 32];
#pragma unroll
    for (int i = 0; i < kCacheMaxCtas / 32; ++i) {
      cut[i] = make_int4(0, 0, -1, 0);
      if (32 * i + lane < n_cuts) cut[i] = __ldcg(cuts + 32 * i + lane);
    }
    int n = 0;
#pragma unroll
    for (int i = 0; i < kCacheMaxCtas / 32; ++i) {
      const unsigned int all = __ballot_sync(0xffffffffu, cut[i].z >= 0);
      cut[i].w = 32 * i + lane;
      if (cut[i].z >= 0) s_cut[n + __popc(all & ((1u << lane) - 1u))] = cut[i];
      n += __popc(all);
    }
    if (lane == 0) s_items = n;
  }
  __syncthreads();
  const int work = s_items * Cfg::kSoft;
  for (int x = blockIdx.x; x < work; x += gridDim.x) {
    const int4 cut = s_cut[x / Cfg::kSoft];
    const int first = cut.w, warp = x % Cfg::kSoft, n = cut.z - first + 1;
    const int row0 = cut.y * Cfg::kRows + warp * 16;
    if (row0 >= nrows) continue;   // (uniform)
    auto part = [&](int p) { return parts + (2ll * (first + p) + (p == 0)) * Cfg::kSlot + warp * 128; };
    // The sums' loads wait for nothing: the first eight parts' are under way while the weights are found.  Sixteen bytes
    // of two units a thread: columns 8 j + 2 (lane % 4), + 1 of rows lane / 4 and lane / 4 + 8.
    const int r8 = lane >> 2, j8 = tid >> 5;
    float4 ahead[8][2];
    auto load = [&](int p0) {
#pragma unroll
      for (int p = 0; p < 8; ++p)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (p0 + p < n) ahead[p][e] = __ldcg((const float4*)(part(p0 + p) + lane * 4 + (long long)(j8 + 8 * e) * Cfg::kSoftThreads * 4));
    };
    load(0);
    {   // weights of the parts for row tid / 16, sixteen parts at a time
      const int r = tid >> 4, l16 = tid & 15;
      const long long at = (long long)(16 + (r >> 3)) * Cfg::kSoftThreads * 4 + (r & 7) * 16;
      // log2 of what separates two references; with biases a logit and the log2 of V's scale that came with it
      auto beyond = [](float a, float av, float b, float bv) { return kBias ? fmaf(a - b, kLog2e, av - bv) : a - b; };
      float top = -INFINITY, topv = 0.f;
      auto raise = [&](float a, float av) {
        if (a != -INFINITY && (top == -INFINITY || beyond(a, av, top, topv) > 0.f)) {
          top = a;
          topv = av;
        }
      };
      float4 mine = make_float4(-INFINITY, 0.f, 0.f, 0.f);   // of the first sixteen parts
      if (l16 < n) mine = __ldcg((const float4*)(part(l16) + at));
      raise(mine.x, mine.y);
      for (int p = l16 + 16; p < n; p += 16) {
        const float2 y = __ldcg((const float2*)(part(p) + at));
        raise(y.x, y.y);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        const float a = __shfl_xor_sync(0xffffffffu, top, o), av = __shfl_xor_sync(0xffffffffu, topv, o);
        raise(a, av);
      }
      float z = 0.f;
      for (int p = l16; p < n; p += 16) {
        const float4 y = p == l16 ? mine : __ldcg((const float4*)(part(p) + at));
        float w = 0.f;
        if (y.x != -INFINITY) {   // (else a part that saw nothing)
          const float by = beyond(y.x, y.y, top, topv);
          w = ex2_approx(by);
          z += scaled(y.z, by);
        }
        s_w[p][r] = w;
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      if (l16 == 0) s_inv[r] = z == 0.f ? 0.f : kVsUnit / z;
    }
    __syncthreads();
    {
      float4 a[2];
      a[0] = a[1] = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p0 = 0; p0 < n; p0 += 8) {
        if (p0 > 0) load(p0);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
          if (p0 + p >= n) break;
          const float w0 = s_w[p0 + p][r8], w1 = s_w[p0 + p][r8 + 8];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 y = ahead[p][e];
            a[e] = make_float4(fmaf(y.x, w0, a[e].x), fmaf(y.y, w0, a[e].y), fmaf(y.z, w1, a[e].z), fmaf(y.w, w1, a[e].w));
          }
        }
      }
      const int s = cut.x / H, h = cut.x - s * H, q0 = row0 + r8, q1 = q0 + 8;
      const long long at0 = (q0 / G) * os.i + (q0 % G) * 128, at1 = (q1 / G) * os.i + (q1 % G) * 128;
      const float i0 = s_inv[r8], i1 = s_inv[r8 + 8];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        store_rows(O + s * os.s + h * os.h + 8 * (j8 + 8 * e) + 2 * (lane & 3), at0, at1, q0 < nrows, q1 < nrows,
                   make_float4(a[e].x * i0, a[e].y * i0, a[e].z * i1, a[e].w * i1), stt);
    }
    __syncthreads();
  }
}

template <int kT, bool kBias>
int launch_tiles(const arckv_cache8& c, const CacheQuery& q, float scale, float* O, RowStrides os, void* ws,
                 cudaStream_t st) {
  using Cfg = TileCfg<kT>;
  CUtensorMap mK, mV;
  if (!encode_u8_map_3d(&mK, c.K, c.cap, (uint64_t)c.S * c.H, kCB) ||
      !encode_u8_map_3d(&mV, c.V, c.cap, (uint64_t)c.S * c.H, kCB))
    return -1;
  TileShape d;
  d.H = c.H;
  d.n_pos = q.n_pos;
  d.G = q.G;
  d.nblk = c.cap / kCB;
  d.tiles = cdiv((long long)q.n_pos * q.G, Cfg::kRows);
  d.causal = q.causal;
  auto kern = cache_tiles_kernel<kT, kBias>;
  const int smem = Cfg::kSmem + (c.S + 1) * (int)sizeof(long long);
  if (set_dyn_smem((const void*)kern, smem) != cudaSuccess) return -1;
  const int ctas = std::min(tc_gemm_sm_count(), kCacheMaxCtas);
  float* parts = (float*)((char*)ws + ARCKV_CACHE_WS_HEADER);
  int4* cuts = (int4*)(parts + kCacheMaxCtas * (2ll * Cfg::kSlot + 64 * Cfg::kSoftThreads));
  DevStatus* stt = (DevStatus*)ws;
  cudaError_t e = launch_pdl(kern, dim3(ctas), Cfg::kThreads, smem, st, mK, mV, c, d, q.Q, q.qs, scale, O, os, parts, cuts, stt);
  if (e != cudaSuccess) return -1;
  e = launch_pdl(cache_join_kernel<kT, kBias>, dim3(4 * ctas), kJoinThreads, 0, st, c.H, q.n_pos, q.G, O, os, parts, cuts,
                 ctas, stt);
  return e == cudaSuccess ? 2 : -1;
}

}  // namespace

size_t cache_tiles_scratch(long long rows) {
  const size_t slot = rows <= 128 ? TileCfg<1>::kSlot : TileCfg<2>::kSlot;
  const size_t sums = 64 * (rows <= 128 ? TileCfg<1>::kSoftThreads : TileCfg<2>::kSoftThreads);
  return kCacheMaxCtas * ((2 * slot + sums) * sizeof(float) + sizeof(int4));
}

int launch_cache_tiles(const arckv_cache8& c, const CacheQuery& q, float scale, float* O, RowStrides os, void* ws,
                       cudaStream_t st) {
  const long long rows = (long long)q.n_pos * q.G;
  // one tile where it holds all rows (128 over 16 x 8 heads of 8K: 129 us; 132 rows, with two, 178)
  if (rows <= 128)
    return c.bias ? launch_tiles<1, true>(c, q, scale, O, os, ws, st) : launch_tiles<1, false>(c, q, scale, O, os, ws, st);
  return c.bias ? launch_tiles<2, true>(c, q, scale, O, os, ws, st) : launch_tiles<2, false>(c, q, scale, O, os, ws, st);
}

}  // namespace arckv
