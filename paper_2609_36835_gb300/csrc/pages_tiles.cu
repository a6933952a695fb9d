// Attention of packed queries over paged 4-bit caches, for requests of many rows
// (prompt chunks): the products of pages_attend.cu on tcgen05.
//
// With n rows a head every code is used n times, so the call is bound by the
// tensor pipe.  A CTA takes 128 or 256 rows of one request and head (one or two
// M = 128 tiles) and goes over the request's pages:
//   pages (1 warp)        a page of the head by one bulk copy into a ring
//   scales (1 warp)       the page's largest magnitudes, as powers of two
//   converters (4 warps)  codes to f16 operands in shared memory, V transposed by
//                         matrix stores, up to three pages ahead
//   MMA warp              S = Q K^T, O += P V, fp32 sums in TMEM
//   softmax (8 warps a tile, 16 rows each, four lanes a row)  turn S into weights
//                         in place; P is the MMA's operand from TMEM
//   items (1 warp)        the CTA's items ahead of the other warps, and the one that
//                         other CTAs go on with
// A tile has two buffers of S in TMEM (four if it is alone): the softmax of one page runs beside the products of its neighbours.  A tile without
// rows is left out.  Work is dealt out in equal shares of pages; an item (request, head, row tile) that several CTAs share is
// added up by pages_join_kernel behind this one.
//
// A key or value m + c s enters the products as f16, in units of a power of two near its page's largest: half a step is
// 2^-11 of an element, an eighth of what the bf16 outputs round to, and elements below 2^-8 of the largest are off by up to
// 2^-17 of it.  K's unit goes into the factor of its page's logits.  V's goes into the exponent of the weights:
//   w_j = 2^{x_j - ref + 7 + ev - eref},  O = 2^eref sum_j w_j v_j 2^-ev / sum_b 2^{eref - ev} sum_{j in b} w_j
// where eref is at least every page's ev and at most 6 above it: O, whose fp32 sums have the range, is scaled whenever the values'
// size leaves that, up or down (down as far as 2^-60 of the largest size met; what lies below that counts as zero).  With a unit that
// only grew, pages behind one of values 2^20 times theirs lost 0.16 of their output, whether or not that one had any weight.
// Weights enter as one f16, 2^-11 of each down to 2^-15 of ref's (2^-26 of ref's weight below, where values are 2^-6 of the unit),
// so that what lies 20 nats below an early token still counts.  They begin at 2^7 and reach 2^15: ref follows the running maximum
// when that has grown by more than 8, and then for all rows that have grown by more than 1, as to scale O is to wait for
// its products.  (Room below costs what jumps of 8 to 15 cost: from one on, 8192 positions 660 us, 695 from 2^7, 706 if rows
// follow by themselves; but 16 nats below a token of no value 0.3 to 0.7 of the output were lost, 4e-3 now, most of which is
// the keys' rounding.)  The pipe's fp32 sums round towards zero: O shrinks by 7e-8 a page.
//
// Bound by shared memory, which the N = 64 products of S read Q from once a page, and by the softmax's issue (a page and 256
// rows take 0.93 us, of which the pipe needs 0.54; steps of two pages with one buffer of S took longer, 295 us against 237;
// a warp for S and one for P V 265).  With one tile a page takes 0.8 us: a chain of waits, whatever the rows.
// Measured (CUDA graph): 2048 rows of 8 heads over 32,768 tokens 242 us, 1.13 PFLOP/s; 256 rows over 8192 34 us with the join;
// 32 rows, 250 x 8 x up to 500 (which pages_attend.cu takes in 122): 202 us, most of it changes of items.
#include "pages.cuh"
#include "tc.cuh"

namespace arckv {
namespace {

constexpr int kHalf = 128 * 128;              // bytes of a 128 x 64 f16 operand tile
constexpr int kKTile = 64 * 128;              // of a 64 x 64 one
constexpr int kSegments = 4;                  // items that are found ahead
constexpr int kStageBytes = 2 * kKTile + kHalf;   // a page (K, V) as operands
constexpr float kGrow = 8.f, kLift = 7.f, kFollow = 1.f;   // see above

struct TileShape {
  int G, N, above, max_count;   // requests of more than `above` rows of a head
  bool causal;
};

template <int kT>
struct TileCfg {
  static constexpr int kRows = 128 * kT;
  static constexpr int kSoft = 8 * kT;                   // softmax warps 0 .. kSoft - 1, then 4 converters, then MMA
  static constexpr int kSoftThreads = 32 * kSoft;
  static constexpr int kMma = kSoft + 4;                 // first warp behind them
  static constexpr int kThreads = 32 * (kMma + 4);       // whole warpgroups: MMA, scales, pages, items
  // registers at launch, and how the warpgroups share them: softmax (2 kT groups), converters, MMA
  static constexpr int kRegs = kT == 2 ? 80 : 128;
  static constexpr int kRegsSoft = kT == 2 ? 88 : 152, kRegsConv = kT == 2 ? 80 : 128, kRegsMma = kT == 2 ? 48 : 80;
  static_assert(2 * kT * kRegsSoft + kRegsConv + kRegsMma <= (2 * kT + 2) * kRegs && kRegs * kThreads <= 65536,
                "the shares are within what the block was launched with");
  // pages as operands, and on their way as codes (two tiles: a third way ahead is in the others' way, 239 us instead of 234 for
  // 2048 rows over 32K)
  static constexpr int kStages = kT == 2 ? 3 : 4, kRaw = kT == 2 ? 2 : 3;
  static constexpr int kBuf = kT == 2 ? 2 : 4;           // buffers of S in TMEM
  static constexpr int kO = kBuf * 64;                   // first column of O
  static_assert(kT == 2 || kBuf == kStages, "see the converters");
  static constexpr int kSmem = kT * 2 * kHalf + kStages * kStageBytes + kRaw * ARCKV_PAGE_BYTES + 1024;
  static_assert(kSmem + 4097 * 8 + 4 * kSoftThreads + 2048 <= 227 * 1024, "shared memory");
  // 32-bit words of a partial result: 64 outputs as f16, of two rows (ref, sum) and what a unit stands for, of each softmax thread
  static constexpr int kSlot = 40 * kSoftThreads;
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
// O (+)= P V: P in TMEM, 16 tokens in 8 columns; V^T 128 x 64.
__device__ __forceinline__ void mma_pv(uint32_t o, uint32_t p, uint64_t v, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, c, y;\n\t.reg .b64 b;\n\t.reg .b32 a;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 c, %4, 0;\n\tsetp.eq.b32 y, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, c;\n\t"
      "add.u32 a, %1, 8;\n\tadd.s64 b, %2, 2;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 16;\n\tadd.s64 b, %2, 4;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, y;\n\t"
      "add.u32 a, %1, 24;\n\tadd.s64 b, %2, 6;\n\t"
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

// 2^e as fp32 for e within the normal range, zero below it.
__device__ __forceinline__ float pow2(int e) { return e < -126 ? 0.f : __uint_as_float((unsigned)(e + 127) << 23); }

// Rows that a request has here, and the first of them in the packed call.
__device__ __forceinline__ int tile_rows(const TileShape& d, const int* starts, int s, int& first, DevStatus* stt) {
  first = min(max(starts[s], 0), d.N);
  const int n = min(max(starts[s + 1], first), d.N) - first;
  if (n > d.max_count) {   // (few-row requests of that kind have their own record)
    set_status(stt, ARCKV_ERR_SHAPE);
    return 0;
  }
  return (long long)n * d.G > d.above ? n : 0;
}
// Tokens that row i of `count` sees in a request of len tokens.
__device__ __forceinline__ int row_sees(bool causal, int len, int count, int i) {
  return causal ? max(0, min(len, len - count + i + 1)) : len;
}
// Pages of a row tile: as far as its last row sees (one at least).
__device__ __forceinline__ int tile_steps(const TileShape& d, int len, int count, int tile, int rows) {
  const int last = min((tile + 1) * rows, count * d.G) - 1;
  return max(1, pages_of(row_sees(d.causal, len, count, last / d.G)));
}

struct Segment {
  long long first;         // unit at which the item begins
  int s, h, tile, step, count;   // from step `step` of `count`
  int rows, row, len;      // rows (tokens) of the request, the first of them in the packed call, its tokens
};

// The item of unit u: units run over requests (pre[s] of a head of the earlier ones), heads, row tiles, steps.
__device__ __forceinline__ Segment segment_of(long long u, const TileShape& d, const arckv_pages4& c, const int* starts,
                                              const long long* pre, int rows, DevStatus* stt) {
  Segment g;
  int lo = 0, hi = c.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] * c.H <= u) lo = mid;
    else hi = mid;
  }
  g.s = lo;
  const long long per = pre[lo + 1] - pre[lo], rest = u - pre[lo] * c.H, h = quotient(rest, per);
  g.h = (int)h;
  g.rows = tile_rows(d, starts, lo, g.row, stt);
  const int len = g.len = pages_len(c, lo), lane = threadIdx.x & 31, tiles = (g.rows * d.G + rows - 1) / rows;
  long long at = rest - h * per;   // (a head's tiles times its pages: up to 2^40; 32 tiles have 2^25 steps at most)
  for (int t0 = 0;; t0 += 32) {   // the tile, 32 at a time
    const int mine = t0 + lane < tiles ? tile_steps(d, len, g.rows, t0 + lane, rows) : 0;
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
      g.step = (int)at - (__shfl_sync(0xffffffffu, x, w) - g.count);
      g.tile = t0 + w;
      break;
    }
    at -= __shfl_sync(0xffffffffu, x, 31);
    if (t0 + 32 >= tiles) {   // not reached: `at` lies within the head's steps
      g.count = 1;
      g.step = 0;
      g.tile = max(0, tiles - 1);
      break;
    }
  }
  g.first = u - g.step;
  return g;
}

constexpr float kLargestBf16 = 3.3895313892515355e38f;

// Of four lanes with four words each, lane c ends with word c of all, in the order of the lanes.
__device__ __forceinline__ void transpose4(uint32_t (&y)[4], int lane) {
  const bool b0 = lane & 1, b1 = lane & 2;
  uint32_t a = __shfl_xor_sync(0xffffffffu, b0 ? y[0] : y[1], 1), b = __shfl_xor_sync(0xffffffffu, b0 ? y[2] : y[3], 1);
  if (b0) y[0] = a, y[2] = b;
  else y[1] = a, y[3] = b;
  a = __shfl_xor_sync(0xffffffffu, b1 ? y[0] : y[2], 2), b = __shfl_xor_sync(0xffffffffu, b1 ? y[1] : y[3], 2);
  if (b1) y[0] = a, y[1] = b;
  else y[2] = a, y[3] = b;
}

// Two columns of two rows of the output, at o + at0 and o + at1.
__device__ __forceinline__ void store_rows(bf16* o, long long at0, long long at1, bool row0, bool row1, float4 x,
                                           DevStatus* stt) {
  const float big = kLargestBf16;
  if (row0) *(__nv_bfloat162*)(o + at0) = __floats2bfloat162_rn(x.x, x.y);
  if (row1) *(__nv_bfloat162*)(o + at1) = __floats2bfloat162_rn(x.z, x.w);
  if ((row0 && !(fabsf(x.x) <= big && fabsf(x.y) <= big)) || (row1 && !(fabsf(x.z) <= big && fabsf(x.w) <= big)))
    set_status(stt, ARCKV_ERR_NONFINITE);
}

// Of a page: the unit of K; ev - eref, 2^{eref - ev}, 2^eref and what O shrinks by before it; the page (-1: none).
struct __align__(16) Meta {
  float ks, dv, undo, unit, shrink;
  int page;
};
struct __align__(16) Units {   // for the converters: 1 / unit of K, of V, and tokens that are held
  float k, v;
  int held;
};
// Codes as f16: a nibble c is the number c 2^-24 by itself, c 2^-20 four bits up.  Both are below the normal range, exact, and
// ordinary operands: one operation makes c s + m of two, with s 2^24 or s 2^20 for the scale.  The latter must stay below
// 2^16, so elements are taken in units that leave them below 2^-6 (kDown): then s < 2^-8.9.
constexpr int kDown = 7;
struct Scale {
  __half2 low, high, m;   // s 2^24, s 2^20, m
  __device__ __forceinline__ Scale(float s0, float s1, float m0, float m1) {
    high = __floats2half2_rn(s0 * 1048576.f, s1 * 1048576.f);
    low = __hmul2(high, __half2{__half_raw{0x4c00}, __half_raw{0x4c00}});   // 16
    m = __floats2half2_rn(m0, m1);
  }
};
__device__ __forceinline__ uint32_t low_pair(uint32_t w, const Scale& s) {
  const uint32_t c = w & 0x000f000fu;
  const __half2 z = __hfma2(*(const __half2*)&c, s.low, s.m);
  return *(const uint32_t*)&z;
}
__device__ __forceinline__ uint32_t high_pair(uint32_t w, const Scale& s) {
  const uint32_t c = w & 0x00f000f0u;
  const __half2 z = __hfma2(*(const __half2*)&c, s.high, s.m);
  return *(const uint32_t*)&z;
}

template <int kT, bool kBias>
__global__ void __launch_bounds__(TileCfg<kT>::kThreads, 1)
    pages_tiles_kernel(const arckv_pages4 c, TileShape d, const bf16* Q, PackedStrides qs, float scale, const int* starts, bf16* O,
                       PackedStrides os, float* parts, int4* cuts, DevStatus* stt) {
  using Cfg = TileCfg<kT>;
  constexpr int kSoft = Cfg::kSoft, kMma = Cfg::kMma, kRows = Cfg::kRows, kRaw = Cfg::kRaw, kStages = Cfg::kStages, kBuf = Cfg::kBuf;
  extern __shared__ unsigned char smraw[];
  unsigned char* sQ = smraw + ((1024u - (tc::smem_u32(smraw) & 1023u)) & 1023u);   // [tile][half][128][128 B]
  unsigned char* sKV = sQ + kT * 2 * kHalf;                                        // [stage][K halves, V]
  unsigned char* sRaw = sKV + kStages * kStageBytes;                               // [raw stage] page
  long long* pre = (long long*)(sRaw + kRaw * ARCKV_PAGE_BYTES);                   // [S + 1] pages of a head's tiles
  // of each buffer of a tile: S written, P written, P V done
  __shared__ __align__(8) uint64_t qfull, full[kStages], empty[kStages], sfull[kT][kBuf], pfull[kT][kBuf], odone[kT][kBuf], drain;
  __shared__ __align__(8) uint64_t raw_full[kRaw], raw_empty[kRaw], scaled[kRaw];
  constexpr int kMetas = kRaw + kStages;
  __shared__ Meta meta[kMetas];   // of the pages that have come and are not done
  __shared__ Units units[kRaw];
  __shared__ int raw_page[kRaw];
  __shared__ uint32_t tmem_slot;
  __shared__ long long s_share[2];
  __shared__ __align__(8) uint64_t seg_full[kSegments], seg_empty[kSegments];
  __shared__ Segment s_first, s_seg[kSegments];   // the CTA's first item; the later ones, in turn
  __shared__ int abort_flag, stop_flag;
  __shared__ uint32_t s_beyond[Cfg::kSoftThreads];   // a softmax thread's own: what its two rows' products are short of, as powers of two
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abortp = &abort_flag;

  if (tid == 0) {
    tc::mbar_init(&qfull, kSoft);
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(&full[i], 4);   // converters
      tc::mbar_init(&empty[i], 1);
    }
    for (int t = 0; t < kT; ++t)
      for (int i = 0; i < kBuf; ++i) {
        tc::mbar_init(&sfull[t][i], 1);
        tc::mbar_init(&pfull[t][i], 8);
        tc::mbar_init(&odone[t][i], 1);
      }
    for (int i = 0; i < kRaw; ++i) {
      tc::mbar_init(&raw_full[i], 1);
      tc::mbar_init(&raw_empty[i], 5);
      tc::mbar_init(&scaled[i], 1);
    }
    for (int i = 0; i < kSegments; ++i) {
      tc::mbar_init(&seg_full[i], 1);
      tc::mbar_init(&seg_empty[i], kSoft + 3);   // softmax, MMA, scales, pages
    }
    tc::mbar_init(&drain, 1);
    abort_flag = 0;
    tc::mbar_fence_init();
  }
  if (warp == kMma) tc::tmem_alloc(&tmem_slot, 512);
  pdl_trigger();
  pdl_wait();
  for (int s = tid; s < c.S; s += Cfg::kThreads) {   // pages of one head's tiles of each request
    int first;
    const int len = pages_len(c, s), rows = tile_rows(d, starts, s, first, stt), tiles = (rows * d.G + kRows - 1) / kRows;
    long long n = 0;
    if (d.causal)
      for (int t = 0; t < tiles; ++t) n += tile_steps(d, len, rows, t, kRows);
    else if (tiles > 0)
      n = (long long)tiles * tile_steps(d, len, rows, 0, kRows);
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
    long long u0 = 0, u1 = 0;
    Segment g = {};
    if (run > 0) {
      const CacheShares sh(run * c.H, gridDim.x);
      u0 = sh.start(min((int)blockIdx.x, sh.ctas));
      u1 = sh.start(min((int)blockIdx.x + 1, sh.ctas));
      if (u0 < u1) g = segment_of(u0, d, c, starts, pre, kRows, stt);
    }
    if (lane == 0) {
      s_share[0] = u0;
      s_share[1] = u1;
      s_first = g;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;   // tile t: buffers of S / P from column 256 t on, O behind them
  const long long u0 = s_share[0], u1 = s_share[1];
  // The CTA's item behind its k-th, which the last warp has found.
  auto next_segment = [&](int k, Segment& g) {
    const int at = k % kSegments;
    const bool ok = __all_sync(0xffffffffu, tc::mbar_wait(&seg_full[at], (k / kSegments) & 1, abortp, stt));
    if (ok) g = s_seg[at];
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&seg_empty[at]);
    return ok;
  };
  // whether the second tile of an item has rows
  auto both = [&](const Segment& g) { return kT == 2 && g.tile * kRows + 128 < g.rows * d.G; };

  if (warp == kMma + 3) {
    // ------------- the CTA's items, ahead of the others; the one that begins here and goes on in other CTAs
    regs_dec<Cfg::kRegsMma>();
    int4 cut = make_int4(0, 0, -1, 0);
    if (u0 < u1) {
      Segment g = s_first;
      bool ok = true;
      int k = 0;
      for (long long u = g.first + g.count; u < u1; u = g.first + g.count, ++k) {
        g = segment_of(u, d, c, starts, pre, kRows, stt);
        const int at = k % kSegments;
        if (k >= kSegments) ok = __all_sync(0xffffffffu, tc::mbar_wait(&seg_empty[at], ((k / kSegments) - 1) & 1, abortp, stt));
        if (!ok) break;
        if (lane == 0) {
          s_seg[at] = g;
          tc::mbar_arrive(&seg_full[at]);
        }
      }
      const CacheShares sh(pre[c.S] * c.H, gridDim.x);
      const long long end = g.first + g.count;
      if (ok && end > u1 && g.first >= u0) cut = make_int4(g.s * c.H + g.h, g.tile, sh.owner(end - 1), 0);
    }
    if (lane == 0) cuts[blockIdx.x] = cut;
  } else if (warp == kMma + 2) {
    // ---------------------------------------------------------------- pages
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int q = 0;   // pages issued
    Segment g = s_first;
    int seg = 0;
    for (long long u = u0; u < u1 && ok;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u), held = pages_of(g.len);
      int page = -1;
      for (int i = 0; i < n; ++i, ++q) {
        const int st = q % kRaw;
        if ((i & 31) == 0) {   // of the next 32 steps, a lane each
          const int b = g.step + i + lane;
          page = i + lane < n && b < held ? c.table[(long long)g.s * c.M + b] : -1;
          if (page >= c.P) {
            set_status(stt, ARCKV_ERR_INVALID_ARG);
            page = -1;
          }
        }
        if (q >= kRaw) ok = __all_sync(0xffffffffu, tc::mbar_wait(&raw_empty[st], ((q / kRaw) - 1) & 1, abortp, stt));
        if (!ok) break;
        if (lane == (i & 31)) {
          raw_page[st] = page;
          if (page >= 0) {
            tc::mbar_arrive_expect_tx(&raw_full[st], ARCKV_PAGE_BYTES);
            tc::bulk_load(sRaw + st * ARCKV_PAGE_BYTES, page_at(c, page, g.h), ARCKV_PAGE_BYTES, &raw_full[st]);
          } else {
            tc::mbar_arrive(&raw_full[st]);
          }
        }
        __syncwarp();
      }
      u += n;
      if (u < u1 && ok) ok = next_segment(seg++, g);
    }
    if (!ok) {   // let the copies in flight land before the CTA's memory goes
      volatile int never = 0;
      for (int p = max(0, q - kRaw); p < q; ++p) tc::mbar_wait(&raw_full[p % kRaw], (p / kRaw) & 1, &never, stt);
    }
  } else if (warp == kMma + 1) {
    // ---------------------------------------------------------------- scales
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int q = 0, seg = 0;
    Segment g = s_first;
    for (long long u = u0; u < u1 && ok;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u), len = g.len;
      int eref = -1000, largest_ref = -1000;
      for (int i = 0; i < n && ok; ++i, ++q) {
        const int rs = q % kRaw;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&raw_full[rs], (q / kRaw) & 1, abortp, stt));
        if (!ok) break;
        const int page = raw_page[rs], held = page < 0 ? 0 : min(kPT, max(0, len - (g.step + i) * kPT));
        const unsigned char* raw = sRaw + rs * ARCKV_PAGE_BYTES;
        auto largest = [](uint32_t w) { return __float_as_uint(fmaxf(fabsf(bf16_hi(w)), fabsf(fmaf(15.f, bf16_lo(w), bf16_hi(w))))); };
        uint32_t k = 0u, v = 0u;   // (as integers, the larger of two magnitudes is the larger float)
#pragma unroll
        for (int x = 0; x < 2; ++x) {   // a lane has tokens lane, lane + 32
          const int tok = lane + 32 * x;
          if (tok < held) {
            const uint4 w = *(const uint4*)(raw + kPageKp + tok * 16);
            k = max(max(max(k, largest(w.x)), max(largest(w.y), largest(w.z))), largest(w.w));
            v = max(v, largest(*(const uint32_t*)(raw + kPageVp + tok * 4)));
          }
        }
        k = __reduce_max_sync(0xffffffffu, k);
        v = __reduce_max_sync(0xffffffffu, v);
        const int ek = min(max((int)(k >> 23) - 127, -100), 70), own = min(max((int)(v >> 23) - 127, -100), 70);
        Meta m;
        m.shrink = 1.f;
        // two bits of room, so that few pages raise it; where a page needs less than 2^-6 of it, it follows down, as far as O's
        // range goes (values of zero need nothing)
        if (own > eref || (own < eref - 6 && v != 0u)) {
          const int to = max(own + 2, largest_ref - 60);
          if (i > 0) m.shrink = pow2(eref - to);
          eref = to;
          largest_ref = max(largest_ref, eref);
        }
        const int ev = max(own, eref - 6);
        m.ks = pow2(ek + kDown);
        m.dv = (float)(ev - eref);
        m.undo = pow2(eref - ev);
        m.unit = pow2(eref + kDown);
        m.page = page;
        if (lane == 0) {   // (the page has come, so the one kRaw before it is converted, and P V of the one kStages before that done)
          meta[q % kMetas] = m;
          units[rs] = Units{pow2(-ek - kDown), pow2(-ev - kDown), held};
          tc::mbar_arrive(&scaled[rs]);
          tc::mbar_arrive(&raw_empty[rs]);
        }
      }
      u += n;
      if (u < u1 && ok) ok = next_segment(seg++, g);
    }
  } else if (warp == kMma) {
    // ------------------------------------------------------------ MMA issuer
    regs_dec<Cfg::kRegsMma>();
    bool ok = true;
    int st = 0, sp = 0, phase = 0;   // stages of the next page for S, for P V
    int base[kT];                    // pages of each tile in earlier items
#pragma unroll
    for (int t = 0; t < kT; ++t) base[t] = 0;
    // warp-wide reductions leave their result in uniform registers
    const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem);
    const uint64_t q_desc = tc::sdesc_k128(tc::smem_u32(sQ)), kv_desc = tc::sdesc_k128(tc::smem_u32(sKV));
    int steps = s_first.count - s_first.step, tiles = both(s_first) ? 2 : 1;   // of this item
    int seg = 0, left = __reduce_max_sync(0xffffffffu, (int)(u1 - u0));   // pages to come
    for (long long u = u0; left > 0 && ok; ++seg) {
      const int n = __reduce_max_sync(0xffffffffu, min(steps, left)), nt = __reduce_max_sync(0xffffffffu, tiles);
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&qfull, seg & 1, abortp, stt));
      // S of page i, then P V of page i - 1
      for (int i = 0; i <= n && ok; ++i) {
        if (i < n) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[st], phase, abortp, stt));
          if (!ok) break;
          tc::fence_after_sync();
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            if (t < nt) {
              const int b = (base[t] + i) % kBuf;
              mma_qk(tm + 256 * t + b * 64, q_desc + t * (2 * kHalf >> 4), kv_desc + (st * kStageBytes >> 4), idesc_f16(64));
              commit_elected(&sfull[t][b]);
            }
          }
          if (++st == kStages) {
            st = 0;
            phase ^= 1;
          }
        }
        if (i > 0) {
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            if (t >= nt) break;
            const int p = base[t] + i - 1, b = p % kBuf;
            ok = __all_sync(0xffffffffu, ok && tc::mbar_wait(&pfull[t][b], (p / kBuf) & 1, abortp, stt));
            if (!ok) break;
            tc::fence_after_sync();
            mma_pv(tm + 256 * t + Cfg::kO, tm + 256 * t + b * 64, kv_desc + ((sp * kStageBytes + 2 * kKTile) >> 4), idesc_f16(128),
                   i > 1);
            commit_elected(&odone[t][b]);
          }
          if (!ok) break;
          if (kT == 2) commit_elected(&empty[sp]);   // (of one tile, P V)
          if (++sp == kStages) sp = 0;
        }
      }
#pragma unroll
      for (int t = 0; t < kT; ++t)
        if (t < nt) base[t] += n;
      left -= n;
      u += n;
      if (left > 0 && ok) {
        Segment next = {};
        ok = next_segment(seg, next);
        steps = next.count - next.step;
        tiles = both(next) ? 2 : 1;
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
    const int cw = warp - kSoft, total = (int)(u1 - u0), g = lane >> 2, t = lane & 3;
    // K: rows r, r + 8 of this warp's 16, eight dims of each group.  Eight lanes have two rows four apart, whose operands
    // meet in no bank (as codes they do, one load for four stores).
    const int kr = cw * 16 + ((g >> 1) | (g & 1) << 2);
    // V: 16 tokens; lane (g, t) has pairs t, t + 4 of them, dims g + 8 x.  Matrices of 8 dims x 8 tokens: lane l gives the
    // address of row l % 8 of matrix l / 8, dims 8 (x + m / 2), tokens 8 (m % 2).
    const int m4 = lane >> 3, v_row = ((m4 >> 1) * 8 + (lane & 7)) * 128 + (((2 * cw + (m4 & 1)) ^ (lane & 7)) << 4);
    const uint32_t kv0 = tc::smem_u32(sKV);
    for (int q = 0; q < total; ++q) {
      const int st = q % kStages, rs = q % kRaw;
      bool ok = tc::mbar_wait(&scaled[rs], (q / kRaw) & 1, abortp, stt);
      if (ok) ok = tc::mbar_wait(&raw_full[rs], (q / kRaw) & 1, abortp, stt);   // (long done: for the copy's visibility)
      // (with one tile and as many stages as buffers, P V is done with both at once)
      if (ok && q >= kStages) ok = tc::mbar_wait(kT == 1 ? &odone[0][st] : &empty[st], ((q / kStages) - 1) & 1, abortp, stt);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const unsigned char* raw = sRaw + rs * ARCKV_PAGE_BYTES;
      const Units un = units[rs];
      unsigned char* Ks = sKV + st * kStageBytes;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = kr + 8 * x;
        const uint4 cw4 = *(const uint4*)(raw + r * 64 + t * 16);
        uint4 pw4 = *(const uint4*)(raw + kPageKp + r * 16);
        if (r >= un.held) pw4 = make_uint4(0u, 0u, 0u, 0u);   // (anything may be there)
        const uint32_t cws[4] = {cw4.x, cw4.y, cw4.z, cw4.w}, pws[4] = {pw4.x, pw4.y, pw4.z, pw4.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float sc = bf16_lo(pws[w]) * un.k, least = bf16_hi(pws[w]) * un.k;
          const Scale z(sc, sc, least, least);
          const uint32_t a = cws[w], b = a >> 8;
          *(uint4*)(Ks + (w >> 1) * kKTile + r * 128 + ((((w & 1) * 4 + t) ^ (r & 7)) << 4)) =
              make_uint4(low_pair(a, z), high_pair(a, z), low_pair(b, z), high_pair(b, z));
        }
      }
      auto pair_scale = [&](int pair) {
        uint2 p = *(const uint2*)(raw + kPageVp + pair * 8);
        if (2 * pair >= un.held) p.x = 0u;
        if (2 * pair + 1 >= un.held) p.y = 0u;
        return Scale(bf16_lo(p.x) * un.v, bf16_lo(p.y) * un.v, bf16_hi(p.x) * un.v, bf16_hi(p.y) * un.v);
      };
      const int pair = cw * 8 + t;
      const Scale z0 = pair_scale(pair), z1 = pair_scale(pair + 4);
      const uint4 va = *(const uint4*)(raw + kPageV + pair * 128 + ((g ^ (t << 1)) << 4));
      const uint4 vb = *(const uint4*)(raw + kPageV + (pair + 4) * 128 + ((g ^ (t << 1)) << 4));
      const uint32_t aw[4] = {va.x, va.y, va.z, va.w}, bw[4] = {vb.x, vb.y, vb.z, vb.w};
      const uint32_t vd = kv0 + st * kStageBytes + 2 * kKTile + v_row;
#pragma unroll
      for (int w = 0; w < 4; ++w) {   // dims 32 w .. + 31, 16 at a time
        const uint32_t a8 = aw[w] >> 8, b8 = bw[w] >> 8;
        store_matrices(vd + w * (32 * 128), low_pair(aw[w], z0), low_pair(bw[w], z1), high_pair(aw[w], z0), high_pair(bw[w], z1));
        store_matrices(vd + w * (32 * 128) + 16 * 128, low_pair(a8, z0), low_pair(b8, z1), high_pair(a8, z0), high_pair(b8, z1));
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
    const uint32_t Sb = tmem + 256 * t + ((uint32_t)(quarter * 32 + half * 16) << 16), Ot = Sb + Cfg::kO;
    bool ok = true;
    // P V of page q is in O.  (The one before it, whose phase this could be taken for, is known to be: S of page
    // q + 1 was issued after it and has come in.)
    auto product_done = [&](int q) {
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&odone[t][q % kBuf], (q / kBuf) & 1, abortp, stt));
      tc::fence_after_sync();
      return ok;
    };
    int it = 0, all = 0, seg = 0;   // pages of this tile, of the CTA, in earlier items; their number
    Segment g = s_first;
    for (long long u = u0; u < u1;) {
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      const int row0 = g.tile * kRows + t * 128, len = g.len, nrows = g.rows * d.G;
      const bool idle = t == 1 && !both(g);
      const bf16* Qh = Q + g.row * qs.i + g.h * qs.h;
      // the products' factor (for powers of two without biases, of e with them) and sight of this thread's two rows
      float fac = 0.f;
      int see[2];
      bool far = false;   // see below
      if (!idle) {
        // This warp's 16 queries as f16, scaled by a power of two that leaves the largest element of all in [2^14, 2^15): a bf16
        // is exact down to 2^-31 of it, and next to nothing below 2^-39.  16 lanes have a row, two rows at a time.
        // Where some four dims of a row are all 2^-12 of that or less, each row gets a power of its own, so that what one row
        // holds, however large or not finite, is nothing to the others.  (A change of items waits for its code, some 20 ns an
        // instruction: powers for each row in every case took 686 us for 8192 positions, 657 with this.)
        uint4 x[8];
        int row = row0 + r_warp + (lane >> 4), i = row / d.G, gq = row - i * d.G;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = make_uint4(0u, 0u, 0u, 0u);
          if (row < nrows) x[e] = *((const uint4*)(Qh + i * qs.i + gq * 128) + (lane & 15));
          row += 2;
          gq += 2;
          while (gq >= d.G) {
            gq -= d.G;
            ++i;
          }
        }
        auto largest = [](const uint4& y) {   // magnitudes of four even and four odd elements, as integers
          return __vmaxu2(__vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu), __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu));
        };
        auto exponent = [](uint32_t m) { return min(max((int)(m >> 7) - 127, -100), 127); };
        uint32_t amax = 0u, amin = 0u;   // of all fours; and of the smallest that is not zero, 0x8000 less it
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t m = largest(x[e]);
          amax = __vmaxu2(amax, m);
          amin = __vmaxu2(amin, (0x80008000u - m) & 0x7fff7fffu);
        }
        amax = __reduce_max_sync(0xffffffffu, max(amax & 0xffffu, amax >> 16));
        amin = __reduce_max_sync(0xffffffffu, max(amin & 0xffffu, amin >> 16));
        int ex = exponent(amax);
        far = (int)(amax + amin) > 0x8000 + (12 << 7);
        s_beyond[tid] = 0u;
        if (far) {   // (rare) all rows to the smallest one's power; their products get the rest, 2^beyond, when they come
          ex = 1000;
          uint32_t own = 0u;   // largest magnitudes of rows lane / 4 and lane / 4 + 8
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint32_t m = largest(x[e]);
              m = max(m & 0xffffu, m >> 16);
#pragma unroll
              for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
              if (pass == 0) {
                const uint32_t y = __shfl_sync(0xffffffffu, m, (lane & 4) << 2);
                if (lane >> 3 == (e & 3)) own |= y << (e < 4 ? 0 : 16);
                ex = min(ex, (int)__reduce_min_sync(0xffffffffu, m ? exponent(m) : 1000));
              } else {   // (in two steps: each power is within fp32's normal range)
                const int by = m ? ex - exponent(m) : 0;
                const float by0 = pow2(by / 2), by1 = pow2(by - by / 2);
                uint32_t y[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const __nv_bfloat162 z = __floats2bfloat162_rn(bf16_lo(y[k]) * by0 * by1, bf16_hi(y[k]) * by0 * by1);
                  y[k] = *(const uint32_t*)&z;
                }
                x[e] = make_uint4(y[0], y[1], y[2], y[3]);
              }
            }
          }
          const uint32_t o0 = own & 0xffffu, o1 = own >> 16;
          s_beyond[tid] = (o0 ? exponent(o0) - ex : 0) | (o1 ? exponent(o1) - ex : 0) << 16;
        }
        const float up = pow2(14 - ex);
        fac = pow2(ex - 14) * scale * (kBias ? 1.f : kLog2e);
        const int c16 = lane & 15;   // chunk of 8 dims
        unsigned char* to = sQ + (t * 2 + (c16 >> 3)) * kHalf;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t y[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
          __half2 z[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) z[k] = __floats2half2_rn(bf16_lo(y[k]) * up, bf16_hi(y[k]) * up);
          const int r = quarter * 32 + half * 16 + 2 * e + (lane >> 4);   // TMEM lane
          *(uint4*)(to + r * 128 + (((c16 & 7) ^ (r & 7)) << 4)) = *(const uint4*)&z[0];
        }
        tc::fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&qfull);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = row0 + r_warp + (lane >> 2) + 8 * i;
        see[i] = row < nrows ? row_sees(d.causal, len, g.rows, row / d.G) : 0;
      }
      const int see_min = far ? 0 : __reduce_min_sync(0xffffffffu, min(see[0], see[1]));   // (zero: every page has an edge)
      // references of O (with biases the logit), sums of weights
      float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, unit = 1.f;
      const bool any_row = row0 + r_warp < nrows;
      for (int i = 0; i < n && !idle; ++i) {
        const int q = it + i, j0 = (g.step + i) * kPT + cl;
        const uint32_t S = Sb + (q % kBuf) * 64;
        // S is in, and with it the page's scales (written before the page was converted)
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&sfull[t][q % kBuf], (q / kBuf) & 1, abortp, stt));
        if (!ok) break;
        if (!any_row) {   // (uniform)
          if (lane == 0) tc::mbar_arrive(&pfull[t][q % kBuf]);
          continue;
        }
        tc::fence_after_sync();
        float v[32];
        tmem_ld_rows64(S, v);
        const Meta m = meta[(all + i) % kMetas];
        // (never zero: a masked product is -inf)
        const float f = fmaxf(fac * m.ks, 0x1p-126f);
        unit = m.unit;
        tmem_wait_ld();
        settle(v);
        const bool edge = j0 - cl + kPT > see_min || m.page < 0;
        if (edge && s_beyond[tid] != 0u) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int by = (int)(s_beyond[tid] >> (16 * k) & 0xffffu);
            const float by0 = pow2(by / 2), by1 = pow2(by - by / 2);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              v[4 * j + 2 * k] = v[4 * j + 2 * k] * by0 * by1;
              v[4 * j + 2 * k + 1] = v[4 * j + 2 * k + 1] * by0 * by1;
            }
          }
        }
        if (kBias && m.page >= 0) {   // logits
          const float* bias = c.bias + ((long long)m.page * c.H + g.h) * kPT + cl;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 x = *(const float2*)(bias + 8 * j);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              v[4 * j + 2 * k] = fmaf(v[4 * j + 2 * k], f, x.x);
              v[4 * j + 2 * k + 1] = fmaf(v[4 * j + 2 * k + 1], f, x.y);
            }
          }
        }
        if (edge) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (m.page < 0 || j0 + 8 * j + (k & 1) >= see[k >> 1]) v[4 * j + k] = -INFINITY;
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
          // in units of log2; with biases differences of logits first, so that the type's lowest value cancels against
          // itself.  (A reference of -inf is past by any logit but -inf.)
          grows |= kBias ? (top[k] - ref[k]) * kLog2e > kGrow : top[k] * f > ref[k] + kGrow;
        }
        grows = __any_sync(0xffffffffu, grows);
        if (grows || m.shrink != 1.f) {
          float alpha[2] = {m.shrink, m.shrink};
          if (grows) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
              top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
              const float to = kBias ? top[k] : top[k] * f;
              // what the sums shrink by, as a power of two
              const float by = ref[k] == -INFINITY ? -INFINITY : kBias ? (ref[k] - to) * kLog2e : ref[k] - to;
              if (to != -INFINITY && -by > kFollow) {
                const float x = ex2_approx(by);
                alpha[k] *= x;
                l[k] *= x;
                ref[k] = to;
              }
            }
          }
          if (i > 0) {   // scale O
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
          const float b = ref[k] == -INFINITY ? 0.f : ref[k], a = (kBias ? 0.f : -b) + m.dv + kLift;
          base[k] = make_float2(-b, -b);
          add[k] = make_float2(a, a);
          sum[k] = make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {   // 32 tokens: 16 columns
          uint32_t hr[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = e & 1, j = ch * 4 + (e >> 1);
            float2 x = make_float2(v[4 * j + 2 * k], v[4 * j + 2 * k + 1]);
            if (kBias)
              x = fma2(add2(x, base[k]), make_float2(kLog2e, kLog2e), add[k]);
            else
              x = fma2(x, make_float2(f, f), add[k]);
            x.x = ex2_approx(x.x);
            x.y = ex2_approx(x.y);
            sum[k] = add2(sum[k], x);
            const __half2 h2 = __floats2half2_rn(x.x, x.y);
            hr[e] = *(const uint32_t*)&h2;
          }
          tmem_st_pairs16(S + ch * 16, hr);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) l[k] = fmaf(sum[k].x + sum[k].y, m.undo, l[k]);
        tmem_wait_st();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&pfull[t][q % kBuf]);
      }
      all += n;
      if (!idle) {
        it += n;
        if (ok) product_done(it - 1);
      }
      if (tid == 0) stop_flag = *abortp;   // one reading for all
      asm volatile("bar.sync 1, %0;" ::"r"(Cfg::kSoftThreads) : "memory");
      if (stop_flag) break;
      if (!idle) {
        const bool whole = g.step == 0 && n == g.count;
        // (a product is exact in its difference from the reference, which is rounded: by half of a power of two at most up to here)
        if (!kBias && ((fabsf(ref[0]) > kLogitMost && ref[0] != -INFINITY) || (fabsf(ref[1]) > kLogitMost && ref[1] != -INFINITY)))
          set_status(stt, ARCKV_ERR_NONFINITE);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
          l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
        }
        int q0 = row0 + r_warp + (lane >> 2);   // (not kept in registers through the loop)
        asm volatile("" : "+r"(q0));
        const int q1 = q0 + 8;
        const long long at0 = (g.row + q0 / d.G) * os.i + (q0 % d.G) * 128, at1 = (g.row + q1 / d.G) * os.i + (q1 % d.G) * 128;
        const float inv0 = l[0] == 0.f ? 0.f : 1.f / l[0], inv1 = l[1] == 0.f ? 0.f : 1.f / l[1];
        // A part goes to memory divided by its sum, as f16 (parts as fp32 took twice the time to write and read, half of them
        // 13.8 us to join).  Each row is taken in a power of two of its own that leaves its largest element in [2^14, 2^15): half a
        // step is 2^-11 of an element, down to 2^-28 of the row's largest.  (O's units would not do: they follow the largest value,
        // and the mean of thousands of values lies far below it.)
        float* slot = parts + (2ll * blockIdx.x + (g.step == 0 ? 1 : 0)) * Cfg::kSlot + tid * 4;
        if (any_row) {
          float2 up = make_float2(inv0, inv1), down = make_float2(unit, unit);
          if (!whole) {
            float most[2] = {0.f, 0.f};
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              float v[16];
              tmem_ld_rows32(Ot + ch * 32, v);
              tmem_wait_ld();
              settle(v);
#pragma unroll
              for (int e = 0; e < 16; e += 2) most[(e >> 1) & 1] = max3(most[(e >> 1) & 1], fabsf(v[e]), fabsf(v[e + 1]));
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float a = most[k] * (k ? inv1 : inv0);
              a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
              a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
              const int e_unit = (int)(__float_as_uint(unit) >> 23) - 127;
              // (what a part's elements stand for stays a multiple of 2^-126)
              const int ex = min(max((int)(__float_as_uint(a) >> 23) - 127, max(-100, -112 - e_unit)), 127);
              (k ? up.y : up.x) *= pow2(14 - ex);
              (k ? down.y : down.x) *= pow2(ex - 14);
            }
          }
#pragma unroll 1
          for (int ch = 0; ch < 4; ++ch) {
            float v[16];
            tmem_ld_rows32(Ot + ch * 32, v);
            tmem_wait_ld();
            settle(v);
            if (whole) {   // four lanes have a row's 32 columns, two of each eight: each takes eight of its own
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const float inv = k ? inv1 : inv0;
                uint32_t y[4];
                bool bad = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // (the unit first: it may be far from one, and the sum as far from it as the values are)
                  const float2 z = make_float2(v[4 * e + 2 * k] * unit * inv, v[4 * e + 2 * k + 1] * unit * inv);
                  bad |= !(fabsf(z.x) <= kLargestBf16 && fabsf(z.y) <= kLargestBf16);
                  const __nv_bfloat162 w = __floats2bfloat162_rn(z.x, z.y);
                  y[e] = *(const uint32_t*)&w;
                }
                transpose4(y, lane);
                if ((k ? q1 : q0) < nrows) {
                  *(uint4*)(O + g.h * os.h + (k ? at1 : at0) + ch * 32 + 8 * (lane & 3)) = make_uint4(y[0], y[1], y[2], y[3]);
                  if (bad) set_status(stt, ARCKV_ERR_NONFINITE);
                }
              }
            } else {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                __half2 y[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                  const float by = f & 1 ? up.y : up.x;
                  y[f] = __floats2half2_rn(v[8 * e + 2 * f] * by, v[8 * e + 2 * f + 1] * by);
                }
                __stcg((uint4*)(slot + (long long)(ch * 2 + e) * Cfg::kSoftThreads * 4), *(const uint4*)&y[0]);
              }
            }
          }
          if (!whole) {   // joined by the kernel behind this one
            __stcg((float4*)(slot + 8ll * Cfg::kSoftThreads * 4), make_float4(ref[0], l[0], ref[1], l[1]));
            __stcg((float2*)(slot + 9ll * Cfg::kSoftThreads * 4), down);
          }
        }
      }
      tc::fence_before_sync();
      u += n;
      if (u < u1 && !next_segment(seg++, g)) {   // a wait gave up: once to the barrier, as the others
        if (tid == 0) stop_flag = *abortp;
        asm volatile("bar.sync 1, %0;" ::"r"(Cfg::kSoftThreads) : "memory");
        break;
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kMma) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, 512);
  }
}

// Adds up the parts of the items that several CTAs of pages_tiles_kernel shared: cuts[c] is {request x head, tile, last
// CTA} of the item that begins in CTA c and goes on, or has a last CTA of -1.  One work unit is the 16 rows that one softmax
// warp had.
constexpr int kJoinThreads = 256;
template <int kT, bool kBias>
__global__ void __launch_bounds__(kJoinThreads) pages_join_kernel(int H, TileShape d, const int* starts, bf16* O, PackedStrides os,
                                                                  const float* parts, const int4* cuts, int n_cuts,
                                                                  DevStatus* stt) {
  using Cfg = TileCfg<kT>;
  __shared__ int4 s_cut[kCacheMaxCtas];   // of the items, in order; w: the CTA in which it begins
  __shared__ int s_items;
  __shared__ float s_w[kCacheMaxCtas][16], s_inv[16];
  const int tid = threadIdx.x, lane = tid & 31;
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
    const int s = cut.x / H, h = cut.x - s * H, row0 = cut.y * Cfg::kRows + warp * 16;
    int row;
    const int nrows = tile_rows(d, starts, s, row, stt) * d.G;
    if (row0 >= nrows) continue;   // (uniform)
    auto part = [&](int p) { return parts + (2ll * (first + p) + (p == 0)) * Cfg::kSlot + warp * 128; };
    // The parts' loads wait for nothing: the first eight parts' are under way while the weights are found.  A thread has 16
    // bytes of each: columns 8 j + 2 (lane % 4), + 1 of rows lane / 4 and lane / 4 + 8, for two j.
    const int r8 = lane >> 2, j8 = tid >> 5;
    uint4 ahead[8];
    auto load = [&](int p0) {
#pragma unroll
      for (int p = 0; p < 8; ++p)
        if (p0 + p < n) ahead[p] = __ldcg((const uint4*)(part(p0 + p) + lane * 4 + (long long)j8 * Cfg::kSoftThreads * 4));
    };
    load(0);
    {   // weights of the parts for row tid / 16, sixteen parts at a time
      const int r = tid >> 4, l16 = tid & 15;
      const long long at = 8ll * Cfg::kSoftThreads * 4 + (r & 7) * 16 + (r >> 3) * 2, unit = 9ll * Cfg::kSoftThreads * 4 + (r & 7) * 16 + (r >> 3);
      float top = -INFINITY;
      float2 mine = make_float2(-INFINITY, 0.f);   // of the first sixteen parts
      if (l16 < n) mine = __ldcg((const float2*)(part(l16) + at));
      top = mine.x;
      for (int p = l16 + 16; p < n; p += 16) top = fmaxf(top, __ldcg(part(p) + at));
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float z = 0.f;
      for (int p = l16; p < n; p += 16) {
        const float2 y = p == l16 ? mine : __ldcg((const float2*)(part(p) + at));
        // log2 of what separates two references; of a part that saw nothing no weight
        const float w = y.x == -INFINITY ? 0.f : ex2_approx(kBias ? (y.x - top) * kLog2e : y.x - top);
        z = fmaf(y.y, w, z);
        s_w[p][r] = y.y * w * __ldcg(part(p) + unit);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      if (l16 == 0) s_inv[r] = z == 0.f ? 0.f : 1.f / z;
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
          const uint32_t y[4] = {ahead[p].x, ahead[p].y, ahead[p].z, ahead[p].w};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 y0 = __half22float2(*(const __half2*)&y[2 * e]), y1 = __half22float2(*(const __half2*)&y[2 * e + 1]);
            a[e] = make_float4(fmaf(y0.x, w0, a[e].x), fmaf(y0.y, w0, a[e].y), fmaf(y1.x, w1, a[e].z), fmaf(y1.y, w1, a[e].w));
          }
        }
      }
      const int q0 = row0 + r8, q1 = q0 + 8;
      const long long at0 = (row + q0 / d.G) * os.i + (q0 % d.G) * 128, at1 = (row + q1 / d.G) * os.i + (q1 % d.G) * 128;
      const float i0 = s_inv[r8], i1 = s_inv[r8 + 8];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        store_rows(O + h * os.h + 8 * (2 * j8 + e) + 2 * (lane & 3), at0, at1, q0 < nrows, q1 < nrows,
                   make_float4(a[e].x * i0, a[e].y * i0, a[e].z * i1, a[e].w * i1), stt);
    }
    __syncthreads();
  }
}

template <int kT, bool kBias>
int launch_tiles(const arckv_pages4& p, const PagesQuery& q, float scale, int above, void* ws, cudaStream_t st) {
  using Cfg = TileCfg<kT>;
  TileShape d;
  d.G = q.G;
  d.N = q.N;
  d.above = above;
  d.max_count = q.max_count;
  d.causal = q.causal;
  auto kern = pages_tiles_kernel<kT, kBias>;
  const int smem = Cfg::kSmem + (p.S + 1) * (int)sizeof(long long);
  if (set_dyn_smem((const void*)kern, smem) != cudaSuccess) return -1;
  const int ctas = std::min(tc_gemm_sm_count(), kCacheMaxCtas);
  float* parts = (float*)((char*)ws + ARCKV_CACHE_WS_HEADER);
  int4* cuts = (int4*)(parts + kCacheMaxCtas * 2ll * Cfg::kSlot);
  DevStatus* stt = (DevStatus*)ws;
  cudaError_t e = launch_pdl(kern, dim3(ctas), Cfg::kThreads, smem, st, p, d, q.Q, q.qs, scale, q.starts, q.O, q.os, parts, cuts, stt);
  if (e != cudaSuccess) return -1;
  e = launch_pdl(pages_join_kernel<kT, kBias>, dim3(4 * ctas), kJoinThreads, 0, st, p.H, d, q.starts, q.O, q.os, parts, cuts, ctas, stt);
  return e == cudaSuccess ? 2 : -1;
}

}  // namespace

size_t pages_tiles_scratch(long long rows) {
  return kCacheMaxCtas * (2 * (pages_tile_rows(rows) == 128 ? TileCfg<1>::kSlot : TileCfg<2>::kSlot) * sizeof(float) + sizeof(int4));
}

int launch_pages_tiles(const arckv_pages4& p, const PagesQuery& q, float scale, int above, void* ws, cudaStream_t st) {
  if (pages_tile_rows((long long)q.max_count * q.G) == 128)   // one tile where it holds all rows
    return p.bias ? launch_tiles<1, true>(p, q, scale, above, ws, st) : launch_tiles<1, false>(p, q, scale, above, ws, st);
  return p.bias ? launch_tiles<2, true>(p, q, scale, above, ws, st) : launch_tiles<2, false>(p, q, scale, above, ws, st);
}

}  // namespace arckv
