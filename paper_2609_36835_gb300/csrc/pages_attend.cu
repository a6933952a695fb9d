// Attention of packed queries over paged 4-bit caches, for requests of few rows
// (decode and draft steps):
//
//   O_r = sum_j e^{x_rj} v_j / sum_j e^{x_rj},  x_rj = scale q_r . k_j + bias_j
//
// 148 bytes a token and head are read once.  That is 9472 bytes for 16384 codes: HBM gives an SM a page every 430 cycles or
// so, in which it can issue 1700 warp instructions, so the work on a code has to stay near one tenth of an instruction
// of a warp.  So:
//  - A page of one head is one contiguous piece, and comes by one bulk copy into a ring of stages in shared memory.  The
//    pages lie in the order in which the lanes take them, 16 bytes at a time and free of bank conflicts.
//  - Products run on mma.sync m16n8k16: tokens (dims for V) are the 16 rows, query rows the 8 columns.  A nibble c is an
//    f16 by itself, c 2^-24, and c 2^-20 four bits up, below the normal range and exact: a mask makes two operands, and a
//    word of eight codes costs a shift and four masks.  (tcgen05 would want 64 to 128 rows and a pass of the codes
//    through shared memory; e4m3 operands, of which a nibble is one too, are converted to f16 by the compiler.)
//  - Scales stay out of the products.  The four groups of a key are four sums, exact but for fp32 roundings, that are
//    scaled and added up afterwards; the least values multiply the sums of the query's elements (one more product, of the
//    words as they are).  A value's scale goes into its weight, what its codes are off by goes into a sum of its own that
//    all dims share.
//  - Work is the list of (request, head, page).  With more items than SMs each warp of the launch takes an equal share of it,
//    and waits for no other: what it has of an item at the ends of its share goes to memory as it lies in
//    registers.  (Shares for CTAs, whose warps then add up every item: 94 us instead of 80 for 64 x 8K, 102 instead of 54 for 250
//    requests of up to 1000 tokens.)  With fewer items they are cut into equal parts, a CTA each, whose warps take pages in
//    turn.  An item in several places is finished by the one that comes last (a ticket), which adds the parts up in order.
//  - Weights enter the tensor cores as f16, times the value's scale in units between two and 2^8 times a page's largest.  They begin at
//    2^7 and reach 2^15 (references lag the maximum by up to 2^8).  Half a step is 2^-11 of a weight, down to 2^-13 of the
//    reference's.  It moves v alone, not the v - m of its code: see below.  Scales may grow or
//    shrink from page to page: the output is then scaled, as for a maximum that grows.
//  - The queries' sums over groups, which the keys' least values multiply, are two bf16 each: 2^-17.
//
// Bound by HBM and by the warps at once: a page is 933 instructions with one tile of 8 rows, 320 of
// them the shifts and masks, and 1519 with two and biases.
// Measured (CUDA graph), 4 rows: 64 ragged requests x 8 heads of up to 8192 tokens 80 us, 5.8 TB/s (copies alone 74); one
// of 131,072 tokens 35 us, 4.4 TB/s.  16 rows 130 us, of which HBM needs 69; 12 with biases, 64 x 8 x 1641: 48 us.
#include "pages.cuh"
#include "tc.cuh"

namespace arckv {
namespace {

constexpr int kRowsMax = 32;                 // rows of a request and head in this kernel
constexpr int kRowO = 132;                   // floats of an output row in shared memory (four: rows in other banks)
constexpr float kGrow = 8.f, kLift = 7.f;    // weights reach 2^15: the range of f16

constexpr int kWarpsMost = 11;               // consumer warps of a CTA
constexpr int kKnown = 256;                  // requests whose rows and lengths every CTA keeps in shared memory
constexpr int kTileSlot = 9 * 32 * 4;        // floats of a tile's partial result in registers' order: 32 outputs a lane, two (m, l)

struct RowsShape {
  int G, N, limit, max_count;   // limit: rows of a head that a request may have here
  bool causal;
};

// Rows of a tile are eight.  With one tile, ten or eleven consumer warps and a producer, three to each quarter of the SM: up to
// 12 warps may have 168 registers each, and shared memory is full.  (With 8, 9 and 10 consumers, 250 requests of up to 1000
// tokens: 57.5, 57.6 and 55.5 us, 54 with 11.)  With two tiles seven, which may have 255 each: a warp unpacks for both (two warps a
// page, a tile each, ten in all: 135 us instead of 126 for 16 rows, 64 x 8K; ten that unpack for both and spill: 131).
template <int kR, bool kBias>
struct RowsCfg {
  static constexpr int kW = kR == 16 ? 7 : kBias ? 10 : kWarpsMost, kThreads = 32 * (kW + 1);
  static constexpr int kTiles = kR / 8;
  static constexpr int kOwn = kTiles == 1 ? 2 : 3, kSt = kW * kOwn;   // stages of a warp, and of the ring
  static constexpr int kSmem = kSt * (ARCKV_PAGE_BYTES + (kBias ? kPT * 4 : 0));
  static_assert(kR * kRowO * 4 <= ARCKV_PAGE_BYTES, "a warp's part of an item fits a stage");
  static_assert(sizeof(DevStatus) + kCacheMaxCtas * kW * 2 <= ARCKV_CACHE_WS_HEADER && kW <= kWarpsMost, "a ticket for each warp");
  // the rest of it beside 4097 sums, what kKnown requests are, and 2 KB of fixed arrays
  static_assert(kSmem + 4097 * 4 + kKnown * 12 + 2048 <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Sums that begin at zero.
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// bf16 operands: the same word for both halves of a row's elements.
__device__ __forceinline__ void mma_bf16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %4, %5}, {%6, %7}, {%8, %8, %8, %8};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(b0), "r"(b1), "f"(0.f));
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
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *(const uint32_t*)&h;
}
// Two codes as f16: a nibble c is the number c 2^-24 by itself, c 2^-20 four bits up.
__device__ __forceinline__ uint32_t pair_low(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t pair_high(uint32_t w) { return w & 0x00f000f0u; }
// Whether the phase of `parity` has ended, without waiting.
__device__ __forceinline__ bool mbar_ended(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(ok)
      : "r"(tc::smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void bar_consumers(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// A run of pages of one item.
struct Run {
  int s, h, part;         // part: kR rows of the request's
  int blk, n;             // pages blk .. blk + n - 1 of the request
  int first, last;        // the takers that share the item
};

// The runs of a taker, in order: a CTA, which has one part of an item, or a warp, which has a share of all pages.
// Items are numbered over requests, heads, then kR rows at a time; pre[s] are the pages (or parts) of one head before request s,
// times as often as its rows want.
template <int kR>
struct Walk {
  const arckv_pages4& c;
  const int* pre;
  const int* known;       // [kKnown] first row, rows, tokens
  const int* starts;
  int G, N;
  bool parts;             // items are cut into equal parts
  int id;                 // of the taker
  int u, u1;              // parts: this CTA's part of all; else units (pages) of its share
  int q, r;               // shares: q units each, one more for the first r takers

  __device__ Walk(const arckv_pages4& c, const int* pre, const int* known, const int* starts, int G, int N, bool parts,
                  int id, int takers)
      : c(c), pre(pre), known(known), starts(starts), G(G), N(N), parts(parts), id(id) {
    const int total = pre[c.S] * c.H;
    // a page a taker, or shares of two at least (64 x 300 tokens: 13.5 us, 14.6 with shares of one and two)
    const int n = max(1, total <= takers ? total : min(takers, total - total / 2));
    q = total / n;
    r = total - q * n;
    u = id < n ? q * id + min(id, r) : total;
    u1 = id < n ? q * (id + 1) + min(id + 1, r) : total;
  }
  __device__ int owner(int unit) const {
    const int big = r * (q + 1);
    return unit < big ? unit / (q + 1) : r + (unit - big) / q;
  }
  __device__ bool next(Run& p) {
    if (u >= u1) return false;
    int lo = 0, hi = c.S;   // last s with pre[s] H <= u: the one with unit u, as those without rows have none
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] * c.H <= u) lo = mid;
      else hi = mid;
    }
    p.s = lo;
    const int span = pre[lo + 1] - pre[lo], rest = u - pre[lo] * c.H;
    p.h = rest / span;
    int cut = span, k = rest - p.h * span;
    p.part = 0;
    if (kR > 8) {
      const int first = lo < kKnown ? 0 : min(max(starts[lo], 0), N);
      const int rows = (lo < kKnown ? known[3 * lo + 1] : min(max(starts[lo + 1], first), N) - first) * G;
      if (rows > kR) {
        cut = span / ((rows + kR - 1) / kR);
        p.part = k / cut;
        k -= p.part * cut;
      }
    }
    if (parts) {
      const int nb = max(1, pages_of(p.s < kKnown ? known[3 * p.s + 2] : pages_len(c, p.s)));
      p.blk = (int)((long long)nb * k / cut);
      p.n = (int)((long long)nb * (k + 1) / cut) - p.blk;
      p.first = u - k;
      p.last = p.first + cut - 1;
      ++u;
      return true;
    }
    p.blk = k;
    p.n = min(cut - k, u1 - u);
    p.first = p.last = id;
    if (p.n < cut) {
      p.first = owner(u - k);
      p.last = owner(u - k + cut - 1);
    }
    u += p.n;
    return true;
  }
};

template <int kR, bool kBias>
__global__ void __launch_bounds__(RowsCfg<kR, kBias>::kThreads, 1)
    pages_rows_kernel(const arckv_pages4 c, RowsShape d, const bf16* Q, PackedStrides qs, float scale, const int* starts, bf16* O,
                      PackedStrides os, float* parts, int* tickets, DevStatus* stt) {
  using Cfg = RowsCfg<kR, kBias>;
  // Fewest pages that are worth a CTA of their own (joining parts takes over 1 us).
  constexpr int kPartMin = 6;
  constexpr int kW = Cfg::kW, kSt = Cfg::kSt;
  extern __shared__ __align__(128) unsigned char smraw[];
  unsigned char* ring = smraw;                                   // [stage][page]
  float* sBias = (float*)(ring + kSt * ARCKV_PAGE_BYTES);        // [stage][64]
  int* known = (int*)(sBias + (kBias ? kSt * kPT : 0));          // [kKnown] first row, rows, tokens of a request
  int* pre = known + 3 * min(c.S, kKnown);                       // [S + 1]
  __shared__ __align__(8) uint64_t full[kSt], empty[kSt];
  __shared__ int sHeld[kSt];                                     // whether the stage has a page
  __shared__ float sM[kW][kR], sL[kW][kR];
  __shared__ int abort_flag, last_flag, stop_flag, s_cut;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile int* abortp = &abort_flag;

  if (tid == 0) {
    for (int s = 0; s < kSt; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    abort_flag = 0;
    tc::mbar_fence_init();
  }
  pdl_trigger();
  pdl_wait();
  // First row, number of rows and tokens of request s, from memory; no rows where it has more than the launch was made for.
  auto look_up = [&](int s, int& first, int& n, int& len) {
    const int a = starts[s], b = starts[s + 1], l = c.len[s];
    first = min(max(a, 0), d.N);
    n = min(max(b, first), d.N) - first;
    len = min(max(l, 0), c.M * kPT);
    if (n > d.max_count) set_status(stt, ARCKV_ERR_SHAPE);
    if ((long long)n * d.G > d.limit) n = 0;
  };
  if (warp == kW) {   // pages, or parts, before each request, by warp scan
    int cut = 0, items = 0;
    auto scan = [&] {
      int run = 0;
      for (int s0 = 0; s0 < c.S; s0 += 32) {
        const int s = s0 + lane;
        int x = 0, rows = 0;
        if (s < c.S) {
          int first, n, len;
          if (cut > 0 && s < kKnown) {
            n = known[3 * s + 1];
            len = known[3 * s + 2];
          } else {
            look_up(s, first, n, len);
          }
          if (cut == 0 && s < kKnown) {
            known[3 * s] = first;
            known[3 * s + 1] = n;
            known[3 * s + 2] = len;
          }
          if (n > 0) x = max(1, pages_of(len));
          rows = n;
        }
        const int times = x > 0 ? (rows * d.G + kR - 1) / kR : 0;
        if (cut == 0) items += __reduce_add_sync(0xffffffffu, times);
        if (cut > 0 && x > 0) x = max(1, min((x + cut - 1) / cut, x / kPartMin));
        x *= times;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (s0 + lane < c.S) pre[s0 + lane + 1] = run + x;
        run += __shfl_sync(0xffffffffu, x, 31);
      }
      return run;
    };
    int all = scan();
    if (all > 0 && items * c.H <= (int)gridDim.x) {   // the smallest parts that the CTAs suffice for
      cut = (all * c.H + (int)gridDim.x - 1) / (int)gridDim.x;
      for (all = scan(); all * c.H > (int)gridDim.x; all = scan())
        cut = max(cut + 1, (int)((long long)cut * all * c.H / (int)gridDim.x));
    }
    if (lane == 0) {
      pre[0] = 0;
      s_cut = cut;
    }
  }
  __syncthreads();
  auto request = [&](int s, int& first, int& n, int& len) {
    if (s >= kKnown) return look_up(s, first, n, len);
    first = known[3 * s];
    n = known[3 * s + 1];
    len = known[3 * s + 2];
  };
  const bool parts_mode = s_cut > 0;
  // Warps of the launch are numbered over CTAs first, so that few of them are spread over the SMs.
  auto walk_of = [&](int w) {
    return Walk<kR>(c, pre, known, starts, d.G, d.N, parts_mode, parts_mode ? (int)blockIdx.x : w * (int)gridDim.x + (int)blockIdx.x,
                (int)gridDim.x * (parts_mode ? 1 : kW));
  };

  if (warp == kW) {
    // ------------------------------------------------------------- producer
    // Lane w fills the stages of warp w as that gives them back, each lane at its own pace (in one order for all, the
    // slowest warp held up the others' pages: 104 us instead of 97 for 64 x 8K).
    const bool feeds = lane < kW;
    constexpr int kOwn = Cfg::kOwn;
    Walk<kR> walk = walk_of(min(lane, kW - 1));
    Run p;
    int i = 0, issued = 0, entry = -1, held = 0;
    const int step = parts_mode ? kW : 1;   // the warps of a CTA with a part take its pages in turn
    auto begin = [&] {
      if (!walk.next(p)) return false;
      int first, n, len;
      request(p.s, first, n, len);
      held = pages_of(len);
      return true;
    };
    bool left = feeds && begin();
    auto settle = [&] {   // from page i on, the next one of this lane's warp
      while (left && i >= p.n) {
        left = begin();
        i = 0;
      }
      // the table's entry, on its way while the page before it is waited for
      if (left) entry = p.blk + i < held ? c.table[(long long)p.s * c.M + p.blk + i] : -1;
    };
    if (parts_mode) i = lane;
    settle();
    unsigned long long since = tc::globaltimer();
    uint32_t spins = 0;
    while (__any_sync(0xffffffffu, left)) {
      bool moved = false;
      if (left) {
        const int st = lane + kW * (issued % kOwn);
        if (issued < kOwn || mbar_ended(&empty[st], (issued / kOwn - 1) & 1)) {
          if (entry >= c.P) {
            set_status(stt, ARCKV_ERR_INVALID_ARG);
            entry = -1;
          }
          sHeld[st] = entry >= 0;
          if (entry >= 0) {
            const long long at = (long long)entry * c.H + p.h;
            tc::mbar_arrive_expect_tx(&full[st], ARCKV_PAGE_BYTES + (kBias ? kPT * 4 : 0));
            tc::bulk_load(ring + st * ARCKV_PAGE_BYTES, c.data + at * ARCKV_PAGE_BYTES, ARCKV_PAGE_BYTES, &full[st]);
            if (kBias) tc::bulk_load(sBias + st * kPT, c.bias + at * kPT, kPT * 4, &full[st]);
          } else {
            tc::mbar_arrive(&full[st]);
          }
          moved = true;
          ++issued;
          i += step;
          settle();
        }
      }
      if (__any_sync(0xffffffffu, moved)) {
        since = tc::globaltimer();
      } else if ((++spins & 63u) == 0) {
        bool stop = *abortp != 0;
        if (!stop && tc::globaltimer() - since > tc::kWaitLimitNs) {
          *abortp = 1;
          set_status(stt, ARCKV_ERR_TIMEOUT);
          stop = true;
        }
        if (__any_sync(0xffffffffu, stop)) break;
      }
    }
    if (*abortp) {   // let the copies in flight land before the CTA's memory goes: a barrier's last phase is complete, or will be
      volatile int never = 0;
      if (feeds)   // (the n-th page of a stage completes its phase n - 1)
        for (int k = 0; k < kOwn; ++k) {
          const int n = (issued + kOwn - 1 - k) / kOwn;   // pages that stage k of this warp's got
          if (n > 0) tc::mbar_wait(&full[lane + k * kW], (n - 1) & 1, &never, stt);
        }
    }
    return;
  }

  // --------------------------------------------------------------- consumers
  const int g = lane >> 2, t = lane & 3;
  constexpr int kT = Cfg::kTiles, kMt = 4 / kT;   // tiles, and 16s of tokens of a pass
  const int step = parts_mode ? kW : 1;
  Walk<kR> walk = walk_of(warp);
  int taken = 0;                 // pages so far
  bool ok = true;
  Run p;
  while (ok && walk.next(p)) {
    int first, count, len;
    request(p.s, first, count, len);
    const int n = p.n, h = p.h, row0 = kR * p.part, nrows = min(kR, count * d.G - row0);
    // query rows: column n is row n of the tile
    uint32_t qf[kT][8][2];
    // what a token's least values multiply beside the codes' sums: the sum of a group's elements as two bf16, row g, group t, and
    // zeros for the scales that are in the same words
    uint32_t q_sum[kT][2];
    float fac[kT][2];                     // 2^e scale (log2 e) of rows 2t, 2t + 1
    int see[kT][2], see_min = 0x7fffffff; // tokens that they see
#pragma unroll
    for (int tt = 0; tt < kT; ++tt) {
      const int r = 8 * tt + g, i = (row0 + r) / d.G;
      const bf16* mine = Q + (first + i) * qs.i + h * qs.h + (row0 + r - i * d.G) * 128;
      uint4 x[4];
      float amax = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        x[w] = make_uint4(0u, 0u, 0u, 0u);
        if (r < nrows) x[w] = *(const uint4*)(mine + 32 * w + 8 * t);
        const uint32_t y[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
#pragma unroll
        for (int f = 0; f < 4; ++f) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(y[f])), fabsf(bf16_hi(y[f]))));
      }
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // exponent of the row's largest element, kept where 2^(14 - ex) and 2^(ex - 14) are normal
      const int ex = min(max((int)((__float_as_uint(amax) >> 23) & 0xff) - 127, -100), 127);
      const float up = __uint_as_float((unsigned)(14 - ex + 127) << 23), down = __uint_as_float((unsigned)(ex - 14 + 127) << 23);
      float sum[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
        sum[w] = 0.f;
#pragma unroll
        for (int f = 0; f < 4; ++f) {   // pair f of the word: dims 32 w + 8 t + 2 f, + 1
          const float by = f & 1 ? up * 0.0625f : up;   // (its codes are 16 times the others')
          qf[tt][2 * w + (f >> 1)][f & 1] = pack_f16(bf16_lo(y[f]) * by, bf16_hi(y[f]) * by);
          sum[w] += bf16_lo(y[f]) * up + bf16_hi(y[f]) * up;
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], o);
      }
      {   // in units of a code, which is 2^-24
        bf16 a, b;
        split_bf16((t == 0 ? sum[0] : t == 1 ? sum[1] : t == 2 ? sum[2] : sum[3]) * 0x1p-24f, a, b);
        q_sum[tt][0] = (uint32_t)__bfloat16_as_ushort(a) << 16;
        q_sum[tt][1] = (uint32_t)__bfloat16_as_ushort(b) << 16;
      }
      const float f = down * 0x1p24f * scale * (kBias ? 1.f : kLog2e);
      const int sees = r < nrows ? (d.causal ? max(0, min(len, len - count + i + 1)) : len) : 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) {   // (a factor is never zero: a masked product is -inf)
        fac[tt][k] = fmaxf(__shfl_sync(0xffffffffu, f, (2 * t + k) * 4), 0x1p-126f);
        see[tt][k] = __shfl_sync(0xffffffffu, sees, (2 * t + k) * 4);
      }
      see_min = min(see_min, (int)__reduce_min_sync(0xffffffffu, r < nrows ? sees : 0x7fffffff));
    }
    float o[kT][8][4], mx[kT][2], l[kT][2], low[kT][2];   // low: sums of weights times least values
    float v_ref = 0.f;                         // unit of o: a power of two
#pragma unroll
    for (int tt = 0; tt < kT; ++tt) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int f = 0; f < 4; ++f) o[tt][k][f] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        mx[tt][k] = -INFINITY;
        l[tt][k] = low[tt][k] = 0.f;
      }
    }
    for (int i = parts_mode ? warp : 0; i < n && ok; i += step, ++taken) {
      const int st = warp + kW * (taken % Cfg::kOwn);
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[st], (taken / Cfg::kOwn) & 1, abortp, stt));
      if (!ok) break;
      if (sHeld[st]) {
        // with two tiles a page is taken in two passes of 32 tokens, as far as registers go
#pragma unroll 1
        for (int pass = 0; pass < kT; ++pass) {
          const unsigned char* page = ring + st * ARCKV_PAGE_BYTES;
          const int m0 = pass * kMt, j0 = (p.blk + i) * kPT + 16 * m0;   // first token of the pass
          // ---- S^T = K Q^T: lane (g, t) has tokens g, g + 8 of 16, and eight dims of each group
          float s[kT][kMt][4];
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt) {
            const int row = (m0 + mt) * 16 + g;
            const uint4 a = *(const uint4*)(page + row * 64 + t * 16);
            const uint4 b = *(const uint4*)(page + (row + 8) * 64 + t * 16);
            const uint4 pa = *(const uint4*)(page + kPageKp + row * 16);
            const uint4 pb = *(const uint4*)(page + kPageKp + (row + 8) * 16);
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
            const uint32_t pw[4] = {pa.x, pa.y, pa.z, pa.w}, pv[4] = {pb.x, pb.y, pb.z, pb.w};
            {   // here lane (g, t) has scale and least value of group t of its tokens
              const uint32_t ma = *(const uint32_t*)(page + kPageKp + row * 16 + 4 * t);
              const uint32_t mb = *(const uint32_t*)(page + kPageKp + (row + 8) * 16 + 4 * t);
#pragma unroll
              for (int tt = 0; tt < kT; ++tt) mma_bf16_zero(s[tt][mt], ma, mb, q_sum[tt][0], q_sum[tt][1]);
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t a8 = aw[w] >> 8, b8 = bw[w] >> 8;
              const uint32_t f0 = pair_low(aw[w]), f1 = pair_low(bw[w]), f2 = pair_high(aw[w]), f3 = pair_high(bw[w]);
              const uint32_t f4 = pair_low(a8), f5 = pair_low(b8), f6 = pair_high(a8), f7 = pair_high(b8);
#pragma unroll
              for (int tt = 0; tt < kT; ++tt) {
                float acc[4];
                mma_f16_zero(acc, f0, f1, f2, f3, qf[tt][2 * w][0], qf[tt][2 * w][1]);
                mma_f16(acc, f4, f5, f6, f7, qf[tt][2 * w + 1][0], qf[tt][2 * w + 1][1]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  s[tt][mt][k] = fmaf(bf16_lo(pw[w]), acc[k], s[tt][mt][k]);
                  s[tt][mt][2 + k] = fmaf(bf16_lo(pv[w]), acc[2 + k], s[tt][mt][2 + k]);
                }
              }
            }
          }
          // ---- softmax of the pass.  References follow the maximum only when it has grown by more than 2^8 (kGrow), so
          // that sums are scaled on few pages.  Without biases the maximum is that of the products, whose factor is
          // positive, and a weight is 2^{product factor - mx}.
          if (kBias) {
#pragma unroll
            for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const float bias = sBias[st * kPT + (m0 + mt) * 16 + hf * 8 + g];
#pragma unroll
                for (int tt = 0; tt < kT; ++tt)
#pragma unroll
                  for (int k = 0; k < 2; ++k) s[tt][mt][2 * hf + k] = fmaf(s[tt][mt][2 * hf + k], fac[tt][k], bias);
              }
          }
          if (j0 + 16 * kMt > see_min) {   // (also where no row has been: anything may be there)
#pragma unroll
            for (int tt = 0; tt < kT; ++tt)
#pragma unroll
              for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
                for (int f = 0; f < 4; ++f)
                  if (j0 + mt * 16 + (f >> 1) * 8 + g >= see[tt][f & 1]) s[tt][mt][f] = -INFINITY;
          }
          float top[kT][2];
          bool grows = false;
#pragma unroll
          for (int tt = 0; tt < kT; ++tt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {   // rows 2t, 2t + 1
              float& x = top[tt][k];
              x = fmaxf(s[tt][0][k], s[tt][0][2 + k]);
#pragma unroll
              for (int mt = 1; mt < kMt; ++mt) x = max3(x, s[tt][mt][k], s[tt][mt][2 + k]);
              if (!kBias) x = fmaf(x, fac[tt][k], -kLift);
              grows |= (kBias ? (x - mx[tt][k]) * kLog2e : x - mx[tt][k]) > kGrow;   // (mx = -inf: by any but -inf)
            }
          if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int tt = 0; tt < kT; ++tt) {
              float alpha[2];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                float& x = top[tt][k];
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
                const float by = kBias ? (mx[tt][k] - x) * kLog2e : mx[tt][k] - x;
                const bool up = x != -INFINITY && (mx[tt][k] == -INFINITY || -by > kGrow);
                alpha[k] = up ? ex2_approx(by) : 1.f;   // (mx = -inf: zero)
                if (up) mx[tt][k] = x;
                l[tt][k] *= alpha[k];
                low[tt][k] *= alpha[k];
              }
#pragma unroll
              for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int f = 0; f < 4; ++f) o[tt][k][f] *= alpha[f & 1];
            }
          }
          // the values' scales and least values; of tokens that are not held, zero
          float vs[2 * kMt], vm[2 * kMt], most = 0.f;
          {
            uint32_t par[2 * kMt];
#pragma unroll
            for (int x = 0; x < 2 * kMt; ++x) par[x] = *(const uint32_t*)(page + kPageVp + (16 * m0 + x * 8 + g) * 4);
            if (j0 + 16 * kMt > len) {
#pragma unroll
              for (int x = 0; x < 2 * kMt; ++x)
                if (j0 + x * 8 + g >= len) par[x] = 0u;
            }
#pragma unroll
            for (int x = 0; x < 2 * kMt; ++x) {
              vs[x] = bf16_lo(par[x]);
              vm[x] = bf16_hi(par[x]);
            }
#pragma unroll
            for (int x = 0; x < 2 * kMt; x += 2) most = max3(most, vs[x], vs[x + 1]);
          }
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, w));
          // (uniform) another unit: between two and four times the scale, so that few pages raise it, and again where a page needs less
          // than 2^-8 of it (one that only grew lost the pages behind larger values, whether or not those had weight).  Sums have
          // fp32's range, which it leaves below 2^-30: down from there it does not follow.
          if (most > v_ref || (most < v_ref * 0x1p-8f && most > 0.f && v_ref > 0x1p-30f)) {
            float to = __uint_as_float((__float_as_uint(most) & 0x7f800000u) + (2u << 23));
            if (most < v_ref) to = fmaxf(to, 0x1p-30f);
            const float by = v_ref / to;
#pragma unroll
            for (int tt = 0; tt < kT; ++tt)
#pragma unroll
              for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int f = 0; f < 4; ++f) o[tt][k][f] *= by;
            v_ref = to;
          }
          const float inv_ref = v_ref > 0.f ? 1.f / v_ref : 0.f;
          // v = s (c - z) + (m + s z): with z = -m / s, the code of zero as far as there is one, the rest is zero where the row has
          // both signs.  The rounded weights multiply c and z, so that their rounding costs what it is of v, however far the row
          // reaches; the rest has the weight as it was.  (With the whole of m in the rest, one channel of 64 times the others' size cost the
          // others up to 1.3e-2 of their outputs, 2e-3 now; 16 rows, 64 x 8K, took 124 us, 130 now.)
          float vz[2 * kMt];   // -z in units of o
          const float2 unit2 = make_float2(inv_ref, inv_ref), most_z = make_float2(-15.f * v_ref, -15.f * v_ref);
#pragma unroll
          for (int x = 0; x < 2 * kMt; x += 2) {
            const float2 s2 = make_float2(vs[x], vs[x + 1]), s15 = mul2(s2, make_float2(15.f, 15.f));
            const float2 t2 = make_float2(__saturatef(-vm[x] * rcp_approx(s15.x)), __saturatef(-vm[x + 1] * rcp_approx(s15.y)));
            const float2 rest = fma2(s15, t2, make_float2(vm[x], vm[x + 1])), z2 = mul2(t2, most_z), u2 = mul2(s2, unit2);
            vm[x] = rest.x, vm[x + 1] = rest.y;
            vz[x] = z2.x, vz[x + 1] = z2.y;
            vs[x] = u2.x, vs[x + 1] = u2.y;
          }
          uint32_t ph[kT][kMt][2];
#pragma unroll
          for (int tt = 0; tt < kT; ++tt) {
            // (nothing visible yet: weights 2^{-inf} = 0)
            const float2 ref = make_float2(mx[tt][0] == -INFINITY ? 0.f : -mx[tt][0], mx[tt][1] == -INFINITY ? 0.f : -mx[tt][1]);
            const float2 fac2 = make_float2(fac[tt][0], fac[tt][1]);
            float2 sum = make_float2(0.f, 0.f), lows = make_float2(low[tt][0], low[tt][1]);
#pragma unroll
            for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                float2 x = make_float2(s[tt][mt][2 * hf], s[tt][mt][2 * hf + 1]);
                // a bias of the type's lowest value cancels against itself before the factor log2 e
                if (kBias) x = fma2(add2(x, ref), make_float2(kLog2e, kLog2e), make_float2(kLift, kLift));
                else x = fma2(x, fac2, ref);
                x.x = ex2_approx(x.x);
                x.y = ex2_approx(x.y);
                sum = add2(sum, x);
                lows = fma2(x, make_float2(vm[2 * mt + hf], vm[2 * mt + hf]), lows);
                x = mul2(x, make_float2(vs[2 * mt + hf], vs[2 * mt + hf]));
                const __half2 p = __floats2half2_rn(x.x, x.y);
                lows = fma2(__half22float2(p), make_float2(vz[2 * mt + hf], vz[2 * mt + hf]), lows);
                ph[tt][mt][hf] = transpose8x8(*(const uint32_t*)&p);   // as f16, transposed to (tokens, row) operands
              }
            l[tt][0] += sum.x;
            l[tt][1] += sum.y;
            low[tt][0] = lows.x;
            low[tt][1] = lows.y;
          }
          // ---- O^T += V^T P^T, 16 dims and 16 tokens a product: lane (g, t) has tokens 2t, 2t + 1 and 8 on, dims g + 8 x
#pragma unroll
          for (int mt = 0; mt < kMt; ++mt) {
            const unsigned char* pairs = page + kPageV + ((m0 + mt) * 8 + t) * 128 + ((g ^ (t << 1)) << 4);
            const uint4 a = *(const uint4*)pairs;
            const uint4 b = *(const uint4*)(pairs + 4 * 128);
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t a8 = aw[x] >> 8, b8 = bw[x] >> 8;
              const uint32_t f0 = pair_low(aw[x]), f1 = pair_high(aw[x]), f2 = pair_low(bw[x]), f3 = pair_high(bw[x]);
              const uint32_t f4 = pair_low(a8), f5 = pair_high(a8), f6 = pair_low(b8), f7 = pair_high(b8);
#pragma unroll
              for (int tt = 0; tt < kT; ++tt) {
                mma_f16(o[tt][2 * x], f0, f1, f2, f3, ph[tt][mt][0], ph[tt][mt][1]);
                mma_f16(o[tt][2 * x + 1], f4, f5, f6, f7, ph[tt][mt][0], ph[tt][mt][1]);
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&empty[st]);
    }
    // ---- the run's end
    if (!kBias) {   // (a product is exact in its difference from the reference, which is rounded: by half of a power of two at most up to here)
      float most = 0.f;
#pragma unroll
      for (int tt = 0; tt < kT; ++tt)
#pragma unroll
        for (int k = 0; k < 2; ++k) most = fmaxf(most, mx[tt][k] == -INFINITY ? 0.f : fabsf(mx[tt][k]));
      if (most > kLogitMost) set_status(stt, ARCKV_ERR_NONFINITE);
    }
#pragma unroll
    for (int tt = 0; tt < kT; ++tt) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          l[tt][k] += __shfl_xor_sync(0xffffffffu, l[tt][k], w);
          low[tt][k] += __shfl_xor_sync(0xffffffffu, low[tt][k], w);
        }
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int f = 0; f < 4; ++f)   // dims 16 x + g are of low nibbles, those 8 on of high ones
          o[tt][x][f] = fmaf(o[tt][x][f] * (f >> 1 ? 0x1p20f : 0x1p24f), v_ref, low[tt][f & 1]);
    }
    const bool whole = p.first == p.last;
    auto weight = [](float m, float top) {   // e^{m - top}; 0 for a part that saw nothing
      return m == -INFINITY ? 0.f : ex2_approx(kBias ? (m - top) * kLog2e : m - top);
    };
    constexpr float kBig = 3.3895313892515355e38f;   // (the largest bf16)
    if (!parts_mode) {   // a share's run: the warp's own affair
      if (!ok) break;    // a wait gave up: write nothing
      if (!whole) {
        // slot 2c holds the item that warp c went on with, 2c + 1 the one it began
        auto slot_of = [&](int w, bool began) { return (float4*)(parts + (2ll * w + began) * kT * kTileSlot) + lane; };
        float4* slot = slot_of(walk.id, p.blk == 0);
#pragma unroll
        for (int tt = 0; tt < kT; ++tt)
          if (8 * tt + 2 * t < nrows) {   // (rows 2t, 2t + 1 of the tile)
#pragma unroll
            for (int x = 0; x < 8; ++x)
              __stcg(slot + (9 * tt + x) * 32, make_float4(o[tt][x][0], o[tt][x][1], o[tt][x][2], o[tt][x][3]));
            __stcg(slot + (9 * tt + 8) * 32, make_float4(mx[tt][0], mx[tt][1], l[tt][0], l[tt][1]));
          }
        __syncwarp();
        int last = 0;
        if (lane == 0) {   // the warp's results before the ticket, the others' after it; tickets are halves of words
          const int shift = 16 * (p.first & 1);
          unsigned int* word = (unsigned int*)tickets + (p.first >> 1);
          unsigned int old;
          asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;" : "=r"(old) : "l"(word), "r"(1u << shift) : "memory");
          last = (int)((old >> shift) & 0xffffu) == p.last - p.first;
          if (last) atomicSub(word, (unsigned int)(p.last - p.first + 1) << shift);
        }
        if (!__shfl_sync(0xffffffffu, last, 0)) continue;
        __syncwarp();
#pragma unroll
        for (int tt = 0; tt < kT; ++tt) {
          if (8 * tt + 2 * t >= nrows) continue;
          float up[2] = {-INFINITY, -INFINITY};   // with a running maximum, so that a part's loads wait for nothing
          l[tt][0] = l[tt][1] = 0.f;
#pragma unroll
          for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int f = 0; f < 4; ++f) o[tt][x][f] = 0.f;
#pragma unroll 1
          for (int cc = p.first; cc <= p.last; ++cc) {
            const float4* from = slot_of(cc, cc == p.first) + 9 * tt * 32;
            float4 y[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) y[x] = __ldcg(from + 32 * x);
            const float4 ml = __ldcg(from + 32 * 8);
            const float m0 = fmaxf(up[0], ml.x), m1 = fmaxf(up[1], ml.y);
            const float f0 = weight(up[0], m0), f1 = weight(up[1], m1), b0 = weight(ml.x, m0), b1 = weight(ml.y, m1);
            up[0] = m0;
            up[1] = m1;
            l[tt][0] = fmaf(l[tt][0], f0, ml.z * b0);
            l[tt][1] = fmaf(l[tt][1], f1, ml.w * b1);
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              o[tt][x][0] = fmaf(o[tt][x][0], f0, y[x].x * b0);
              o[tt][x][1] = fmaf(o[tt][x][1], f1, y[x].y * b1);
              o[tt][x][2] = fmaf(o[tt][x][2], f0, y[x].z * b0);
              o[tt][x][3] = fmaf(o[tt][x][3], f1, y[x].w * b1);
            }
          }
        }
      }
#pragma unroll
      for (int tt = 0; tt < kT; ++tt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = 8 * tt + 2 * t + k;
          if (r >= nrows) continue;   // (a tile without rows masks nothing: it may have met anything behind the end)
          const int i = (row0 + r) / d.G;
          bf16* to = O + (first + i) * os.i + h * os.h + (row0 + r - i * d.G) * 128 + g;
          const float inv = l[tt][k] == 0.f ? 0.f : 1.f / l[tt][k];
          bool fine = true;
#pragma unroll
          for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float v = o[tt][x][2 * z + k] * inv;
              to[16 * x + 8 * z] = __float2bfloat16_rn(v);
              fine &= fabsf(v) <= kBig;
            }
          if (!fine) set_status(stt, ARCKV_ERR_NONFINITE);
        }
      continue;
    }
    // a part of an item: add the CTA's warps up.  A warp's part lies where its pages were, all of which it has taken
    auto out_of = [&](int w, int r) { return (float*)(ring + w * ARCKV_PAGE_BYTES) + r * kRowO; };
    __syncwarp();
#pragma unroll
    for (int tt = 0; tt < kT; ++tt)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = 8 * tt + 2 * t + k;
        if (g == 0) {
          sM[warp][r] = mx[tt][k];
          sL[warp][r] = l[tt][k];
        }
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int z = 0; z < 2; ++z) out_of(warp, r)[16 * x + 8 * z + g] = o[tt][x][2 * z + k];
      }
    if (tid == 0) stop_flag = *abortp;   // one reading for all: the producer may raise the flag at any time
    bar_consumers(kW * 32);
    if (stop_flag) break;   // a wait gave up: write nothing
    auto store = [&](int r, int dim, float4 v, float z) {
      const float inv = z == 0.f ? 0.f : 1.f / z;
      v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      if (r >= nrows) return;
      const int i = (row0 + r) / d.G;
      __nv_bfloat162 y[2] = {__floats2bfloat162_rn(v.x, v.y), __floats2bfloat162_rn(v.z, v.w)};
      *(uint2*)(O + (first + i) * os.i + h * os.h + (row0 + r - i * d.G) * 128 + dim) = *(const uint2*)&y[0];
      if (!(fabsf(v.x) <= kBig && fabsf(v.y) <= kBig && fabsf(v.z) <= kBig && fabsf(v.w) <= kBig))
        set_status(stt, ARCKV_ERR_NONFINITE);
    };
    // partial results: slot 2c holds the item that CTA c went on with, 2c + 1 the one it began
    constexpr int kSlot = kR * 132;   // 128 outputs, m, l (and two unused) for each row
    for (int x = tid; x < kR * 32; x += kW * 32) {
      const int r = x >> 5, dim = (x & 31) * 4;
      float up = -INFINITY, z = 0.f;
#pragma unroll
      for (int w = 0; w < kW; ++w)
        if (w < n) up = fmaxf(up, sM[w][r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        if (w >= n) break;   // (these warps had no page)
        const float f = weight(sM[w][r], up);
        const float4 y = *(const float4*)(out_of(w, r) + dim);
        z = fmaf(sL[w][r], f, z);
        v = make_float4(fmaf(y.x, f, v.x), fmaf(y.y, f, v.y), fmaf(y.z, f, v.z), fmaf(y.w, f, v.w));
      }
      if (whole) store(r, dim, v, z);
      else {
        float* slot = parts + (2ll * blockIdx.x + (p.blk == 0 ? 1 : 0)) * kSlot + r * 132;
        __stcg((float4*)(slot + dim), v);
        if (dim == 0) __stcg((float2*)(slot + 128), make_float2(up, z));
      }
    }
    if (!whole) {
      bar_consumers(kW * 32);
      if (tid == 0) {
        // the CTA's results before the ticket, the others' after it
        int ticket;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(ticket) : "l"(&tickets[p.first]) : "memory");
        last_flag = ticket == p.last - p.first;
        if (last_flag) tickets[p.first] = 0;
      }
      bar_consumers(kW * 32);
      if (last_flag) {
        for (int x = tid; x < kR * 32; x += kW * 32) {
          const int r = x >> 5, dim = (x & 31) * 4;
          // with a running maximum, so that a part's loads wait for nothing
          float up0 = -INFINITY, z = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int cc = p.first; cc <= p.last; ++cc) {
            const float* slot = parts + (2ll * cc + (cc == p.first)) * kSlot + r * 132;
            const float2 ml = __ldcg((const float2*)(slot + 128));
            const float4 y = __ldcg((const float4*)(slot + dim));
            const float up = fmaxf(up0, ml.x), f = weight(ml.x, up), f0 = weight(up0, up);
            up0 = up;
            z = fmaf(z, f0, ml.y * f);
            v = make_float4(fmaf(v.x, f0, y.x * f), fmaf(v.y, f0, y.y * f), fmaf(v.z, f0, y.z * f), fmaf(v.w, f0, y.w * f));
          }
          store(r, dim, v, z);
        }
      }
    }
    break;   // (the only one)
  }
}

template <int kR, bool kBias>
int launch_rows(const arckv_pages4& p, const PagesQuery& q, float scale, int limit, void* ws, cudaStream_t st) {
  RowsShape d;
  d.G = q.G;
  d.N = q.N;
  d.limit = limit;
  d.max_count = q.max_count;
  d.causal = q.causal;
  auto kern = pages_rows_kernel<kR, kBias>;
  const int smem = RowsCfg<kR, kBias>::kSmem + (3 * std::min(p.S, kKnown) + p.S + 1) * (int)sizeof(int);
  if (set_dyn_smem((const void*)kern, smem) != cudaSuccess) return -1;
  const int ctas = std::min(tc_gemm_sm_count(), kCacheMaxCtas);
  const cudaError_t e = launch_pdl(kern, dim3(ctas), RowsCfg<kR, kBias>::kThreads, smem, st, p, d, q.Q, q.qs, scale, q.starts, q.O, q.os,
                                   (float*)((char*)ws + ARCKV_CACHE_WS_HEADER), ws_tickets(ws), (DevStatus*)ws);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace

// Whether requests of so many rows of a head are all for pages_rows_kernel.  Up to 32: its items are 16 rows, whose pages' second
// reading L2 serves, and a change of items costs it next to nothing (32 rows, 250 x 8 x up to 500: 122 us, where the kernel for many
// rows takes 202; 20 rows, 64 x 8 x up to 8192: 241 and 277; 32 over one request of 300: 9.2 and 14.3), while their units are numbers of 31 bits.
static bool few_rows(int S, int H, int M, long long rows) {
  return rows <= 16 || (rows <= kRowsMax && (long long)S * H * M < (1LL << 30));
}

size_t pages_attend_scratch(int S, int H, int M, int max_count, int G) {
  // partial results of CTAs, or of the warps of each: of 7 warps with two tiles, or 11 with one.  A workspace serves calls of fewer
  // rows too, so the size never falls as rows become more.
  const long long all = (long long)max_count * G;
  const int slots = all > 8 ? std::max(2 * RowsCfg<16, false>::kW, kWarpsMost) : kWarpsMost;
  const size_t rows = (size_t)2 * kCacheMaxCtas * std::max(16 * 132, slots * kTileSlot) * sizeof(float);
  return few_rows(S, H, M, all) ? rows : std::max(rows, pages_tiles_scratch(all));
}

int launch_pages_attend(const arckv_pages4& p, const PagesQuery& q, float scale, void* ws, cudaStream_t st) {
  const long long rows = (long long)q.max_count * q.G;
  const bool few = few_rows(p.S, p.H, p.M, rows);
  // Beside requests of more rows, those of 9 and more go with them (a mixed batch of one chunk and 16 single tokens: 115 us with
  // 16 rows a request here)
  const int limit = few ? (int)rows : (int)std::min(rows, 8LL);
  const int n = limit <= 8 ? (p.bias ? launch_rows<8, true>(p, q, scale, limit, ws, st) : launch_rows<8, false>(p, q, scale, limit, ws, st))
                           : (p.bias ? launch_rows<16, true>(p, q, scale, limit, ws, st) : launch_rows<16, false>(p, q, scale, limit, ws, st));
  if (n < 0 || few) return n;
  const int more = launch_pages_tiles(p, q, scale, limit, ws, st);
  return more < 0 ? -1 : n + more;
}

}  // namespace arckv
