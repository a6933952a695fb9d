// Attention of few query rows over an 8-bit cache (decode and draft steps, and
// every sparse call):
//
//   O_r = sum_j e^{x_rj} v_j / sum_j e^{x_rj},  x_rj = scale q_r . k_j + bias_j
//
// over all visible tokens j, or over the listed blocks.  256 bytes of codes a
// token and head are read once: the call is bound by HBM, and the work per byte
// has to stay small.  So:
//  - Work is the list of (item, block) pairs, an item being (sequence, KV head,
//    up to 16 query rows[, position]).  With more items than SMs each SM's CTA
//    takes an equal share of it, whatever the lengths; with fewer, items are cut
//    into equal parts, a CTA each, as many as there are SMs for: a CTA then meets
//    one item only.  An item in several CTAs is finished by the one that comes
//    last (a ticket), which adds the parts up in CTA order.
//  - Two producer warps stream the blocks' keys and values (64 x 128 codes, 8 KB
//    each, 128-byte swizzle) through rings in shared memory by TMA.  Each
//    consumer warp takes whole blocks of its own, with its own running maximum,
//    sum and output: no barrier between warps until the item ends.  A warp gives
//    its keys' stage back before the softmax, so that the next block's keys come
//    in while it works on the values, and its values while on those keys.
//  - Products run on mma.sync m16n8k16 with f16 operands: keys (dims for V) are
//    the 16 rows and the query rows the 8 columns, so four to eight rows fill
//    an instruction; tcgen05 would want 64 to 128 rows and a pass of the
//    codes through shared memory as f16.  A code becomes an f16 with one byte permute
//    and one subtraction a pair (1024 + u is 0x6400 | u); codes are exact in f16.
//    So are bf16 queries once each row is scaled by a power of two (elements
//    under 2^-32 of the row's largest lose bits, far below fp32 rounding).
//    Softmax weights, of up to 2^15, enter as f16 pairs hi + lo: 22 bits.  With
//    four rows, hi and lo are columns 0-3 and 4-7 of the same instruction.
//  - S^T and O^T are what the instructions give (keys x rows, dims x rows), so
//    weights go from one product to the other by an 8 x 8 transpose in registers;
//    V's operand comes by transposed loads of 16-bit units, two dims of a key each.
//  - V's scales enter 2^-15 as large (kValues): a token then adds at most its value to O, which overflows only where the
//    values' magnitude times the tokens does.
//
// Measured: 64 ragged sequences x 8 heads, up to 8K, 4 rows: 118 us, 6.6 TB/s (97 % of
// a copy's rate); one of 128K 48 us (5.6 TB/s: 6 us are start and join).  12 rows with
// biases over 64 x 8 x 1641: 65 us, 3.4 TB/s, bound by two warps' dequantising and
// products of a block (44 without arithmetic).  32 listed blocks for each of 128
// positions x 8 heads: 76 us, 7.1 TB/s of codes from L2 (50 us without arithmetic).
#include "cache8.cuh"
#include "tc.cuh"

namespace arckv {
namespace {

// More rows of a head go to the tcgen05 kernel (32 x 8 heads of 8K: 16 rows take 117 us here, 17 there 215).
constexpr int kRowsMax = 16;
constexpr float kValues = 0x1p-15f;          // O's unit: 1 / the largest weight
constexpr int kRowO = 132;                   // floats of an output row in shared memory (four: rows in other banks)

struct RowsShape {
  int H, n_pos, G, nblk, cap;   // nblk: blocks of the capacity
  int groups;                   // sparse: row groups of a position
  int m;                        // blocks listed for an item (sparse)
  bool causal;
};

// Consumer warps: with the two producers at most 12 warps, as registers are dealt out to the SM's quarters (168 a
// thread).  Ten where HBM is the bound; eight for 9 to 16 rows, where the warps' own work is and ten would leave two
// quarters of the SM a third consumer (12 rows over 64 x 8 compact caches of 1641: 73.6 us with ten, 70.5 with eight;
// 64 x 8K decode of 4 rows: 123.9 and 127.2).
// Stages of a ring: one for each consumer warp (two for each pair of warps that share blocks), so that a stage is
// always consumed by the same warps.  A warp that came to a stage while an earlier block of another warp was still on
// its way there would take the phase before that one for its own (a wait sees a phase's parity only).
template <int kR>
struct RowsCfg {
  static constexpr int kW = kR == 16 ? 8 : 10, kSt = kW, kThreads = 32 * (kW + 2);
  static constexpr int kTiles = kR == 16 ? 2 : 1;   // tiles of 8 rows; warps w and w + kW / 2 share blocks, a tile each
  static constexpr int kTeams = kW / kTiles;        // warps, or pairs, that take blocks in turn
  static constexpr int kTileRows = kR < 8 ? kR : 8;
  static constexpr int kSmem = kSt * (2 * kTileBytes + kCB * 4) + kW * kTileRows * kRowO * 4 + 2 * kR * 256 + 1024;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *(const uint32_t*)&h;
}
__device__ __forceinline__ void bar_consumers(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// A CTA's run of blocks (entries of the block list) of one item.
struct Run {
  int s, h, sh;           // sequence, head, both
  int pos, group, list;   // sparse: position, row group, row of the block lists
  int blk, n;             // blocks blk .. blk + n - 1
  int first, last;        // the CTAs that share the item
};

// The runs of a CTA, in order.  Items are numbered over sequences, then heads (sparse: positions, row groups); dense,
// pre[s] are the blocks (or parts) before sequence s of one head.
template <bool kSparse>
struct Walk {
  const RowsShape& d;
  const int* pre;
  int S, cta;
  bool parts;             // items are cut into equal parts
  int u, u1;              // parts: this CTA's part of all; else units (blocks) of its share
  int q, r;               // shares: q units each, one more for the first r CTAs
  int per;                // sparse: parts of an item
  const int* len;

  __device__ int owner(int unit) const {
    const int big = r * (q + 1);
    return unit < big ? unit / (q + 1) : r + (unit - big) / q;
  }
  __device__ int blocks_of(int s) const { return max(1, (min(max(len[s], 0), d.cap) + kCB - 1) / kCB); }
  // last s with pre[s] * H <= x
  __device__ int sequence_of(int x) const {
    int lo = 0, hi = S;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] * d.H <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  }
  __device__ bool next(Run& p) {
    if (u >= u1) return false;
    if (kSparse) {
      const int cut = parts ? per : d.m, item = u / cut, k = u - item * cut;
      p.group = item % d.groups;
      p.list = item / d.groups;
      p.pos = p.list % d.n_pos;
      p.sh = p.list / d.n_pos;
      p.s = p.sh / d.H;
      p.h = p.sh - p.s * d.H;
      if (parts) {
        p.blk = (int)((long long)d.m * k / per);
        p.n = (int)((long long)d.m * (k + 1) / per) - p.blk;
        p.first = item * per;
        p.last = p.first + per - 1;
        ++u;
      } else {
        take(p, k, d.m);
      }
      return true;
    }
    p.s = sequence_of(u);
    const int cut = pre[p.s + 1] - pre[p.s], rest = u - pre[p.s] * d.H;
    p.h = rest / cut;
    p.sh = p.s * d.H + p.h;
    p.pos = p.group = p.list = 0;
    const int k = rest - p.h * cut;
    if (parts) {
      const int nb = blocks_of(p.s);
      p.blk = (int)((long long)nb * k / cut);
      p.n = (int)((long long)nb * (k + 1) / cut) - p.blk;
      p.first = u - k;
      p.last = p.first + cut - 1;
      ++u;
    } else {
      take(p, k, cut);
    }
    return true;
  }
  // block k of an item of `count`, and as many as the share holds
  __device__ void take(Run& p, int k, int count) {
    p.blk = k;
    p.n = min(count - k, u1 - u);
    p.first = p.last = cta;
    if (p.n < count) {
      p.first = owner(u - k);
      p.last = owner(u - k + count - 1);
    }
    u += p.n;
  }
};

template <int kR, bool kBias, bool kSparse>
__global__ void __launch_bounds__(RowsCfg<kR>::kThreads, 1)
    cache_rows_kernel(const __grid_constant__ CUtensorMap mK, const __grid_constant__ CUtensorMap mV,
                      const arckv_cache8 c, RowsShape d, const bf16* Q, RowStrides qs, float scale, const int* blocks,
                      float* O, RowStrides os, float* parts, int* tickets, DevStatus* stt) {
  using Cfg = RowsCfg<kR>;
  // Fewest blocks that are worth a CTA of their own: joining parts takes over 1 us, in which the warps of one CTA, with a
  // block each, get further.  4 rows of 8 heads with 6 and with 4: 450 tokens 5.9 us and 7.1, 4 x 500 6.2 and 7.7, 4000
  // 8.9 and 9.7, but 1000 7.5 and 7.1, 4 x 1000 8.1 and 7.9 (8 rows alike).  12 rows of 4 x 8 heads, 1000 tokens: 10.9
  // with 6, 9.4 with 4.
  constexpr int kPartMin = kR == 16 ? 4 : 6;
  constexpr int kTR = Cfg::kTileRows, kTeams = Cfg::kTeams, kW = Cfg::kW, kSt = Cfg::kSt;
  extern __shared__ __align__(1024) unsigned char smraw[];
  unsigned char* ringK = smraw + ((1024u - (tc::smem_u32(smraw) & 1023u)) & 1023u);
  unsigned char* ringV = ringK + kSt * kTileBytes;
  float* sBias = (float*)(ringV + kSt * kTileBytes);
  float* sO = sBias + kSt * kCB;                                 // [warp][row of its tile][kRowO]
  bf16* sQ = (bf16*)(sO + kW * kTR * kRowO);                     // [parity of the run][row][128]
  int* pre = (int*)(sQ + 2 * kR * 128);                       // dense: [S + 1]
  __shared__ __align__(8) uint64_t fullK[kSt], emptyK[kSt], fullV[kSt], emptyV[kSt], fullQ[2], emptyQ[2];
  __shared__ float sKs[kSt], sVs[kSt];
  __shared__ int sBlk[kSt];
  __shared__ float sM[kW][kTR], sL[kW][kTR];
  __shared__ int abort_flag, last_flag, stop_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  volatile int* abortp = &abort_flag;

  if (tid == 0) {
    for (int s = 0; s < kSt; ++s) {
      tc::mbar_init(&fullK[s], 1);
      tc::mbar_init(&emptyK[s], Cfg::kTiles);
      tc::mbar_init(&fullV[s], 1);
      tc::mbar_init(&emptyV[s], Cfg::kTiles);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&fullQ[i], 1);
      tc::mbar_init(&emptyQ[i], kW);
    }
    abort_flag = 0;
    tc::mbar_fence_init();
  }
  pdl_trigger();
  pdl_wait();
  __shared__ int s_cut;   // blocks of a part (0: equal shares)
  if (warp == kW) {   // blocks, or parts, before each sequence, by warp scan
    if (lane == 0) {
      tc::tma_prefetch(&mK);
      tc::tma_prefetch(&mV);
    }
    if (!kSparse) {
      int cut = 0;
      auto scan = [&] {
        int run = 0;
        for (int s0 = 0; s0 < c.S; s0 += 32) {
          int x = s0 + lane < c.S ? max(1, (cache_len(c, s0 + lane) + kCB - 1) / kCB) : 0;
          if (cut > 0 && x > 0) x = max(1, min((x + cut - 1) / cut, x / kPartMin));
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
      if (c.S * d.H <= (int)gridDim.x) {   // the smallest parts that the CTAs suffice for
        cut = (all * d.H + (int)gridDim.x - 1) / (int)gridDim.x;
        for (all = scan(); all * d.H > (int)gridDim.x; all = scan())
          cut = max(cut + 1, (int)((long long)cut * all * d.H / (int)gridDim.x));
      }
      if (lane == 0) {
        pre[0] = 0;
        s_cut = cut;
      }
    }
  }
  __syncthreads();
  Walk<kSparse> walk{d, pre, c.S, (int)blockIdx.x};
  walk.len = c.len;
  int total;
  if (kSparse) {
    const int items = c.S * d.H * d.n_pos * d.groups;
    walk.parts = items <= (int)gridDim.x;
    walk.per = walk.parts ? max(1, min((int)gridDim.x / items, d.m / kPartMin)) : 1;
    total = items * (walk.parts ? walk.per : d.m);
  } else {
    walk.parts = s_cut > 0;
    total = pre[c.S] * d.H;
  }
  const int ctas = min((int)gridDim.x, total), me = blockIdx.x;
  if (me >= ctas) return;
  walk.q = total / ctas;
  walk.r = total - walk.q * ctas;
  walk.u = walk.q * me + min(me, walk.r);
  walk.u1 = walk.q * (me + 1) + min(me + 1, walk.r);

  if (warp >= kW) {
    // ------------------------------------- producers: keys (with scales and biases); queries and values
    const bool keys = warp == kW;
    uint64_t *full = keys ? fullK : fullV, *empty = keys ? emptyK : emptyV;
    unsigned char* ring = keys ? ringK : ringV;
    const CUtensorMap* map = keys ? &mK : &mV;
    const float* scales = keys ? c.k_scale : c.v_scale;
    float* sScale = keys ? sKs : sVs;
    int it = 0, run = 0;   // blocks and runs issued
    bool ok = true;
    for (Run p; ok && walk.next(p); ++run) {
      const int n = p.n, len = cache_len(c, p.s);
      if (!keys && !walk.parts) {   // a run ahead, as far as the ring reaches
        const int buf = run & 1, r = p.group * kR + lane, nrows = kSparse ? d.G : d.n_pos * d.G;
        if (run >= 2) ok = __all_sync(0xffffffffu, tc::mbar_wait(&emptyQ[buf], ((run >> 1) - 1) & 1, abortp, stt));
        if (!ok) {
          ++it;   // (as where a block's wait gives up: `it` is one more than were issued)
          break;
        }
        if (lane == 0) tc::mbar_arrive_expect_tx(&fullQ[buf], 256 * min(kR, nrows - p.group * kR));
        if (lane < kR && r < nrows) {
          const int pos = kSparse ? p.pos : r / d.G, gq = kSparse ? r : r - pos * d.G;
          tc::bulk_load(sQ + (buf * kR + lane) * 128, Q + p.s * qs.s + p.h * qs.h + pos * qs.i + gq * 128, 256, &fullQ[buf]);
        }
      }
      for (int k0 = 0; k0 < n && ok; k0 += 32) {
        const int k = k0 + lane;
        int b = -1;
        if (k < n) {
          b = kSparse ? blocks[(long long)p.list * d.m + p.blk + k] : p.blk + k;
          if (kSparse && b >= d.nblk) {
            set_status(stt, ARCKV_ERR_INVALID_ARG);
            b = -1;
          }
          if (b >= 0 && b * kCB >= len) b = -1;   // nothing of it is held
        }
        const float sc = b >= 0 ? scales[(long long)p.sh * d.nblk + b] : 0.f;
        const int cnt = min(32, n - k0);
        const bool with_bias = kBias && keys;
        auto load = [&](int st) {   // this lane's block into stage st
          tc::tma_load_3d(ring + st * kTileBytes, map, 0, b * kCB, p.sh, &full[st]);
          if (with_bias)
            tc::bulk_load(sBias + st * kCB, c.bias + (long long)p.sh * c.cap + b * kCB, kCB * 4, &full[st]);
        };
        auto announce = [&](int st) {
          sScale[st] = sc;
          if (keys) sBlk[st] = b;
          if (b >= 0) tc::mbar_arrive_expect_tx(&full[st], kTileBytes + (with_bias ? kCB * 4 : 0));
          else tc::mbar_arrive(&full[st]);
        };
        int j = 0;
        if (it < kSt) {   // the ring's first round: copies start before the scales have come
          const int first = min(cnt, kSt - it);
          if (lane < first && b >= 0) load(it + lane);
          if (lane < first) announce(it + lane);
          __syncwarp();
          j = first;
        }
        for (; j < cnt && ok; ++j) {
          const int q = it + j, st = q % kSt;
          ok = tc::mbar_wait(&empty[st], ((q / kSt) - 1) & 1, abortp, stt);
          ok = __all_sync(0xffffffffu, ok);
          if (ok && lane == j) {
            if (b >= 0) load(st);
            announce(st);
          }
        }
        it += j;
      }
    }
    if (!ok) {   // let the copies in flight land before the CTA's memory goes
      volatile int never = 0;
      for (int q = max(0, it - 1 - kSt); q < it - 1; ++q) tc::mbar_wait(&full[q % kSt], (q / kSt) & 1, &never, stt);
      if (!keys && !walk.parts)
        for (int q = max(0, run - 2); q < run; ++q) tc::mbar_wait(&fullQ[q & 1], (q >> 1) & 1, &never, stt);
    }
    return;
  }

  // --------------------------------------------------------------- consumers
  const int g = lane >> 2, t = lane & 3;
  const int team = warp % kTeams, tile0 = warp / kTeams * 8;   // first row of this warp's tile
  // this lane's row of a V tile (key lane & 15), and its 16-byte chunk (dims 32j + 16 (lane >> 4)) as stored for j = 0
  const uint32_t v_row = (lane & 15) * 128, v_chunk = ((lane >> 4) ^ (lane & 7)) << 4;
  constexpr float kGrow = 8.f, kLift = 7.f;   // weights reach 2^15: the range of f16
  int base = 0, run = 0;         // blocks of earlier runs, and their number
  bool ok = true;
  for (Run p; walk.next(p); ++run) {
    const int n = p.n, len = cache_len(c, p.s), h = p.h, nrows = kSparse ? d.G : d.n_pos * d.G;
    // query rows: column n is row n of the tile (four rows: twice the same four)
    uint32_t qf[8][2];
    float fac[2];           // 2^e scale (log2 e) of rows 2t, 2t + 1
    int see[2], see_min;    // tokens that they see
    {
      const int rt = tile0 + (kR == 4 ? (g & 3) : g), r = p.group * kR + rt, pos = kSparse ? p.pos : r / d.G;
      float x[32], amax = 0.f;
      // Queries of a CTA's only run are read here, beside its first copies; of several runs, they have come to shared
      // memory (64 x 8K decode 117 us; read from memory 120; 8 heads of 300 tokens 6.0 us by way of shared memory, 5.7)
      const bf16* mine = sQ + ((run & 1) * kR + rt) * 128;
      if (walk.parts) mine = Q + p.s * qs.s + h * qs.h + pos * qs.i + (kSparse ? r : r - pos * d.G) * 128;
      else ok = __all_sync(0xffffffffu, tc::mbar_wait(&fullQ[run & 1], (run >> 1) & 1, abortp, stt));
      if (r < nrows) {
        const uint4* src = (const uint4*)(mine + 32 * t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint4 v = src[e];
          const __nv_bfloat162* y = (const __nv_bfloat162*)&v;
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            const float2 z = __bfloat1622float2(y[f]);
            x[8 * e + 2 * f] = z.x;
            x[8 * e + 2 * f + 1] = z.y;
          }
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) amax = fmaxf(amax, fabsf(x[e]));
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = 0.f;
      }
      __syncwarp();
      if (!walk.parts && lane == 0) tc::mbar_arrive(&emptyQ[run & 1]);
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // exponent of the row's largest element, kept where 2^(14 - e) and 2^(e - 14) are normal
      const int e = max((int)((__float_as_uint(amax) >> 23) & 0xff) - 127, -100);
      const float up = __uint_as_float((unsigned)(14 - e + 127) << 23), down = __uint_as_float((unsigned)(e - 14 + 127) << 23);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        qf[k][0] = pack_f16(x[4 * k] * up, x[4 * k + 1] * up);
        qf[k][1] = pack_f16(x[4 * k + 2] * up, x[4 * k + 3] * up);
      }
      const float f = down * scale * (kBias ? 1.f : kLog2e);
      const int sees = r < nrows ? visible_tokens(len, d.n_pos, pos, d.causal) : 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fac[i] = __shfl_sync(0xffffffffu, f, (2 * t + i) * 4);
        see[i] = __shfl_sync(0xffffffffu, sees, (2 * t + i) * 4);
      }
      see_min = __reduce_min_sync(0xffffffffu, r < nrows ? sees : 0x7fffffff);
    }
    float o[8][4], mx[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[k][e] = 0.f;
    // block base + i of the CTA belongs to team (base + i) % kTeams
    for (int i = (team - base % kTeams + kTeams) % kTeams; i < n && ok; i += kTeams) {
      const int q = base + i, st = q % kSt;
      ok = __all_sync(0xffffffffu, tc::mbar_wait(&fullK[st], (q / kSt) & 1, abortp, stt));
      if (!ok) break;
      const int b = sBlk[st];
      if (b >= 0) {
        const float ks = sKs[st];
        const unsigned char* Kt = ringK + st * kTileBytes;
        // ---- S^T = K Q^T: lane (g, t) has keys g, g + 8 and dims 32t .. 32t + 31
        // (four independent chains of products: the 16-key tiles)
        float s[4][4];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][e] = 0.f;
#pragma unroll
        for (int ch = 0; ch < 2; ++ch) {
          uint4 a[4], a8[4];
#pragma unroll
          for (int mt = 0; mt < 4; ++mt) {
            const int off = (mt * 16 + g) * 128 + (((2 * t + ch) ^ g) << 4);
            a[mt] = *(const uint4*)(Kt + off);
            a8[mt] = *(const uint4*)(Kt + off + 8 * 128);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
              const uint32_t w = k == 0 ? a[mt].x : k == 1 ? a[mt].y : k == 2 ? a[mt].z : a[mt].w;
              const uint32_t w8 = k == 0 ? a8[mt].x : k == 1 ? a8[mt].y : k == 2 ? a8[mt].z : a8[mt].w;
              mma_f16(s[mt], codes_f16<0x4140>(w), codes_f16<0x4140>(w8), codes_f16<0x4342>(w), codes_f16<0x4342>(w8), qf[4 * ch + k][0],
                      qf[4 * ch + k][1]);
            }
          }
        }
        // ---- softmax of the block.  References follow the maximum only when it has grown by more than 2^8 (kGrow), so
        // that sums are scaled on few blocks.  Without biases the maximum is that of the products, whose factor is
        // positive (and never zero: a masked product is -inf), and a weight is 2^{product factor - mx}.
        const float f[2] = {fmaxf(fac[0] * ks, 0x1p-126f), fmaxf(fac[1] * ks, 0x1p-126f)};
        if (kBias) {
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const float bias = sBias[st * kCB + mt * 16 + hf * 8 + g];
#pragma unroll
              for (int e2 = 0; e2 < 2; ++e2) s[mt][2 * hf + e2] = fmaf(s[mt][2 * hf + e2], f[e2], bias);
            }
        }
        if ((b + 1) * kCB > see_min) {
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (b * kCB + mt * 16 + (e >> 1) * 8 + g >= see[e & 1]) s[mt][e] = -INFINITY;
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&emptyK[st]);   // the next block's keys may come
        // each lane looks whether one of its own logits is past what the reference allows; the rows' maxima are taken
        // where one is
        float top[2];
        bool grows = false;
#pragma unroll
        for (int e2 = 0; e2 < 2; ++e2) {   // rows 2t, 2t + 1
          top[e2] = max3(s[0][e2], s[0][2 + e2], s[1][e2]);
          top[e2] = fmaxf(max3(top[e2], s[1][2 + e2], s[2][e2]), max3(s[2][2 + e2], s[3][e2], s[3][2 + e2]));
          if (!kBias) top[e2] = fmaf(top[e2], f[e2], -kLift);
          grows |= (kBias ? (top[e2] - mx[e2]) * kLog2e : top[e2] - mx[e2]) > kGrow;   // (mx = -inf: by any but -inf)
        }
        if (__any_sync(0xffffffffu, grows)) {
          float alpha[2];
#pragma unroll
          for (int e2 = 0; e2 < 2; ++e2) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) top[e2] = fmaxf(top[e2], __shfl_xor_sync(0xffffffffu, top[e2], w));
            const float by = kBias ? (mx[e2] - top[e2]) * kLog2e : mx[e2] - top[e2];
            const bool up = top[e2] != -INFINITY && (mx[e2] == -INFINITY || -by > kGrow);
            alpha[e2] = up ? ex2_approx(by) : 1.f;   // (mx = -inf: zero)
            if (up) mx[e2] = top[e2];
            l[e2] *= alpha[e2];
          }
#pragma unroll
          for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][e] *= alpha[e & 1];
        }
#pragma unroll
        for (int e2 = 0; e2 < 2; ++e2) {
          const float ref = mx[e2] == -INFINITY ? 0.f : mx[e2];   // nothing visible yet: weights 2^{-inf} = 0
          float sum = 0.f;
#pragma unroll
          for (int mt = 0; mt < 4; ++mt)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              float& x = s[mt][2 * hf + e2];
              // a bias of the type's lowest value cancels against itself before the factor log2 e
              x = ex2_approx(kBias ? fmaf(x - ref, kLog2e, kLift) : fmaf(x, f[e2], -ref));
              sum += x;
            }
          l[e2] += sum;
        }
        // f16 pairs, transposed to (keys, row) operands
        uint32_t ph[4][2], pl[4][2];
#pragma unroll
        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float2 x = make_float2(s[mt][2 * hf], s[mt][2 * hf + 1]);
            const uint32_t hi = pack_f16(x.x, x.y);
            const float2 rest = minus_f16(x, *(const __half2*)&hi);
            const uint32_t lo = pack_f16(rest.x, rest.y);
            if (kR == 4) {   // columns 4 .. 7 carry lo of the same rows
              ph[mt][hf] = transpose8x8(t >= 2 ? lo : hi);
            } else {
              ph[mt][hf] = transpose8x8(hi);
              pl[mt][hf] = transpose8x8(lo);
            }
          }
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&fullV[st], (q / kSt) & 1, abortp, stt));
        if (!ok) break;
        const float vs = sVs[st] * kValues;   // (2^-122 at least; by the producer it would hold up the first copies)
        const uint32_t vt = tc::smem_u32(ringV) + st * kTileBytes + v_row;
        // ---- O^T += V^T P^T, 16 dims and 16 keys a product: a transposed 16-bit load gives lane (g, t) dims 2g, 2g + 1
        // of keys 2t, 2t + 1 in one word; even dims are the product's rows 0 .. 7, odd ones 8 .. 15
        float acc[8][4];
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[k][e] = 0.f;
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {   // dims 32j .. 32j + 31
            uint32_t w[4];
            load_transposed(w, vt + mt * (16 * 128) + ((j << 5) ^ v_chunk));
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const uint32_t f0 = codes_f16<0x4240>(w[2 * z]), f1 = codes_f16<0x4341>(w[2 * z]);
              const uint32_t f2 = codes_f16<0x4240>(w[2 * z + 1]), f3 = codes_f16<0x4341>(w[2 * z + 1]);
              mma_f16(acc[2 * j + z], f0, f1, f2, f3, ph[mt][0], ph[mt][1]);
              if (kR != 4) mma_f16(acc[2 * j + z], f0, f1, f2, f3, pl[mt][0], pl[mt][1]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&emptyV[st]);
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[k][e] = fmaf(vs, acc[k][e], o[k][e]);
      } else {   // an entry that names no block
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&fullV[st], (q / kSt) & 1, abortp, stt));
        if (!ok) break;
        if (lane == 0) {
          tc::mbar_arrive(&emptyK[st]);
          tc::mbar_arrive(&emptyV[st]);
        }
      }
    }
    base += n;
    // ---- the item's end (or this CTA's part of it): add the warps up
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
      const int r = 2 * t + i;
      if (g == 0 && r < kTR) {
        sM[warp][r] = mx[i];
        sL[warp][r] = l[i];
      }
      if (kR == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int z = 0; z < 2; ++z) o[k][2 * z + i] += __shfl_xor_sync(0xffffffffu, o[k][2 * z + i], 2);   // hi + lo
      }
      if (r < kTR) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          *(float2*)(sO + (warp * kTR + r) * kRowO + 16 * k + 2 * g) = make_float2(o[k][i], o[k][2 + i]);
      }
    }
    if (tid == 0) stop_flag = *abortp;   // one reading for all: the producers may raise the flag at any time
    bar_consumers(kW * 32);
    if (stop_flag) break;   // a wait gave up: write nothing
    const bool whole = p.first == p.last;
    auto weight = [](float m, float top) {   // e^{m - top}; 0 for a part that saw nothing
      return m == -INFINITY ? 0.f : ex2_approx(kBias ? (m - top) * kLog2e : m - top);
    };
    auto store = [&](int r, int dim, float4 v, float z) {
      const float inv = z == 0.f ? 0.f : 1.f / kValues / z;
      v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      const int row = p.group * kR + r, pos = kSparse ? p.pos : row / d.G, gq = kSparse ? row : row - pos * d.G;
      if (row >= nrows) return;   // (a tile without rows masks nothing: it may have met anything behind the end)
      *(float4*)(O + p.s * os.s + h * os.h + pos * os.i + gq * 128 + dim) = v;
      const float big = 3.402823466e38f;
      if (!(fabsf(v.x) <= big && fabsf(v.y) <= big && fabsf(v.z) <= big && fabsf(v.w) <= big))
        set_status(stt, ARCKV_ERR_NONFINITE);
    };
    // partial results: slot 2c holds the item that CTA c went on with, 2c + 1 the one it began
    constexpr int kSlot = kR * 132;   // 128 outputs, m, l (and two unused) for each row
    for (int x = tid; x < kR * 32; x += kW * 32) {
      const int r = x >> 5, dim = (x & 31) * 4, w0 = r / kTR * kTeams, rr = r % kTR;
      float up = -INFINITY, z = 0.f;
#pragma unroll
      for (int w = 0; w < kTeams; ++w) up = fmaxf(up, sM[w0 + w][rr]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kTeams; ++w) {
        const float f = weight(sM[w0 + w][rr], up);
        const float4 y = *(const float4*)(sO + ((w0 + w) * kTR + rr) * kRowO + dim);
        z = fmaf(sL[w0 + w][rr], f, z);
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
          float top = -INFINITY, z = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int cc = p.first; cc <= p.last; ++cc) {
            const float* slot = parts + (2ll * cc + (cc == p.first)) * kSlot + r * 132;
            const float2 ml = __ldcg((const float2*)(slot + 128));
            const float4 y = __ldcg((const float4*)(slot + dim));
            const float up = fmaxf(top, ml.x), f = weight(ml.x, up), f0 = weight(top, up);
            top = up;
            z = fmaf(z, f0, ml.y * f);
            v = make_float4(fmaf(v.x, f0, y.x * f), fmaf(v.y, f0, y.y * f), fmaf(v.z, f0, y.z * f), fmaf(v.w, f0, y.w * f));
          }
          store(r, dim, v, z);
        }
      }
    }
    bar_consumers(kW * 32);   // sO, sM, sL are free
  }
}

template <int kR, bool kBias, bool kSparse>
int launch_rows(const arckv_cache8& c, const CacheQuery& q, float scale, const int* blocks, int m, float* O,
                RowStrides os, void* ws, cudaStream_t st) {
  CUtensorMap mK, mV;
  if (!encode_u8_map_3d(&mK, c.K, c.cap, (uint64_t)c.S * c.H, kCB) ||
      !encode_u8_map_3d(&mV, c.V, c.cap, (uint64_t)c.S * c.H, kCB))
    return -1;
  RowsShape d;
  d.H = c.H;
  d.n_pos = q.n_pos;
  d.G = q.G;
  d.cap = c.cap;
  d.nblk = c.cap / kCB;
  d.groups = kSparse ? cdiv(q.G, kR) : 1;   // dense calls with more rows go elsewhere
  d.m = m;
  d.causal = q.causal;
  auto kern = cache_rows_kernel<kR, kBias, kSparse>;
  const int smem = RowsCfg<kR>::kSmem + (kSparse ? 0 : (c.S + 1) * (int)sizeof(int));
  if (set_dyn_smem((const void*)kern, smem) != cudaSuccess) return -1;
  const int ctas = std::min(tc_gemm_sm_count(), kCacheMaxCtas);
  const cudaError_t e = launch_pdl(kern, dim3(ctas), RowsCfg<kR>::kThreads, smem, st, mK, mV, c, d, q.Q, q.qs, scale, blocks, O, os,
                                   (float*)((char*)ws + ARCKV_CACHE_WS_HEADER), ws_tickets(ws), (DevStatus*)ws);
  return e == cudaSuccess ? 1 : -1;
}

template <int kR>
int launch_rows_r(const arckv_cache8& c, const CacheQuery& q, float scale, const int* blocks, int m, float* O,
                  RowStrides os, void* ws, cudaStream_t st) {
  if (c.bias)
    return blocks ? launch_rows<kR, true, true>(c, q, scale, blocks, m, O, os, ws, st)
                  : launch_rows<kR, true, false>(c, q, scale, blocks, m, O, os, ws, st);
  return blocks ? launch_rows<kR, false, true>(c, q, scale, blocks, m, O, os, ws, st)
                : launch_rows<kR, false, false>(c, q, scale, blocks, m, O, os, ws, st);
}

}  // namespace

size_t cache_attend_scratch(int, int, int, int n_pos, int G) {
  const size_t rows = (size_t)2 * kCacheMaxCtas * 16 * 132 * sizeof(float);
  return (long long)n_pos * G > kRowsMax ? std::max(rows, cache_tiles_scratch((long long)n_pos * G)) : rows;
}

int launch_cache_attend(const arckv_cache8& c, const CacheQuery& q, float scale, const int* blocks, int m, float* O,
                        RowStrides os, void* ws, cudaStream_t st) {
  const long long rows = blocks ? q.G : (long long)q.n_pos * q.G;   // rows that read the same blocks
  if (rows <= 4) return launch_rows_r<4>(c, q, scale, blocks, m, O, os, ws, st);
  if (rows <= 8) return launch_rows_r<8>(c, q, scale, blocks, m, O, os, ws, st);
  if (blocks || rows <= kRowsMax) return launch_rows_r<16>(c, q, scale, blocks, m, O, os, ws, st);
  return launch_cache_tiles(c, q, scale, O, os, ws, st);
}

}  // namespace arckv
