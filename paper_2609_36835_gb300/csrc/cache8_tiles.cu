// Attention of many query rows over an 8-bit cache (prompt chunks, reference
// queries): the products of cache8_attend.cu on tcgen05.
//
// With n rows a head every code is used n times, so the call is bound by the
// tensor pipe.  A CTA takes 128 or 256 rows of one head (one or two M = 128
// tiles) and goes over the keys 128 at a time:
//   converters (4 warps)  read the codes of K and V from HBM and leave them in
//                         shared memory as f16 operands, V transposed; a code
//                         costs about one instruction for 256 rows
//   MMA warp              S = Q K^T (f16, exact products, fp32 sums in TMEM), O += P V
//   softmax (4 warps a tile, one row a thread)  turn S into weights in place: the
//                         f16 pair hi + lo of 32 keys takes the 32 columns that
//                         their logits had; P is the MMA's operand from TMEM
// P V runs once for hi and once for lo, which keeps 22 bits of a weight: three
// units of MMA work where f16 weights would do with two, so 2/3 of the pipe's
// peak is the most that the fp32 output allows.  With two tiles the pipe works
// on one while the other's softmax runs.
//
// The weight of key j of block b carries the block's scale of V:
//   w_j = 2^{x_j + log2 vs_b - ref + 7},  O = sum_j w_j c_j / sum_b (sum_{j in b} w_j) / vs_b
// so codes go into the product as they are and no partial sum depends on how
// far apart the blocks' scales lie.  ref follows the running maximum of x_j +
// log2 vs_b only when that has grown by more than 8 (weights then stay below
// 2^15, in the range of f16): O is read, scaled and written back on few steps.
//
// The pipe's fp32 sums round towards zero, and O would shrink by 1.4e-7 a step:
// after 16 steps it is added to sums in the workspace (L2) and starts again.
#include "cache8.cuh"
#include "tc.cuh"

#include <cuda_fp16.h>

namespace arckv {
namespace {

constexpr int kStep = 128;                    // keys of a step (two blocks)
constexpr int kHalf = 128 * 128;              // bytes of a 128 x 64 f16 operand tile
constexpr int kFlush = 16;                    // steps that O is summed up over in TMEM
constexpr float kFar = 60.f;                  // growth of ref (log2) past which the flushed sums are scaled down
constexpr float kGrow = 8.f, kLift = 7.f;     // see above
constexpr float kVsUnit = 0x1p-20f;           // sums are in units of kVsUnit / vs: the least vs, 2^-107, stays in range

struct TileShape {
  int H, n_pos, G, nblk, cap, tiles;   // tiles: row tiles of a head
  bool causal;
};

template <int kT>
struct TileCfg {
  static constexpr int kRows = 128 * kT;
  static constexpr int kSoft = 4 * kT;                   // softmax warps 0 .. kSoft - 1, then 4 converters, then MMA
  static constexpr int kThreads = 32 * (kSoft + 8);      // (whole warpgroups: three warps idle)
  // registers at launch (65536 / kThreads, a multiple of 8), and how the warpgroups share them:
  // kT kRegsSoft + 2 kRegsRest = (kT + 2) kRegs
  static constexpr int kRegs = kT == 2 ? 128 : 168, kRegsRest = kT == 2 ? 72 : 136, kRegsSoft = kT == 2 ? 184 : 232;
  static_assert(kT * kRegsSoft + 2 * kRegsRest == (kT + 2) * kRegs && kRegs * kThreads <= 65536, "register shares");
  static constexpr int kSmem = kT * 2 * kHalf + 2 * 4 * kHalf + 1024;   // Q, then two stages of (K, V)
  static constexpr int kSlot = 131 * kRows;              // floats of a partial result: O, ref, log2 vs of ref, sum
};

// D[tmem] (+)= A[tmem] * B[smem]^T, kind::f16, one CTA.
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// 32 columns of this warp's lanes, not waited for.
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Nothing that uses v moves above this point (behind a wait).
__device__ __forceinline__ void settle32(float* v) {
  asm volatile(""
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                 "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]),
                 "+f"(v[30]), "+f"(v[31]));
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
      "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// kind::f16 with A = B = f16, D = fp32, both K-major, M = 128, N = 128.
constexpr uint32_t kIdescF16 = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);

template <int kHi>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {   // bytes (0, 1) or (2, 3), codes + 128, as two f16 codes
  const uint32_t y = __byte_perm(w, 0x64646464u, kHi ? 0x4342 : 0x4140);
  const __half2 z = __hsub2(*(const __half2*)&y, __half2{__half_raw{0x6480}, __half_raw{0x6480}});
  return *(const uint32_t*)&z;
}

// Steps of a row tile: as far as its last row sees (one at least).
__device__ __forceinline__ int tile_steps(const TileShape& d, int len, int tile, int rows) {
  const int last = min((tile + 1) * rows, d.n_pos * d.G) - 1;
  return max(1, (visible_tokens(len, d.n_pos, last / d.G, d.causal) + kStep - 1) / kStep);
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
  const long long per = pre[lo + 1] - pre[lo], rest = u - pre[lo] * d.H, h = rest / per;
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

struct Meta {   // of a step's two blocks
  float ks[2], lv[2], iv[2];   // scale of K, log2 and inverse (in units of kVsUnit) of V's
};

template <int kT, bool kBias>
__global__ void __launch_bounds__(TileCfg<kT>::kThreads, 1)
    cache_tiles_kernel(const arckv_cache8 c, TileShape d, const bf16* Q, RowStrides qs, float scale, float* O,
                       RowStrides os, float* parts, int* tickets, DevStatus* stt) {
  using Cfg = TileCfg<kT>;
  constexpr int kSoft = Cfg::kSoft, kRows = Cfg::kRows;
  extern __shared__ unsigned char smraw[];
  unsigned char* sQ = smraw + ((1024u - (tc::smem_u32(smraw) & 1023u)) & 1023u);   // [tile][half][128][128 B]
  unsigned char* sKV = sQ + kT * 2 * kHalf;                                        // [stage][K, V][half]
  long long* pre = (long long*)(sKV + 8 * kHalf);                                  // [S + 1] steps of a head
  __shared__ __align__(8) uint64_t qfull, kfull[2], vfull[2], kempty[2], vempty[2], sfull[kT], pfull[kT], odone[kT],
      drain;
  __shared__ Meta meta[4];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, stop_flag, last_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abortp = &abort_flag;

  if (tid == 0) {
    tc::mbar_init(&qfull, kRows);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&kfull[i], 128);
      tc::mbar_init(&vfull[i], 128);
      tc::mbar_init(&kempty[i], 1);
      tc::mbar_init(&vempty[i], 1);
    }
    for (int t = 0; t < kT; ++t) {
      tc::mbar_init(&sfull[t], 1);
      tc::mbar_init(&pfull[t], 128);
      tc::mbar_init(&odone[t], 1);
    }
    tc::mbar_init(&drain, 1);
    abort_flag = 0;
    tc::mbar_fence_init();
  }
  if (warp == kSoft + 4) tc::tmem_alloc(&tmem_slot, 256 * kT);
  for (int s = tid; s < c.S; s += Cfg::kThreads) {   // steps of one head of each sequence
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
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_slot;   // tile t: S / P at columns 256 t, O at 256 t + 128
  CacheShares sh;
  sh.total = pre[c.S] * d.H;
  sh.ctas = (int)min((long long)gridDim.x, sh.total);
  const bool active = (int)blockIdx.x < sh.ctas;
  const long long u0 = active ? sh.start(blockIdx.x) : 0, u1 = active ? sh.start(blockIdx.x + 1) : 0;

  if (warp >= kSoft) regs_dec<Cfg::kRegsRest>();
  else regs_inc<Cfg::kRegsSoft>();

  if (warp > kSoft + 4) {
    // idle
  } else if (warp == kSoft + 4) {
    // ------------------------------------------------------------ MMA issuer
    bool ok = true;
    int it = 0, seg = 0;   // steps and items so far
    for (long long u = u0; u < u1 && ok; ++seg) {
      const Segment g = segment_of(u, d, c, pre, kRows);
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      ok = tc::mbar_wait(&qfull, seg & 1, abortp, stt);
      for (int i = 0; i <= n && ok; ++i) {
        const int q = it + i;
        if (i < n) ok = tc::mbar_wait(&kfull[q & 1], (q >> 1) & 1, abortp, stt);
        if (ok && i > 0) ok = tc::mbar_wait(&vfull[(q - 1) & 1], ((q - 1) >> 1) & 1, abortp, stt);
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          if (ok && i > 0) ok = tc::mbar_wait(&pfull[t], (q - 1) & 1, abortp, stt);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc::fence_after_sync();
          if (lane == 0) {
            const uint32_t S = tmem + 256 * t, Ot = S + 128;
            if (i > 0) {   // O += P V of the step before
              const uint32_t v = tc::smem_u32(sKV + ((q - 1) & 1) * 4 * kHalf + 2 * kHalf);
#pragma unroll
              for (int ks = 0; ks < 8; ++ks) {
                const uint64_t bd = tc::sdesc_k128(v + (ks >> 2) * kHalf + (ks & 3) * 32);
                const uint32_t a = S + (ks >> 1) * 32 + (ks & 1) * 8;   // hi; lo is 16 columns on
                mma_f16_ts(Ot, a, bd, kIdescF16, ((i - 1) % kFlush != 0 || ks > 0) ? 1u : 0u);
                mma_f16_ts(Ot, a + 16, bd, kIdescF16, 1u);
              }
              if (i == n) tc::mma_commit(&odone[t]);
            }
            if (i < n) {   // S = Q K^T
              const uint32_t a = tc::smem_u32(sQ + t * 2 * kHalf), k = tc::smem_u32(sKV + (q & 1) * 4 * kHalf);
#pragma unroll
              for (int ks = 0; ks < 8; ++ks)
                tc::mma_f16(S, tc::sdesc_k128(a + (ks >> 2) * kHalf + (ks & 3) * 32),
                            tc::sdesc_k128(k + (ks >> 2) * kHalf + (ks & 3) * 32), kIdescF16, ks > 0 ? 1u : 0u);
              tc::mma_commit(&sfull[t]);
            }
          }
          __syncwarp();
        }
        if (ok && lane == 0) {
          if (i < n) tc::mma_commit(&kempty[q & 1]);
          if (i > 0) tc::mma_commit(&vempty[(q - 1) & 1]);
        }
        __syncwarp();
      }
      it += n;
      u += n;
    }
    if (lane == 0) {   // every MMA done before TMEM and shared memory go
      tc::mma_commit(&drain);
      volatile int never = 0;
      tc::mbar_wait(&drain, 0, &never, stt);
    }
    __syncwarp();
  } else if (warp >= kSoft) {
    // ------------------------------------------------------------ converters
    const int cw = warp - kSoft, ct = tid - kSoft * 32;
    // K: eight lanes a row, 16 dims each.  V: keys 8 ko .. 8 ko + 7, dims 16 dg .. 16 dg + 15 (eight lanes with
    // different ko write one dim's chunks: no bank conflicts)
    const int kc = lane & 7, kr = cw * 32 + (lane >> 3);
    const int ko = (lane & 7) + 8 * (cw & 1), dg = (lane >> 3) + 4 * (cw >> 1);
    bool ok = true;
    int it = 0;
    for (long long u = u0; u < u1 && ok;) {
      const Segment g = segment_of(u, d, c, pre, kRows);
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      const uint8_t* Kh = c.K + g.sh * c.cap * 128;
      const uint8_t* Vh = c.V + g.sh * c.cap * 128;
      const uint4 zero = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
      uint4 raw[8];
      auto load_k = [&](int i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = (g.step + i) * kStep + kr + 4 * j;
          raw[j] = key < c.cap ? __ldg((const uint4*)(Kh + (long long)key * 128 + kc * 16)) : zero;
        }
      };
      auto load_v = [&](int i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = (g.step + i) * kStep + ko * 8 + j;
          raw[j] = key < c.cap ? __ldg((const uint4*)(Vh + (long long)key * 128 + dg * 16)) : zero;
        }
      };
      for (int i = 0; i < n && ok; ++i) {
        const int q = it + i, st = q & 1;
        unsigned char* Ks = sKV + st * 4 * kHalf;
        unsigned char* Vs = Ks + 2 * kHalf;
        load_k(i);   // in flight while the stage is waited for
        if (q >= 2) ok = tc::mbar_wait(&kempty[st], ((q >> 1) - 1) & 1, abortp, stt);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = kr + 4 * j;
          const uint4 x = make_uint4(codes_f16<0>(raw[j].x), codes_f16<1>(raw[j].x), codes_f16<0>(raw[j].y),
                                     codes_f16<1>(raw[j].y));
          const uint4 y = make_uint4(codes_f16<0>(raw[j].z), codes_f16<1>(raw[j].z), codes_f16<0>(raw[j].w),
                                     codes_f16<1>(raw[j].w));
          unsigned char* row = Ks + (kc >> 2) * kHalf + r * 128;
          // the two chunks in an order that keeps the eight lanes of a row on different banks
          const int q0 = (kc & 3) * 2 + (kc >> 2), q1 = (kc & 3) * 2 + 1 - (kc >> 2);
          *(uint4*)(row + ((q0 ^ (r & 7)) << 4)) = (kc >> 2) ? y : x;
          *(uint4*)(row + ((q1 ^ (r & 7)) << 4)) = (kc >> 2) ? x : y;
        }
        if (ct < 2) {
          const int b = (g.step + i) * 2 + ct;
          float ks = 1.f, vs = 1.f;   // of blocks that hold nothing: their keys are masked
          if (b * kCB < cache_len(c, g.s)) {
            ks = c.k_scale[g.sh * d.nblk + b];
            vs = c.v_scale[g.sh * d.nblk + b];
          }
          Meta& m = meta[q & 3];
          m.ks[ct] = ks;
          m.lv[ct] = log2f(vs);
          m.iv[ct] = kVsUnit / vs;
        }
        tc::fence_proxy_async_smem();
        tc::mbar_arrive(&kfull[st]);
        load_v(i);
        if (q >= 2) ok = tc::mbar_wait(&vempty[st], ((q >> 1) - 1) & 1, abortp, stt);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
#pragma unroll
        for (int w = 0; w < 4; ++w) {   // dims 16 dg + 4 w ..
          uint32_t f[4][4];             // [dim][key pair]
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint32_t a = w == 0 ? raw[2 * p].x : w == 1 ? raw[2 * p].y : w == 2 ? raw[2 * p].z : raw[2 * p].w;
            const uint32_t b = w == 0 ? raw[2 * p + 1].x : w == 1 ? raw[2 * p + 1].y : w == 2 ? raw[2 * p + 1].z : raw[2 * p + 1].w;
            const uint32_t y = __byte_perm(a, b, 0x5140), z = __byte_perm(a, b, 0x7362);
            f[0][p] = codes_f16<0>(y);
            f[1][p] = codes_f16<1>(y);
            f[2][p] = codes_f16<0>(z);
            f[3][p] = codes_f16<1>(z);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int dim = dg * 16 + w * 4 + e;
            *(uint4*)(Vs + (ko >> 3) * kHalf + dim * 128 + (((ko & 7) ^ (dim & 7)) << 4)) =
                make_uint4(f[e][0], f[e][1], f[e][2], f[e][3]);
          }
        }
        tc::fence_proxy_async_smem();
        tc::mbar_arrive(&vfull[st]);
      }
      it += n;
      u += n;
    }
  } else {
    // --------------------------------------------------------------- softmax
    const int t = warp >> 2, row_t = (warp & 3) * 32 + lane;   // this thread's row of its tile
    const uint32_t S = tmem + 256 * t + ((uint32_t)(warp & 3) * 32 << 16), Ot = S + 128;
    const int nrows = d.n_pos * d.G;
    bool ok = true;
    int it = 0, seg = 0;
    for (long long u = u0; u < u1; ++seg) {
      const Segment g = segment_of(u, d, c, pre, kRows);
      const int n = (int)min((long long)(g.count - g.step), u1 - u);
      const int row = g.tile * kRows + t * 128 + row_t, pos = row / d.G, gq = row - pos * d.G;
      const int h = (int)(g.sh - (long long)g.s * d.H);
      const bool mine = row < nrows;
      const int see = mine ? visible_tokens(cache_len(c, g.s), d.n_pos, pos, d.causal) : 0;
      float fac;   // of this row's products, in powers of two without biases, of e with them
      {            // the query row as f16, scaled by a power of two
        const uint4* src = (const uint4*)(Q + g.s * qs.s + h * qs.h + pos * qs.i + gq * 128);
        float amax = 0.f;
        if (mine)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint4 v = __ldg(src + e);
            const __nv_bfloat162* y = (const __nv_bfloat162*)&v;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              const float2 z = __bfloat1622float2(y[f]);
              amax = fmaxf(amax, fmaxf(fabsf(z.x), fabsf(z.y)));
            }
          }
        const int ex = max((int)((__float_as_uint(amax) >> 23) & 0xff) - 127, -100);
        const float up = __uint_as_float((unsigned)(14 - ex + 127) << 23);
        fac = __uint_as_float((unsigned)(ex - 14 + 127) << 23) * scale * (kBias ? 1.f : kLog2e);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (mine) {
            v = __ldg(src + e);
            const __nv_bfloat162* y = (const __nv_bfloat162*)&v;
            __half2 z[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              const float2 a = __bfloat1622float2(y[f]);
              z[f] = __floats2half2_rn(a.x * up, a.y * up);
            }
            v = *(const uint4*)&z[0];
          }
          *(uint4*)(sQ + (t * 2 + (e >> 3)) * kHalf + row_t * 128 + (((e & 7) ^ (row_t & 7)) << 4)) = v;
        }
        tc::fence_proxy_async_smem();
        tc::mbar_arrive(&qfull);
      }
      float* sums = parts + 2ll * kCacheMaxCtas * Cfg::kSlot + (long long)blockIdx.x * kRows * 128 + t * 128 + row_t;
      float bref = -INFINITY, brefv = 0.f;          // reference of the flushed sums
      float ref = -INFINITY, refv = 0.f, l = 0.f;   // with biases ref is the logit and refv the log2 vs that came with it
      const float* bias = kBias ? c.bias + g.sh * c.cap : nullptr;
      for (int i = 0; i < n; ++i) {
        const int q = it + i, j0 = (g.step + i) * kStep;
        // S is in; so are the product of the step before (issued earlier by the same thread) and the step's scales
        // (written before kfull, which the MMA warp waited for)
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&sfull[t], q & 1, abortp, stt));
        if (!ok) break;
        tc::fence_after_sync();
        const Meta m = meta[q & 3];
        if (i > 0 && i % kFlush == 0) {
          // O goes to this row's sums in memory and starts again at zero (see above)
          const float d = kBias ? fmaf(ref - bref, kLog2e, refv - brefv) : ref - bref;   // NaN, inf: nothing there yet
          const bool none = bref == -INFINITY, far = !none && d > kFar;
          const float up = none || far ? 1.f : ex2_approx(d), down = far ? ex2_approx(-d) : 1.f;
          const bool redo = __any_sync(0xffffffffu, none || far);
#pragma unroll 1
          for (int ch = 0; ch < 8; ++ch) {
            float o[16];
            tc::tmem_ld16(Ot + ch * 16, o);
            float* b = sums + ch * 16 * kRows;
            if (redo) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float old = none ? 0.f : __ldcg(b + e * kRows);
                __stcg(b + e * kRows, fmaf(old, down, o[e] * up));
              }
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                asm volatile("red.global.add.f32 [%0], %1;" ::"l"(b + e * kRows), "f"(o[e] * up) : "memory");
            }
          }
          if (none || far) {
            bref = ref;
            brefv = refv;
          }
          tc::fence_before_sync();
        }
        float v[128];
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) tmem_ld32_async(S + ch * 32, v + ch * 32);
        tmem_wait_ld();
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) settle32(v + ch * 32);
        const int lim = see - j0;   // keys of the step that the row sees
        const bool edge = __any_sync(0xffffffffu, lim < kStep);
        const float f[2] = {fac * m.ks[0], fac * m.ks[1]};
        if (kBias) {   // logits; biases are read four at a time where the row sees something, within the capacity
#pragma unroll
          for (int e = 0; e < kStep; e += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (e < lim) x = __ldg((const float4*)(bias + j0 + e));
            v[e] = fmaf(v[e], f[e >> 6], x.x);
            v[e + 1] = fmaf(v[e + 1], f[e >> 6], x.y);
            v[e + 2] = fmaf(v[e + 2], f[e >> 6], x.z);
            v[e + 3] = fmaf(v[e + 3], f[e >> 6], x.w);
          }
        }
        if (edge) {
#pragma unroll
          for (int e = 0; e < kStep; ++e)
            if (e >= lim) v[e] = -INFINITY;
        }
        // largest of each block
        float top[2];
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          float a = v[hb * 64], b = v[hb * 64 + 1];
#pragma unroll
          for (int e = 2; e < 64; e += 2) {
            a = fmaxf(a, v[hb * 64 + e]);
            b = fmaxf(b, v[hb * 64 + e + 1]);
          }
          a = fmaxf(a, b);
          top[hb] = kBias ? a : fmaf(a, f[hb], m.lv[hb]);   // f > 0: the largest product is the largest logit
        }
        float alpha = 1.f;
        bool grow;
        if (kBias) {
          // in units of log2: (x - ref) log2 e + lv - refv; differences of logits first, so that the type's lowest
          // value cancels against itself
          float nr = ref, nv = refv;
#pragma unroll
          for (int hb = 0; hb < 2; ++hb)
            if (top[hb] != -INFINITY && (nr == -INFINITY || fmaf(top[hb] - nr, kLog2e, m.lv[hb] - nv) > 0.f)) {
              nr = top[hb];
              nv = m.lv[hb];
            }
          grow = nr != -INFINITY && (ref == -INFINITY || fmaf(nr - ref, kLog2e, nv - refv) > kGrow);
          if (grow) {
            alpha = ref == -INFINITY ? 0.f : ex2_approx(fmaf(ref - nr, kLog2e, refv - nv));
            ref = nr;
            refv = nv;
          }
        } else {
          const float nr = fmaxf(top[0], top[1]);
          grow = nr > ref + kGrow || (ref == -INFINITY && nr != -INFINITY);
          if (grow) {
            alpha = ref == -INFINITY ? 0.f : ex2_approx(ref - nr);
            ref = nr;
          }
        }
        if (i % kFlush != 0 && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
          for (int ch = 0; ch < 8; ++ch) {
            float o[16];
            tc::tmem_ld16(Ot + ch * 16, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= alpha;
            tmem_st16(Ot + ch * 16, o);
          }
          tmem_wait_st();
        }
        l *= alpha;
        const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          const float add = kBias ? m.lv[hb] - refv + kLift : m.lv[hb] - base + kLift;
          const float2 add_2 = make_float2(add, add);
          float2 sum = make_float2(0.f, 0.f);
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            uint32_t r[32];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const int k = hb * 64 + ch * 32 + e;
              float2 x = make_float2(v[k], v[k + 1]);
              if (kBias)
                x = fma2(add2(x, make_float2(-base, -base)), make_float2(kLog2e, kLog2e), add_2);
              else
                x = fma2(x, make_float2(f[hb], f[hb]), add_2);
              x.x = ex2_approx(x.x);
              x.y = ex2_approx(x.y);
              sum = add2(sum, x);
              // hi: the leading 11 bits, exact in f16; lo: the rest, at most 2^-10 of w, rounded to 11 bits
              const float2 hi = make_float2(__uint_as_float(__float_as_uint(x.x) & 0xffffe000u),
                                            __uint_as_float(__float_as_uint(x.y) & 0xffffe000u));
              const float2 lo = add2(x, make_float2(-hi.x, -hi.y));
              const __half2 h2 = __floats2half2_rn(hi.x, hi.y), l2 = __floats2half2_rn(lo.x, lo.y);
              r[e >> 1] = *(const uint32_t*)&h2;
              r[16 + (e >> 1)] = *(const uint32_t*)&l2;
            }
            tmem_st32(S + hb * 64 + ch * 32, r);
          }
          l = fmaf(sum.x + sum.y, m.iv[hb], l);
        }
        tmem_wait_st();
        tc::fence_before_sync();
        tc::mbar_arrive(&pfull[t]);
      }
      it += n;
      if (ok) ok = __all_sync(0xffffffffu, tc::mbar_wait(&odone[t], seg & 1, abortp, stt));
      tc::fence_after_sync();
      if (tid == 0) stop_flag = *abortp;   // one reading for all
      asm volatile("bar.sync 1, %0;" ::"r"(kRows) : "memory");
      if (stop_flag) break;
      const bool whole = g.step == 0 && n == g.count;
      auto store4 = [&](int dim, float4 v, float inv) {
        v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        const float big = 3.402823466e38f;
        if (!(fabsf(v.x) <= big && fabsf(v.y) <= big && fabsf(v.z) <= big && fabsf(v.w) <= big))
          set_status(stt, ARCKV_ERR_NONFINITE);
        *(float4*)(O + g.s * os.s + h * os.h + pos * os.i + gq * 128 + dim) = v;
      };
      const float inv = l == 0.f ? 0.f : kVsUnit / l;
      const bool flushed = bref != -INFINITY;
      const float bw = flushed ? ex2_approx(kBias ? fmaf(bref - ref, kLog2e, brefv - refv) : bref - ref) : 0.f;
      float* slot = parts + (2ll * blockIdx.x + (g.step == 0 ? 1 : 0)) * Cfg::kSlot + t * 128 + row_t;
#pragma unroll
      for (int ch = 0; ch < 4; ++ch) {
        float v[32];
        tc::tmem_ld32(Ot + ch * 32, v);
        if (flushed) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(__ldcg(sums + (ch * 32 + e) * kRows), bw, v[e]);
        }
        if (whole) {
          if (mine)
#pragma unroll
            for (int e = 0; e < 32; e += 4) store4(ch * 32 + e, make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]), inv);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) __stcg(slot + (ch * 32 + e) * kRows, v[e]);
        }
      }
      tc::fence_before_sync();
      if (!whole) {
        __stcg(slot + 128 * kRows, ref);
        __stcg(slot + 129 * kRows, refv);
        __stcg(slot + 130 * kRows, l);
        const int c_first = sh.owner(g.first), c_last = sh.owner(g.first + g.count - 1);
        __threadfence();
        asm volatile("bar.sync 1, %0;" ::"r"(kRows) : "memory");
        if (tid == 0) {
          last_flag = atomicAdd(&tickets[c_first], 1) == c_last - c_first;
          if (last_flag) tickets[c_first] = 0;
          __threadfence();
        }
        asm volatile("bar.sync 1, %0;" ::"r"(kRows) : "memory");
        if (last_flag && mine) {
          auto part = [&](int cc) { return parts + (2ll * cc + (cc == c_first)) * Cfg::kSlot + t * 128 + row_t; };
          float top = -INFINITY, topv = 0.f, z = 0.f;
          for (int cc = c_first; cc <= c_last; ++cc) {
            const float r = __ldcg(part(cc) + 128 * kRows), rv = __ldcg(part(cc) + 129 * kRows);
            if (r != -INFINITY && (top == -INFINITY || (kBias ? fmaf(r - top, kLog2e, rv - topv) : r - top) > 0.f)) {
              top = r;
              topv = rv;
            }
          }
          auto weight = [&](int cc) {
            const float r = __ldcg(part(cc) + 128 * kRows), rv = __ldcg(part(cc) + 129 * kRows);
            return r == -INFINITY ? 0.f : ex2_approx(kBias ? fmaf(r - top, kLog2e, rv - topv) : r - top);
          };
          for (int cc = c_first; cc <= c_last; ++cc) z = fmaf(__ldcg(part(cc) + 130 * kRows), weight(cc), z);
          const float zinv = z == 0.f ? 0.f : kVsUnit / z;
          for (int ch = 0; ch < 4; ++ch) {
            float v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.f;
            for (int cc = c_first; cc <= c_last; ++cc) {
              const float w = weight(cc);
              const float* p = part(cc) + ch * 32 * kRows;
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = fmaf(__ldcg(p + e * kRows), w, v[e]);
            }
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              store4(ch * 32 + e, make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]), zinv);
          }
        }
      }
      u += n;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kSoft + 4) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem, 256 * kT);
  }
}

template <int kT, bool kBias>
int launch_tiles(const arckv_cache8& c, const CacheQuery& q, float scale, float* O, RowStrides os, void* ws,
                 cudaStream_t st) {
  using Cfg = TileCfg<kT>;
  TileShape d;
  d.H = c.H;
  d.n_pos = q.n_pos;
  d.G = q.G;
  d.nblk = c.cap / kCB;
  d.cap = c.cap;
  d.tiles = cdiv((long long)q.n_pos * q.G, Cfg::kRows);
  d.causal = q.causal;
  auto kern = cache_tiles_kernel<kT, kBias>;
  const int smem = Cfg::kSmem + (c.S + 1) * (int)sizeof(long long);
  if (set_dyn_smem((const void*)kern, smem) != cudaSuccess) return -1;
  kern<<<std::min(tc_gemm_sm_count(), kCacheMaxCtas), Cfg::kThreads, smem, st>>>(
      c, d, q.Q, q.qs, scale, O, os, (float*)((char*)ws + ARCKV_CACHE_WS_HEADER), ws_tickets(ws), (DevStatus*)ws);
  return 1;
}

}  // namespace

size_t cache_tiles_scratch(long long rows) {
  const size_t slot = rows <= 128 ? TileCfg<1>::kSlot : TileCfg<2>::kSlot;
  return kCacheMaxCtas * (2 * slot + (rows <= 128 ? TileCfg<1>::kRows : TileCfg<2>::kRows) * 128) * sizeof(float);
}

int launch_cache_tiles(const arckv_cache8& c, const CacheQuery& q, float scale, float* O, RowStrides os, void* ws,
                       cudaStream_t st) {
  const long long rows = (long long)q.n_pos * q.G;
  if (rows <= 128)
    return c.bias ? launch_tiles<1, true>(c, q, scale, O, os, ws, st) : launch_tiles<1, false>(c, q, scale, O, os, ws, st);
  return c.bias ? launch_tiles<2, true>(c, q, scale, O, os, ws, st) : launch_tiles<2, false>(c, q, scale, O, os, ws, st);
}

}  // namespace arckv
