// Block selection for sparse attention over an 8-bit cache.
//
// The logits of block b's keys are at most scale_b sum_e max(q_e lo_be, q_e hi_be)
// with lo, hi the least and largest key codes of dimension e.  With the query
// quantised to 8 bits too, the sum is sum_e (q_e^+ hi_be + q_e^- lo_be), an exact
// integer below 2^21: scores are the same in whatever order they are added up.
//
// Two kernels.  Scores: 260 bytes a block and head are read once and take 64
// four-way integer dot products a query row; one thread has one block's bounds
// in registers and goes over the CTA's rows, whose codes it reads by broadcast.
// Choice: a group of threads (a warp for short lists, up to 1024 threads for
// long ones) holds one position's scores in registers and bisects for the m-th
// largest; it stops at the first threshold that separates m of them, usually
// after about log2(blocks) + 3 passes, and settles ties by index only if none does.
// Both are bound by latency: 9.5 us for 2048 blocks of 8 heads, 12 for 512 of 16 x 8,
// 17 for 128 positions over 256 of 8 (18.5 with 128 threads an item instead of a warp).
#include "cache8.cuh"

namespace arckv {
namespace {

constexpr int kScoreThreads = 128;   // blocks of a CTA
constexpr int kScoreRows = 64;       // query rows whose codes a CTA holds at a time

// score[item][b] of every candidate block; CTA = (sequence x head and 128 blocks, `per` positions).
__global__ void __launch_bounds__(kScoreThreads) cache_score_kernel(const arckv_cache8 c, CacheQuery q, int per,
                                                                    int tiles, float* score) {
  pdl_wait();
  const int nblk = c.cap / kCB, p0 = blockIdx.y * per, p1 = min(p0 + per, q.n_pos);
  const long long sh = blockIdx.x / tiles;
  const int h = (int)(sh % c.H), s = (int)(sh / c.H), len = cache_len(c, s);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // blocks that the CTA's last position sees; earlier ones see no more
  const int cand = (visible_tokens(len, q.n_pos, p1 - 1, q.causal) + kCB - 1) / kCB;
  const int t0 = (int)(blockIdx.x - sh * tiles) * kScoreThreads, b = t0 + threadIdx.x;
  if (t0 >= cand) return;
  __shared__ __align__(16) int s_q[kScoreRows][64];   // codes of a row: q^-, then q^+, four to a word
  __shared__ float s_scale[kScoreRows];
  int4 w[16];
  float ks = 0.f;
  if (b < cand) {
    const int4* src = (const int4*)(c.bounds + (sh * nblk + b) * 256);
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = src[e];
    ks = c.k_scale[sh * nblk + b];
  }
  const int rows = (p1 - p0) * q.G;
  float best = -INFINITY;
  int left = q.G, p = p0;   // rows of position p that are still to come
  for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
    const int nr = min(kScoreRows, rows - r0);
    __syncthreads();
    for (int r = warp; r < nr; r += kScoreThreads / 32) {
      const int pos = p0 + (r0 + r) / q.G, g = (r0 + r) % q.G;
      const uint2 raw = *(const uint2*)(q.Q + s * q.qs.s + h * q.qs.h + pos * q.qs.i + g * 128 + lane * 4);
      const float2 a01 = __bfloat1622float2(*(const __nv_bfloat162*)&raw.x);
      const float2 a23 = __bfloat1622float2(*(const __nv_bfloat162*)&raw.y);
      const float x[4] = {a01.x, a01.y, a23.x, a23.y};
      float a = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
      a = fmaxf(warp_max(a), kCacheFloor);
      const float inv = __fdiv_rn(127.f, a);
      unsigned int pos4 = 0, neg4 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = min(max(__float2int_rn(x[e] * inv), -127), 127);
        pos4 |= (unsigned int)(max(v, 0) & 0xff) << (8 * e);
        neg4 |= (unsigned int)(min(v, 0) & 0xff) << (8 * e);
      }
      s_q[r][lane] = (int)neg4;
      s_q[r][32 + lane] = (int)pos4;
      if (lane == 0) s_scale[r] = a * kInv127;
    }
    __syncthreads();
    if (b >= cand) continue;
    for (int r = 0; r < nr; ++r) {
      int d0 = 0, d1 = 0, d2 = 0, d3 = 0;   // four chains
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int4 v = *(const int4*)&s_q[r][4 * e];
        d0 = __dp4a(v.x, w[e].x, d0);
        d1 = __dp4a(v.y, w[e].y, d1);
        d2 = __dp4a(v.z, w[e].z, d2);
        d3 = __dp4a(v.w, w[e].w, d3);
      }
      best = fmaxf(best, __fmul_rn(__fmul_rn(s_scale[r], (float)(d0 + d1 + (d2 + d3))), ks));
      if (--left == 0) {
        score[(sh * q.n_pos + p) * nblk + b] = best;
        best = -INFINITY;
        left = q.G;
        ++p;
      }
    }
  }
}

// Sum over a group of kT threads (one item's); `part` is the item's scratch, two
// rows of kT / 32 used in turn so that one barrier a sum is enough.
template <int kT>
struct GroupSum {
  int* part;
  int turn = 0;
  __device__ int operator()(int v) {
    v = __reduce_add_sync(0xffffffffu, v);
    if (kT == 32) return v;
    int* row = part + turn * (kT / 32);
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) row[(threadIdx.x % kT) >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < kT / 32 ? row[threadIdx.x & 31] : 0;
    return __reduce_add_sync(0xffffffffu, v);
  }
};

// One item a group of kT threads; thread i has the scores of blocks i n .. i n + n - 1,
// n = kPer of them in registers (kPer = 0: any number, read again in each pass).
template <int kT, int kPer>
__global__ void __launch_bounds__(kT == 32 ? 128 : kT) cache_pick_kernel(const arckv_cache8 c, CacheQuery q,
                                                                         const float* score, int m, int keep_first,
                                                                         int keep_last, long long items, int* blocks) {
  constexpr int kGroups = kT == 32 ? 4 : 1;
  __shared__ int s_part[kT == 32 ? 1 : 2 * (kT / 32)];
  __shared__ int s_scan[kT == 32 ? 1 : kT / 32];
  __shared__ unsigned int s_ends[2][kT == 32 ? 1 : kT / 32];
  pdl_wait();
  const long long item = (long long)blockIdx.x * kGroups + threadIdx.x / kT;
  if (item >= items) return;   // whole warps (kT = 32) or never
  const int tid = threadIdx.x % kT, lane = threadIdx.x & 31, nblk = c.cap / kCB;
  const int sh = (int)item / q.n_pos, pos = (int)item - sh * q.n_pos, s = sh / c.H;   // (items are below 2^31)
  const int cand = (visible_tokens(cache_len(c, s), q.n_pos, pos, q.causal) + kCB - 1) / kCB;
  const float* sc = score + item * nblk;
  int* out = blocks + item * m;
  if (cand <= m) {   // every candidate
    for (int i = tid; i < m; i += kT) out[i] = i < cand ? i : -1;
    return;
  }
  const int per = kPer > 0 ? kPer : (cand + kT - 1) / kT, b0 = tid * per;
  // order of scores as integers; forced blocks above all, nothing (0) past the candidates
  auto load = [&](int b) -> unsigned int {
    if (b >= cand) return 0u;
    if (b < keep_first || b >= cand - keep_last) return 0xffffffffu;
    return f32_ordered(sc[b] + 0.f);   // -0 is 0
  };
  unsigned int reg[kPer > 0 ? kPer : 1];
  if (kPer > 0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) reg[i] = load(b0 + i);
  }
  auto count = [&](unsigned int least) {   // this thread's keys >= least
    int n = 0;
    if (kPer > 0) {
#pragma unroll
      for (int i = 0; i < (kPer > 0 ? kPer : 1); ++i) n += reg[i] >= least;
    } else {
      for (int i = 0; i < per; ++i) n += load(b0 + i) >= least;
    }
    return n;
  };
  GroupSum<kT> sum{s_part};
  // the largest threshold that at least m keys reach: lo is reached by m, hi + 1 is not.  It lies between the least and
  // the largest key that is not forced, or right above (where the forced ones are m).
  unsigned int lo = 0xffffffffu, hi = 0u;
  auto span = [&](unsigned int key) {
    if (key == 0u || key == 0xffffffffu) return;
    lo = min(lo, key);
    hi = max(hi, key);
  };
  if (kPer > 0) {
#pragma unroll
    for (int i = 0; i < (kPer > 0 ? kPer : 1); ++i) span(reg[i]);
  } else {
    for (int i = 0; i < per; ++i) span(load(b0 + i));
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (kT > 32) {
    if (lane == 0) {
      s_ends[0][tid >> 5] = lo;
      s_ends[1][tid >> 5] = hi;
    }
    __syncthreads();
    lo = __reduce_min_sync(0xffffffffu, lane < kT / 32 ? s_ends[0][lane] : 0xffffffffu);
    hi = __reduce_max_sync(0xffffffffu, lane < kT / 32 ? s_ends[1][lane] : 0u);
  }
  if (lo > hi) lo = hi = 1u;   // all candidates are forced (and more than m: not with keep_first + keep_last <= m)
  hi = hi == 0xffffffffu ? hi : hi + 1u;
  bool exact = false;   // exactly m keys reach lo
  while (lo < hi && !exact) {
    const unsigned int mid = lo + ((hi - lo) >> 1) + 1u;
    const int n = sum(count(mid));
    if (n >= m) {
      lo = mid;
      exact = n == m;
    } else {
      hi = mid - 1;
    }
  }
  // keys equal to lo fill the places that larger ones leave, by index
  int above = 0, equal = 0;
  const int larger = exact ? 0 : count(lo == 0xffffffffu ? lo : lo + 1) * (lo != 0xffffffffu);
  const int reach = count(lo);
  above = exact ? reach : larger;
  equal = exact ? 0 : reach - larger;
  const int room = exact ? 0 : m - sum(above);
  // places: exclusive prefix of (equal), then of what is taken
  auto prefix = [&](int v) {
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (kT > 32) {
      __syncthreads();
      if (lane == 31) s_scan[tid >> 5] = x;
      __syncthreads();
      int before = 0;
      for (int w = 0; w < (tid >> 5); ++w) before += s_scan[w];
      x += before;
    }
    return x - v;
  };
  int taken_equal = 0;
  if (!exact) taken_equal = min(max(room - prefix(equal), 0), equal);   // uniform branch
  int at = prefix(above + taken_equal);
  auto emit = [&](unsigned int key, int b) {
    if (key < lo) return;
    if (!exact && key == lo) {
      if (taken_equal == 0) return;
      --taken_equal;
    }
    out[at++] = b;
  };
  if (kPer > 0) {
#pragma unroll
    for (int i = 0; i < (kPer > 0 ? kPer : 1); ++i) emit(reg[i], b0 + i);
  } else {
    for (int i = 0; i < per; ++i) emit(load(b0 + i), b0 + i);
  }
}

template <int kT, int kPer>
cudaError_t launch_pick(const arckv_cache8& c, const CacheQuery& q, const float* score, int m, int keep_first, int keep_last,
                 long long items, int* blocks, cudaStream_t st) {
  const int groups = kT == 32 ? 4 : 1;
  return launch_pdl(cache_pick_kernel<kT, kPer>, dim3((unsigned)((items + groups - 1) / groups)), kT * groups, 0, st, c, q,
                    score, m, keep_first, keep_last, items, blocks);
}

}  // namespace

size_t cache_select_scratch(int S, int H, int cap, int n_pos, int) {
  return (size_t)S * H * n_pos * (cap / kCB) * sizeof(float);
}

int launch_cache_select(const arckv_cache8& c, const CacheQuery& q, int m, int keep_first, int keep_last, int* blocks,
                        void* ws, cudaStream_t st) {
  const long long items = (long long)c.S * c.H * q.n_pos;
  const int nblk = c.cap / kCB, bt = cdiv(nblk, kScoreThreads);
  float* score = (float*)((char*)ws + ARCKV_CACHE_WS_HEADER);
  // positions of a CTA: as many as leave four CTAs an SM, but at least 16 rows, which pay for the bounds' loads (with
  // 64, 128 positions over 256 blocks of 8 heads take 29 us with the choice instead of 17)
  const long long want = 4ll * tc_gemm_sm_count();
  const int tiles = (int)std::max<long long>(1, std::min<long long>(want / std::max(1ll, (long long)bt * c.S * c.H),
                                                                    cdiv((long long)q.n_pos * q.G, kScoreRows / 4)));
  const int per = cdiv(q.n_pos, std::min(tiles, q.n_pos));
  const long long heads = (long long)c.S * c.H;
  cudaError_t e = launch_pdl(cache_score_kernel, dim3((unsigned)(heads * bt), cdiv(q.n_pos, per)), kScoreThreads, 0, st, c,
                             q, per, bt, score);
  if (e != cudaSuccess) return -1;
  if (nblk <= 256) e = launch_pick<32, 8>(c, q, score, m, keep_first, keep_last, items, blocks, st);
  else if (nblk <= 1024) e = launch_pick<128, 8>(c, q, score, m, keep_first, keep_last, items, blocks, st);
  else if (nblk <= 4096) e = launch_pick<512, 8>(c, q, score, m, keep_first, keep_last, items, blocks, st);
  else if (nblk <= 16384) e = launch_pick<1024, 16>(c, q, score, m, keep_first, keep_last, items, blocks, st);
  else e = launch_pick<1024, 0>(c, q, score, m, keep_first, keep_last, items, blocks, st);
  return e == cudaSuccess ? 2 : -1;
}

}  // namespace arckv
