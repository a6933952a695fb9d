// Page tables and slot maps from request lengths.
//
//   need_s = ceil((len_s + c_s) / 64) - ceil(len_s / 64),  the k-th page of a call is free[n_free - 1 - k]
//
// Two prefix sums over the requests (rows and pages) and a search in them for
// every row.  A few hundred bytes decide everything, so each CTA does the sums
// by itself in shared memory and fills its share of the rows from the state
// before the call; the CTA that comes last (a ticket) then writes the new state.
// One launch, bound by its chain of dependent loads.  Measured (CUDA graph): with
// the truncation behind it 5.5 us for 64 requests of a token each, 9.0 for 250
// requests and 16,000 rows (of which the look for missing pages takes 0.5).
#include "pages.cuh"

namespace arckv {
namespace {

constexpr int kTT = 512;       // threads
constexpr int kTRows = 512;    // rows of a CTA, one a thread (250 requests, 16,000 rows: 4.4 us, 6.5 with 2048)

// Exclusive prefix sums of x[0 .. n) in place over the block, at most `most` (sums stay below 2^62); returns the total.
// kTT threads take n / kTT consecutive entries each.
template <typename F>
__device__ __forceinline__ long long block_scan(int n, F value, int* out, int most) {
  __shared__ long long warp_sums[kTT / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = (n + kTT - 1) / kTT;
  const int i0 = min(tid * per, n), i1 = min(i0 + per, n);
  long long sum = 0;
  for (int i = i0; i < i1; ++i) sum += value(i);
  long long x = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    long long w = lane < kTT / 32 ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < kTT / 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    if (lane < kTT / 32) warp_sums[lane] = w;
  }
  __syncthreads();
  long long run = x - sum + (warp > 0 ? warp_sums[warp - 1] : 0);
  for (int i = i0; i < i1; ++i) {
    out[i] = (int)min(run, (long long)most);
    run += value(i);
  }
  const long long total = warp_sums[kTT / 32 - 1];
  __syncthreads();
  if (tid == 0) out[n] = (int)min(total, (long long)most);
  __syncthreads();
  return total;
}

// last i < n with sums[i] <= x (sums ascend from 0)
__device__ __forceinline__ int last_at(const int* sums, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kTT) pages_extend_kernel(const arckv_pages4 p, const int* counts, int N, int* starts,
                                                           int* slots, int* positions) {
  extern __shared__ int sm[];
  const int S = p.S, tid = threadIdx.x;
  int* start = sm;                  // [S + 1] rows before a request, at most N
  int* before = start + S + 1;      // [S + 1] pages before it
  int* len = before + S + 1;        // [S]
  int* take = len + S;              // [S] its count, -1 where it is refused
  __shared__ int s_new, s_last, s_free;
  DevStatus* stt = (DevStatus*)p.state;
  pdl_trigger();
  pdl_wait();
  if (tid == 0) {
    s_new = 0;
    s_free = min(max(p.n_free[0], 0), p.P);
  }
  for (int s = tid; s < S; s += kTT) {
    len[s] = pages_len(p, s);
    take[s] = counts[s];
    if (take[s] < 0) {
      set_status(stt, ARCKV_ERR_INVALID_ARG);
      take[s] = 0;
    }
  }
  __syncthreads();
  block_scan(S, [&](int s) { return take[s]; }, start, 0x7fffffff);
  // requests whose rows and length fit
  auto fits = [&](int s) { return (long long)start[s] + take[s] <= N && (long long)len[s] + take[s] <= (long long)p.M * kPT; };
  auto need = [&](int s) { return fits(s) ? pages_of(len[s] + take[s]) - pages_of(len[s]) : 0; };
  block_scan(S, need, before, 0x7fffffff);
  for (int s = tid; s < S; s += kTT) {
    const int n = need(s);
    if (!fits(s) || (n > 0 && (long long)before[s] + n > s_free)) {
      set_status(stt, ARCKV_ERR_SHAPE);
      take[s] = -1;
    } else if (n > 0) {
      atomicMax(&s_new, before[s] + n);
    }
  }
  __syncthreads();
  auto page_of = [&](int s, int j) {   // page j of request s, which is served
    const int held = pages_of(len[s]);
    return j < held ? p.table[(long long)s * p.M + j] : p.free[s_free - 1 - (before[s] + j - held)];
  };
  const int r0 = blockIdx.x * kTRows, r1 = min(r0 + kTRows, N);
  for (int i = r0 + tid; i < r1; i += kTT) {
    int slot = -1, pos = -1;
    if (i < start[S]) {
      const int s = last_at(start, S, i);   // (requests of no rows come before the one that has row i)
      if (take[s] >= 0) {
        pos = len[s] + i - start[s];
        const int page = page_of(s, pos / kPT);
        if (page >= 0 && page < p.P) slot = page * kPT + pos % kPT;
        else set_status(stt, ARCKV_ERR_INVALID_ARG);
      }
    }
    slots[i] = slot;
    positions[i] = pos;
  }
  // the state, once every CTA has read it
  __syncthreads();
  if (tid == 0) {
    s_last = 1;
    if (gridDim.x > 1) {
      unsigned int* ticket = state_ticket(stt);
      unsigned int t;
      asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(t) : "l"(ticket) : "memory");
      s_last = t == gridDim.x - 1;
      if (s_last) *ticket = 0;
    }
  }
  __syncthreads();
  if (!s_last) return;
  for (int k = tid; k < s_new; k += kTT) {   // new pages: the one whose sum holds k (those that need none come before it)
    const int s = last_at(before, S, k), held = pages_of(len[s]), j = held + k - before[s];
    if (take[s] >= 0) p.table[(long long)s * p.M + j] = p.free[s_free - 1 - k];
  }
  for (int s = tid; s <= S; s += kTT) {
    starts[s] = min(start[s], N);
    if (s < S && take[s] > 0) p.len[s] = len[s] + take[s];
  }
  if (tid == 0) p.n_free[0] = s_free - s_new;
}

__global__ void __launch_bounds__(kTT) pages_truncate_kernel(const arckv_pages4 p, const int* lens) {
  extern __shared__ int sm[];
  const int S = p.S, tid = threadIdx.x;
  int* before = sm;               // [S + 1] pages given back before a request
  int* keep = before + S + 1;     // [S] pages that it keeps
  int* back = keep + S;           // [S] pages that it gives back
  DevStatus* stt = (DevStatus*)p.state;
  pdl_trigger();
  pdl_wait();
  const int n_free = min(max(p.n_free[0], 0), p.P);
  for (int s = tid; s < S; s += kTT) {
    const int len = pages_len(p, s);
    int to = lens[s];
    if (to < 0 || to > len) {
      set_status(stt, ARCKV_ERR_INVALID_ARG);
      to = len;
    }
    keep[s] = pages_of(to);
    back[s] = pages_of(len) - keep[s];
    p.len[s] = to;
  }
  __syncthreads();
  const int total = (int)min(block_scan(S, [&](int s) { return back[s]; }, before, 0x7fffffff), (long long)0x7fffffff);
  const int room = p.P - n_free;   // more pages than the pool has are not given back (a damaged table)
  auto entry_of = [&](int k) {
    const int s = last_at(before, S, k);
    return p.table + (long long)s * p.M + keep[s] + k - before[s];
  };
  // Entries without a page of the pool are passed over.  They are rare: all are looked at first, a thread's first one kept.
  int first = -1, held = 0;
  bool rare = total > room;
  for (int k = tid; k < total; k += kTT) {
    const int page = *entry_of(k);
    if (k == tid) first = page;
    if (page >= p.P) set_status(stt, ARCKV_ERR_INVALID_ARG);
    if (page >= 0 && page < p.P) ++held;
    else rare = true;
  }
  if (!__syncthreads_or(rare)) {
    for (int k = tid; k < total; k += kTT) {
      int* entry = entry_of(k);
      p.free[n_free + total - 1 - k] = k == tid ? first : *entry;
      *entry = -1;
    }
    if (tid == 0) p.n_free[0] = n_free + total;
    return;
  }
  __shared__ int s_held, s_warp[kTT / 32];
  if (tid == 0) s_held = 0;
  __syncthreads();
  atomicAdd(&s_held, held);
  __syncthreads();
  const int n = min(s_held, room), lane = tid & 31, warp = tid >> 5;
  if (tid == 0 && s_held > room) set_status(stt, ARCKV_ERR_INVALID_ARG);
  int done = 0;   // pages of earlier rounds
  for (int k0 = 0; k0 < total; k0 += kTT) {
    const int k = k0 + tid;
    int* entry = k < total ? entry_of(k) : nullptr;
    const int page = entry ? *entry : -1;
    const bool held_one = page >= 0 && page < p.P;
    const unsigned int mine = __ballot_sync(0xffffffffu, held_one);
    if (lane == 0) s_warp[warp] = __popc(mine);
    __syncthreads();
    int at = done + __popc(mine & ((1u << lane) - 1u));
    for (int w = 0; w < kTT / 32; ++w) {
      if (w < warp) at += s_warp[w];
      done += s_warp[w];
    }
    if (held_one && at < n) p.free[n_free + n - 1 - at] = page;
    if (entry) *entry = -1;
    __syncthreads();
  }
  if (tid == 0) p.n_free[0] = n_free + n;
}

}  // namespace

int launch_pages_extend(const arckv_pages4& p, const int* counts, int N, int* starts, int* slots, int* positions,
                        cudaStream_t st) {
  const int smem = (4 * p.S + 2) * (int)sizeof(int);
  if (set_dyn_smem((const void*)pages_extend_kernel, smem) != cudaSuccess) return -1;
  const int ctas = std::max(1, cdiv(N, kTRows));
  return launch_pdl(pages_extend_kernel, dim3(ctas), kTT, smem, st, p, counts, N, starts, slots, positions) == cudaSuccess
             ? 1 : -1;
}

int launch_pages_truncate(const arckv_pages4& p, const int* lens, cudaStream_t st) {
  const int smem = (3 * p.S + 1) * (int)sizeof(int);
  if (set_dyn_smem((const void*)pages_truncate_kernel, smem) != cudaSuccess) return -1;
  return launch_pdl(pages_truncate_kernel, dim3(1), kTT, smem, st, p, lens) == cudaSuccess ? 1 : -1;
}

}  // namespace arckv
