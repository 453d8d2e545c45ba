// bdkv_tables: block tables, slot map and positions from the requests'
// lengths.
//
// Every output follows from three prefix sums over the requests (tokens added,
// pages needed, pages given back). They are a few thousand additions, so every
// CTA computes all of them for itself in shared memory, which takes one launch
// and no waiting between CTAs; added tokens and pages that change hands are
// then divided evenly among all threads, which find their request by bisection.
// A page just taken is read from the ring again where its token's slot is
// written, so no thread depends on another's block-table stores. Bound by
// latency: two trips to memory and two scans (replayed from a graph: 8 requests
// 3.5 us, 256 of 512 new tokens 5.1 us).
#include "cache.h"

namespace bdkv {
namespace {

constexpr int THREADS = 512;

struct Sums {
  int add, need, give;
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return {a.add + b.add, a.need + b.need, a.give + b.give}; }

struct Request {
  int old, add, held, want_pages, want;  // tokens before, tokens added, pages before and after, tokens after
  bool fits;
  int need, give;
};

__device__ __forceinline__ Request request(const bdkv_tables_args& a, int shift, int s) {
  Request r;
  const int n = a.new_tokens[s], page1 = a.page_size - 1;
  r.old = max(a.lens[s], 0);
  r.add = max(n, 0);
  const int drop = n < 0 ? (n == INT32_MIN ? r.old : min(-n, r.old)) : 0;
  r.want = r.old + r.add - drop;
  r.held = static_cast<int>((static_cast<uint32_t>(r.old) + page1) >> shift);
  r.want_pages = static_cast<int>((static_cast<uint32_t>(r.want) + page1) >> shift);
  r.fits = max(r.held, r.want_pages) <= a.max_blocks;
  r.need = r.fits ? max(r.want_pages - r.held, 0) : 0;
  r.give = r.fits ? max(r.held - r.want_pages, 0) : 0;
  return r;
}

__device__ __forceinline__ Sums warp_scan(Sums v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums o = {__shfl_up_sync(~0u, v.add, d), __shfl_up_sync(~0u, v.need, d), __shfl_up_sync(~0u, v.give, d)};
    if (lane >= d) v = v + o;
  }
  return v;
}

// The last of n entries of `before` (ascending) that is at most i.
template <class F>
__device__ __forceinline__ int last_at_most(F before, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (before(mid) <= i) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Shared memory: starts[n_seq + 1] (tokens added before a request), taken_at[n_seq] (pages needed before it; ~that where it
// is not served), given_at[n_seq] (pages given back before it).
__global__ void __launch_bounds__(THREADS) tables_kernel(bdkv_tables_args a, int shift) {
  extern __shared__ int sh[];
  int* starts = sh;
  int* taken_at = sh + a.n_seq + 1;
  int* given_at = taken_at + a.n_seq;
  __shared__ Sums warp_sum[THREADS / 32];
  __shared__ int taken_sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t head = a.pool_in[0], tail = a.pool_in[1];
  const int R = static_cast<int>(a.ring_size);
  const int64_t avail = min(tail - head, a.ring_size);
  if (tid == 0) taken_sh = 0;

  Sums base = {0, 0, 0};
  for (int s0 = 0; s0 < a.n_seq; s0 += THREADS) {
    const int s = s0 + tid;
    Request r = {};
    if (s < a.n_seq) r = request(a, shift, s);
    const Sums own = {r.add, r.need, r.give};
    Sums inc = warp_scan(own, lane);
    __syncthreads();  // warp_sum of the round before has been read
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    Sums before = base;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before = before + warp_sum[w];
      base = base + warp_sum[w];
    }
    inc = before + inc;
    if (s < a.n_seq) {
      const bool ok = r.fits && (r.need == 0 || inc.need <= avail);
      starts[s] = inc.add - r.add;
      taken_at[s] = ok ? inc.need - r.need : ~(inc.need - r.need);
      given_at[s] = inc.give - r.give;
      if (ok && r.need > 0) atomicMax(&taken_sh, inc.need);
      if (blockIdx.x == 0) {
        a.kv_lens[s] = ok ? r.want : r.old;
        a.query_start[s] = inc.add - r.add;
        a.status[s] = ok ? 0 : r.fits ? 1 : 2;
      }
    }
  }
  const int total = base.add, given = base.give;
  __syncthreads();
  const int taken = taken_sh;
  if (blockIdx.x == 0 && tid == 0) {
    a.query_start[a.n_seq] = total;
    a.pool_out[0] = head + taken;
    a.pool_out[1] = tail + given;
  }
  // ring indices by one remainder each (heads of either sign)
  const int head_at = static_cast<int>((head % R + R) % R), tail_at = static_cast<int>((tail % R + R) % R);
  const auto ring = [&](int at, int i) {  // 0 <= i < R
    const int64_t x = static_cast<int64_t>(at) + i;
    return a.free_pages + (x >= R ? x - R : x);
  };
  const auto pages = [&](int n) { return static_cast<int>((static_cast<uint32_t>(n) + a.page_size - 1) >> shift); };
  const auto taken_before = [&](int s) { return taken_at[s] < 0 ? ~taken_at[s] : taken_at[s]; };
  const int64_t gtid = static_cast<int64_t>(blockIdx.x) * THREADS + tid, threads = static_cast<int64_t>(gridDim.x) * THREADS;

  for (int64_t i = gtid; i < static_cast<int64_t>(taken) + given; i += threads) {
    if (i < taken) {
      const int p = static_cast<int>(i), s = last_at_most(taken_before, a.n_seq, p);
      a.block_table[s * a.table_stride + pages(max(a.lens[s], 0)) + p - taken_before(s)] = *ring(head_at, p);
    } else {
      const int p = static_cast<int>(i - taken), s = last_at_most([&](int k) { return given_at[k]; }, a.n_seq, p);
      const int old = max(a.lens[s], 0), n = a.new_tokens[s];
      const int left = n == INT32_MIN || -n >= old ? 0 : old + n;  // tokens it keeps
      *ring(tail_at, p % R) = a.block_table[s * a.table_stride + pages(left) + p - given_at[s]];
    }
  }
  for (int64_t i = gtid; i < a.max_tokens; i += threads) {
    int64_t slot = -1;
    int pos = -1;
    if (i < total) {
      const int s = last_at_most([&](int k) { return starts[k]; }, a.n_seq, static_cast<int>(i));
      const int old = max(a.lens[s], 0);
      pos = old + static_cast<int>(i) - starts[s];
      if (taken_at[s] >= 0) {
        const int held = pages(old), j = pos >> shift;
        const int page = j < held ? a.block_table[s * a.table_stride + j] : *ring(head_at, taken_at[s] + j - held);
        slot = (static_cast<int64_t>(page) << shift) + (pos & (a.page_size - 1));
      }
    }
    a.slot_map[i] = slot;
    a.positions[i] = pos;
  }
}

}  // namespace

cudaError_t launch_tables(const bdkv_tables_args& a, int sm_count, cudaStream_t st) {
  int shift = 0;
  while ((1 << shift) < a.page_size) ++shift;
  const int64_t work = a.max_tokens > a.n_seq ? a.max_tokens : a.n_seq;
  int64_t grid = (work + THREADS - 1) / THREADS;
  if (grid < 1) grid = 1;
  if (grid > sm_count) grid = sm_count;
  const size_t smem = (3 * static_cast<size_t>(a.n_seq) + 1) * sizeof(int);
  static std::atomic<bool> ready[64];  // by device
  if (smem > 40 * 1024)
    if (cudaError_t e = allow_smem(tables_kernel, (3 * MAX_SEQ_TABLES + 1) * sizeof(int), ready); e != cudaSuccess)
      return e;
  tables_kernel<<<static_cast<unsigned>(grid), THREADS, smem, st>>>(a, shift);
  return cudaGetLastError();
}

}  // namespace bdkv
