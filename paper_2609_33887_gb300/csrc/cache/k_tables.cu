// bdkv_tables: block tables, slot map and positions from the requests'
// lengths.
//
// Every output follows from three prefix sums over the requests (tokens added,
// pages needed, pages given back). They are a few thousand additions, so every
// CTA computes all of them for itself in shared memory, which takes one launch
// and no waiting between CTAs; the added tokens are then divided evenly among
// the CTAs and the page lists among their warps. A page just taken is read
// from the ring again where its token's slot is written, so no CTA depends on
// another's block-table stores.
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

// Shared memory: starts[n_seq + 1] (tokens before a request), first[n_seq]
// (index of its first new page behind the ring's head, -1: not served).
__global__ void __launch_bounds__(THREADS) tables_kernel(bdkv_tables_args a, int shift) {
  extern __shared__ int sh[];
  int* starts = sh;
  int* first = sh + a.n_seq + 1;
  __shared__ Sums warp_sum[THREADS / 32];
  __shared__ int taken;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t head = a.pool_in[0], tail = a.pool_in[1];
  const int64_t avail = tail - head;
  if (tid == 0) taken = 0;

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
      first[s] = ok ? inc.need - r.need : -1;
      if (ok && r.need > 0) atomicMax(&taken, inc.need);
      if (blockIdx.x == 0) {
        a.kv_lens[s] = ok ? r.want : r.old;
        a.query_start[s] = inc.add - r.add;
        a.status[s] = ok ? 0 : r.fits ? 1 : 2;
      }
      // pages that change hands, a request per thread of one CTA in turn
      if (s % gridDim.x == blockIdx.x) {
        int32_t* row = a.block_table + s * a.table_stride;
        if (ok)
          for (int j = 0; j < r.need; ++j)
            row[r.held + j] = a.free_pages[(head + inc.need - r.need + j) % a.ring_size];
        for (int j = 0; j < r.give; ++j)
          a.free_pages[(tail + inc.give - r.give + j) % a.ring_size] = row[r.want_pages + j];
      }
    }
  }
  const int total = base.add;
  if (tid == 0) starts[a.n_seq] = total;
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    a.query_start[a.n_seq] = total;
    a.pool_out[0] = head + taken;
    a.pool_out[1] = tail + base.give;
  }

  for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + tid; i < a.max_tokens;
       i += static_cast<int64_t>(gridDim.x) * THREADS) {
    int64_t slot = -1;
    int pos = -1;
    if (i < total) {
      int lo = 0, hi = a.n_seq - 1;  // the last request whose tokens start at or before i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= i) lo = mid; else hi = mid - 1;
      }
      const int old = max(a.lens[lo], 0);
      pos = old + static_cast<int>(i) - starts[lo];
      if (first[lo] >= 0) {
        const int held = static_cast<int>((static_cast<uint32_t>(old) + a.page_size - 1) >> shift), j = pos >> shift;
        const int page = j < held ? a.block_table[lo * a.table_stride + j]
                                  : a.free_pages[(head + first[lo] + j - held) % a.ring_size];
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
  const size_t smem = (2 * static_cast<size_t>(a.n_seq) + 1) * sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (2 * MAX_SEQ_TABLES + 1) * sizeof(int));
    if (e != cudaSuccess) return e;
  }
  tables_kernel<<<static_cast<unsigned>(grid), THREADS, smem, st>>>(a, shift);
  return cudaGetLastError();
}

}  // namespace bdkv
