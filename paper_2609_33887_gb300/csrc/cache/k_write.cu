// bdkv_write: rows of keys and values into the cache, quantised to E4M3 with a
// power-of-two scale for each page and head.
//
// A CTA takes one head of a few rows (a chunk), and does every run that starts
// among them, to the run's end: half of its threads the keys, half the values.
// A run's rows are read once: they stay in registers between the reduction
// that gives the scale and the conversion (64 rows of 128 elements; longer
// runs read the rest again). Which rows belong to a run follows from their
// slots alone: row r0 + t does if its slot is the first one's plus t. Bound by
// the bytes moved; few registers (one tensor's pointers to a thread) keep four
// CTAs' loads on their way on an SM. 131072 tokens of 8 heads of 128 take 157 us,
// 5.1 TB/s (0.76 of a copy); 64 tokens 5.4 us (replayed from a graph), latency.
#include "write_rows.cuh"

namespace bdkv {
namespace {

template <class T>
__global__ void __launch_bounds__(WRITE_THREADS, 4) write_kernel(WriteArgs a) {
  write_rows<T>(a, PlainRows(), blockIdx.x);
}

}  // namespace

cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, int sm_count, cudaStream_t st) {
  int64_t grid = 0;
  const WriteArgs a = write_args(c, k, v, slot_map, n_tokens, sm_count, &grid);
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  if (k.dtype == BDKV_BF16)
    write_kernel<Bf16><<<static_cast<unsigned>(grid), WRITE_THREADS, 0, st>>>(a);
  else
    write_kernel<F16><<<static_cast<unsigned>(grid), WRITE_THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace bdkv
