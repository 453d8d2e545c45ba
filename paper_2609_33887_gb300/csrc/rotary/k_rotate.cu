// bdrot_rotate: rows of queries or keys turned by their positions.
//
// A thread takes eight pairs of a token (16 elements, two 16-byte loads) and goes through a group of heads with their
// sines and cosines in registers. Bound by the bytes moved: 131072 tokens of 32 heads of 128 take 307 us, 7.0 TB/s (a copy
// 6.8); 64 tokens 4.2 us (replayed from a graph), latency.
#include "rotary/rotary.cuh"

namespace bdrot {
namespace {

template <class T>
__global__ void __launch_bounds__(ROTATE_THREADS) rotate_kernel(RotateArgs a) {
  rotate_rows<T, 4>(a, blockIdx.x, threadIdx.x);
}

}  // namespace

RotateArgs rotate_args(const bdkv_rows& x, const bdkv_rows& out, int n_heads, int head_dim, const Turn& turn,
                       int64_t n_tokens, int sm_count, int64_t* blocks) {
  RotateArgs a = {};
  a.turn = turn;
  a.x = static_cast<const uint16_t*>(x.data), a.x_tok = x.stride_token, a.x_head = x.stride_head;
  a.out = static_cast<uint16_t*>(out.data), a.o_tok = out.stride_token, a.o_head = out.stride_head;
  a.n_tokens = n_tokens, a.n_heads = n_heads, a.units = head_dim / 16;
  a.in_place = x.data == out.data;
  // heads of a thread: as many as leave two blocks to each SM
  const int tokens = ROTATE_THREADS / a.units;
  const int64_t spans = (n_tokens + tokens - 1) / tokens;
  a.per = 8;
  while (a.per > 1 && spans * ((n_heads + a.per - 1) / a.per) < 2 * sm_count) a.per /= 2;
  a.groups = (n_heads + a.per - 1) / a.per;
  *blocks = spans * a.groups;
  return a;
}

cudaError_t launch_rotate(const RotateArgs& a, int64_t blocks, bool f16, cudaStream_t st) {
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  if (f16)
    rotate_kernel<F16><<<static_cast<unsigned>(blocks), ROTATE_THREADS, 0, st>>>(a);
  else
    rotate_kernel<Bf16><<<static_cast<unsigned>(blocks), ROTATE_THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace bdrot
