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

constexpr int HALF = WRITE_THREADS / 2;  // threads of a tensor
constexpr int MAX_PAGE = 256;
constexpr int HELD = 8;  // rows of a thread that stay in registers

template <class T>
__global__ void __launch_bounds__(WRITE_THREADS, 4) write_kernel(WriteArgs a) {
  // the patterns of infinities and NaN are the ones from here on
  constexpr uint32_t INF = std::is_same<T, Bf16>::value ? 0x7f80u : 0x7c00u;
  __shared__ int64_t sl[MAX_PAGE + 64 + MAX_PAGE];  // slots, from page_size rows before the chunk to as many behind
  __shared__ uint32_t top[2][2][HALF / 32];         // of the runs in turn: the tensors' warps' largest patterns
  __shared__ uint8_t bad[MAX_PAGE];                 // a run's rows with something that is not finite
  // heads vary fastest: the CTAs that run together then read whole rows
  const int tid = threadIdx.x, lane = tid & 31, h = static_cast<int>(blockIdx.x % a.c.n_heads);
  const int w = tid / HALF, page_size = a.c.page_size;  // w: 0 keys, 1 values
  const int64_t r0 = static_cast<int64_t>(blockIdx.x / a.c.n_heads) * a.chunk, first = r0 - page_size;
  for (int i = tid; i < 2 * page_size + a.chunk; i += WRITE_THREADS) {
    const int64_t r = first + i;
    const int64_t s = r >= 0 && r < a.n_tokens ? a.slots[r] : -1;
    sl[i] = s < a.n_slots ? s : -1;
  }
  __syncthreads();
  uint64_t starts = 0;  // rows of the chunk that start a run
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int t = part * 32 + lane;
    const int64_t s = t < a.chunk ? sl[page_size + t] : -1;
    bool begins = s >= 0;
    if (begins) {
      const int off = static_cast<int>(s & (page_size - 1));
      int d = 1;  // to the row before that is stored at all
      while (d <= off && sl[page_size + t - d] < 0) ++d;
      begins = d > off || sl[page_size + t - d] != s - d;
    }
    starts |= static_cast<uint64_t>(__ballot_sync(~0u, begins)) << (part * 32);
  }

  // a thread's eight elements of every step-th row
  const int per_row = a.c.head_dim <= 32 ? 4 : a.c.head_dim <= 64 ? 8 : 16;
  const int step = HALF / per_row, sub = tid % per_row, mine = tid % HALF / per_row;
  const bool live = sub * 8 < a.c.head_dim;
  const int64_t tok = w == 0 ? a.k_tok : a.v_tok;
  const uint16_t* rows = (w == 0 ? a.k + h * a.k_head : a.v + h * a.v_head) + first * tok + sub * 8;
  const int64_t* stride = w == 0 ? a.c.k_stride : a.c.v_stride;
  uint8_t* codes = (w == 0 ? a.c.k : a.c.v) + h * stride[2] + sub * 8;
  const int64_t cell = stride[1];
  for (int run = 0; starts != 0; starts &= starts - 1, run ^= 1) {
    const int at = page_size + __ffsll(static_cast<long long>(starts)) - 1;
    const int64_t slot = sl[at], page = slot >> a.shift;
    const int off = static_cast<int>(slot & (page_size - 1)), n = page_size - off;
    const uint16_t* src = rows + at * tok;
    uint8_t* scale = w == 0 ? a.c.k_scale + page * a.c.k_scale_stride + h : a.c.v_scale + page * a.c.v_scale_stride + h;
    const auto there = [&](int t) { return t < n && sl[at + t] == slot + t; };
    const auto read = [&](int t) {
      return live && there(t) ? *reinterpret_cast<const uint4*>(src + t * tok) : make_uint4(0, 0, 0, 0);
    };
    const int before = off != 0 ? *scale : 0;

    uint4 held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = read(mine + i * step);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) most = __vmaxu2(most, top_of(held[i]));
    for (int t = mine + HELD * step; t < n; t += step) most = __vmaxu2(most, top_of(read(t)));
    most = max(most & 0xffffu, most >> 16);
    const uint32_t warp_top = __reduce_max_sync(~0u, most);
    if (lane == 0) top[run][w][tid % HALF / 32] = warp_top;
    const bool some_bad = __syncthreads_or(most >= INF);
    if (some_bad) {  // such rows do not count for either tensor's scale: find them, and the largest of the others
      for (int t = tid; t < n; t += WRITE_THREADS) bad[t] = 0;
      __syncthreads();
      for (int t = mine; t < n; t += step) {
        const uint32_t m = top_of(read(t));
        if ((m & 0xffffu) >= INF || (m >> 16) >= INF) bad[t] = 1;
      }
      __syncthreads();
      most = 0;
      for (int t = mine; t < n; t += step)
        if (!bad[t]) most = __vmaxu2(most, top_of(read(t)));
      const uint32_t good_top = __reduce_max_sync(~0u, max(most & 0xffffu, most >> 16));
      if (lane == 0) top[run][w][tid % HALF / 32] = good_top;
      __syncthreads();
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < HALF / 32; ++i) m = max(m, top[run][w][i]);
    const int e = max(scale_byte(T::to_float2(m).x), before);
    uint8_t* dst = codes + page * stride[0];
    const float f = pow2i(127 - e);
    const auto write = [&](int t, uint4 x) {
      uint2 y = {e4m3x4(scaled(T::to_float2(x.x), f), scaled(T::to_float2(x.y), f)),
                 e4m3x4(scaled(T::to_float2(x.z), f), scaled(T::to_float2(x.w), f))};
      if (some_bad && bad[t]) y.x = y.y = w == 0 ? 0x7f7f7f7fu : 0u;
      *reinterpret_cast<uint2*>(dst + (off + t) * cell) = y;
    };
    if (live) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (there(mine + i * step)) write(mine + i * step, held[i]);
      for (int t = mine + HELD * step; t < n; t += step)
        if (there(t)) write(t, read(t));
      if (off != 0 && e > before) {  // the tokens that the page holds already
        const float g = before - e < -126 ? 0.f : pow2i(before - e);
        for (int t = mine; t < off; t += step) {
          uint2* p = reinterpret_cast<uint2*>(dst + t * cell);
          const uint2 x = *p;
          uint32_t y[4];
          decode4(x.x, y[0], y[1]);
          decode4(x.y, y[2], y[3]);
          *p = make_uint2(e4m3x4(scaled(F16::to_float2(y[0]), g), scaled(F16::to_float2(y[1]), g)),
                          e4m3x4(scaled(F16::to_float2(y[2]), g), scaled(F16::to_float2(y[3]), g)));
        }
      }
    }
    if (tid % HALF == 0 && e != before) *scale = static_cast<uint8_t>(e);  // (read by all before the barrier above)
    if (some_bad) __syncthreads();  // `bad` is free again; `top` alternates
  }
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
