// bdkv_write: rows of keys and values into the cache, quantised to E4M3 with a
// power-of-two scale for each page and head.
//
// A CTA takes one head of a few rows (a chunk), and does every run that starts
// among them, to the run's end. A run's rows are read once: they stay in
// registers between the reduction that gives the scale and the conversion
// (64 rows of 128 elements of both tensors; longer runs read the rest again).
// Which rows belong to a run follows from their slots alone: row r0 + t does
// if its slot is the first one's plus t.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int THREADS = 256;
constexpr int WARPS = THREADS / 32;
constexpr int MAX_PAGE = 256;
constexpr int HELD = 4;  // rows of a thread that stay in registers

struct WriteArgs {
  bdkv_cache c;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_tok, k_head, v_tok, v_head;
  const int64_t* slots;
  int64_t n_tokens, n_slots;
  int shift, chunk;
};

__device__ __forceinline__ uint32_t e4m3x4(float2 a, float2 b) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 scaled(float2 x, float f) { return make_float2(x.x * f, x.y * f); }

// Two elements' magnitudes as 16-bit patterns (they order as the values do).
__device__ __forceinline__ uint32_t umax2(uint32_t a, uint32_t b) { return __vmaxu2(a, b & 0x7fff7fffu); }

struct Row {
  uint4 x[2];  // eight elements of the key and of the value
};

// The largest magnitude pattern of eight elements, in each half of a word.
__device__ __forceinline__ uint32_t top_of(uint4 x) { return umax2(umax2(umax2(x.x & 0x7fff7fffu, x.y), x.z), x.w); }

template <class T>
__global__ void __launch_bounds__(THREADS, 4) write_kernel(WriteArgs a) {
  // the patterns of infinities and NaN are the ones from here on
  constexpr uint32_t INF = std::is_same<T, Bf16>::value ? 0x7f80u : 0x7c00u;
  __shared__ int64_t sl[MAX_PAGE + 64 + MAX_PAGE];  // slots of the rows from `page_size` before the chunk to as many behind
  __shared__ uint32_t starts[2];                    // rows of the chunk that start a run
  __shared__ uint32_t top[2][WARPS];
  __shared__ uint8_t bad[MAX_PAGE];  // a run's rows behind the held ones: not finite
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y;
  const int page_size = a.c.page_size;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * a.chunk, first = r0 - page_size;

  for (int i = tid; i < 2 * page_size + a.chunk; i += THREADS) {
    const int64_t r = first + i;
    int64_t s = r >= 0 && r < a.n_tokens ? a.slots[r] : -1;
    sl[i] = s < a.n_slots ? s : -1;
  }
  if (tid < 2) starts[tid] = 0;
  __syncthreads();
  if (tid < a.chunk) {
    const int64_t s = sl[page_size + tid];
    if (s >= 0) {
      const int off = static_cast<int>(s & (page_size - 1));
      int d = 1;  // the row before that is stored at all
      while (d <= off && sl[page_size + tid - d] < 0) ++d;
      if (d > off || sl[page_size + tid - d] != s - d) atomicOr(&starts[tid >> 5], 1u << (tid & 31));
    }
  }
  __syncthreads();

  // a thread's eight elements of every (THREADS / per_row)-th row
  const int per_row = a.c.head_dim <= 32 ? 4 : a.c.head_dim <= 64 ? 8 : 16;
  const int step = THREADS / per_row, sub = tid % per_row, mine = tid / per_row;
  const bool live = sub * 8 < a.c.head_dim;
  const uint32_t group = ((1u << per_row) - 1) << (lane & ~(per_row - 1));
  const int64_t row_of[2] = {a.k_tok, a.v_tok};
  for (int half = 0; half < 2; ++half) {
    for (uint32_t left = starts[half]; left != 0; left &= left - 1) {
      const int at = page_size + half * 32 + __ffs(left) - 1;
      const int64_t slot = sl[at], page = slot >> a.shift;
      const int off = static_cast<int>(slot & (page_size - 1)), n = page_size - off;
      const uint16_t* src[2] = {a.k + (first + at) * a.k_tok + h * a.k_head + sub * 8,
                                a.v + (first + at) * a.v_tok + h * a.v_head + sub * 8};
      uint8_t* scale[2] = {a.c.k_scale + page * a.c.k_scale_stride + h, a.c.v_scale + page * a.c.v_scale_stride + h};
      int before[2] = {0, 0};
      if (off != 0) before[0] = *scale[0], before[1] = *scale[1];

      Row held[HELD];
      bool in[HELD], ok[HELD];
      uint32_t most[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        const int t = mine + i * step;
        in[i] = t < n && sl[at + t] == slot + t;
        held[i] = Row{};
        if (in[i] && live)
#pragma unroll
          for (int w = 0; w < 2; ++w) held[i].x[w] = *reinterpret_cast<const uint4*>(src[w] + t * row_of[w]);
      }
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        const uint32_t m0 = top_of(held[i].x[0]), m1 = top_of(held[i].x[1]);
        const uint32_t m = __vmaxu2(m0, m1);
        const bool fin = (m & 0xffffu) < INF && (m >> 16) < INF;
        ok[i] = (__ballot_sync(~0u, fin) & group) == group;
        if (ok[i]) most[0] = __vmaxu2(most[0], m0), most[1] = __vmaxu2(most[1], m1);
      }
      for (int t = mine + HELD * step; t - mine < n; t += step) {
        const bool there = t < n && sl[at + t] == slot + t;
        Row r{};
        if (there && live)
#pragma unroll
          for (int w = 0; w < 2; ++w) r.x[w] = *reinterpret_cast<const uint4*>(src[w] + t * row_of[w]);
        const uint32_t m0 = top_of(r.x[0]), m1 = top_of(r.x[1]), m = __vmaxu2(m0, m1);
        const bool fine = (__ballot_sync(~0u, (m & 0xffffu) < INF && (m >> 16) < INF) & group) == group;
        if (fine) most[0] = __vmaxu2(most[0], m0), most[1] = __vmaxu2(most[1], m1);
        if (there && sub == 0) bad[t] = !fine;
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t m = __reduce_max_sync(~0u, max(most[w] & 0xffffu, most[w] >> 16));
        if (lane == 0) top[w][warp] = m;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) m = max(m, top[w][i]);
        const int e = max(scale_byte(T::to_float2(m).x), before[w]);
        const int64_t* stride = w == 0 ? a.c.k_stride : a.c.v_stride;
        uint8_t* dst = (w == 0 ? a.c.k : a.c.v) + page * stride[0] + h * stride[2] + sub * 8;
        const float f = pow2i(127 - e);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const int t = mine + i * step;
          if (!in[i] || !live) continue;
          const uint4 x = held[i].x[w];
          uint2 y = {e4m3x4(scaled(T::to_float2(x.x), f), scaled(T::to_float2(x.y), f)),
                     e4m3x4(scaled(T::to_float2(x.z), f), scaled(T::to_float2(x.w), f))};
          if (!ok[i]) y.x = y.y = w == 0 ? 0x7f7f7f7fu : 0u;
          *reinterpret_cast<uint2*>(dst + (off + t) * stride[1]) = y;
        }
        for (int t = mine + HELD * step; t < n; t += step) {
          if (sl[at + t] != slot + t || !live) continue;
          const uint4 x = *reinterpret_cast<const uint4*>(src[w] + t * row_of[w]);
          uint2 y = {e4m3x4(scaled(T::to_float2(x.x), f), scaled(T::to_float2(x.y), f)),
                     e4m3x4(scaled(T::to_float2(x.z), f), scaled(T::to_float2(x.w), f))};
          if (bad[t]) y.x = y.y = w == 0 ? 0x7f7f7f7fu : 0u;
          *reinterpret_cast<uint2*>(dst + (off + t) * stride[1]) = y;
        }
        if (off != 0 && e > before[w]) {  // the tokens that the page holds already
          const float g = before[w] - e < -126 ? 0.f : pow2i(before[w] - e);
          if (live)
            for (int t = mine; t < off; t += step) {
              uint2* p = reinterpret_cast<uint2*>(dst + t * stride[1]);
              const uint2 x = *p;
              const auto two = [&](uint32_t c) { return scaled(F16::to_float2(bd::e4m3x2_to_f16x2(c & 0xffffu)), g); };
              *p = make_uint2(e4m3x4(two(x.x), two(x.x >> 16)), e4m3x4(two(x.y), two(x.y >> 16)));
            }
        }
        if (tid == 0 && e != before[w]) *scale[w] = static_cast<uint8_t>(e);
      }
      __syncthreads();  // `top` and `bad` are free again
    }
  }
}

}  // namespace

cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, int sm_count, cudaStream_t st) {
  WriteArgs a;
  a.c = c;
  a.k = static_cast<const uint16_t*>(k.data);
  a.v = static_cast<const uint16_t*>(v.data);
  a.k_tok = k.stride_token;
  a.k_head = k.stride_head;
  a.v_tok = v.stride_token;
  a.v_head = v.stride_head;
  a.slots = slot_map;
  a.n_tokens = n_tokens;
  a.n_slots = c.n_pages * c.page_size;
  a.shift = 0;
  while ((1 << a.shift) < c.page_size) ++a.shift;
  // rows per CTA: as many as a page (64 at most), fewer while the CTAs would not fill the SMs twice
  a.chunk = c.page_size < 64 ? c.page_size : 64;
  while (a.chunk > 1 && (n_tokens + a.chunk - 1) / a.chunk * c.n_heads < 2 * sm_count) a.chunk /= 2;
  const dim3 grid(static_cast<unsigned>((n_tokens + a.chunk - 1) / a.chunk), static_cast<unsigned>(c.n_heads));
  if (k.dtype == BDKV_BF16)
    write_kernel<Bf16><<<grid, THREADS, 0, st>>>(a);
  else
    write_kernel<F16><<<grid, THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace bdkv
