// The write of rows into the 8-bit cache, for the kernels that store them as they are and turned.
#pragma once

#include "cache.h"

namespace bdkv {
namespace {

constexpr int WRITE_THREADS = 256;
constexpr int HALF = WRITE_THREADS / 2;  // threads of a tensor
constexpr int MAX_PAGE = 256;
constexpr int HELD = 8;  // rows of a thread that stay in registers

struct WriteArgs {
  bdkv_cache c;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_tok, k_head, v_tok, v_head;
  const int64_t* slots;
  int64_t n_tokens, n_slots;
  int shift, chunk;
};

// The arguments of a write, and how many CTAs it takes.
inline WriteArgs write_args(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                            int64_t n_tokens, int sm_count, int64_t* grid) {
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
  *grid = (n_tokens + a.chunk - 1) / a.chunk * c.n_heads;
  return a;
}

#ifdef __CUDACC__
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

// The largest magnitude pattern of eight elements, in each half of a word.
__device__ __forceinline__ uint32_t top_of(uint4 x) { return umax2(umax2(umax2(x.x & 0x7fff7fffu, x.y), x.z), x.w); }

// How eight elements of a row are read: at their address, of row `row`, elements 8 sub and on, of keys (w = 0) or values.
struct PlainRows {
  __device__ __forceinline__ uint4 operator()(const uint16_t* p, int64_t /*row*/, int /*sub*/, int /*w*/) const {
    return *reinterpret_cast<const uint4*>(p);
  }
};

template <class T, class Rows>
__device__ __forceinline__ void write_rows(const WriteArgs& a, const Rows& rows_of, uint32_t block) {
  // the patterns of infinities and NaN are the ones from here on
  constexpr uint32_t INF = std::is_same<T, Bf16>::value ? 0x7f80u : 0x7c00u;
  __shared__ int64_t sl[MAX_PAGE + 64 + MAX_PAGE];  // slots, from page_size rows before the chunk to as many behind
  __shared__ uint32_t top[2][2][HALF / 32];         // of the runs in turn: the tensors' warps' largest patterns
  __shared__ uint8_t bad[MAX_PAGE];                 // a run's rows with something that is not finite
  // heads vary fastest: the CTAs that run together then read whole rows
  const int tid = threadIdx.x, lane = tid & 31, h = static_cast<int>(block % a.c.n_heads);
  const int w = tid / HALF, page_size = a.c.page_size;  // w: 0 keys, 1 values
  const int64_t r0 = static_cast<int64_t>(block / a.c.n_heads) * a.chunk, first = r0 - page_size;
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
      return live && there(t) ? rows_of(src + t * tok, first + at + t, sub, w) : make_uint4(0, 0, 0, 0);
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
#endif

}  // namespace
}  // namespace bdkv
