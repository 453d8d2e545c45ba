// What the kernels that write rows into the 8-bit cache share, of rows as they are and of keys turned on their way.
#pragma once

#include "cache.h"

namespace bdkv {
namespace {

constexpr int WRITE_THREADS = 256;

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
#endif

}  // namespace
}  // namespace bdkv
