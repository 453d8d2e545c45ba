// Internal interface of libbdcache: what the entry points (cache_api.cu) hand
// the kernel translation units, and the device helpers they share.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "bdcache.h"
#include "common.cuh"

namespace bdkv {

constexpr int E_MIN = 27, E_MAX = 247;  // E8M0 bytes a write stores (2^-100 .. 2^120)
constexpr int MAX_SEQ_TABLES = 8192;

cudaError_t launch_tables(const bdkv_tables_args& a, int sm_count, cudaStream_t st);
cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, int sm_count, cudaStream_t st);

// What the attention kernels read of one call.
struct AttnArgs {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* ks;
  const uint8_t* vs;
  int64_t k_page, k_tok, k_head, v_page, v_tok, v_head, ks_page, vs_page;
  int64_t n_pages;
  int page_shift, dim, n_kv, group;  // group: query heads per key/value head
  const void* q;
  int64_t q_tok, q_head;
  void* out;
  int64_t o_tok, o_head;
  float* lse;
  const int32_t* table;
  int64_t table_stride;
  int max_blocks;
  const int32_t* kv_lens;
  const int32_t* q_start;
  int n_seq, max_q, max_kv, mask_block;
  float coef;  // scale * log2(e)
  bool f16;
};

cudaError_t launch_attn_rows(const AttnArgs& a, int sm_count, cudaStream_t st);

#ifdef __CUDACC__
// 2^k for whole k in -126..127.
__device__ __forceinline__ float pow2i(int k) { return __int_as_float((k + 127) << 23); }

// E8M0 byte of the smallest power of two that brings amax (finite, >= 0) to at
// most 448 = 1.75 * 2^8, within the bytes a write stores.
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = static_cast<int>(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, E_MIN), E_MAX);
}

// The 16-bit element types of rows.
struct Bf16 {
  static __device__ __forceinline__ float2 to_float2(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t from_float2(float2 x) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
};
struct F16 {
  static __device__ __forceinline__ float2 to_float2(uint32_t x) {
    return __half22float2(*reinterpret_cast<const __half2*>(&x));
  }
  static __device__ __forceinline__ uint32_t from_float2(float2 x) {
    const __half2 h = __floats2half2_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
__device__ __forceinline__ uint32_t f16x2(float2 x) { return F16::from_float2(x); }

// One request's lengths, cut to the call's bounds.
struct Seq {
  int q0, q_len, kv_len, shown;  // shown: kv_len - the request's whole q_len, what its first query has before it
};
__device__ __forceinline__ Seq load_seq(const AttnArgs& a, int s) {
  Seq r;
  r.q0 = a.q_start[s];
  const int q_len = max(a.q_start[s + 1] - r.q0, 0);
  r.q_len = min(q_len, a.max_q);
  const int kv = max(a.kv_lens[s], 0);
  r.shown = kv - q_len;
  r.kv_len = min(kv, a.max_kv);
  return r;
}
// Tokens that query i of the request sees.
__device__ __forceinline__ int visible(const AttnArgs& a, const Seq& s, int q_len_all, int i) {
  if (a.mask_block == 0) return s.kv_len;
  const int64_t end = (static_cast<int64_t>(i) / a.mask_block + 1) * a.mask_block;
  const int n = s.shown + static_cast<int>(end < q_len_all ? end : q_len_all);
  return min(max(n, 0), s.kv_len);
}

// Exponent s with amax * 2^s in [2^14, 2^15), for query rows held in f16: a bf16 element keeps its eight
// significant bits down to 2^-31 of the row's largest.
__device__ __forceinline__ int row_shift(float amax) {
  const int e = static_cast<int>(__float_as_uint(amax) >> 23);  // 0 for subnormals and zero
  return amax > 0.f ? min(max(141 - e, -112), 120) : 0;
}
#endif

}  // namespace bdkv
