// Internal interface of libbdcache: what the entry points (cache_api.cu) hand
// the kernel translation units, and the device helpers they share.
#pragma once

#include <atomic>
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
  bool one_tile;       // of rows to a CTA of the tile kernel
  bool longest_first;  // CTAs take the requests in that order (see ranked_seq)
  float coef;  // scale * log2(e)
  bool f16;
  // Work split along the cache: part p of n_split takes tokens [p chunk, (p + 1) chunk). A row that sees at most `chunk`
  // tokens is written by part 0; of the others each part leaves its output (fp32, divided by its sum of weights) and
  // log2-sum-exp in part_o [row, part, dim] and part_l [row, part], row = (seq max_q + query) n_q + head.
  int chunk, n_split;
  float* part_o;
  float* part_l;
};

constexpr int ROWS_TILE = 16;    // rows of a CTA of the two attention kernels (the second: one or two tiles of as many)
constexpr int TILES_TILE = 128;
cudaError_t launch_attn_rows(const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attn_tiles(const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attn_join(const AttnArgs& a, cudaStream_t st);
// Reads and clears the device status bits of the current device.
cudaError_t tiles_status(cudaStream_t st, uint32_t* bits);

#ifdef __CUDACC__
// Lets `kernel` use `bytes` of dynamic shared memory on the current device, once per device.
template <class K>
cudaError_t allow_smem(K kernel, size_t bytes, std::atomic<bool> (&ready)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || ready[dev].load(std::memory_order_relaxed)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (e == cudaSuccess) ready[dev].store(true, std::memory_order_relaxed);
  return e;
}

// 2^k for whole k in -126..127.
__device__ __forceinline__ float pow2i(int k) { return __int_as_float((k + 127) << 23); }

// E8M0 byte of the smallest power of two that brings amax (finite, >= 0) to at
// most 448 = 1.75 * 2^8, within the bytes a write stores.
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = static_cast<int>(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, E_MIN), E_MAX);
}

// Four E4M3 codes of a word to f16, two words.
__device__ __forceinline__ void decode4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
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

// One request's lengths; q_len and kv_len cut to the call's bounds.
struct Seq {
  int q0, q_len, kv_len;
  int q_all, shown;  // its whole q_len, and what its first query has before it
};
__device__ __forceinline__ Seq make_seq(const AttnArgs& a, int q0, int q1, int kv) {
  Seq r;
  r.q0 = q0;
  r.q_all = max(q1 - q0, 0);
  r.q_len = min(r.q_all, a.max_q);
  r.shown = max(kv, 0) - r.q_all;
  r.kv_len = min(max(kv, 0), a.max_kv);
  return r;
}
__device__ __forceinline__ Seq load_seq(const AttnArgs& a, int s) {
  return make_seq(a, a.q_start[s], a.q_start[s + 1], a.kv_lens[s]);
}
// The request with the nth longest cache (equal ones in their order). With more CTAs than the device runs at once, the
// long ones then start first and the short ones fill up the end. The host does not know the lengths, so each CTA ranks
// them itself, in `lens`, shared memory of MAX_ORDERED + 4 words, free again afterwards.
constexpr int MAX_ORDERED = 256;
template <int THREADS>
__device__ __forceinline__ Seq ranked_seq(const AttnArgs& a, int n, int* lens, int& seq) {
  constexpr int PER = (MAX_ORDERED + THREADS - 1) / THREADS;
  const int n4 = (a.n_seq + 3) / 4 * 4;
  int q0[PER], q1[PER], kv[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int t = threadIdx.x + i * THREADS;
    q0[i] = q1[i] = kv[i] = -1;
    if (t < a.n_seq) {
      kv[i] = max(a.kv_lens[t], 0);
      q0[i] = a.q_start[t];
      q1[i] = a.q_start[t + 1];
    }
    if (t < n4) lens[t] = kv[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int t = threadIdx.x + i * THREADS;
    if (t >= a.n_seq) break;
    int rank = 0;
    for (int u = 0; u < n4; u += 4) {
      const int4 x = *reinterpret_cast<const int4*>(lens + u);
      rank += (x.x > kv[i] - (u < t)) + (x.y > kv[i] - (u + 1 < t)) + (x.z > kv[i] - (u + 2 < t)) +
              (x.w > kv[i] - (u + 3 < t));
    }
    if (rank == n) *reinterpret_cast<int4*>(lens + MAX_ORDERED) = make_int4(t, q0[i], q1[i], kv[i]);
  }
  __syncthreads();
  const int4 x = *reinterpret_cast<const int4*>(lens + MAX_ORDERED);
  __syncthreads();
  seq = x.x;
  return make_seq(a, x.y, x.z, x.w);
}
// Tokens that query i of the request sees (no fewer for a later query).
__device__ __forceinline__ int visible(const AttnArgs& a, const Seq& s, int i) {
  if (a.mask_block == 0) return s.kv_len;
  const int64_t end = (static_cast<int64_t>(i / a.mask_block) + 1) * a.mask_block;
  return min(max(s.shown + static_cast<int>(end < s.q_all ? end : s.q_all), 0), s.kv_len);
}

// Where a part's result for one row goes: the call's outputs, the workspace, or nowhere.
struct RowOut {
  uint16_t* out;  // null: a partial result
  float* o;
  float* l;  // the log-sum-exp (null: none wanted)
};
__device__ __forceinline__ RowOut row_out(const AttnArgs& a, const Seq& s, int seq, int part, int i, int h, int vis) {
  RowOut r = {nullptr, nullptr, nullptr};
  const int64_t n_q = static_cast<int64_t>(a.n_kv) * a.group, tok = static_cast<int64_t>(s.q0) + i;
  if (vis <= a.chunk) {
    if (part == 0) {
      r.out = static_cast<uint16_t*>(a.out) + tok * a.o_tok + h * a.o_head;
      if (a.lse != nullptr) r.l = a.lse + tok * n_q + h;
    }
  } else {
    const int64_t at = ((static_cast<int64_t>(seq) * a.max_q + i) * n_q + h) * a.n_split + part;
    r.o = a.part_o + at * a.dim;
    r.l = a.part_l + at;
  }
  return r;
}
template <class T>
__device__ __forceinline__ void store4(const RowOut& r, int d, float4 x) {
  if (r.out != nullptr)
    *reinterpret_cast<uint2*>(r.out + d) =
        make_uint2(T::from_float2(make_float2(x.x, x.y)), T::from_float2(make_float2(x.z, x.w)));
  else if (r.o != nullptr)
    *reinterpret_cast<float4*>(r.o + d) = x;
}
__device__ __forceinline__ void store_lse(const RowOut& r, float lse2) {
  if (r.l != nullptr) *r.l = r.out != nullptr ? lse2 / bd::LOG2E : lse2;
}

// Exponent s with amax * 2^s in [2^14, 2^15), for query rows held in f16: a bf16 element keeps its eight
// significant bits down to 2^-31 of the row's largest.
__device__ __forceinline__ int row_shift(float amax) {
  const int e = static_cast<int>(__float_as_uint(amax) >> 23);  // 0 for subnormals and zero
  return amax > 0.f ? min(max(141 - e, -112), 120) : 0;
}
#endif

}  // namespace bdkv
