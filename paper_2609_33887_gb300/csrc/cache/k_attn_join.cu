// Joins the parts of rows whose cache was split: the parts' normalised outputs
// weighted by 2^(lse_p - max). One to eight warps take a row, so that a few
// rows of very many parts (a long cache read by one query) are not left to a
// few warps: 64 rows of 147 parts took 71 us with a warp each.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int WARPS = 8;

template <class T>
__global__ void __launch_bounds__(WARPS * 32) attn_join_kernel(AttnArgs a, int per_row) {
  __shared__ float4 sums[WARPS][32];
  __shared__ float totals[WARPS];
  const int n_q = a.n_kv * a.group, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % per_row;
  const int row = blockIdx.x * (WARPS / per_row) + warp / per_row, seq = blockIdx.y;
  const int i = row / n_q, h = row - i * n_q;
  const Seq sq = load_seq(a, seq);
  const int vis = i < sq.q_len ? visible(a, sq, i) : 0;
  const bool mine = vis > a.chunk;  // else part 0 has written the row
  const int n = mine ? (vis - 1) / a.chunk + 1 : 0, d = lane * 4;
  bd::griddep_wait();

  const int64_t at = ((static_cast<int64_t>(seq) * a.max_q + i) * n_q + h) * a.n_split;
  const float* l = a.part_l + at;
  const float* src = a.part_o + at * a.dim + d;
  float top = -INFINITY;
  for (int p = lane; p < n; p += 32) top = fmaxf(top, l[p]);
#pragma unroll
  for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
  const float ref = top == -INFINITY ? 0.f : top;
  float4 o = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
  const bool in_row = d < a.dim;
  for (int p0 = sub; p0 < n; p0 += 8 * per_row) {
    float4 x[8];
    float w[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int p = p0 + u * per_row;
      x[u] = p < n && in_row ? *reinterpret_cast<const float4*>(src + static_cast<int64_t>(p) * a.dim)
                             : make_float4(0.f, 0.f, 0.f, 0.f);
      w[u] = p < n ? l[p] : -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float f = bd::ex2_approx(w[u] - ref);
      total += f;
      o.x = fmaf(f, x[u].x, o.x), o.y = fmaf(f, x[u].y, o.y), o.z = fmaf(f, x[u].z, o.z), o.w = fmaf(f, x[u].w, o.w);
    }
  }
  if (per_row > 1) {
    sums[warp][lane] = o;
    if (lane == 0) totals[warp] = total;
    __syncthreads();
    if (sub != 0) return;
    for (int s = 1; s < per_row; ++s) {
      const float4 x = sums[warp + s][lane];
      o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
      total += totals[warp + s];
    }
  }
  if (!mine) return;
  const float f = 1.f / total;  // (0 * inf, NaN, where all scores of the row are -inf)
  const int64_t tok = static_cast<int64_t>(sq.q0) + i;
  const RowOut dst = {static_cast<uint16_t*>(a.out) + tok * a.o_tok + h * a.o_head, nullptr,
                      a.lse == nullptr ? nullptr : a.lse + tok * n_q + h};
  if (in_row) store4<T>(dst, d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
  if (lane == 0) store_lse(dst, total == 0.f ? -INFINITY : ref + log2f(total));
}

}  // namespace

cudaError_t launch_attn_join(const AttnArgs& a, cudaStream_t st) {
  const int per_row = a.n_split <= 4 ? 1 : a.n_split <= 8 ? 2 : a.n_split <= 16 ? 4 : 8;  // two to four parts a warp, or more
  const int rows = WARPS / per_row;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((static_cast<unsigned>(a.max_q) * a.n_kv * a.group + rows - 1) / rows, a.n_seq);
  cfg.blockDim = dim3(WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];  // scheduled while the parts still run; it waits for them before it reads
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return a.f16 ? cudaLaunchKernelEx(&cfg, attn_join_kernel<F16>, a, per_row)
               : cudaLaunchKernelEx(&cfg, attn_join_kernel<Bf16>, a, per_row);
}

}  // namespace bdkv
