// Joins the parts of rows whose cache was split: a warp per row, the parts'
// normalised outputs weighted by 2^(lse_p - max). Reads each partial once.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int WARPS = 4;

template <class T>
__global__ void __launch_bounds__(WARPS * 32) attn_join_kernel(AttnArgs a) {
  const int n_q = a.n_kv * a.group, lane = threadIdx.x & 31;
  const int row = blockIdx.x * WARPS + (threadIdx.x >> 5), seq = blockIdx.y;
  const int i = row / n_q, h = row - i * n_q;
  const Seq sq = load_seq(a, seq);
  if (i >= sq.q_len) return;
  const int vis = visible(a, sq, i);
  if (vis <= a.chunk) return;
  const int n = (vis - 1) / a.chunk + 1, d = lane * 4;
  bd::griddep_wait();

  const int64_t at = ((static_cast<int64_t>(seq) * a.max_q + i) * n_q + h) * a.n_split;
  float top = -INFINITY;
  for (int p = lane; p < n; p += 32) top = fmaxf(top, a.part_l[at + p]);
#pragma unroll
  for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
  const float ref = top == -INFINITY ? 0.f : top;
  float4 o = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    const float w = bd::ex2_approx(a.part_l[at + p] - ref);
    total += w;
    if (d < a.dim) {
      const float4 x = *reinterpret_cast<const float4*>(a.part_o + (at + p) * a.dim + d);
      o.x = fmaf(w, x.x, o.x), o.y = fmaf(w, x.y, o.y), o.z = fmaf(w, x.z, o.z), o.w = fmaf(w, x.w, o.w);
    }
  }
  const float f = total == 0.f ? 0.f : 1.f / total;
  const int64_t tok = static_cast<int64_t>(sq.q0) + i;
  const RowOut dst = {static_cast<uint16_t*>(a.out) + tok * a.o_tok + h * a.o_head, nullptr,
                      a.lse == nullptr ? nullptr : a.lse + tok * n_q + h};
  if (d < a.dim) store4<T>(dst, d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
  if (lane == 0) store_lse(dst, total == 0.f ? -INFINITY : ref + log2f(total));
}

}  // namespace

cudaError_t launch_attn_join(const AttnArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((static_cast<unsigned>(a.max_q) * a.n_kv * a.group + WARPS - 1) / WARPS, a.n_seq);
  cfg.blockDim = dim3(WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];  // scheduled while the parts still run; it waits for them before it reads
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return a.f16 ? cudaLaunchKernelEx(&cfg, attn_join_kernel<F16>, a) : cudaLaunchKernelEx(&cfg, attn_join_kernel<Bf16>, a);
}

}  // namespace bdkv
