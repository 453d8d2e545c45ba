// Joins the parts of rows whose cache was split: the parts' normalised outputs
// weighted by their sums of weights, brought to one reference. A CTA takes a row, a thread four dims of it.
#include "rotary/latent.h"

namespace bdrot {
namespace {

constexpr int THREADS = 128, AHEAD = 8;

template <class T>
__global__ void __launch_bounds__(THREADS) latent_join_kernel(bdkv::AttnArgs a) {
  const int row = blockIdx.x, seq = blockIdx.y, i = row / a.group, h = row - i * a.group, lane = threadIdx.x & 31;
  const bdkv::Seq sq = bdkv::load_seq(a, seq);
  const int vis = i < sq.q_len ? bdkv::visible(a, sq, i) : 0;
  if (vis <= a.chunk) return;  // part 0 has written the row
  const int n = (vis - 1) / a.chunk + 1, d = threadIdx.x * 4;
  bd::griddep_wait();

  const int64_t at = (static_cast<int64_t>(seq) * a.max_q * a.group + row) * a.n_split;
  const float2* l = reinterpret_cast<const float2*>(a.part_l) + at;  // reference, sum
  const float* src = a.part_o + at * a.dim + d;
  const bool in_row = d < a.dim;
  float top = -INFINITY;
  for (int p = lane; p < n; p += 32) top = fmaxf(top, l[p].x);
#pragma unroll
  for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
  const float ref = top == -INFINITY ? 0.f : top;
  float4 o = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
  for (int p0 = 0; p0 < n; p0 += AHEAD) {
    float4 x[AHEAD];
    float2 w[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int p = p0 + u;
      x[u] = p < n && in_row ? *reinterpret_cast<const float4*>(src + static_cast<int64_t>(p) * a.dim)
                             : make_float4(0.f, 0.f, 0.f, 0.f);
      w[u] = p < n ? l[p] : make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float f = w[u].y * bd::ex2_approx(w[u].x - ref);
      total += f;
      o.x = fmaf(f, x[u].x, o.x), o.y = fmaf(f, x[u].y, o.y), o.z = fmaf(f, x[u].z, o.z), o.w = fmaf(f, x[u].w, o.w);
    }
  }
  const float f = 1.f / total;  // (0 * inf, NaN, where all scores of the row are -inf)
  const int64_t tok = static_cast<int64_t>(sq.q0) + i;
  const bdkv::RowOut dst = {static_cast<uint16_t*>(a.out) + tok * a.o_tok + h * a.o_head, nullptr,
                            a.lse == nullptr ? nullptr : a.lse + tok * a.group + h};
  if (in_row) bdkv::store4<T>(dst, d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
  if (threadIdx.x == 0) bdkv::store_lse(dst, total == 0.f ? -INFINITY : ref + log2f(total));
}

}  // namespace

cudaError_t launch_latent_join(const LatentArgs& p, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.a.max_q) * p.a.group, p.a.n_seq);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];  // scheduled while the parts still run; it waits for them before it reads
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return p.a.f16 ? cudaLaunchKernelEx(&cfg, latent_join_kernel<F16>, p.a)
                 : cudaLaunchKernelEx(&cfg, latent_join_kernel<Bf16>, p.a);
}

}  // namespace bdrot
