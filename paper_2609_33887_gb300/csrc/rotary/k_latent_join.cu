// Joins the parts of units whose tiles went to several CTAs: the parts'
// normalised outputs weighted by their sums of weights, brought to one reference.
// A warp takes 128 dims of a row; where there are so few of them that the units
// have many parts, eight warps share the parts. Latency: the plan, then all loads
// of a warp at once, then the store; 512 CTAs 7 us, 64 CTAs 5 (from cold caches).
// 16 CTAs to an SM at most, each for several items: with 4, 2 us more for 80 units
// of 64 rows; with a CTA to every eight items, 2 us more where no unit is split.
#include <algorithm>

#include "rotary/latent.h"

namespace bdrot {
namespace {

constexpr int WARPS = 8;

template <class T, bool MANY>
__global__ void __launch_bounds__(WARPS * 32, MANY ? 3 : 4) latent_join_kernel(const LatentArgs p) {
  constexpr int AHEAD = MANY ? 8 : 4;  // parts of a warp that are loaded at once
  const bdkv::AttnArgs& a = p.a;
  __shared__ float4 sums[MANY ? WARPS : 1][32];
  constexpr int STEP = MANY ? WARPS : 1;
  __shared__ float2 totals[WARPS];  // references, sums
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunks = (a.dim + 127) / 128, per_unit = p.rows * chunks, units = a.n_seq * p.row_tiles;
  bd::griddep_wait();
  const bool none = p.plan[units].x < 0;
  for (int item = MANY ? blockIdx.x : blockIdx.x * WARPS + warp; item < units * per_unit;
       item += gridDim.x * (MANY ? 1 : WARPS)) {
    const int unit = item / per_unit, in_unit = item - unit * per_unit;
    const int seq = unit / p.row_tiles, tile = unit - seq * p.row_tiles;
    const int in_tile = in_unit / chunks, c = in_unit - in_tile * chunks, row = tile * p.rows + in_tile;
    const int i = row / a.group, h = row - i * a.group;
    const int2 plan = p.plan[unit];  // (of a unit without rows: anything)
    const bdkv::Seq sq = bdkv::load_seq(a, seq);
    if (none) return;
    if (i >= sq.q_len || plan.x < 0) continue;  // (of all a CTA's threads, where they share the item)
    const int vis = bdkv::visible(a, sq, i);
    const int first = plan.x >> 1, n = plan.y - first + 1;
    const auto part = [&](int k) { return static_cast<int64_t>(k == 0 ? plan.x : 2 * (first + k)) * p.rows + in_tile; };

    const float2* l = reinterpret_cast<const float2*>(a.part_l);  // reference, sum
    const int64_t tok = static_cast<int64_t>(sq.q0) + i;
    const bdkv::RowOut dst = {static_cast<uint16_t*>(a.out) + tok * a.o_tok + h * a.o_head, nullptr,
                              a.lse == nullptr ? nullptr : a.lse + tok * a.group + h};
    const float4 zero = {0.f, 0.f, 0.f, 0.f};
    const auto scaled = [](float4 x, float f) { return make_float4(x.x * f, x.y * f, x.z * f, x.w * f); };
    const auto add = [](float4& o, float f, float4 x) {
      o.x = fmaf(f, x.x, o.x), o.y = fmaf(f, x.y, o.y), o.z = fmaf(f, x.z, o.z), o.w = fmaf(f, x.w, o.w);
    };
    // Sums under the largest reference so far (-inf: nothing yet), as in the attention itself; `by` brings what is held to a
    // new one.
    float ref = -INFINITY, total = 0.f;
    const auto raise = [&](float to) {
      const float most = fmaxf(ref, to), by = most == ref ? 1.f : bd::ex2_approx(ref - most);
      ref = most;
      total *= by;
      return by;
    };
    const auto weight = [&](float2 w) { return ref == -INFINITY ? w.y : w.y * bd::ex2_approx(w.x - ref); };  // (w.y: 0 or NaN)
    const int d = c * 128 + lane * 4;
    float4 o = zero;
    for (int k0 = MANY ? warp : 0; k0 < n; k0 += AHEAD * STEP) {
      float4 x[AHEAD];
      float2 w[AHEAD];
      float most = -INFINITY;
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int k = k0 + u * STEP;
        x[u] = k < n && d < a.dim ? *reinterpret_cast<const float4*>(a.part_o + part(k) * a.dim + d) : zero;
        w[u] = k < n ? l[part(k)] : make_float2(-INFINITY, 0.f);
        most = fmaxf(most, w[u].x);
      }
      o = scaled(o, raise(most));
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const float f = weight(w[u]);
        total += f;
        add(o, f, x[u]);
      }
    }
    if constexpr (MANY) {
      sums[warp][lane] = o;
      if (lane == 0) totals[warp] = make_float2(ref, total);
      __syncthreads();
      if (warp == 0) {
        for (int s = 1; s < WARPS; ++s) {
          const float2 w = totals[s];
          o = scaled(o, raise(w.x));
          const float f = ref == -INFINITY ? 1.f : bd::ex2_approx(w.x - ref);
          total += w.y * f;
          add(o, f, sums[s][lane]);
        }
      }
      __syncthreads();
      if (warp != 0) continue;
    }
    // (0 * inf, NaN, where all scores of the row are -inf; 0 where it sees nothing)
    if (d < a.dim) bdkv::store4<T>(dst, d, scaled(o, vis > 0 ? 1.f / total : 0.f));
    if (c == 0 && lane == 0) bdkv::store_lse(dst, total == 0.f ? -INFINITY : ref + log2f(total));
  }
}

}  // namespace

cudaError_t launch_latent_join(const LatentArgs& p, int sm_count, cudaStream_t st) {
  const int items = p.a.n_seq * p.row_tiles * p.rows * ((p.a.dim + 127) / 128);
  const bool many = items <= 2 * sm_count;  // (8 units of 16 rows of 512 dims: 20.6 us with eight warps to an item, 16.5 with one)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(many ? items : std::min((items + WARPS - 1) / WARPS, 16 * sm_count));
  cfg.blockDim = dim3(WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];  // scheduled while the parts still run; it waits for them before it reads
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const auto kernel = p.a.f16 ? (many ? latent_join_kernel<F16, true> : latent_join_kernel<F16, false>)
                              : (many ? latent_join_kernel<Bf16, true> : latent_join_kernel<Bf16, false>);
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace bdrot
