// bdkv_attention for few query rows per key/value head: single tokens, drafts.
//
// The rows of a request that share a key/value head (queries x the group's
// heads) are the M side of m16n8k16 products, so the head's cache is read
// once for all of them. Each warp walks its own 16-token steps of the cache
// through a ring of asynchronous copies, with the running statistics of an
// online softmax, and the warps' states are merged at the end:
//     S = Q K^T, w = 2^(S coef + e_v), O = sum w code_v, L = sum 2^(S coef)
// where e_v is the exponent of the page's value scale, so values are
// multiplied as the codes they are (exact in f16). O and L have a reference
// of their own each (M and m), so pages of very different value scales, all
// zeros among them, cost neither range.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int WARPS = 8;
constexpr int STAGES = 4;
constexpr int STEP = 16;       // tokens a warp takes at once
constexpr float P_SHIFT = 12;  // weights are held as f16 times 2^12: 11 bits down to 2^-26 of the largest
constexpr float P_SLACK = 3;   // ... and may exceed it by 2^3 before O is rescaled (2^15 < 65504)

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint2 ld_shared_v2(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

// 16-byte chunk of a token's row in a stage: the readers of a quarter warp (keys: two tokens' halves, values: four
// pairs of tokens) then meet in different banks.
template <int D>
__device__ __forceinline__ int k_chunk(int token, int chunk) {
  return D == 128 ? chunk ^ ((token & 1) << 2) : chunk;
}
template <int D>
__device__ __forceinline__ int v_chunk(int token, int chunk) {
  return D == 128 ? chunk ^ (token & 6) : chunk ^ ((token >> 1) & 3);
}

template <int D>
constexpr size_t smem_bytes() {
  const size_t ring = size_t(WARPS) * STAGES * STEP * D * 2, merge = size_t(WARPS) * 16 * (D + 4) * 4;
  return ring > merge ? ring : merge;
}

// One CTA: 16 rows of a request's key/value head, one part of its cache.
template <class T, int D>
__global__ void __launch_bounds__(WARPS * 32, 1) attn_rows_kernel(AttnArgs a) {
  constexpr int CH = D / 16;  // 16-byte chunks of a token's row; also k-steps
  constexpr int VB = D / 8;   // bytes of a value row a lane reads; also n-tiles of O
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float sm_m[WARPS][16], sm_M[WARPS][16], sm_L[WARPS][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = lane >> 2, c = lane & 3;
  const int seq = blockIdx.z, part = blockIdx.y;
  const int head = blockIdx.x % a.n_kv, row0 = blockIdx.x / a.n_kv * ROWS_TILE;
  const Seq sq = load_seq(a, seq);
  const int rows = sq.q_len * a.group;
  if (row0 >= rows) return;
  // later queries see at least as much, so the CTA's last row bounds it
  const int begin = part * a.chunk;
  const int end = min(visible(a, sq, (min(rows, row0 + ROWS_TILE) - 1) / a.group), begin + a.chunk);
  if (part > 0 && end <= begin) return;
  bd::griddep_launch_dependents();

  // queries as A fragments, in f16 times a power of two per row
  uint32_t qf[CH][4];
  float coef[2];
  int vis[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + n + 8 * r, i = row / a.group;
    const bool live = row < rows;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(sq.q0 + i) * a.q_tok +
                        (static_cast<int64_t>(head) * a.group + row - i * a.group) * a.q_head;
    vis[r] = live ? visible(a, sq, i) : 0;
    float2 x[CH][2];
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int d = (j / 4) * 64 + c * 16 + (j % 4) * 4;
      uint2 w = {0, 0};
      if (live && d < a.dim) w = *reinterpret_cast<const uint2*>(q + d);
      x[j][0] = T::to_float2(w.x);
      x[j][1] = T::to_float2(w.y);
      amax = fmaxf(amax, fmaxf(fmaxf(fabsf(x[j][0].x), fabsf(x[j][0].y)), fmaxf(fabsf(x[j][1].x), fabsf(x[j][1].y))));
    }
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
    const int s = row_shift(amax);
    const float f = pow2i(s);
    coef[r] = a.coef * pow2i(-s);
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int p = 0; p < 2; ++p) qf[j][r + 2 * p] = f16x2(make_float2(x[j][p].x * f, x[j][p].y * f));
  }

  float O[VB][4] = {};
  float m[2] = {-INFINITY, -INFINITY}, M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f};
  const int n_steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;
  const uint32_t ring = bd::smem_u32(smem) + warp * (STAGES * STEP * D * 2);
  int scales[STAGES];  // of the steps in flight: key byte, value byte << 8

  auto fetch = [&](int step, int stage) -> int {
    int got = 0;
    if (step < n_steps) {
      const int t0 = begin + step * STEP, col = t0 >> a.page_shift;
      const int64_t page = col < a.max_blocks ? a.table[seq * a.table_stride + col] : -1;
      const bool ok = page >= 0 && page < a.n_pages;
      const int64_t p = ok ? page : 0;
      got = ok ? a.ks[p * a.ks_page + head] | (a.vs[p * a.vs_page + head] << 8) : 127 | (127 << 8);
      const uint8_t* k = a.k + p * a.k_page + head * a.k_head;
      const uint8_t* v = a.v + p * a.v_page + head * a.v_head;
      const int in = t0 & ((1 << a.page_shift) - 1);
      const uint32_t dst = ring + stage * (STEP * D * 2);
#pragma unroll
      for (int u = 0; u < STEP * CH / 32; ++u) {
        const int t = (u * 32 + lane) / CH, ch = (u * 32 + lane) % CH;
        const bool live = ok && t0 + t < end && ch * 16 < a.dim;
        const int64_t ko = live ? (in + t) * a.k_tok + ch * 16 : 0, vo = live ? (in + t) * a.v_tok + ch * 16 : 0;
        cp_async16(dst + (t * CH + k_chunk<D>(t, ch)) * 16, k + ko, live);
        cp_async16(dst + STEP * D + (t * CH + v_chunk<D>(t, ch)) * 16, v + vo, live);
      }
    }
    cp_async_commit();
    return got;
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) scales[s] = fetch(warp + s * WARPS, s);

  int stage = 0;
  for (int step = warp; step < n_steps; step += WARPS) {
    cp_async_wait<STAGES - 2>();
    __syncwarp();
    const int sc = scales[0];
#pragma unroll
    for (int s = 0; s < STAGES - 2; ++s) scales[s] = scales[s + 1];
    scales[STAGES - 2] = fetch(step + (STAGES - 1) * WARPS, (stage + STAGES - 1) % STAGES);
    const uint32_t kb = ring + stage * (STEP * D * 2), vb = kb + STEP * D;
    stage = (stage + 1) % STAGES;

    float S[2][4] = {};
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const int t = nt * 8 + n;
#pragma unroll
      for (int q4 = 0; q4 < CH / 4; ++q4) {
        const uint4 w = bd::ld_shared_v4(kb + (t * CH + k_chunk<D>(t, q4 * 4 + c)) * 16);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          mma_f16(S[nt], qf[q4 * 4 + j], bd::e4m3x2_to_f16x2(ww[j] & 0xffffu), bd::e4m3x2_to_f16x2(ww[j] >> 16));
      }
    }

    const float ks = pow2i((sc & 255) - 127);
    const float ve = static_cast<float>((sc >> 8) - 127);
    uint32_t pf[4];
    bool grown = false;
    float newM[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float f = coef[r] * ks;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = begin + step * STEP + (e >> 1) * 8 + 2 * c + (e & 1);
        x[e] = t < min(vis[r], end) ? S[e >> 1][2 * r + (e & 1)] * f : -INFINITY;
      }
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
      if (top > m[r]) {
        L[r] *= bd::ex2_approx(m[r] - top);  // m = -inf: L is 0
        m[r] = top;
      }
      newM[r] = top + ve > M[r] + P_SLACK || M[r] == -INFINITY ? top + ve : M[r];
      grown |= newM[r] != M[r];
      const float mr = m[r] == -INFINITY ? 0.f : m[r];
      const float Mr = (newM[r] == -INFINITY ? 0.f : newM[r]) - ve - P_SHIFT;
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        L[r] += bd::ex2_approx(x[e] - mr);
        w[e] = bd::ex2_approx(x[e] - Mr);
      }
      pf[r] = f16x2(make_float2(w[0], w[1]));
      pf[r + 2] = f16x2(make_float2(w[2], w[3]));
    }
    if (__any_sync(~0u, grown)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float f = newM[r] == M[r] ? 1.f : bd::ex2_approx(M[r] - newM[r]);
        M[r] = newM[r];
#pragma unroll
        for (int j = 0; j < VB; ++j) {
          O[j][2 * r] *= f;
          O[j][2 * r + 1] *= f;
        }
      }
    }

    // values: this lane's bytes n * VB .. of tokens 2c, 2c + 1, 8 + 2c, 9 + 2c
    uint32_t w[4][VB / 4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = (u >> 1) * 8 + 2 * c + (u & 1);
      if constexpr (D == 128) {
        const uint4 x = bd::ld_shared_v4(vb + (t * CH + v_chunk<D>(t, n)) * 16);
        w[u][0] = x.x, w[u][1] = x.y, w[u][2] = x.z, w[u][3] = x.w;
      } else {
        const uint2 x = ld_shared_v2(vb + (t * CH + v_chunk<D>(t, n >> 1)) * 16 + (n & 1) * 8);
        w[u][0] = x.x, w[u][1] = x.y;
      }
    }
#pragma unroll
    for (int j = 0; j < VB / 4; ++j) {
      const uint32_t a0 = __byte_perm(w[0][j], w[1][j], 0x5140), a1 = __byte_perm(w[0][j], w[1][j], 0x7362);
      const uint32_t b0 = __byte_perm(w[2][j], w[3][j], 0x5140), b1 = __byte_perm(w[2][j], w[3][j], 0x7362);
      mma_f16(O[4 * j], pf, bd::e4m3x2_to_f16x2(a0 & 0xffffu), bd::e4m3x2_to_f16x2(b0 & 0xffffu));
      mma_f16(O[4 * j + 1], pf, bd::e4m3x2_to_f16x2(a0 >> 16), bd::e4m3x2_to_f16x2(b0 >> 16));
      mma_f16(O[4 * j + 2], pf, bd::e4m3x2_to_f16x2(a1 & 0xffffu), bd::e4m3x2_to_f16x2(b1 & 0xffffu));
      mma_f16(O[4 * j + 3], pf, bd::e4m3x2_to_f16x2(a1 >> 16), bd::e4m3x2_to_f16x2(b1 >> 16));
    }
  }
  cp_async_wait<0>();
  __syncthreads();  // the ring becomes the merge buffer

  constexpr int LD = D + 4;
  float* acc = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    L[r] += __shfl_xor_sync(~0u, L[r], 1);
    L[r] += __shfl_xor_sync(~0u, L[r], 2);
    if (c == 0) {
      sm_m[warp][n + 8 * r] = m[r];
      sm_M[warp][n + 8 * r] = M[r];
      sm_L[warp][n + 8 * r] = L[r];
    }
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e)  // column n of tile j is element n * VB + j
        acc[(warp * 16 + n + 8 * r) * LD + (2 * c + e) * VB + j] = O[j][2 * r + e];
  }
  __syncthreads();
  for (int u = tid; u < 16 * D / 4; u += WARPS * 32) {
    const int r = u / (D / 4), d = u % (D / 4) * 4, row = row0 + r;
    if (row >= rows) continue;
    float mt = -INFINITY, Mt = -INFINITY, Lt = 0.f;
    for (int w = 0; w < WARPS; ++w) {
      mt = fmaxf(mt, sm_m[w][r]);
      Mt = fmaxf(Mt, sm_M[w][r]);
    }
    const float ms = mt == -INFINITY ? 0.f : mt, Ms = Mt == -INFINITY ? 0.f : Mt;
    float4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < WARPS; ++w) {
      Lt += sm_L[w][r] * bd::ex2_approx(sm_m[w][r] - ms);
      const float f = bd::ex2_approx(sm_M[w][r] - Ms);
      const float4 x = *reinterpret_cast<const float4*>(acc + (w * 16 + r) * LD + d);
      o.x += x.x * f, o.y += x.y * f, o.z += x.z * f, o.w += x.w * f;
    }
    const float f = Lt == 0.f ? 0.f : bd::ex2_approx(Ms - P_SHIFT - ms) / Lt;
    const int i = row / a.group;
    const RowOut dst = row_out(a, sq, seq, part, i, head * a.group + row - i * a.group, visible(a, sq, i));
    if (d < a.dim) store4<T>(dst, d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    if (d == 0) store_lse(dst, Lt == 0.f ? -INFINITY : ms + log2f(Lt));
  }
}

template <class T, int D>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  if (cudaError_t e = allow_smem(attn_rows_kernel<T, D>, smem_bytes<D>(), ready); e != cudaSuccess) return e;
  const dim3 grid((a.max_q * a.group + ROWS_TILE - 1) / ROWS_TILE * a.n_kv, a.n_split, a.n_seq);
  attn_rows_kernel<T, D><<<grid, WARPS * 32, smem_bytes<D>(), st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attn_rows(const AttnArgs& a, cudaStream_t st) {
  if (a.dim <= 64) return a.f16 ? launch<F16, 64>(a, st) : launch<Bf16, 64>(a, st);
  return a.f16 ? launch<F16, 128>(a, st) : launch<Bf16, 128>(a, st);
}

}  // namespace bdkv
