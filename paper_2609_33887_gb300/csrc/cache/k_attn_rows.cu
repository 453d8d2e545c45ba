// bdkv_attention for few query rows per key/value head: single tokens, drafts.
//
// The rows of a request that share a key/value head (queries x the group's
// heads) are the M side of m16n8k16 products, so the head's cache is read
// once for all of them. Each warp walks its own 32-token steps of the cache
// through a ring of asynchronous copies, with the running statistics of an
// online softmax, and the warps' states are merged at the end:
//     S = Q K^T, w = 2^(S coef + e_v), O = sum w code_v, L = sum 2^(S coef)
// where e_v is the exponent of the page's value scale, so values are
// multiplied as the codes they are (exact in f16). O and L have a reference
// of their own each, 2^(r + d) and 2^m, so pages of very different value scales,
// all zeros among them, cost neither range. O's is in two parts, r a score and
// d an exponent of values: added up, a large score would leave the exponent no
// bits (scores of 2^24 made results wrong by powers of two).
//
// Bound by the cache's bytes while a head has few rows: one token of each of 64
// requests of 57 to 8189 tokens, 8 heads of 128, takes 87 us, 6.2 TB/s (0.92 of
// a copy). Legacy products do for that: 16 rows leave 7/8 of a tcgen05 tile
// empty, and registers feed them without a round through shared memory.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int WARPS = 4;       // two CTAs to an SM: one's start and merge run beside the other's products
constexpr int STAGES = 3;
constexpr int STEP = 32;       // tokens a warp takes at once
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

// One CTA: 16 rows of a request's key/value head (R = 1: at most 8 of them exist), one part of its cache. BIG: a step's
// tokens share a page (pages of 32 and more). ORDERED: the longest caches first; a kernel of its own, since the code for it,
// even where it is not taken, costs a call of one request 1.7 of 8.6 us.
template <class T, int D, int R, bool BIG, bool ORDERED>
__global__ void __launch_bounds__(WARPS * 32, 2) attn_rows_kernel(AttnArgs a) {
  constexpr int CH = D / 16;  // 16-byte chunks of a token's row; also k-steps
  constexpr int VB = D / 8;   // bytes of a value row a lane reads; also n-tiles of O
  constexpr int STAGE = STEP * D * 2;
  constexpr int GROUPS = BIG ? 1 : 2;  // pages of a step
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float sm_m[WARPS][16], sm_r[WARPS][16], sm_d[WARPS][16], sm_L[WARPS][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = lane >> 2, c = lane & 3;
  int seq = blockIdx.z;
  Seq sq;
  if constexpr (ORDERED)
    sq = ranked_seq<WARPS * 32>(a, blockIdx.z, reinterpret_cast<int*>(smem), seq);
  else
    sq = load_seq(a, seq);
  const int part = blockIdx.y;
  const int head = blockIdx.x % a.n_kv, row0 = blockIdx.x / a.n_kv * ROWS_TILE;
  const int rows = sq.q_len * a.group;
  if (row0 >= rows) return;
  // later queries see at least as much, so the CTA's last row bounds it
  const int begin = part * a.chunk;
  const int end = min(visible(a, sq, (min(rows, row0 + ROWS_TILE) - 1) / a.group), begin + a.chunk);
  if (part > 0 && end <= begin) return;
  bd::griddep_launch_dependents();
  const int n_steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;

  // Copies: a lane has a 16-byte chunk of every (32 / CH)-th token of a step. What is not there (past the last token, past
  // the row's end, on no page of the cache) is filled with zeros.
  const int my_t = lane / CH, my_ch = lane % CH;
  const bool in_row = my_ch * 16 < a.dim;
  const uint32_t ring = bd::smem_u32(smem) + warp * (STAGES * STAGE);
  const int32_t* table = a.table + seq * a.table_stride;
  const uint8_t* k0 = a.k + head * a.k_head + my_t * a.k_tok + my_ch * 16;
  const uint8_t* v0 = a.v + head * a.v_head + my_t * a.v_tok + my_ch * 16;
  const int mask = (1 << a.page_shift) - 1, n_pages = static_cast<int>(a.n_pages);
  int pages[GROUPS];  // of the step to be fetched next (-1: nothing to read)
  const auto find = [&](int step) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int t = begin + step * STEP + g * 16, col = t >> a.page_shift;
      pages[g] = t < end && col < a.max_blocks ? table[col] : -1;
    }
  };
  const auto fetch = [&](int step, int stage, int (&ks)[GROUPS], int (&vs)[GROUPS]) {
    const int t0 = begin + step * STEP;
    const uint32_t dst = ring + stage * STAGE;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const bool ok = pages[g] >= 0 && pages[g] < n_pages;
      const int64_t page = ok ? pages[g] : 0;
      ks[g] = vs[g] = 127;
      if (ok) {
        ks[g] = a.ks[page * a.ks_page + head];
        vs[g] = a.vs[page * a.vs_page + head];
      }
      const int in = (t0 + g * 16) & mask;
      const uint8_t* k = k0 + page * a.k_page + in * a.k_tok;
      const uint8_t* v = v0 + page * a.v_page + in * a.v_tok;
      if (step < n_steps) {
#pragma unroll
        for (int u = 0; u < STEP * CH / 32 / GROUPS; ++u) {
          const int t = u * (32 / CH) + my_t;  // of the group's tokens
          const bool live = ok && in_row && t0 + g * 16 + t < end;
          cp_async16(dst + ((g * 16 + t) * CH + k_chunk<D>(t, my_ch)) * 16, live ? k + u * (32 / CH) * a.k_tok : a.k, live);
          cp_async16(dst + STEP * D + ((g * 16 + t) * CH + v_chunk<D>(t, my_ch)) * 16,
                     live ? v + u * (32 / CH) * a.v_tok : a.v, live);
        }
      }
    }
    cp_async_commit();
    find(step + WARPS);
  };
  int ks[STAGES][GROUPS], vs[STAGES][GROUPS];
  find(warp);
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(warp + s * WARPS, s, ks[s], vs[s]);

  // queries as A fragments, in f16 times a power of two per row
  uint32_t qf[CH][4] = {};
  float coef[R];
  int vis[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + n + 8 * r, i = row / a.group;
    const bool live = row < rows;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(sq.q0 + i) * a.q_tok +
                        (static_cast<int64_t>(head) * a.group + row - i * a.group) * a.q_head;
    vis[r] = live ? min(visible(a, sq, i), end) : 0;
    uint2 w[CH];
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int d = (j / 4) * 64 + c * 16 + (j % 4) * 4;
      w[j] = make_uint2(0, 0);
      if (live && d < a.dim) w[j] = *reinterpret_cast<const uint2*>(q + d);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const float2 x = T::to_float2(w[j].x), y = T::to_float2(w[j].y);
      amax = bd::max3(bd::max3(amax, fabsf(x.x), fabsf(x.y)), fabsf(y.x), fabsf(y.y));
    }
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
    const int s = row_shift(amax);
    const float f = pow2i(s);
    coef[r] = a.coef * pow2i(-s);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const float2 x = T::to_float2(w[j].x), y = T::to_float2(w[j].y);
      qf[j][r] = f16x2(make_float2(x.x * f, x.y * f));
      qf[j][r + 2] = f16x2(make_float2(y.x * f, y.y * f));
    }
  }

  float O[VB][4] = {};
  float m[R], ro[R], d[R], L[R];  // ro, d: O's reference (d = -inf: O holds nothing yet)
#pragma unroll
  for (int r = 0; r < R; ++r) m[r] = d[r] = -INFINITY, ro[r] = L[r] = 0.f;

  for (int step0 = warp; step0 < n_steps; step0 += STAGES * WARPS) {
#pragma unroll
    for (int stage = 0; stage < STAGES; ++stage) {
      const int step = step0 + stage * WARPS;
      if (step >= n_steps) break;
      cp_async_wait<STAGES - 2>();
      __syncwarp();
      constexpr int AHEAD = STAGES - 1;
      fetch(step + AHEAD * WARPS, (stage + AHEAD) % STAGES, ks[(stage + AHEAD) % STAGES], vs[(stage + AHEAD) % STAGES]);
      const uint32_t kb = ring + stage * STAGE, vb = kb + STEP * D;
      const int t0 = begin + step * STEP;

      float S[4][4] = {};
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const int t = nt * 8 + n;
#pragma unroll
        for (int q4 = 0; q4 < CH / 4; ++q4) {
          const uint4 w = bd::ld_shared_v4(kb + (t * CH + k_chunk<D>(t, q4 * 4 + c)) * 16);
          const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t b0, b1;
            decode4(ww[j], b0, b1);
            mma_f16(S[nt], qf[q4 * 4 + j], b0, b1);
          }
        }
      }

      uint32_t pf[2][4] = {};  // weights as A fragments of two products
      float new_ro[R], new_d[R];
      bool grown = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x[8], ve[GROUPS], top[GROUPS];
        constexpr int E = 8 / GROUPS;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          const float f = coef[r] * pow2i(ks[stage][g] - 127);
          ve[g] = static_cast<float>(vs[stage][g] - 127);
          top[g] = -INFINITY;
#pragma unroll
          for (int e = g * E; e < g * E + E; ++e) x[e] = __fmul_rn(S[e >> 1][2 * r + (e & 1)], f);  // (its own maximum less itself is 0)
          if (t0 + STEP > vis[r])
#pragma unroll
            for (int e = g * E; e < g * E + E; ++e)
              if (t0 + (e >> 1) * 8 + 2 * c + (e & 1) >= vis[r]) x[e] = -INFINITY;
#pragma unroll
          for (int e = g * E; e < g * E + E; e += 2) top[g] = bd::max3(top[g], x[e], x[e + 1]);
          top[g] = fmaxf(top[g], __shfl_xor_sync(~0u, top[g], 1));
          top[g] = fmaxf(top[g], __shfl_xor_sync(~0u, top[g], 2));
        }
        float m_new = m[r], u_top = -INFINITY;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          m_new = fmaxf(m_new, top[g]);
          u_top = fmaxf(u_top, (top[g] - ro[r]) + ve[g]);
        }
        L[r] *= m_new == m[r] ? 1.f : bd::ex2_approx(m[r] - m_new);
        m[r] = m_new;
        const bool grow = u_top > d[r] + P_SLACK || (d[r] == -INFINITY && u_top > d[r]);
        new_ro[r] = grow ? m_new : ro[r];
        new_d[r] = grow ? -INFINITY : d[r];
        if (grow)
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) new_d[r] = fmaxf(new_d[r], (top[g] - m_new) + ve[g]);
        grown |= grow;
        const float mr = m_new == -INFINITY ? 0.f : m_new, dr = new_d[r] == -INFINITY ? 0.f : new_d[r];
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          L[r] += bd::ex2_approx(x[e] - mr);
          w[e] = bd::ex2_approx((x[e] - new_ro[r]) - (dr - ve[e / E] - P_SHIFT));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          pf[k][r] = f16x2(make_float2(w[4 * k], w[4 * k + 1]));
          pf[k][r + 2] = f16x2(make_float2(w[4 * k + 2], w[4 * k + 3]));
        }
      }
      if (__any_sync(~0u, grown)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float f = bd::ex2_approx((ro[r] - new_ro[r]) + (d[r] == new_d[r] ? 0.f : d[r] - new_d[r]));
          ro[r] = new_ro[r];
          d[r] = new_d[r];
#pragma unroll
          for (int j = 0; j < VB; ++j) {
            O[j][2 * r] *= f;
            O[j][2 * r + 1] *= f;
          }
        }
      }

      // values: this lane's bytes n * VB .. of tokens 2c, 2c + 1, 8 + 2c, 9 + 2c of each half of the step
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[4][VB / 4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int t = k * 16 + (u >> 1) * 8 + 2 * c + (u & 1);
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
          uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
          decode4(__byte_perm(w[0][j], w[1][j], 0x5140), a0, a1);
          decode4(__byte_perm(w[0][j], w[1][j], 0x7362), a2, a3);
          decode4(__byte_perm(w[2][j], w[3][j], 0x5140), b0, b1);
          decode4(__byte_perm(w[2][j], w[3][j], 0x7362), b2, b3);
          mma_f16(O[4 * j], pf[k], a0, b0);
          mma_f16(O[4 * j + 1], pf[k], a1, b1);
          mma_f16(O[4 * j + 2], pf[k], a2, b2);
          mma_f16(O[4 * j + 3], pf[k], a3, b3);
        }
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();  // the ring becomes the merge buffer

  constexpr int LD = D + 4;
  float* acc = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    L[r] += __shfl_xor_sync(~0u, L[r], 1);
    L[r] += __shfl_xor_sync(~0u, L[r], 2);
    if (c == 0) {
      sm_m[warp][n + 8 * r] = m[r];
      sm_r[warp][n + 8 * r] = ro[r];
      sm_d[warp][n + 8 * r] = d[r];
      sm_L[warp][n + 8 * r] = L[r];
    }
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e)  // column n of tile j is element n * VB + j
        acc[(warp * 16 + n + 8 * r) * LD + (2 * c + e) * VB + j] = O[j][2 * r + e];
  }
  __syncthreads();
  for (int u = tid; u < 8 * R * D / 4; u += WARPS * 32) {
    const int r = u / (D / 4), d = u % (D / 4) * 4, row = row0 + r;
    if (row >= rows) continue;
    float mt = -INFINITY, Lt = 0.f;
    for (int w = 0; w < WARPS; ++w) mt = fmaxf(mt, sm_m[w][r]);
    const float ms = mt == -INFINITY ? 0.f : mt;
    for (int w = 0; w < WARPS; ++w) Lt += sm_L[w][r] * bd::ex2_approx(sm_m[w][r] - ms);
    const int i = row / a.group, see = visible(a, sq, i);
    const RowOut dst = row_out(a, sq, seq, part, i, head * a.group + row - i * a.group, see);
    // a row's whole result: 0 where it sees nothing, NaN where all of its scores are -inf (a part may well hold nothing)
    const float inv = Lt != 0.f ? 1.f / Lt : dst.out != nullptr && see > 0 ? NAN : 0.f;
    float4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < WARPS; ++w) {
      const float f = bd::ex2_approx((sm_r[w][r] - ms) + (sm_d[w][r] - P_SHIFT)) * inv;
      const float4 x = *reinterpret_cast<const float4*>(acc + (w * 16 + r) * LD + d);
      o.x += x.x * f, o.y += x.y * f, o.z += x.z * f, o.w += x.w * f;
    }
    if (d < a.dim) store4<T>(dst, d, o);
    if (d == 0) store_lse(dst, Lt == 0.f ? -INFINITY : ms + log2f(Lt));
  }
}

template <class T, int D, int R, bool BIG, bool ORDERED>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  const auto kernel = attn_rows_kernel<T, D, R, BIG, ORDERED>;
  if (cudaError_t e = allow_smem(kernel, smem_bytes<D>(), ready); e != cudaSuccess) return e;
  const dim3 grid((a.max_q * a.group + ROWS_TILE - 1) / ROWS_TILE * a.n_kv, a.n_split, a.n_seq);
  kernel<<<grid, WARPS * 32, smem_bytes<D>(), st>>>(a);
  return cudaGetLastError();
}

template <class T, int D, int R>
cudaError_t launch_pages(const AttnArgs& a, cudaStream_t st) {
  if ((1 << a.page_shift) >= STEP)
    return a.longest_first ? launch<T, D, R, true, true>(a, st) : launch<T, D, R, true, false>(a, st);
  return a.longest_first ? launch<T, D, R, false, true>(a, st) : launch<T, D, R, false, false>(a, st);
}

template <class T, int D>
cudaError_t launch_rows(const AttnArgs& a, cudaStream_t st) {
  return a.max_q * a.group <= 8 ? launch_pages<T, D, 1>(a, st) : launch_pages<T, D, 2>(a, st);
}

}  // namespace

cudaError_t launch_attn_rows(const AttnArgs& a, cudaStream_t st) {
  if (a.dim <= 64) return a.f16 ? launch_rows<F16, 64>(a, st) : launch_rows<Bf16, 64>(a, st);
  return a.f16 ? launch_rows<F16, 128>(a, st) : launch_rows<Bf16, 128>(a, st);
}

}  // namespace bdkv
