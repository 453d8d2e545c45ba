// bdrot_latent_attention: tcgen05 products of 64 rows (queries x heads) with
// tiles of 128 cached tokens, the tokens along the instruction's 128 rows.
//
//   S^T [tokens, rows] = C Q^T     C the tile: 128 tokens x (latent, key part),
//                                  in 128-byte columns as the TMA loads it
//   O^T [dims, rows] += C_l^T P    the same bytes, read with the token index
//                                  along K: a latent is loaded once for both
// Rows as columns of the accumulators keep O in half of tensor memory (512 dims
// x 64 rows are 4 x 64 columns), where rows as its rows would fill all of it,
// and cost a few rows no more products than they fill columns.
// Warps: one loads, one issues the products, eight hold the softmax: a thread
// has one token and 32 rows, so maxima over tokens are taken across threads, and
// only when some score exceeds its row's reference by more than 2^7; sums stay
// with the threads until the end.
#include "rotary/latent.h"

namespace bdrot {
namespace {

using bdkv::Seq;

constexpr int SOFT_WARPS = 8, THREADS = (SOFT_WARPS + 2) * 32;
constexpr int SOFT = SOFT_WARPS * 32;
constexpr uint32_t CHUNK = TOKENS * 128, PAIR = 2 * CHUNK;  // bytes of 64 and of 128 elements of a tile
constexpr uint32_t Q_CHUNK = ROWS * 128;
constexpr int S_COL = 0, O_COL = 64;  // tensor memory: scores, then O's dims by 128
constexpr int MAX_PAIRS = 4;
// Weights are held times 2^8 and may exceed that by 2^7 before O is rescaled: 2^15 at most, which f16 holds, with 11 bits
// down to 2^-22 of the reference.
constexpr float P_SHIFT = 8, P_SLACK = 7;

__device__ uint32_t g_status;  // bd::DEV_* bits

struct Ctl {
  uint64_t q_full, pair_full[MAX_PAIRS], pair_empty[MAX_PAIRS], rope_full, rope_empty;
  uint64_t s_full, p_full, o_done, drain;
  alignas(16) float ref[ROWS];    // a row's weights are 2^(score - ref)
  alignas(16) float limit[ROWS];  // scores above it make the reference grow
  alignas(16) float factor[ROWS];
  float part[4][ROWS];            // of the warps of a token quarter: maxima, at the end sums
  float scale[ROWS];
  int visible[ROWS];
  uint64_t out[ROWS];             // where a row goes (0: nowhere); lowest bit: fp32 parts
  uint32_t tmem_base;
  int abort_flag;
};

// Shared memory: the queries' columns, pairs of columns of a tile's latents in a ring of n_pairs, and one place for the
// tile's key parts, which the weights take over once the scores are done.
__host__ __device__ constexpr size_t smem_bytes(int n_pairs) {
  return size_t(2 * n_pairs + 1) * Q_CHUNK + size_t(n_pairs) * PAIR + CHUNK + sizeof(Ctl) + 1024;
}
// (a power of two; CTAs of small latents share an SM, and none waits for another's columns)
__device__ constexpr uint32_t tmem_columns(int n_pairs) { return n_pairs == 1 ? 128 : n_pairs < 4 ? 256 : 512; }
static_assert(smem_bytes(MAX_PAIRS) <= 232448, "shared memory of a CTA");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// D[tmem] (+)= A[smem] * B[smem]; `hi` is the upper word of both descriptors. Issued by predicate in the elected lane.
__device__ __forceinline__ void mma(uint32_t issue, uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t hi_a, uint32_t hi_b,
                                    uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %7};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(issue), "r"(hi_a), "r"(hi_b)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t issue, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(issue)
      : "memory");
}
constexpr uint32_t A_MN_MAJOR = 1u << 15, B_MN_MAJOR = 1u << 16;
// Low word of a descriptor whose operand has M or N contiguous: `lead` bytes between blocks of 64 along it; 1 KB between
// groups of eight along K.
__device__ __forceinline__ uint32_t mn_low(uint32_t saddr, uint32_t lead) {
  return ((saddr & 0x3FFFFu) >> 4) | ((lead >> 4) << 16);
}
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);  // 1 KB stride, version, 128-byte swizzle

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// The 128 threads that share the tile's rows 32 h .. 32 h + 31: a barrier, and one that says whether any of them has `some`.
__device__ __forceinline__ void half_sync(int h) { bd::named_barrier_sync(1 + h, SOFT / 2); }
__device__ __forceinline__ bool half_any(int h, bool some) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(some)), "r"(1 + h), "r"(SOFT / 2)
      : "memory");
  return r != 0;
}

// A row's reference for a largest score of `most`: scores so large that 8 is about a rounding of theirs go without the shift.
__device__ __forceinline__ float reference(float most) { return fabsf(most) < 1048576.f ? most - P_SHIFT : most; }

// v[c] of all lanes combined: lane l returns column l's.
template <class Op>
__device__ __forceinline__ float across_lanes(const float (&v)[32], int lane, Op op) {
  float w[16];
  const auto step = [&](auto width, const auto& from) {
    constexpr int H = decltype(width)::value;
    const bool upper = lane & H;
#pragma unroll
    for (int u = 0; u < H; ++u) {
      const float lo = from[u], hi = from[u + H];
      const float other = __shfl_xor_sync(~0u, upper ? lo : hi, H);
      w[u] = op(upper ? hi : lo, other);
    }
  };
  step(std::integral_constant<int, 16>(), v);
  step(std::integral_constant<int, 8>(), w);
  step(std::integral_constant<int, 4>(), w);
  step(std::integral_constant<int, 2>(), w);
  step(std::integral_constant<int, 1>(), w);
  return w[0];
}

__global__ void __launch_bounds__(THREADS, 1)
    latent_attn_kernel(const LatentArgs p, const __grid_constant__ CUtensorMap latent_map,
                       const __grid_constant__ CUtensorMap rope_map) {
  const bdkv::AttnArgs& a = p.a;
  extern __shared__ __align__(16) uint8_t raw[];
  const int n_pairs = (a.dim + 127) / 128;
  const uint32_t base = (bd::smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, kv_at = q_at + (2 * n_pairs + 1) * Q_CHUNK, rope_at = kv_at + n_pairs * PAIR;
  Ctl* ctl = reinterpret_cast<Ctl*>(raw + (rope_at + CHUNK - bd::smem_u32(raw)));
  const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(bd::warp_uniform(tid >> 5));

  int seq = blockIdx.z;
  const Seq sq = a.longest_first ? bdkv::ranked_seq<THREADS>(a, blockIdx.z, reinterpret_cast<int*>(raw), seq)
                                 : bdkv::load_seq(a, seq);
  // the last rows first: under a causal mask they see the most
  const int row0 = (gridDim.x - 1 - blockIdx.x) * ROWS, part = blockIdx.y, rows = sq.q_len * a.group;
  if (row0 >= rows) return;
  // later queries see at least as much: the CTA's last row bounds it, and all of its rows see what its first one does
  const int i_first = row0 / a.group, i_last = (min(rows, row0 + ROWS) - 1) / a.group;
  const int begin = part * a.chunk, end = min(bdkv::visible(a, sq, i_last), begin + a.chunk);
  if (part > 0 && end <= begin) return;
  const int n = end > begin ? (end - begin + TOKENS - 1) / TOKENS : 0;
  const int all_see = bdkv::visible(a, sq, i_first);

  if (tid == 0) {
    bd::mbar_init(bd::smem_u32(&ctl->q_full), SOFT);
    for (int i = 0; i < MAX_PAIRS; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->pair_full[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->pair_empty[i]), 1);
    }
    bd::mbar_init(bd::smem_u32(&ctl->rope_full), 1);
    bd::mbar_init(bd::smem_u32(&ctl->rope_empty), 1);
    bd::mbar_init(bd::smem_u32(&ctl->s_full), 1);
    bd::mbar_init(bd::smem_u32(&ctl->p_full), SOFT);
    bd::mbar_init(bd::smem_u32(&ctl->o_done), 1);
    bd::mbar_init(bd::smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    bd::fence_mbar_init();
  }
  if (tid < ROWS) {
    ctl->ref[tid] = -P_SHIFT;
    ctl->limit[tid] = -INFINITY;
    const int row = row0 + tid, i = row / a.group, h = row - i * a.group;
    const int vis = row < rows ? bdkv::visible(a, sq, i) : 0;
    ctl->visible[tid] = row < rows ? min(vis, end) : 0;
    uint64_t to = 0;
    if (row < rows) {
      const bdkv::RowOut o = bdkv::row_out(a, sq, seq, part, i, h, vis);
      to = o.out != nullptr ? reinterpret_cast<uint64_t>(o.out) : o.o != nullptr ? reinterpret_cast<uint64_t>(o.o) | 1u : 0u;
    }
    ctl->out[tid] = to;
  }
  constexpr int LOAD_WARP = SOFT_WARPS, MMA_WARP = SOFT_WARPS + 1;
  if (warp == MMA_WARP) {
    bd::tmem_alloc(bd::smem_u32(&ctl->tmem_base), tmem_columns(n_pairs));
    bd::tmem_relinquish();
  }
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  const uint32_t tmem = bd::warp_uniform(ctl->tmem_base);
  volatile int* abort_flag = &ctl->abort_flag;
  const auto wait = [&](uint64_t& bar, int phase) {
    return bd::mbar_wait_warp(bd::smem_u32(&bar), static_cast<uint32_t>(phase & 1), abort_flag, &g_status);
  };
  bd::griddep_launch_dependents();

  if (warp == LOAD_WARP) {
    // ---------------------------------------------------------------- loads
    // Lane b has box b of a tile: a page's tokens, or 128 tokens of a larger page. What is not there (a column behind the
    // table, a page outside the cache, tokens that no row sees) is read from behind the cache's last page, as zeros.
    const int page_size = 1 << a.page_shift, step = min(page_size, TOKENS), boxes = TOKENS / step;
    const int32_t* table = a.table + seq * a.table_stride;
    const int outside = static_cast<int>(max(a.n_pages, static_cast<int64_t>(1)));
    const auto find = [&](int j) {
      const int t = begin + j * TOKENS + lane * step, col = t >> a.page_shift;
      int page = lane < boxes && t < end && col < a.max_blocks ? table[col] : -1;
      return page >= 0 && page < a.n_pages ? page : outside;
    };
    int page = n > 0 ? find(0) : 0, issued = 0, ropes = 0;
    bool ok = true;
    for (int j = 0; ok && j < n; ++j) {
      const int y = (begin + j * TOKENS + lane * step) & (page_size - 1);
      for (int s = 0; s < n_pairs; ++s) {
        if (!(ok = wait(ctl->pair_empty[s], j + 1))) break;
        const uint32_t bar = bd::smem_u32(&ctl->pair_full[s]), dst = kv_at + s * PAIR + lane * step * 128;
        if (lane == 0) bd::mbar_expect_tx(bar, PAIR);
        __syncwarp();
        if (lane < boxes) {
          tma_load_3d(dst, &latent_map, bar, s * 128, y, page);
          tma_load_3d(dst + CHUNK, &latent_map, bar, s * 128 + 64, y, page);
        }
        ++issued;
      }
      if (!ok || !(ok = wait(ctl->rope_empty, j + 1))) break;
      const uint32_t bar = bd::smem_u32(&ctl->rope_full);
      if (lane == 0) bd::mbar_expect_tx(bar, CHUNK);
      __syncwarp();
      if (lane < boxes) tma_load_3d(rope_at + lane * step * 128, &rope_map, bar, 0, y, page);
      ++ropes;
      if (j + 1 < n) page = find(j + 1);
    }
    // nothing is on its way when the CTA ends (all of it has been waited for, unless a wait gave up)
    __syncwarp();
    for (int s = 0; s < n_pairs; ++s) {
      const int loads = (issued - s + n_pairs - 1) / n_pairs;
      if (loads > 0) bd::mbar_drain(bd::smem_u32(&ctl->pair_full[s]), (loads - 1) & 1);
    }
    if (ropes > 0) bd::mbar_drain(bd::smem_u32(&ctl->rope_full), (ropes - 1) & 1);
    __syncwarp();
  } else if (warp == MMA_WARP) {
    // ------------------------------------------------------------- products
    const uint32_t issue = bd::elect_one();
    const uint32_t type = a.f16 ? 0u : (1u << 7) | (1u << 10);
    const uint32_t idesc_s = bd::warp_uniform(bd::idesc_f16_f32(TOKENS, ROWS) | type);
    const uint32_t idesc_o = bd::warp_uniform(bd::idesc_f16_f32(128, ROWS) | type | A_MN_MAJOR | B_MN_MAJOR);
    const uint32_t q_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(q_at)));
    const uint32_t k_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(kv_at)));
    const uint32_t r_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(rope_at)));
    const uint32_t v_lo = bd::warp_uniform(mn_low(kv_at, CHUNK)), p_lo = bd::warp_uniform(mn_low(rope_at, CHUNK));
    const uint32_t s_at = tmem + S_COL;
    bool ok = n > 0 && wait(ctl->q_full, 0);
    for (int j = 0; ok && j < n; ++j) {
      for (int s = 0; s < n_pairs; ++s) {
        if (!(ok = wait(ctl->pair_full[s], j))) break;
        bd::tc_fence_after();
        const uint32_t kd = bd::warp_uniform(k_lo + s * (PAIR >> 4)), qd = bd::warp_uniform(q_lo + s * (2 * Q_CHUNK >> 4));
#pragma unroll
        for (int k = 0; k < 8; ++k)
          mma(issue, s_at, kd + (k / 4) * (CHUNK >> 4) + 2u * (k % 4), qd + (k / 4) * (Q_CHUNK >> 4) + 2u * (k % 4), DESC_HI,
              DESC_HI, idesc_s, (s | k) != 0);
      }
      if (!ok || !(ok = wait(ctl->rope_full, j))) break;
      bd::tc_fence_after();
      const uint32_t qr = bd::warp_uniform(q_lo + n_pairs * (2 * Q_CHUNK >> 4));
#pragma unroll
      for (int k = 0; k < 4; ++k) mma(issue, s_at, r_lo + 2u * k, qr + 2u * k, DESC_HI, DESC_HI, idesc_s, 1);
      mma_commit(issue, bd::smem_u32(&ctl->s_full));
      if (!(ok = wait(ctl->p_full, j))) break;
      bd::tc_fence_after();
      for (int s = 0; s < n_pairs; ++s) {
        const uint32_t vd = bd::warp_uniform(v_lo + s * (PAIR >> 4)), od = bd::warp_uniform(tmem + O_COL + s * ROWS);
#pragma unroll
        for (int k = 0; k < TOKENS / 16; ++k)
          mma(issue, od, vd + k * (2048u >> 4), p_lo + k * (2048u >> 4), DESC_HI, DESC_HI, idesc_o, (j | k) != 0);
        mma_commit(issue, bd::smem_u32(&ctl->pair_empty[s]));
      }
      mma_commit(issue, bd::smem_u32(&ctl->rope_empty));
    }
    mma_commit(issue, bd::smem_u32(&ctl->o_done));
    mma_commit(issue, bd::smem_u32(&ctl->drain));  // all MMAs issued have completed once it flips
    __syncwarp();
    bd::mbar_drain(bd::smem_u32(&ctl->drain), 0);
    __syncwarp();
  } else {
    // -------------------------------------------------------------- softmax
    // A wait that gives up (`ok`) ends no warp's loop: the barriers below count all of them.
    const int quarter = warp & 3, half = warp >> 2;  // tokens and rows, by 32
    if (n > 0) {
      const int wide = a.dim + p.rope_dim, units = (2 * n_pairs + 1) * 8;  // units of eight elements
      const uint16_t* q = static_cast<const uint16_t*>(a.q);
      for (int x = tid; x < ROWS * units; x += SOFT) {
        const int r = x / units, u = x - r * units, row = row0 + r;
        // the key part's columns begin behind the padded latents'
        const int e = u < 16 * n_pairs ? (u * 8 < a.dim ? u * 8 : wide) : a.dim + (u - 16 * n_pairs) * 8;
        uint4 w = {0, 0, 0, 0};
        if (row < rows && e < wide) {
          const int i = row / a.group, h = row - i * a.group;
          w = *reinterpret_cast<const uint4*>(q + static_cast<int64_t>(sq.q0 + i) * a.q_tok + h * a.q_head + e);
        }
        st_shared_v4(q_at + (u / 8) * Q_CHUNK + r * 128 + (((u % 8) ^ (r & 7)) << 4), w.x, w.y, w.z, w.w);
      }
      fence_proxy_async();
      bd::mbar_arrive(bd::smem_u32(&ctl->q_full));
    }
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t s_at = tmem + lanes + S_COL + half * 32, o_at = tmem + lanes + O_COL + half * 32;
    const int token = quarter * 32 + lane;
    // the weights of a token, its row of the second operand: 64 rows contiguous
    const uint32_t p_at = rope_at + (token / 8) * 1024 + (token % 8) * 128;
    float L[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) L[c] = 0.f;
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      const int t0 = begin + j * TOKENS;
      if (ok) ok = wait(ctl->s_full, j);
      bd::tc_fence_after();
      float v[32];
      __syncwarp();
      bd::tmem_ld32(s_at, v);
      const bool cut = t0 + TOKENS > min(all_see, end);  // some row does not see all of the tile
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = __fmul_rn(v[c], a.coef);
      if (cut) {
#pragma unroll
        for (int c = 0; c < 32; ++c)
          if (t0 + token >= ctl->visible[half * 32 + c]) v[c] = -INFINITY;
      }
      bool grow = false;
#pragma unroll
      for (int c = 0; c < 32; ++c) grow |= v[c] > ctl->limit[half * 32 + c];
      if (half_any(half, grow)) {
        const float top = across_lanes(v, lane, [](float x, float y) { return fmaxf(x, y); });
        const int col = half * 32 + lane;
        ctl->part[quarter][col] = top;
        half_sync(half);
        const float most = fmaxf(fmaxf(ctl->part[0][col], ctl->part[1][col]), fmaxf(ctl->part[2][col], ctl->part[3][col]));
        const float limit = ctl->limit[col], before = ctl->ref[col];
        half_sync(half);
        if (quarter == 0) {
          const bool up = most > limit;  // (a limit of -inf: there is no reference yet)
          ctl->factor[col] = !up ? 1.f : limit == -INFINITY ? 0.f : bd::ex2_approx(before - reference(most));
          if (up) ctl->ref[col] = reference(most), ctl->limit[col] = most + P_SLACK;
        }
        half_sync(half);
        float f[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) f[c] = ctl->factor[half * 32 + c], L[c] *= f[c];
        if (j > 0) {  // the products of the tile before came before this tile's scores: O is at rest
          for (int s = 0; s < n_pairs; ++s) {
            float o[32];
            uint32_t y[32];
            __syncwarp();
            bd::tmem_ld32(o_at + s * ROWS, o);
#pragma unroll
            for (int c = 0; c < 32; ++c) y[c] = __float_as_uint(o[c] * f[c]);
            bd::tmem_st32(o_at + s * ROWS, y);
          }
          bd::tmem_st_wait();
        }
      }
      uint32_t w[16];
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        const float2 ref = *reinterpret_cast<const float2*>(&ctl->ref[half * 32 + c]);
        const float2 x = make_float2(bd::ex2_approx(v[c] - ref.x), bd::ex2_approx(v[c + 1] - ref.y));
        L[c] += x.x, L[c + 1] += x.y;
        w[c / 2] = a.f16 ? F16::from_float2(x) : Bf16::from_float2(x);
      }
      // (the scores are done, so the key parts that lay here have been read)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        st_shared_v4(p_at + (((half * 4 + i) ^ (token & 7)) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      if (t0 + TOKENS > end) {
        // What a page holds behind the last token may be anything, and zero times it NaN: its latents become zeros.
        const int from = end - t0, units = (TOKENS - from) * n_pairs * 16;
        for (int x = tid; x < units; x += SOFT) {
          const int r = from + x / (n_pairs * 16), u = x % (n_pairs * 16);
          st_shared_v4(kv_at + (u / 8) * CHUNK + r * 128 + ((u % 8) << 4), 0, 0, 0, 0);
        }
      }
      fence_proxy_async();
      bd::tc_fence_before();
      bd::mbar_arrive(bd::smem_u32(&ctl->p_full));
    }

    // a row's sum: over the lanes, then over the four warps that have its tokens
    ctl->part[quarter][half * 32 + lane] = across_lanes(L, lane, [](float x, float y) { return x + y; });
    half_sync(half);
    if (quarter == 0) {
      const int col = half * 32 + lane, row = row0 + col;
      const float sum = (ctl->part[0][col] + ctl->part[1][col]) + (ctl->part[2][col] + ctl->part[3][col]);
      const uint64_t to = ctl->out[col];
      // a whole row is 0 where it sees nothing, NaN where all of its scores are -inf (a part may well hold nothing)
      ctl->scale[col] = sum == 0.f ? (to != 0 && (to & 1) == 0 && ctl->visible[col] > 0 ? NAN : 0.f) : 1.f / sum;
      if (row < rows) {
        const int i = row / a.group, h = row - i * a.group;
        const bdkv::RowOut o = bdkv::row_out(a, sq, seq, part, i, h, bdkv::visible(a, sq, i));
        if (o.o != nullptr)  // a part's reference and sum: their log-sum-exp in one number would lose the sum of large scores
          reinterpret_cast<float2*>(a.part_l)[o.l - a.part_l] = make_float2(sum == 0.f ? -INFINITY : ctl->ref[col], sum);
        else
          bdkv::store_lse(o, sum == 0.f ? -INFINITY : ctl->ref[col] + log2f(sum));
      }
    }
    half_sync(half);
    if (n > 0 && ok) ok = wait(ctl->o_done, 0);
    bd::tc_fence_after();
    for (int s = 0; s < n_pairs; ++s) {
      float o[32];
      __syncwarp();
      if (n > 0)
        bd::tmem_ld32(o_at + s * ROWS, o);
      else
#pragma unroll
        for (int c = 0; c < 32; ++c) o[c] = 0.f;
      const int d = s * 128 + token;
      if (d < a.dim)
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          const uint64_t to = ctl->out[half * 32 + c];
          const float x = o[c] * ctl->scale[half * 32 + c];
          if (to & 1)
            reinterpret_cast<float*>(to & ~uint64_t(1))[d] = x;
          else if (to != 0)
            reinterpret_cast<uint16_t*>(to)[d] = static_cast<uint16_t>(a.f16 ? F16::from_float2(make_float2(x, 0.f))
                                                                            : Bf16::from_float2(make_float2(x, 0.f)));
        }
    }
  }

  __syncwarp();
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  if (warp == MMA_WARP) bd::tmem_dealloc(tmem, tmem_columns(n_pairs));
}

}  // namespace

cudaError_t launch_latent_attn(const LatentArgs& p, const CUtensorMap& latent, const CUtensorMap& rope, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  if (cudaError_t e = bdkv::allow_smem(latent_attn_kernel, smem_bytes(MAX_PAIRS), ready); e != cudaSuccess) return e;
  const dim3 grid((p.a.max_q * p.a.group + ROWS - 1) / ROWS, p.a.n_split, p.a.n_seq);
  latent_attn_kernel<<<grid, THREADS, smem_bytes((p.a.dim + 127) / 128), st>>>(p, latent, rope);
  return cudaGetLastError();
}

cudaError_t latent_status(cudaStream_t st, uint32_t* bits) {
  cudaError_t e = cudaMemcpyFromSymbolAsync(bits, g_status, sizeof *bits, 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess || *bits == 0) return e;
  const uint32_t zero = 0;
  e = cudaMemcpyToSymbolAsync(g_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

}  // namespace bdrot
