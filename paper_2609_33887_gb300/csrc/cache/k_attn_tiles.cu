// bdkv_attention for many query rows per key/value head: windows of blocks,
// prompts. tcgen05 products on tiles of 128 rows.
//
// A CTA holds NM x 128 rows of a request's key/value head (queries x the
// group's heads, so the head's cache is read once for all of them) and walks
// the cache in tiles of 128 tokens (64 with one half of rows, NM = 1):
//   converter warps   codes from global memory to f16 (exact), into shared
//                     memory in the 128-byte swizzle, in stages; a request's
//                     tail is zeros, so its values times zero weights stay zero
//   MMA warp          S = Q K^T (both operands in shared memory) and O += P V
//                     (P in tensor memory, V read with the token index along
//                     K). With two halves the products of one run while the
//                     softmax of the other does; with one, S of two tiles is
//                     made ahead
//   softmax warps     two threads per row, each half of a tile's columns:
//                     running maxima, weights to f16, written over S in tensor
//                     memory; O is rescaled only when a row's maximum has grown
//                     by more than 2^7, which the two warps of 32 rows agree
//                     on in a barrier that carries the vote
// Scales of pages come in through the exponent: w = 2^(S coef k_scale + e_v),
// see k_attn_rows.cu; O and the sum L have a reference maximum of their own.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int TILE = TILES_TILE;  // rows of an MMA
// Weights are held as f16 times 2^8, with 11 bits down to 2^-22 of the reference, and may exceed it by 2^7 before O is
// rescaled (2^15 < 65504): a rescale costs a warp about as much as a tile.
constexpr float P_SHIFT = 8, P_SLACK = 7;
constexpr int CONV_WARPS = 8;

template <int NM>
struct Shape {
  static constexpr int TOK = NM == 2 ? 128 : 64;    // tokens of a tile
  static constexpr int STAGES = NM == 2 ? 2 : 4;    // tiles of keys and of values in shared memory
  static constexpr int AHEAD = NM == 2 ? 1 : 2;     // tiles whose S is held at once
  static constexpr int W = TOK / 2;                 // columns of a softmax thread
  static constexpr int SOFT_WARPS = 8 * NM;
  // Converters are warpgroups too, and so are the MMA warp, the one that looks up scales and two idle ones, so that
  // registers can be moved: with two halves 896 threads start with 72 each, 512 x 80 + 256 x 64 + 128 x 56 = 64512; with
  // one, 640 threads have 96.
  static constexpr int THREADS = (SOFT_WARPS + CONV_WARPS + 4) * 32;
};

__device__ uint32_t g_status;  // bd::DEV_* bits

struct Ctl {
  uint64_t q_full, k_full[4], k_empty[4], v_full[4], v_empty[4];
  uint64_t s_full[2][2], p_full[2][2];     // by half and parity of the tile
  uint64_t o_before[2], o_done[2], drain;  // by half: O without (AHEAD = 2), and with its last product
  float ks[8][8], ve[8][8];                // page scales of a tile's groups of 16 tokens: factor, exponent
  float2 row[2][2][TILE];                  // what the two threads of a row tell each other, by half and side
  int q_shift[2][2][4];                    // by half, side and quarter of the rows
  uint32_t tmem_base;
  int abort_flag;
};

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// The MMA warp issues in the elected lane by predicate, not by branch, and its descriptors' low words come through
// warp_uniform: they then stay in uniform registers. D[tmem] (+)= A[smem] * B[smem]^T, f16; `hi` is the upper word of both
// descriptors.
__device__ __forceinline__ void mma_ss(uint32_t issue, uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t hi,
                                       uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(issue), "r"(hi)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], f16: row i of A in lane i, two elements per 32-bit column.
__device__ __forceinline__ void mma_ts(uint32_t issue, uint32_t d_tmem, uint32_t a_tmem, uint32_t b, uint32_t hi,
                                       uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b), "r"(idesc), "r"(accumulate), "r"(issue), "r"(hi)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t issue, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(issue)
      : "memory");
}

// B operand stored with N contiguous (128-byte swizzle, atoms of 64 elements of
// N by 8 of K): `lead` bytes between atoms along N, 1 KB along K.
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t saddr, uint32_t lead) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(lead >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}
constexpr uint32_t B_MN_MAJOR = 1u << 16;

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}

// Moves registers between the warpgroups (all four warps execute it).
template <int N>
__device__ __forceinline__ void take_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void give_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// Loads that happen where `live` says so, without a branch that would hold up the loads behind them.
__device__ __forceinline__ int ld_global_if(const int32_t* p, bool live, int other) {
  int x = other;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p ld.global.b32 %0, [%1];\n\t}"
               : "+r"(x)
               : "l"(p), "r"(static_cast<int>(live)));
  return x;
}
__device__ __forceinline__ int ld_global_byte_if(const uint8_t* p, bool live) {
  int x = 127;  // a scale of 1
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p ld.global.u8 %0, [%1];\n\t}"
               : "+r"(x)
               : "l"(p), "r"(static_cast<int>(live)));
  return x;
}
__device__ __forceinline__ void ld_global_over(uint4& x, const uint8_t* p, bool live) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "+r"(x.x), "+r"(x.y), "+r"(x.z), "+r"(x.w)
               : "l"(p), "r"(static_cast<int>(live)));
}

// A barrier of the two warps that share 32 rows, which tells both whether some thread of either says so.
__device__ __forceinline__ bool pair_any(int id, bool says) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\t"
      "barrier.cta.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(id), "r"(static_cast<int>(says))
      : "memory");
  return any != 0;
}

template <int NM, int D>
constexpr size_t smem_bytes() {
  return size_t(NM * TILE + 2 * Shape<NM>::STAGES * Shape<NM>::TOK) * D * 2 + sizeof(Ctl) + 1024;
}

// BIG: pages of 64 tokens and more (a softmax thread's columns share a page), else 16 or 32.
template <int NM, int D, bool BIG>
__global__ void __launch_bounds__(Shape<NM>::THREADS, 1) attn_tiles_kernel(AttnArgs a) {
  using Sh = Shape<NM>;
  constexpr int TOK = Sh::TOK, STAGES = Sh::STAGES, AHEAD = Sh::AHEAD, W = Sh::W;
  constexpr int ATOMS = D / 64;                                 // 128-byte column blocks of a row
  constexpr uint32_t Q_ATOM = TILE * 128, KV_ATOM = TOK * 128;  // bytes of one
  constexpr uint32_t Q_HALF = ATOMS * Q_ATOM, KV_TILE = ATOMS * KV_ATOM;
  constexpr int CH = D / 16;                                    // 16-code chunks of a token's row
  constexpr int O_COL = 256;  // tensor memory: S and P of half x at 128 x (and of parity b at 64 b), O behind
  extern __shared__ uint8_t raw[];
  const uint32_t base = (bd::smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + NM * Q_HALF, v_at = k_at + STAGES * KV_TILE;
  Ctl* ctl = reinterpret_cast<Ctl*>(raw + (v_at + STAGES * KV_TILE - bd::smem_u32(raw)));
  const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(bd::warp_uniform(tid >> 5));
  const int n_tiles_rows = gridDim.x / a.n_kv;
  const int head = blockIdx.x / n_tiles_rows, row0 = (n_tiles_rows - 1 - blockIdx.x % n_tiles_rows) * (NM * TILE);
  const int seq = blockIdx.z, part = blockIdx.y;
  const Seq sq = load_seq(a, seq);
  const int rows = sq.q_len * a.group;
  if (row0 >= rows) return;
  // later queries see at least as much, so the CTA's last row bounds it
  const int i_last = (min(rows, row0 + NM * TILE) - 1) / a.group;
  const int begin = part * a.chunk, end = min(visible(a, sq, i_last), begin + a.chunk);
  if (part > 0 && end <= begin) return;
  const int n = end > begin ? (end - begin + TOK - 1) / TOK : 0;

  if (tid == 0) {
    bd::mbar_init(bd::smem_u32(&ctl->q_full), Sh::SOFT_WARPS);  // a warp's arrival, like that of every barrier with warps
    for (int i = 0; i < STAGES; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->k_full[i]), CONV_WARPS + 1);
      bd::mbar_init(bd::smem_u32(&ctl->v_full[i]), CONV_WARPS);
      bd::mbar_init(bd::smem_u32(&ctl->k_empty[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->v_empty[i]), 1);
    }
    for (int x = 0; x < 2; ++x) {
      for (int b = 0; b < 2; ++b) {
        bd::mbar_init(bd::smem_u32(&ctl->s_full[x][b]), 1);
        bd::mbar_init(bd::smem_u32(&ctl->p_full[x][b]), 8);
      }
      bd::mbar_init(bd::smem_u32(&ctl->o_before[x]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->o_done[x]), 1);
    }
    bd::mbar_init(bd::smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    bd::fence_mbar_init();
  }
  constexpr int MMA_WARP = Sh::SOFT_WARPS + CONV_WARPS;
  if (warp == MMA_WARP) {
    bd::tmem_alloc(bd::smem_u32(&ctl->tmem_base), 512);
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
  const auto arrive = [&](uint64_t& bar) {  // for the warp, whose lanes are done with what they hand on
    __syncwarp();
    if (lane == 0) bd::mbar_arrive(bd::smem_u32(&bar));
  };
  bd::griddep_launch_dependents();

  if (warp >= MMA_WARP) {
    // ---------------------------------------------------------- MMA issuer
    if constexpr (NM == 2) give_registers<56>();
    if (warp == MMA_WARP) {
      const uint32_t issue = bd::elect_one();
      constexpr uint32_t IDESC_S = bd::idesc_f16_f32(TILE, TOK), IDESC_O = bd::idesc_f16_f32(TILE, D) | B_MN_MAJOR;
      // low words of the descriptors (addresses count 16 bytes) and their common upper word: 1 KB stride, version, swizzle
      const uint32_t q_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(q_at)));
      const uint32_t k_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(k_at)));
      const uint32_t v_lo = bd::warp_uniform(static_cast<uint32_t>(sw128_mnmajor_desc(v_at, KV_ATOM)));
      constexpr uint32_t HI = (1024u >> 4) | (1u << 14) | (2u << 29);
      const auto scores = [&](int x, int u) {  // S of half x, a tile of stage u
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_ss(issue, tmem + x * TILE + u % AHEAD * TOK, q_lo + x * (Q_HALF >> 4) + (k / 4) * (Q_ATOM >> 4) + 2u * (k % 4),
                 k_lo + u * (KV_TILE >> 4) + (k / 4) * (KV_ATOM >> 4) + 2u * (k % 4), HI, IDESC_S, k != 0);
        mma_commit(issue, bd::smem_u32(&ctl->s_full[x][u % AHEAD]));
        if (x == NM - 1) mma_commit(issue, bd::smem_u32(&ctl->k_empty[u]));
      };
      bool ok = n > 0 && wait(ctl->q_full, 0);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (!ok || u >= n) break;
        ok = wait(ctl->k_full[u], 0);
        if (!ok) break;
        bd::tc_fence_after();
#pragma unroll
        for (int x = 0; x < NM; ++x) scores(x, u);
      }
      for (int j0 = 0; ok && j0 < n; j0 += STAGES) {
#pragma unroll
        for (int u = 0; u < STAGES; ++u) {  // stages by number: every address is a constant away from its base
          const int j = j0 + u;
          if (!ok || j >= n) break;
#pragma unroll
          for (int x = 0; x < NM; ++x) {
            if (!ok || !(ok = wait(ctl->p_full[x][u % AHEAD], j / AHEAD))) break;
            if (x == 0 && !(ok = wait(ctl->v_full[u], j / STAGES))) break;
            bd::tc_fence_after();
#pragma unroll
            for (int k = 0; k < TOK / 16; ++k)  // a side's weights lie over the first half of its scores
              mma_ts(issue, tmem + O_COL + x * TILE,
                     tmem + x * TILE + u % AHEAD * TOK + k * 16 / W * W + k * 16 % W / 2,
                     v_lo + u * (KV_TILE >> 4) + k * (2048u >> 4), HI, IDESC_O, (j | k) != 0);
            if (x == NM - 1) mma_commit(issue, bd::smem_u32(&ctl->v_empty[u]));
            if (j + AHEAD < n) {  // over the weights that the products above read: the tensor pipe takes them in order
              if (x == 0 && !(ok = wait(ctl->k_full[(u + AHEAD) % STAGES], (j + AHEAD) / STAGES))) break;
              bd::tc_fence_after();
              scores(x, (u + AHEAD) % STAGES);
            } else {
              mma_commit(issue, bd::smem_u32(j + 1 < n ? &ctl->o_before[x] : &ctl->o_done[x]));
            }
          }
        }
      }
      mma_commit(issue, bd::smem_u32(&ctl->drain));  // all MMAs issued have completed once it flips
      __syncwarp();
      bd::mbar_drain(bd::smem_u32(&ctl->drain), 0);
    } else if (warp == MMA_WARP + 1) {
      // ------------------------------------------------------- page scales
      // a lane has 16 tokens of a tile: their page and, a tile ahead, its scales
      const int32_t* table = a.table + seq * a.table_stride;
      int page = -1, ks_byte = 127, vs_byte = 127;
      const auto find_page = [&](int j) {
        const int t = begin + j * TOK + lane * 16, col = t >> a.page_shift;
        page = ld_global_if(table + col, lane < TOK / 16 && t < end && col < a.max_blocks, -1);
      };
      const auto find_scales = [&](int j) {  // of tile j, whose pages were found; then the pages of the next
        const bool in = page >= 0 && page < a.n_pages;
        ks_byte = ld_global_byte_if(a.ks + page * a.ks_page + head, in);
        vs_byte = ld_global_byte_if(a.vs + page * a.vs_page + head, in);
        find_page(j + 1);
      };
      if (n > 0) {
        find_page(0);
        find_scales(0);
      }
      for (int j = 0; j < n && wait(ctl->k_empty[j % STAGES], j / STAGES + 1); ++j) {
        if (lane < TOK / 16) {
          ctl->ks[j & 7][lane] = pow2i(ks_byte - 127);
          ctl->ve[j & 7][lane] = static_cast<float>(vs_byte - 127);
        }
        arrive(ctl->k_full[j % STAGES]);
        find_scales(j + 1);
      }
    }
    __syncwarp();
  } else if (warp >= Sh::SOFT_WARPS) {
    // ---------------------------------------------------------- converters
    if constexpr (NM == 2) give_registers<64>();
    const int ct = tid - Sh::SOFT_WARPS * 32;
    constexpr int PER = TOK * CH / (CONV_WARPS * 32);  // chunks of a thread and tile
    constexpr int STEP = CONV_WARPS * 32 / CH;         // rows between them
    constexpr int DEPTH = NM == 2 ? 1 : 2;             // tiles on their way in registers
    // eight lanes take four chunks each of two rows, which the swizzle puts into different banks
    const int sub = (ct & 3) | (CH == 8 ? (ct >> 1) & 4 : 0), mine = ct / (2 * CH) * 2 + ((ct >> 2) & 1);
    const int32_t* table = a.table + seq * a.table_stride;
    const int mask = (1 << a.page_shift) - 1, n_pages = static_cast<int>(a.n_pages);
    const uint8_t* k0 = a.k + head * a.k_head + mine * a.k_tok + sub * 16;
    const uint8_t* v0 = a.v + head * a.v_head + mine * a.v_tok + sub * 16;
    const bool in_row = sub * 16 < a.dim;
    uint4 kx[DEPTH][PER] = {}, vx[DEPTH][PER] = {};
    constexpr int PAGES = BIG ? TOK / 64 : PER;
    int pages[PAGES];  // of the tile to be loaded next (-1: nothing to read)
    const auto find = [&](int j) {
#pragma unroll
      for (int u = 0; u < PAGES; ++u) {
        const int t = begin + j * TOK + (BIG ? u * 64 : mine + u * STEP);
        pages[u] = ld_global_if(table + (t >> a.page_shift), t < end && (t >> a.page_shift) < a.max_blocks, -1);
        if (pages[u] >= n_pages) pages[u] = -1;
      }
    };
    // One of keys and values of tile j, whose pages were found. Lanes past a row's end keep the zeros they began with; what
    // is not there in a tile (past the last token, on no page of the cache) becomes zeros.
    const auto load = [&](const uint8_t* p, int64_t page_stride, int64_t tok_stride, int j, uint4 (&x)[PER]) {
      const int t0 = begin + j * TOK;
      bool whole = t0 + TOK <= end;
#pragma unroll
      for (int u = 0; u < PAGES; ++u) whole = whole && pages[u] >= 0;
      if (BIG && whole) {
#pragma unroll
        for (int g = 0; g < PAGES; ++g) {
          const uint8_t* at = p + pages[g] * page_stride + ((t0 + g * 64) & mask) * tok_stride;
#pragma unroll
          for (int u = 0; u < PER / PAGES; ++u) ld_global_over(x[g * (PER / PAGES) + u], at + u * STEP * tok_stride, in_row);
        }
      } else {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int page = pages[BIG ? u * STEP / 64 : u], t = t0 + u * STEP;
          const int in = ((t + mine) & mask) - mine;  // tokens from this thread's first to its chunk's in the page
          x[u] = make_uint4(0, 0, 0, 0);
          ld_global_over(x[u], p + page * page_stride + in * tok_stride, in_row && page >= 0 && t + mine < end);
        }
      }
    };
    const auto store = [&](uint32_t at, const uint4 (&x)[PER]) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int r = mine + u * STEP;
        uint32_t y[8];
        decode4(x[u].x, y[0], y[1]);
        decode4(x[u].y, y[2], y[3]);
        decode4(x[u].z, y[4], y[5]);
        decode4(x[u].w, y[6], y[7]);
        const uint32_t rowp = at + (sub / 4) * KV_ATOM + r * 128, c0 = (sub % 4) * 2;
        st_shared_v4(rowp + ((c0 ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
        st_shared_v4(rowp + (((c0 + 1) ^ (r & 7)) << 4), y[4], y[5], y[6], y[7]);
      }
    };
    if (n > 0) {
#pragma unroll
      for (int b = 0; b < DEPTH; ++b) {
        find(b);
        load(k0, a.k_page, a.k_tok, b, kx[b]);
        load(v0, a.v_page, a.v_tok, b, vx[b]);
      }
      find(DEPTH);
    }
    bool ok = true;
    for (int j0 = 0; ok && j0 < n; j0 += DEPTH) {
#pragma unroll
      for (int b = 0; b < DEPTH; ++b) {
        const int j = j0 + b;
        if (j >= n || !(ok = wait(ctl->k_empty[j % STAGES], j / STAGES + 1))) break;
        store(k_at + (j % STAGES) * KV_TILE, kx[b]);
        fence_proxy_async();
        arrive(ctl->k_full[j % STAGES]);
        load(k0, a.k_page, a.k_tok, j + DEPTH, kx[b]);
        if (!(ok = wait(ctl->v_empty[j % STAGES], j / STAGES + 1))) break;
        store(v_at + (j % STAGES) * KV_TILE, vx[b]);
        fence_proxy_async();
        arrive(ctl->v_full[j % STAGES]);
        load(v0, a.v_page, a.v_tok, j + DEPTH, vx[b]);
        find(j + DEPTH + 1);
      }
    }
  } else {
    // ------------------------------------------------------------- softmax
    if constexpr (NM == 2) take_registers<80>();
    const int x = warp >> 3, side = (warp >> 2) & 1, warp_row = (warp & 3) * 32;  // half of rows, half of columns
    const int pair = 1 + x * 4 + (warp & 3);                                      // the two warps' barrier
    const int r = warp_row + lane, row = row0 + x * TILE + r, i = row / a.group;
    const bool live = row < rows;
    const int h = head * a.group + row - i * a.group;
    const int vis = live ? min(visible(a, sq, i), end) : end;  // rows that do not exist never need a mask
    float coef = 0.f;
    if (n > 0) {
      // Queries: a warp moves 16 of its 32 rows, LANES lanes to a row (16 bytes each). f16, with the sign of the scale; bf16
      // ones times a power of two that brings the largest finite element of the 16 rows into [2^14, 2^15): elements down to
      // 2^-32 of it keep their eight bits.
      constexpr int LANES = D / 8, ROWS = 32 / LANES;
      const int my_c = lane % LANES, my_r = lane / LANES;
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(sq.q0 + i) * a.q_tok + h * a.q_head;
      uint4 w[16 / ROWS] = {};
#pragma unroll
      for (int u = 0; u < 16 / ROWS; ++u) {
        const int rr = side * 16 + u * ROWS + my_r;
        const uint64_t src = __shfl_sync(~0u, reinterpret_cast<uint64_t>(q), rr);
        ld_global_over(w[u], reinterpret_cast<const uint8_t*>(src) + my_c * 16, row - lane + rr < rows && my_c * 8 < a.dim);
      }
      int shift = 0;
      if (!a.f16) {
        uint32_t most = 0;  // magnitudes' patterns, two to a word
#pragma unroll
        for (int u = 0; u < 16 / ROWS; ++u) {
          const uint32_t t = __vmaxu2(__vmaxu2(w[u].x & 0x7fff7fffu, w[u].y & 0x7fff7fffu),
                                      __vmaxu2(w[u].z & 0x7fff7fffu, w[u].w & 0x7fff7fffu));
          if ((t & 0xffffu) < 0x7f80u && t < 0x7f800000u) most = __vmaxu2(most, t);
        }
        most = __reduce_max_sync(~0u, max(most & 0xffffu, most >> 16));
        shift = row_shift(__uint_as_float(most << 16));
      }
      const float f = a.coef < 0.f ? -pow2i(shift) : pow2i(shift);
      const uint32_t flip = a.coef < 0.f ? 0x80008000u : 0u;
#pragma unroll
      for (int u = 0; u < 16 / ROWS; ++u) {
        const int rr = warp_row + side * 16 + u * ROWS + my_r;
        uint32_t y[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 g = Bf16::to_float2(y[e]);
          y[e] = a.f16 ? y[e] ^ flip : f16x2(make_float2(g.x * f, g.y * f));
        }
        st_shared_v4(q_at + x * Q_HALF + (my_c / 8) * Q_ATOM + rr * 128 + (((my_c % 8) ^ (rr & 7)) << 4), y[0], y[1], y[2],
                     y[3]);
      }
      if (lane == 0) ctl->q_shift[x][side][warp & 3] = shift;
      fence_proxy_async();
      arrive(ctl->q_full);
      pair_any(pair, false);
      coef = fabsf(a.coef) * pow2i(-ctl->q_shift[x][lane >> 4][warp & 3]);
    }

    const uint32_t lanes = static_cast<uint32_t>(warp_row) << 16;
    const uint32_t o_at = tmem + lanes + O_COL + x * TILE + side * (D / 2);  // this side's columns of O
    const bool any_live = __any_sync(~0u, live);
    float m = -INFINITY, M = -INFINITY, L = 0.f;
    // After a wait that gave up the warp goes through the rest without waiting (the products have stopped, the results are
    // invalid): it meets its pair's barriers as often as the other warp does.
    bool ok = true;
    // One tile: the thread's scores become weights, over themselves in tensor memory. CUT: some row of the warp does not
    // see all tokens of the tile.
    const auto softmax = [&](auto cut, int j) {
      constexpr bool CUT = decltype(cut)::value;
      constexpr int GROUPS = BIG ? 1 : W / 16, GW = W / GROUPS;  // runs of columns that share a scale
      const uint32_t s_at = tmem + lanes + x * TILE + j % AHEAD * TOK + side * W;
      const float* ks = ctl->ks[j & 7] + side * (W / 16);
      const float* ve = ctl->ve[j & 7] + side * (W / 16);
      const int left = vis - (begin + j * TOK) - side * W;  // columns this row sees
      float s_top = -INFINITY, u_top = -INFINITY;
      __syncwarp();
#pragma unroll
      for (int c = 0; c < W / 32; ++c) {
        float v[32];
        bd::tmem_ld32(s_at + c * 32, v);
        constexpr int CG = GW < 32 ? GW : 32;  // columns of a run in this load
#pragma unroll
        for (int b = 0; b < 32 / CG; ++b) {
          float t = -INFINITY, t1 = -INFINITY;
#pragma unroll
          for (int e = b * CG; e < b * CG + CG; e += 4) {
            if (CUT)
#pragma unroll
              for (int k = e; k < e + 4; ++k)
                if (c * 32 + k >= left) v[k] = -INFINITY;
            t = bd::max3(t, v[e], v[e + 1]);
            t1 = bd::max3(t1, v[e + 2], v[e + 3]);
          }
          t = fmaxf(t, t1);
          const int g = (c * 32 + b * CG) / GW;
          const float s2 = CUT && t == -INFINITY ? t : t * (coef * ks[g]);
          s_top = fmaxf(s_top, s2);
          u_top = fmaxf(u_top, s2 + ve[g]);
        }
      }
      const float m_new = fmaxf(m, s_top);
      L *= m_new == m ? 1.f : bd::ex2_approx(m - m_new);
      m = m_new;
      if (pair_any(pair, u_top > M + P_SLACK || (M == -INFINITY && u_top > M))) {
        ctl->row[x][side][r].x = u_top;
        pair_any(pair, false);
        u_top = fmaxf(u_top, ctl->row[x][side ^ 1][r].x);
        const bool grow = u_top > M + P_SLACK || (M == -INFINITY && u_top > M);
        if (j > 0 && __any_sync(~0u, grow)) {
          // O's product of the tile before is done where scores issued behind it are: this tile's, or with two tiles ahead
          // the next one's
          if (AHEAD == 2)
            ok = ok && (j + 1 < n ? wait(ctl->s_full[x][(j + 1) & 1], (j + 1) >> 1) : wait(ctl->o_before[x], 0));
          bd::tc_fence_after();
          const float f = grow ? bd::ex2_approx(M - u_top) : 1.f;
          __syncwarp();  // tensor-memory accesses take the whole warp at once
#pragma unroll 1
          for (int c = 0; c < D / 64; ++c) {
            float o[32];
            bd::tmem_ld32(o_at + c * 32, o);
            uint32_t y[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(o[e] * f);
            bd::tmem_st32(o_at + c * 32, y);
          }
        }
        M = grow ? u_top : M;
      }
      const float ms = m == -INFINITY ? 0.f : m, Ms = M == -INFINITY ? 0.f : M;
      // The weights' sum times 2^(ref - m) is the thread's share of L, unless the weights may have gone to zero where that
      // share has not (this side's scores, or a page's values, are far below the row's): then L is summed for itself.
      bool apart = false;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) apart |= Ms - ve[g] - P_SHIFT - ms > 60.f;
      apart = __any_sync(~0u, apart);
      if (apart) {
        float own = 0.f;
#pragma unroll 1
        for (int c = 0; c < W / 32; ++c) {
          float v[32];
          bd::tmem_ld32(s_at + c * 32, v);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (c * 32 + e < left) own += bd::ex2_approx(fmaf(v[e], coef * ks[(c * 32 + e) / GW], -ms));
        }
        L += own;
      }
      float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
      __syncwarp();
#pragma unroll
      for (int c = 0; c < W / 32; ++c) {
        float v[32];
        bd::tmem_ld32(s_at + c * 32, v);
        uint32_t p[16];
#pragma unroll
        for (int col = 0; col < 32; col += 2) {
          const int at = c * 32 + col, g = at / GW;
          const float f = coef * ks[g], ref = Ms - ve[g] - P_SHIFT;
          const float2 y = bd::fma2(make_float2(v[col], v[col + 1]), make_float2(f, f), make_float2(-ref, -ref));
          float2 w = make_float2(bd::ex2_approx(y.x), bd::ex2_approx(y.y));
          if (CUT) {
            if (at >= left) w.x = 0.f;
            if (at + 1 >= left) w.y = 0.f;
          }
          sum[col / 2 & 1] = bd::add2(sum[col / 2 & 1], w);
          p[col / 2] = f16x2(w);
          if (at % GW == GW - 2) {
            const float2 t = bd::add2(sum[0], sum[1]);
            L += (t.x + t.y) * (apart ? 0.f : bd::ex2_approx(ref - ms));
            sum[0] = sum[1] = make_float2(0.f, 0.f);
          }
        }
        tmem_st16(s_at + c * 16, p);
      }
      bd::tmem_st_wait();
    };

    const int whole = __reduce_min_sync(~0u, max(vis - begin, 0)) / TOK;  // tiles that all rows of the warp see all of
    for (int j = 0; j < n; ++j) {
      ok = ok && wait(ctl->s_full[x][j % AHEAD], j / AHEAD);
      bd::tc_fence_after();
      if (any_live) {
        if (j < whole) softmax(std::false_type(), j); else softmax(std::true_type(), j);
      }
      bd::tc_fence_before();
      arrive(ctl->p_full[x][j % AHEAD]);
    }

    if (n > 0 && ok) wait(ctl->o_done[x], 0);
    bd::tc_fence_after();
    if (any_live) {  // (for both warps of a pair alike)
      ctl->row[x][side][r] = make_float2(m, L);
      pair_any(pair, false);
      const float2 other = ctl->row[x][side ^ 1][r];
      const float mt = fmaxf(m, other.x), ms = mt == -INFINITY ? 0.f : mt, Ms = M == -INFINITY ? 0.f : M;
      const float Lt = L * bd::ex2_approx(m - ms) + other.y * bd::ex2_approx(other.x - ms);
      const float f = Lt == 0.f ? 0.f : bd::ex2_approx(Ms - P_SHIFT - ms) / Lt;
      RowOut o = {nullptr, nullptr, nullptr};
      if (live) o = row_out(a, sq, seq, part, i, h, visible(a, sq, i));
      if (side == 0) store_lse(o, Lt == 0.f ? -INFINITY : ms + log2f(Lt));
      // This side's columns go through shared memory that no product reads any more (the queries' for one side, the keys'
      // for the other): lanes write their rows, the warp stores them row by row.
      const uint32_t stage = (side == 0 ? q_at : k_at) + x * Q_HALF + warp_row * (D * 2);
      const auto give = [&](auto chunks, const void* mine, int elements) {
        constexpr int C = decltype(chunks)::value;  // 16-byte chunks of a row
        const int my_c = lane % C, my_r = lane / C;
        const bool there = side * (D / 2) + my_c * elements < a.dim;
        __syncwarp();
#pragma unroll 4
        for (int u = 0; u < C; ++u) {
          const int rr = u * (32 / C) + my_r;
          const uint64_t dst = __shfl_sync(~0u, reinterpret_cast<uint64_t>(mine), rr);
          const uint4 w = bd::ld_shared_v4(stage + rr * (C * 16) + ((my_c ^ (rr & (C < 8 ? C - 1 : 7))) << 4));
          if (dst != 0 && there) *reinterpret_cast<uint4*>(dst + my_c * 16) = w;
        }
        __syncwarp();
      };
      const auto put = [&](auto chunks, int c, uint32_t y0, uint32_t y1, uint32_t y2, uint32_t y3) {
        constexpr int C = decltype(chunks)::value;
        st_shared_v4(stage + lane * (C * 16) + ((c ^ (lane & (C < 8 ? C - 1 : 7))) << 4), y0, y1, y2, y3);
      };
      const bool direct = __any_sync(~0u, o.out != nullptr), parts = __any_sync(~0u, o.o != nullptr);
      const std::integral_constant<int, D / 16> half;
      const std::integral_constant<int, D / 8> full;
      for (int kind = 0; kind < 2; ++kind) {
        if (!(kind == 0 ? direct : parts)) continue;
#pragma unroll 1
        for (int c = 0; c < D / 64; ++c) {
          float v[32];
          if (n > 0)
            bd::tmem_ld32(o_at + c * 32, v);
          else
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] *= f;
          if (kind == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t y[4];
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const float2 g = make_float2(v[e * 8 + u * 2], v[e * 8 + u * 2 + 1]);
                y[u] = a.f16 ? F16::from_float2(g) : Bf16::from_float2(g);
              }
              put(half, c * 4 + e, y[0], y[1], y[2], y[3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              put(full, c * 8 + e, __float_as_uint(v[e * 4]), __float_as_uint(v[e * 4 + 1]), __float_as_uint(v[e * 4 + 2]),
                  __float_as_uint(v[e * 4 + 3]));
          }
        }
        if (kind == 0)
          give(half, o.out == nullptr ? nullptr : o.out + side * (D / 2), 8);
        else
          give(full, o.o == nullptr ? nullptr : o.o + side * (D / 2), 4);
      }
    }
  }

  __syncwarp();
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  if (warp == MMA_WARP) bd::tmem_dealloc(tmem, 512);
}

template <int NM, int D, bool BIG>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  const auto kernel = attn_tiles_kernel<NM, D, BIG>;
  if (cudaError_t e = allow_smem(kernel, smem_bytes<NM, D>(), ready); e != cudaSuccess) return e;
  const int tiles = (a.max_q * a.group + NM * TILE - 1) / (NM * TILE);
  const dim3 grid(tiles * a.n_kv, a.n_split, a.n_seq);
  kernel<<<grid, Shape<NM>::THREADS, smem_bytes<NM, D>(), st>>>(a);
  return cudaGetLastError();
}

template <int NM, int D>
cudaError_t launch_pages(const AttnArgs& a, cudaStream_t st) {
  return a.page_shift >= 6 ? launch<NM, D, true>(a, st) : launch<NM, D, false>(a, st);
}

}  // namespace

cudaError_t launch_attn_tiles(const AttnArgs& a, cudaStream_t st) {
  const bool one = a.max_q * a.group <= TILE;
  if (a.dim <= 64) return one ? launch_pages<1, 64>(a, st) : launch_pages<2, 64>(a, st);
  return one ? launch_pages<1, 128>(a, st) : launch_pages<2, 128>(a, st);
}

cudaError_t tiles_status(cudaStream_t st, uint32_t* bits) {
  cudaError_t e = cudaMemcpyFromSymbolAsync(bits, g_status, sizeof *bits, 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess || *bits == 0) return e;
  const uint32_t zero = 0;
  e = cudaMemcpyToSymbolAsync(g_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

}  // namespace bdkv
