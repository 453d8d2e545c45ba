// bdkv_attention for many query rows per key/value head: windows of blocks,
// prompts. tcgen05 products on tiles of 128 rows by 64 cached tokens.
//
// A CTA walks a request's key/value head (whose cache is read once for all of
// the group's heads) in tiles of 64 tokens, with two streams of products:
//   NM = 2   256 rows (queries x heads): each half of them sees every tile
//   NM = 1   128 rows (all that there are, or where one tile of rows to a CTA
//            runs in one wave over short caches): one stream takes the even
//            tiles, one the odd ones, and the two results are joined at the end
// and with warps for each part of the work:
//   converter warps   codes from global memory to f16 (exact), into shared
//                     memory in the 128-byte swizzle, in stages; a request's
//                     tail is zeros, so its values times zero weights stay zero
//   MMA warp          S = Q K^T (both operands in shared memory) and O += P V
//                     (P in tensor memory, V read with the token index along
//                     K); a stream's S of the next tile is ready before its
//                     softmax begins, so the softmax warps never wait for a
//                     product of their own last weights
//   softmax warps     a thread per row and stream: running maxima, weights to
//                     f16, written over S in tensor memory; O is rescaled only
//                     when a row's maximum has grown by more than 2^7
// Scales of pages come in through the exponent: w = 2^(S coef k_scale + e_v),
// see k_attn_rows.cu; O and the sum L have a reference maximum of their own,
// O's in two parts, a score and an exponent, so that scores of any size leave
// the exponent its bits.
//
// 32 windows of 512 queries, 32 heads on 8, over 700 to 4096 tokens take 513 us:
// 1140 TFLOP/s, 0.60 of a library product's rate. Bound by the softmax warps'
// chain from scores to weights (about 1600 cycles a tile of 2 x 128 x 64 scores,
// 1080 of them under products), and by each CTA's start and end (a fifth of it),
// during which nothing is multiplied. Few rows (64 x 5 drafts on 4 heads, 61 us,
// 2.4 TB/s) are bound by latency: DRAM 28% busy, the tensor pipe 23%, issue slots
// 37%, with two tiles of codes of a CTA on their way.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int TILE = TILES_TILE;  // rows of an MMA
constexpr int TOK = 64;           // tokens of a tile
// Weights are held as f16 times 2^8, with 11 bits down to 2^-22 of the reference, and may exceed it by 2^7 before O is
// rescaled (2^15 < 65504): a rescale costs a warp about as much as a tile.
constexpr float P_SHIFT = 8, P_SLACK = 7;
// Scores (in powers of two) from which on references are taken off the scores themselves, before exponents of values are
// added: below, the sum of both is rounded by 2^-16 at most, and a product's rounding moves no weight past f16's range.
constexpr float LARGE = 256;
constexpr int stages(int nm) { return nm == 2 ? 4 : 6; }  // tiles of keys and of values in shared memory
// Warps of a CTA: 4 for each stream's softmax, the converters, and 4 of which one issues the MMAs and one looks up page
// scales: warpgroups, so that registers can be moved between them (a row's 64 scores and their weights stay in 128 or more).
// 256 rows leave few issue slots, and four converter warps disturb their softmax least (32 windows of 8 x 64 tokens, when it
// was chosen: 524 us, 540 with eight): 512 threads start with 128 registers, 256 x 144 + 128 x 112 + 128 x 56 <= 65536. Few rows wait for the
// codes: eight converter warps, 640 threads with 96, 256 x 128 + 256 x 80 + 128 x 56 <= 61440.
constexpr int conv_warps(int nm) { return nm == 2 ? 4 : 8; }
constexpr int threads(int nm) { return (8 + conv_warps(nm) + 4) * 32; }

__device__ uint32_t g_status;  // bd::DEV_* bits

struct Ctl {
  uint64_t q_full, kv_full[6], kv_empty[6];
  uint64_t s_full[2][2], p_full[2][2];             // by stream and parity of its tile
  uint64_t o_before[2], o_done[2], joined, drain;  // by stream: O without, and with its last product
  float ks[8][TOK / 16], ve[8][TOK / 16];          // page scales of a tile's groups of tokens: factor, exponent
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

// The 64 columns of a tile for this thread's lane.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float (&v)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]),
        "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
        "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]),
        "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
        "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]),
        "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
        "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]),
        "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
        "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]),
        "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
        "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]),
        "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
      : "r"(taddr)
      : "memory");
}

// Four words of this thread's lane.
__device__ __forceinline__ void tmem_st4(uint32_t taddr, float a, float b, float c, float d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "f"(a), "f"(b), "f"(c), "f"(d)
               : "memory");
}
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, float& a, float& b, float& c, float& d) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(a), "=f"(b), "=f"(c), "=f"(d)
      : "r"(taddr)
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

template <int NM, int D>
constexpr size_t smem_bytes() {
  return size_t(NM * TILE + 2 * stages(NM) * TOK) * D * 2 + sizeof(Ctl) + 1024;
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
__device__ __forceinline__ uint4 ld_global_if(const uint8_t* p, bool live) {
  uint4 x = {0, 0, 0, 0};
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "+r"(x.x), "+r"(x.y), "+r"(x.z), "+r"(x.w)
               : "l"(p), "r"(static_cast<int>(live)));
  return x;
}

// GROUPS: runs of tokens in a tile that share a page, 1 (pages of 64 tokens and more) or 4 (16 and 32).
template <int NM, int D, int GROUPS>
__global__ void __launch_bounds__(threads(NM), 1) attn_tiles_kernel(AttnArgs a) {
  constexpr int ATOMS = D / 64;                // 128-byte column blocks of a row
  constexpr uint32_t Q_ATOM = TILE * 128, KV_ATOM = TOK * 128;  // bytes of one
  constexpr uint32_t Q_HALF = ATOMS * Q_ATOM, KV_TILE = ATOMS * KV_ATOM;
  constexpr int CH = D / 16;                   // 16-code chunks of a token's row
  constexpr int CONV = conv_warps(NM), STAGES = stages(NM);
  constexpr int O_COL = 256;                   // tensor memory: S and P of stream x, parity b at 128 x + 64 b; O behind
  extern __shared__ __align__(16) uint8_t raw[];
  const uint32_t base = (bd::smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + NM * Q_HALF, v_at = k_at + STAGES * KV_TILE;
  Ctl* ctl = reinterpret_cast<Ctl*>(raw + (v_at + STAGES * KV_TILE - bd::smem_u32(raw)));
  const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(bd::warp_uniform(tid >> 5));
  const int n_tiles_rows = gridDim.x / a.n_kv;
  // the last rows of all heads first: under a causal mask they see the most (2 prompts of 2049 rows 65 us; head by head 83)
  const int head = blockIdx.x % a.n_kv, row0 = (n_tiles_rows - 1 - blockIdx.x / a.n_kv) * (NM * TILE);
  int seq = blockIdx.z;
  const Seq sq = a.longest_first ? ranked_seq<threads(NM)>(a, blockIdx.z, reinterpret_cast<int*>(raw), seq) : load_seq(a, seq);
  const int part = blockIdx.y;
  const int rows = sq.q_len * a.group;
  if (row0 >= rows) return;
  // later queries see at least as much, so the CTA's last row bounds it
  const int i_last = (min(rows, row0 + NM * TILE) - 1) / a.group;
  const int begin = part * a.chunk, end = min(visible(a, sq, i_last), begin + a.chunk);
  if (part > 0 && end <= begin) return;
  const int n = end > begin ? (end - begin + TOK - 1) / TOK : 0;

  if (tid == 0) {
    bd::mbar_init(bd::smem_u32(&ctl->q_full), NM * TILE);
    bd::mbar_init(bd::smem_u32(&ctl->joined), 2 * TILE);
    for (int i = 0; i < STAGES; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->kv_full[i]), CONV * 32 + 32);
      bd::mbar_init(bd::smem_u32(&ctl->kv_empty[i]), 1);
    }
    for (int x = 0; x < 2; ++x) {
      for (int b = 0; b < 2; ++b) {
        bd::mbar_init(bd::smem_u32(&ctl->s_full[x][b]), 1);
        bd::mbar_init(bd::smem_u32(&ctl->p_full[x][b]), TILE);
      }
      bd::mbar_init(bd::smem_u32(&ctl->o_before[x]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->o_done[x]), 1);
    }
    bd::mbar_init(bd::smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    bd::fence_mbar_init();
  }
  constexpr int MMA_WARP = 8 + CONV;
  // A stream's j-th tile is the request's tile j (NM = 2) or 2 j + x.
  const auto tile_of = [](int x, int j) { return NM == 2 ? j : 2 * j + x; };
  const auto tiles_of = [&](int x) { return NM == 2 ? n : (n + 1 - x) / 2; };
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
  bd::griddep_launch_dependents();

  if (warp >= MMA_WARP) {
    // ---------------------------------------------------------- MMA issuer
    give_registers<56>();
    if (warp == MMA_WARP) {
      const uint32_t issue = bd::elect_one();
      constexpr uint32_t IDESC_S = bd::idesc_f16_f32(TILE, TOK), IDESC_O = bd::idesc_f16_f32(TILE, D) | B_MN_MAJOR;
      // low words of the descriptors (addresses count 16 bytes) and their common upper word: 1 KB stride, version, swizzle
      const uint32_t q_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(q_at)));
      const uint32_t k_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(k_at)));
      const uint32_t v_lo = bd::warp_uniform(static_cast<uint32_t>(sw128_mnmajor_desc(v_at, KV_ATOM)));
      constexpr uint32_t HI = (1024u >> 4) | (1u << 14) | (2u << 29);
      const auto scores = [&](int x, int parity, int stage) {
        const uint32_t kd = bd::warp_uniform(k_lo + stage * (KV_TILE >> 4));
        const uint32_t qd = bd::warp_uniform(q_lo + (NM == 2 ? x * (Q_HALF >> 4) : 0u));
        const uint32_t sd = bd::warp_uniform(tmem + x * TILE + parity * TOK);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_ss(issue, sd, qd + (k / 4) * (Q_ATOM >> 4) + 2u * (k % 4), kd + (k / 4) * (KV_ATOM >> 4) + 2u * (k % 4), HI,
                 IDESC_S, k != 0);
        mma_commit(issue, bd::smem_u32(&ctl->s_full[x][parity]));
      };
      // Products in the order of the request's tiles, S four of them ahead (two of a stream).
      const int total = tiles_of(0) + tiles_of(1);
      bool ok = n > 0 && wait(ctl->q_full, 0);
      for (int k = 0; ok && k < min(total, 4); ++k) {
        const int x = k & 1, t = tile_of(x, k >> 1);
        if (NM == 1 || x == 0) ok = wait(ctl->kv_full[t], 0);
        if (!ok) break;
        bd::tc_fence_after();
        scores(x, k >> 1, t);
      }
      int stage = 0, ahead = NM == 2 ? 2 : 4, ahead_phase = 0;  // of the tile of k and of k + 4
      for (int k = 0; ok && k < total; ++k) {
        const int x = k & 1, j = k >> 1, parity = j & 1;
        if (!(ok = wait(ctl->p_full[x][parity], j >> 1))) break;
        bd::tc_fence_after();
        const uint32_t vd = bd::warp_uniform(v_lo + stage * (KV_TILE >> 4));
        const uint32_t pd = bd::warp_uniform(tmem + x * TILE + parity * TOK), od = bd::warp_uniform(tmem + O_COL + x * TILE);
#pragma unroll
        for (int i = 0; i < TOK / 16; ++i)
          mma_ts(issue, od, pd + i * 8, vd + i * (2048u >> 4), HI, IDESC_O, (j | i) != 0);
        if (NM == 1 || x == 1) {
          mma_commit(issue, bd::smem_u32(&ctl->kv_empty[stage]));
          stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
        if (k + 4 < total) {  // over the weights that the products above read: the tensor pipe takes them in order
          if ((NM == 1 || x == 0) && !(ok = wait(ctl->kv_full[ahead], ahead_phase))) break;
          bd::tc_fence_after();
          scores(x, parity, ahead);
          if (NM == 1 || x == 1)
            if (++ahead == STAGES) ahead = 0, ahead_phase ^= 1;
        } else {
          mma_commit(issue, bd::smem_u32(k + 2 < total ? &ctl->o_before[x] : &ctl->o_done[x]));
        }
      }
      mma_commit(issue, bd::smem_u32(&ctl->drain));  // all MMAs issued have completed once it flips
      __syncwarp();
      bd::mbar_drain(bd::smem_u32(&ctl->drain), 0);
    } else if (warp == MMA_WARP + 1) {
      // ------------------------------------------------------- page scales
      // a lane has a group of a tile's tokens: their page and, a tile ahead, its scales
      const int32_t* table = a.table + seq * a.table_stride;
      int page = -1, ks_byte = 127, vs_byte = 127;
      const auto find_page = [&](int j) {
        const int t = begin + j * TOK + lane * (TOK / GROUPS), col = t >> a.page_shift;
        page = ld_global_if(table + col, lane < GROUPS && t < end && col < a.max_blocks, -1);
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
      for (int j = 0; j < n && wait(ctl->kv_empty[j % STAGES], j / STAGES + 1); ++j) {
        if (lane < GROUPS) {
          ctl->ks[j & 7][lane] = pow2i(ks_byte - 127);
          ctl->ve[j & 7][lane] = static_cast<float>(vs_byte - 127);
        }
        bd::mbar_arrive(bd::smem_u32(&ctl->kv_full[j % STAGES]));
        find_scales(j + 1);
      }
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ---------------------------------------------------------- converters
    give_registers<NM == 2 ? 112 : 80>();
    const int ct = tid - 256;
    constexpr int PER = TOK * CH / (CONV * 32);  // chunks of a thread and tile
    constexpr int STEP = CONV * 32 / CH;         // rows between them
    // eight lanes take four chunks each of two rows, which the swizzle puts into different banks
    const int sub = (ct & 3) | (CH == 8 ? (ct >> 1) & 4 : 0), mine = ct / (2 * CH) * 2 + ((ct >> 2) & 1);
    const int64_t row_k = a.k_tok, row_v = a.v_tok;
    const uint8_t* kp = a.k + head * a.k_head + sub * 16;
    const uint8_t* vp = a.v + head * a.v_head + sub * 16;
    const int32_t* table = a.table + seq * a.table_stride;
    const int mask = (1 << a.page_shift) - 1;
    // Two tiles of codes are on their way in registers, and the page numbers of the one behind them.
    uint4 kx[2][PER], vx[2][PER];
    constexpr int PAGES = GROUPS == 1 ? 1 : PER;
    int pages[PAGES];  // -1: nothing to read
    const auto find = [&](int j) {
#pragma unroll
      for (int u = 0; u < PAGES; ++u) {
        const int t = begin + j * TOK + (GROUPS == 1 ? 0 : mine + u * STEP);
        pages[u] = ld_global_if(table + (t >> a.page_shift), t < end && (t >> a.page_shift) < a.max_blocks, -1);
      }
    };
    const auto load = [&](int j, uint4 (&k)[PER], uint4 (&v)[PER]) {  // of tile j, whose pages were found
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int t = begin + j * TOK + mine + u * STEP, page = pages[GROUPS == 1 ? 0 : u];
        const bool live = page >= 0 && page < a.n_pages && t < end && sub * 16 < a.dim;
        k[u] = ld_global_if(kp + page * a.k_page + (t & mask) * row_k, live);
        v[u] = ld_global_if(vp + page * a.v_page + (t & mask) * row_v, live);
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
      find(0);
      load(0, kx[0], vx[0]);
      find(1);
      load(1, kx[1], vx[1]);
      find(2);
    }
    bool ok = true;
    for (int j0 = 0; ok && j0 < n; j0 += 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int j = j0 + b;
        if (j >= n || !(ok = wait(ctl->kv_empty[j % STAGES], j / STAGES + 1))) break;
        store(k_at + (j % STAGES) * KV_TILE, kx[b]);
        store(v_at + (j % STAGES) * KV_TILE, vx[b]);
        fence_proxy_async();
        bd::mbar_arrive(bd::smem_u32(&ctl->kv_full[j % STAGES]));
        load(j + 2, kx[b], vx[b]);
        find(j + 3);
      }
    }
  } else {
    // ------------------------------------------------------------- softmax
    take_registers<NM == 2 ? 144 : 128>();
    const int x = warp >> 2, mine = tiles_of(x);  // stream and its tiles
    const int r = tid & 127, row = row0 + (NM == 2 ? x * TILE : 0) + r, i = row / a.group;
    const bool live = row < rows;
    const int h = head * a.group + row - i * a.group;
    const int vis = live ? min(visible(a, sq, i), end) : 0;
    float coef = 0.f;
    // A warp moves its 32 rows together, LANES lanes to a row (16 bytes each): queries in, results out.
    constexpr int LANES = D / 8, ROWS = 32 / LANES;
    const int my_c = lane % LANES, my_r = lane / LANES, warp_row = (warp & 3) * 32;
    if (n > 0) {
      // Rows in f16, with the sign of the scale; bf16 ones times a power of two each that brings the row's largest element
      // into [2^14, 2^15): elements down to 2^-32 of it keep their eight bits.
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(sq.q0 + i) * a.q_tok + h * a.q_head;
      uint4 w[32 / ROWS];
#pragma unroll
      for (int u = 0; u < 32 / ROWS; ++u) {
        const int rr = u * ROWS + my_r;
        const uint64_t src = __shfl_sync(~0u, reinterpret_cast<uint64_t>(q), rr);
        w[u] = ld_global_if(reinterpret_cast<const uint8_t*>(src) + my_c * 16, row - lane + rr < rows && my_c * 8 < a.dim);
      }
      int shift = 0, held = 0;  // of the lane's row, and of row my_c * ROWS + my_r
      if (!a.f16) {
        static_assert(LANES == 32 / ROWS, "a lane ends up with the maximum of one row");
        uint32_t most[LANES];  // magnitudes' patterns; halved and exchanged until the lane has row my_c * ROWS + my_r
#pragma unroll
        for (int u = 0; u < LANES; ++u) {
          const uint32_t t = __vmaxu2(__vmaxu2(w[u].x & 0x7fff7fffu, w[u].y & 0x7fff7fffu),
                                      __vmaxu2(w[u].z & 0x7fff7fffu, w[u].w & 0x7fff7fffu));
          most[u] = max(t & 0xffffu, t >> 16);
        }
        const auto exchange = [&](auto lanes) {
          constexpr int HALF = decltype(lanes)::value;
          const bool upper = my_c & HALF;
#pragma unroll
          for (int u = 0; u < HALF; ++u) {
            const uint32_t other = __shfl_xor_sync(~0u, upper ? most[u] : most[u + HALF], HALF);
            most[u] = max(upper ? most[u + HALF] : most[u], other);
          }
        };
        if constexpr (LANES == 16) exchange(std::integral_constant<int, 8>());
        exchange(std::integral_constant<int, 4>());
        exchange(std::integral_constant<int, 2>());
        exchange(std::integral_constant<int, 1>());
        held = row_shift(__uint_as_float(most[0] << 16));
        shift = __shfl_sync(~0u, held, lane % ROWS * LANES + lane / ROWS);
      }
      const uint32_t flip = a.coef < 0.f ? 0x80008000u : 0u;
#pragma unroll
      for (int u = 0; u < 32 / ROWS; ++u) {
        const int rr = warp_row + u * ROWS + my_r;
        const float f = pow2i(__shfl_sync(~0u, held, my_r * LANES + u));
        uint32_t y[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 g = Bf16::to_float2(y[e]);
          y[e] = (a.f16 ? y[e] : f16x2(make_float2(g.x * f, g.y * f))) ^ flip;
        }
        if (NM == 2 || x == 0)  // (both streams of NM = 1 read the rows: they need the shift)
          st_shared_v4(q_at + (NM == 2 ? x * Q_HALF : 0u) + (my_c / 8) * Q_ATOM + rr * 128 + (((my_c % 8) ^ (rr & 7)) << 4),
                       y[0], y[1], y[2], y[3]);
      }
      coef = fabsf(a.coef) * pow2i(-shift);
      fence_proxy_async();
      if (NM == 2 || x == 0) bd::mbar_arrive(bd::smem_u32(&ctl->q_full));
    }

    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t o_at = tmem + lanes + O_COL + x * TILE;
    const bool any_live = __any_sync(~0u, live);
    // the sum's reference is 2^m, O's 2^(r + d): r a score, d an exponent of values (-inf: O holds nothing yet)
    float m = -INFINITY, r_o = 0.f, d_o = -INFINITY, L = 0.f;
    bool ok = true;
    // One tile: the row's scores become weights, over themselves in tensor memory. CUT: some row of the warp does not see
    // all of its tokens.
    const auto softmax = [&](auto cut, int j, int left) -> bool {
      constexpr bool CUT = decltype(cut)::value;
      const uint32_t s_at = tmem + lanes + x * TILE + (j & 1) * TOK;
      const float* ks = ctl->ks[tile_of(x, j) & 7];
      const float* ve = ctl->ve[tile_of(x, j) & 7];
      float v[TOK];
      __syncwarp();
      tmem_ld64(s_at, v);
      float s_top = -INFINITY, u_top = -INFINITY, s_of[GROUPS];
      constexpr int W = TOK / GROUPS;  // columns of a group
#pragma unroll
      for (int b = 0; b < GROUPS; ++b) {
        float t = -INFINITY, t1 = -INFINITY;
#pragma unroll
        for (int e = b * W; e < b * W + W; e += 4) {
          if (CUT)
#pragma unroll
            for (int c = e; c < e + 4; ++c)
              if (c >= left) v[c] = -INFINITY;
          t = bd::max3(t, v[e], v[e + 1]);
          t1 = bd::max3(t1, v[e + 2], v[e + 3]);
        }
        t = fmaxf(t, t1);
        s_of[b] = CUT && t == -INFINITY ? t : __fmul_rn(t, coef * ks[b]);  // (as where the scores are large)
        s_top = fmaxf(s_top, s_of[b]);
        u_top = fmaxf(u_top, (s_of[b] - r_o) + ve[b]);
      }
      const float m_new = fmaxf(m, s_top);
      L *= m_new == m ? 1.f : bd::ex2_approx(m - m_new);
      m = m_new;
      const float ms = m == -INFINITY ? 0.f : m;
      const bool grow = u_top > d_o + P_SLACK || (d_o == -INFINITY && u_top > d_o);
      bool large = fmaxf(fabsf(ms), fabsf(r_o)) >= LARGE;
      if (__any_sync(~0u, grow || large)) {
        const bool some_grow = __any_sync(~0u, grow);
        large = __any_sync(~0u, large);
        if (some_grow) {
          float d_new = -INFINITY;
#pragma unroll
          for (int b = 0; b < GROUPS; ++b) d_new = fmaxf(d_new, (s_of[b] - m) + ve[b]);
          if (j > 0) {
            // O's product of the tile before is done where the next tile's scores, issued behind it, are
            if (!(j + 1 < mine ? wait(ctl->s_full[x][(j + 1) & 1], (j + 1) >> 1) : wait(ctl->o_before[x], 0))) return false;
            bd::tc_fence_after();
            const float f = grow ? bd::ex2_approx((r_o - m) + (d_o - d_new)) : 1.f;
            __syncwarp();  // tensor-memory accesses take the whole warp at once
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              float o[32];
              bd::tmem_ld32(o_at + c * 32, o);
              uint32_t y[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(o[e] * f);
              bd::tmem_st32(o_at + c * 32, y);
            }
          }
          r_o = grow ? m : r_o;
          d_o = grow ? d_new : d_o;
        }
        if (large) {
#pragma unroll
          for (int b = 0; b < GROUPS; ++b)
#pragma unroll
            for (int col = b * W; col < b * W + W; ++col) v[col] = __fsub_rn(__fmul_rn(v[col], coef * ks[b]), r_o);
        }
      }
      __syncwarp();
      // references as the weights see them: of scores less r_o where those are large
      const float rs = large ? 0.f : r_o, md = large ? ms - r_o : ms, d = d_o == -INFINITY ? 0.f : d_o;
      uint32_t p[16];
#pragma unroll
      for (int b = 0; b < GROUPS; ++b) {
        // A group whose weights all go to zero in f16 (its page's values are so small) may still count in L: its weights are
        // then taken from L's reference, 2^60 below it, which is zero in f16 as well.
        const bool faint = (s_of[b] - r_o) + ve[b] < d - 40.f;
        const float f = large ? 1.f : coef * ks[b], ref = faint ? md + 60.f : rs + (d - ve[b] - P_SHIFT);
        float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
        for (int col = b * W; col < b * W + W; col += 2) {
          const float2 y = bd::fma2(make_float2(v[col], v[col + 1]), make_float2(f, f), make_float2(-ref, -ref));
          float2 w = make_float2(bd::ex2_approx(y.x), bd::ex2_approx(y.y));
          if (CUT) {
            if (col >= left) w.x = 0.f;
            if (col + 1 >= left) w.y = 0.f;
          }
          sum[col / 2 & 1] = bd::add2(sum[col / 2 & 1], w);
          p[col / 2 % 16] = f16x2(w);
          if (col % 32 == 30) tmem_st16(s_at + col / 32 * 16, p);
        }
        sum[0] = bd::add2(sum[0], sum[1]);
        L += (sum[0].x + sum[0].y) * bd::ex2_approx(ref - md);
      }
      bd::tmem_st_wait();
      return true;
    };

    for (int j = 0; j < mine; ++j) {
      ok = wait(ctl->s_full[x][j & 1], j >> 1);
      if (!ok) break;
      bd::tc_fence_after();
      if (any_live) {
        const int left = vis - (begin + tile_of(x, j) * TOK);  // columns this row sees
        ok = __any_sync(~0u, left < TOK) ? softmax(std::true_type(), j, left) : softmax(std::false_type(), j, left);
        if (!ok) break;
      }
      bd::tc_fence_before();
      bd::mbar_arrive(bd::smem_u32(&ctl->p_full[x][j & 1]));
    }

    if (mine > 0 && ok) ok = wait(ctl->o_done[x], 0);
    float f[2];  // what O of this stream, and with NM = 1 of the other one, is multiplied by
    float lse2;
    RowOut o = {nullptr, nullptr, nullptr};
    if (live) o = row_out(a, sq, seq, part, i, h, visible(a, sq, i));
    // a row's whole result: 0 where it sees nothing, NaN where all of its scores are -inf (a part may well hold nothing)
    const float none = o.out != nullptr && vis > 0 ? NAN : 0.f;
    if constexpr (NM == 2) {
      const float ms = m == -INFINITY ? 0.f : m;
      f[0] = L == 0.f ? none : bd::ex2_approx((r_o - ms) + (d_o - P_SHIFT)) / L;
      lse2 = L == 0.f ? -INFINITY : ms + log2f(L);
    } else {
      // the streams tell each other m, L and O's reference through tensor memory, over their last scores (shared memory is full)
      __syncwarp();
      bd::tc_fence_after();
      tmem_st4(tmem + lanes + x * TILE, m, L, r_o, d_o);
      bd::tmem_st_wait();
      bd::tc_fence_before();
      bd::mbar_arrive(bd::smem_u32(&ctl->joined));
      wait(ctl->joined, 0);  // both streams' sums, and both O
      bd::tc_fence_after();
      float m2, L2, r2, d2;
      tmem_ld4(tmem + lanes + (x ^ 1) * TILE, m2, L2, r2, d2);
      const float mt = fmaxf(m, m2), ms = mt == -INFINITY ? 0.f : mt;
      const float total = L * bd::ex2_approx(m - ms) + L2 * bd::ex2_approx(m2 - ms);
      f[0] = none, f[1] = 0.f;
      if (total != 0.f) {
        f[0] = bd::ex2_approx((r_o - ms) + (d_o - P_SHIFT)) / total;  // (d is -inf where a stream's tiles hold nothing for the row)
        f[1] = bd::ex2_approx((r2 - ms) + (d2 - P_SHIFT)) / total;
      }
      lse2 = total == 0.f ? -INFINITY : ms + log2f(total);
    }
    bd::tc_fence_after();
    // Through shared memory that no product reads any more (the queries', for the odd stream of NM = 1 the keys'): lanes
    // write their rows, the warp stores them row by row. The streams of NM = 1 share the rows: each has half of the columns.
    const int c0 = NM == 2 ? 0 : x * (D / 64), c1 = NM == 2 ? D / 32 : c0 + D / 64;
    const auto in_half = [&](int d) { return NM == 2 || d / (D / 2) == x; };
    const uint32_t stage = q_at + x * Q_HALF + warp_row * (D * 2);
    const auto give = [&](const void* mine, bool there) {  // a row's D * 2 bytes to where its lane says
#pragma unroll 4
      for (int u = 0; u < 32 / ROWS; ++u) {
        const int rr = u * ROWS + my_r;
        const uint64_t dst = __shfl_sync(~0u, reinterpret_cast<uint64_t>(mine), rr);
        const uint4 w = bd::ld_shared_v4(stage + rr * (D * 2) + ((my_c ^ (rr & 7)) << 4));
        if (dst != 0 && there) *reinterpret_cast<uint4*>(dst + my_c * 16) = w;
      }
    };
    const auto take = [&](int c, float (&v)[32]) {  // 32 elements of the lane's row
      if (mine > 0)
        bd::tmem_ld32(o_at + c * 32, v);
      else
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] *= f[0];
      if (NM == 1 && tiles_of(x ^ 1) > 0) {
        float w[32];
        bd::tmem_ld32(tmem + lanes + O_COL + (x ^ 1) * TILE + c * 32, w);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = fmaf(w[e], f[1], v[e]);
      }
    };
    if (__any_sync(~0u, o.out != nullptr)) {
#pragma unroll 1
      for (int c = c0; c < c1; ++c) {
        float v[32];
        take(c, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t y[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float2 g = make_float2(v[e * 8 + u * 2], v[e * 8 + u * 2 + 1]);
            y[u] = a.f16 ? F16::from_float2(g) : Bf16::from_float2(g);
          }
          st_shared_v4(stage + lane * (D * 2) + (((c * 4 + e) ^ (lane & 7)) << 4), y[0], y[1], y[2], y[3]);
        }
      }
      __syncwarp();
      give(o.out, my_c * 8 < a.dim && in_half(my_c * 8));
      __syncwarp();
    }
    if (__any_sync(~0u, o.o != nullptr)) {  // fp32: half of the elements at a time
#pragma unroll 1
      for (int c = c0; c < c1; ++c) {
        float v[32];
        take(c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          st_shared_v4(stage + lane * (D * 2) + (((c * 8 + e) % LANES ^ (lane & 7)) << 4), __float_as_uint(v[e * 4]),
                       __float_as_uint(v[e * 4 + 1]), __float_as_uint(v[e * 4 + 2]), __float_as_uint(v[e * 4 + 3]));
        if ((c + 1) % (D / 64) == 0) {
          const int d = (c * 32 + 32) / (D / 2) * (D / 2) - D / 2;  // the half's first element
          __syncwarp();
          give(o.o == nullptr ? nullptr : o.o + d, d + my_c * 4 < a.dim);
          __syncwarp();
        }
      }
    }
    if (live && (NM == 2 || x == 0)) store_lse(o, lse2);
  }

  __syncwarp();
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  if (warp == MMA_WARP) bd::tmem_dealloc(tmem, 512);
}

template <int NM, int D, int GROUPS>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  const auto kernel = attn_tiles_kernel<NM, D, GROUPS>;
  if (cudaError_t e = allow_smem(kernel, smem_bytes<NM, D>(), ready); e != cudaSuccess) return e;
  const int tiles = (a.max_q * a.group + NM * TILE - 1) / (NM * TILE);
  const dim3 grid(tiles * a.n_kv, a.n_split, a.n_seq);
  kernel<<<grid, threads(NM), smem_bytes<NM, D>(), st>>>(a);
  return cudaGetLastError();
}

template <int NM, int D>
cudaError_t launch_pages(const AttnArgs& a, cudaStream_t st) {
  return (1 << a.page_shift) >= TOK ? launch<NM, D, 1>(a, st) : launch<NM, D, 4>(a, st);
}

}  // namespace

cudaError_t launch_attn_tiles(const AttnArgs& a, cudaStream_t st) {
  if (a.dim <= 64) return a.one_tile ? launch_pages<1, 64>(a, st) : launch_pages<2, 64>(a, st);
  return a.one_tile ? launch_pages<1, 128>(a, st) : launch_pages<2, 128>(a, st);
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
