// bdkv_attention for many query rows per key/value head: windows of blocks,
// prompts. tcgen05 products on tiles of 128 rows by 128 cached tokens.
//
// A CTA holds NM x 128 rows of a request's key/value head (queries x the
// group's heads, so the head's cache is read once for all of them) and walks
// the cache in tiles of 128 tokens:
//   converter warps   codes from global memory to f16 (exact), into shared
//                     memory in the 128-byte swizzle, double buffered; a
//                     request's tail is zeros, so its values times zero
//                     weights stay zero
//   MMA warp          S = Q K^T (both operands in shared memory) and O += P V
//                     (P in tensor memory, V read with the token index along
//                     K); S of one half runs while the other half's softmax does
//   softmax warps     a thread per row: running maxima, weights to f16, written
//                     over S in tensor memory; O is rescaled only when a row's
//                     maximum has grown by more than 2^3
// Scales of pages come in through the exponent: w = 2^(S coef k_scale + e_v),
// see k_attn_rows.cu; O and the sum L have a reference maximum of their own.
#include "cache.h"

namespace bdkv {
namespace {

constexpr int TILE = TILES_TILE;  // rows of an MMA, tokens of a tile
constexpr float P_SHIFT = 12, P_SLACK = 3;
constexpr int CONV_WARPS = 4;
// Warps of a CTA: 4 for each half's softmax, 4 converters, 4 of which one issues the MMAs: warpgroups, so that registers
// can be moved between them. With two halves, 512 threads start with 128 each: 2 x 128 x 184 (a row's 128 scores stay in
// registers) + 128 x 104 + 128 x 40 = 65536; with one, 384 threads with 168.
constexpr int threads(int nm) { return (nm + 2) * 128; }

__device__ uint32_t g_status;  // bd::DEV_* bits

struct Ctl {
  uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], pv_done[2], drain;
  float ks[4][8], ve[4][8];  // page scales of a tile's eight groups of 16 tokens: factor, exponent
  uint32_t tmem_base;
  int abort_flag;
};

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// The MMA warp issues in the elected lane by predicate, not by branch: its addresses and descriptors then stay in uniform
// registers. D[tmem] (+)= A[smem] * B[smem]^T, f16.
__device__ __forceinline__ void mma_ss(uint32_t issue, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(issue)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], f16: row i of A in lane i, two elements per 32-bit column.
__device__ __forceinline__ void mma_ts(uint32_t issue, uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(issue)
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

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// All 128 columns of a tile for this thread's lane.
__device__ __forceinline__ void tmem_ld128(uint32_t taddr, float (&v)[128]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%128];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, %76, %77, %78, %79, "
      "%80, %81, %82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95, "
      "%96, %97, %98, %99, %100, %101, %102, %103, %104, %105, %106, %107, %108, %109, %110, %111, "
      "%112, %113, %114, %115, %116, %117, %118, %119, %120, %121, %122, %123, %124, %125, %126, %127}, [%129];\n\t"
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
        "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]),
        "=f"(v[64]), "=f"(v[65]), "=f"(v[66]), "=f"(v[67]),
        "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]),
        "=f"(v[72]), "=f"(v[73]), "=f"(v[74]), "=f"(v[75]),
        "=f"(v[76]), "=f"(v[77]), "=f"(v[78]), "=f"(v[79]),
        "=f"(v[80]), "=f"(v[81]), "=f"(v[82]), "=f"(v[83]),
        "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]),
        "=f"(v[88]), "=f"(v[89]), "=f"(v[90]), "=f"(v[91]),
        "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]),
        "=f"(v[96]), "=f"(v[97]), "=f"(v[98]), "=f"(v[99]),
        "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]),
        "=f"(v[104]), "=f"(v[105]), "=f"(v[106]), "=f"(v[107]),
        "=f"(v[108]), "=f"(v[109]), "=f"(v[110]), "=f"(v[111]),
        "=f"(v[112]), "=f"(v[113]), "=f"(v[114]), "=f"(v[115]),
        "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]),
        "=f"(v[120]), "=f"(v[121]), "=f"(v[122]), "=f"(v[123]),
        "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
      : "r"(taddr), "r"(taddr + 64)
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
  return size_t(NM + 4) * TILE * D * 2 + sizeof(Ctl) + 1024;
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
  int x = 0;
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

// Sixteen codes to f16, two 16-byte chunks.
__device__ __forceinline__ void decode16(uint4 x, uint32_t (&y)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = bd::e4m3x2_to_f16x2(w[i] & 0xffffu);
    y[2 * i + 1] = bd::e4m3x2_to_f16x2(w[i] >> 16);
  }
}

template <class T, int NM, int D>
__global__ void __launch_bounds__(threads(NM), 1) attn_tiles_kernel(AttnArgs a) {
  constexpr int ATOMS = D / 64;             // 128-byte column blocks of a row
  constexpr uint32_t ATOM = TILE * 128;     // bytes of one, 128 rows
  constexpr uint32_t OPERAND = ATOMS * ATOM;
  constexpr int CH = D / 16;                // 16-code chunks of a token's row
  constexpr int O_COL = 256;                // tensor memory: S and P at 0 and 128, O behind
  extern __shared__ uint8_t raw[];
  const uint32_t base = (bd::smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + NM * OPERAND, v_at = k_at + 2 * OPERAND;
  Ctl* ctl = reinterpret_cast<Ctl*>(raw + (v_at + 2 * OPERAND - bd::smem_u32(raw)));
  const int tid = threadIdx.x, warp = static_cast<int>(bd::warp_uniform(tid >> 5));
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
  const int n = end > begin ? (end - begin + TILE - 1) / TILE : 0;

  if (tid == 0) {
    bd::mbar_init(bd::smem_u32(&ctl->q_full), NM * TILE);
    for (int i = 0; i < 2; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->k_full[i]), CONV_WARPS * 32);
      bd::mbar_init(bd::smem_u32(&ctl->v_full[i]), CONV_WARPS * 32);
      bd::mbar_init(bd::smem_u32(&ctl->k_empty[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->v_empty[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->s_full[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->p_full[i]), TILE);
      bd::mbar_init(bd::smem_u32(&ctl->pv_done[i]), 1);
    }
    bd::mbar_init(bd::smem_u32(&ctl->drain), 1);
    ctl->abort_flag = 0;
    bd::fence_mbar_init();
  }
  constexpr int MMA_WARP = 4 * NM + CONV_WARPS;
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
    give_registers<40>();
    if (warp == MMA_WARP) {
      const uint32_t issue = bd::elect_one();
      constexpr uint32_t IDESC_S = bd::idesc_f16_f32(TILE, TILE), IDESC_O = bd::idesc_f16_f32(TILE, D) | B_MN_MAJOR;
      const uint64_t q_desc = bd::sw128_kmajor_desc(q_at), k_desc = bd::sw128_kmajor_desc(k_at);
      const uint64_t v_desc = sw128_mnmajor_desc(v_at, ATOM);
      const auto scores = [&](int x, int j) {  // S in slot x; addresses in descriptors count 16 bytes
        const uint64_t qd = q_desc + (NM == 2 ? x * (OPERAND >> 4) : 0u), kd = k_desc + (j & 1) * (OPERAND >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t at = (k / 4) * (ATOM >> 4) + 2u * (k % 4);
          mma_ss(issue, tmem + x * TILE, qd + at, kd + at, IDESC_S, k != 0);
        }
        mma_commit(issue, bd::smem_u32(&ctl->s_full[x]));
        if (NM == 1 || x == NM - 1) mma_commit(issue, bd::smem_u32(&ctl->k_empty[j & 1]));
      };
      bool ok = n > 0 && wait(ctl->q_full, 0);
      for (int j = 0; ok && j < (NM == 1 ? min(n, 2) : 1); ++j) {
        ok = wait(ctl->k_full[j & 1], 0);
        bd::tc_fence_after();
        if (ok)
          for (int x = 0; x < NM; ++x) scores(NM == 1 ? j : x, j);
      }
      for (int j = 0; ok && j < n; ++j) {
#pragma unroll
        for (int x = 0; x < NM; ++x) {
          const int slot = NM == 1 ? j & 1 : x;
          ok = ok && wait(ctl->p_full[slot], NM == 1 ? j >> 1 : j);
          if (x == 0) ok = ok && wait(ctl->v_full[j & 1], j >> 1);
          if (!ok) break;
          bd::tc_fence_after();
          const uint64_t vd = v_desc + (j & 1) * (OPERAND >> 4);
#pragma unroll
          for (int k = 0; k < TILE / 16; ++k)
            mma_ts(issue, tmem + O_COL + x * TILE, tmem + slot * TILE + k * 8, vd + k * (2048u >> 4), IDESC_O,
                   (j | k) != 0);
          mma_commit(issue, bd::smem_u32(&ctl->pv_done[x]));
          if (x == NM - 1) mma_commit(issue, bd::smem_u32(&ctl->v_empty[j & 1]));
          const int next = NM == 1 ? j + 2 : j + 1;
          if (next < n) {
            if (x == 0) ok = wait(ctl->k_full[next & 1], next >> 1);
            if (!ok) break;
            bd::tc_fence_after();
            scores(slot, next);
          }
        }
      }
      mma_commit(issue, bd::smem_u32(&ctl->drain));  // all MMAs issued have completed once it flips
      __syncwarp();
      bd::mbar_drain(bd::smem_u32(&ctl->drain), 0);
    }
    __syncwarp();
  } else if (warp >= 4 * NM) {
    // ---------------------------------------------------------- converters
    give_registers<104>();
    const int ct = tid - 4 * NM * 32;
    constexpr int PER = TILE * CH / (CONV_WARPS * 32);  // chunks of a thread and tile
    constexpr int STEP = CONV_WARPS * 32 / CH;          // rows between them
    const int sub = ct % CH, mine = ct / CH;
    const int64_t row_k = a.k_tok, row_v = a.v_tok;
    const uint8_t* kp = a.k + head * a.k_head + sub * 16;
    const uint8_t* vp = a.v + head * a.v_head + sub * 16;
    const int32_t* table = a.table + seq * a.table_stride;
    const int mask = (1 << a.page_shift) - 1;
    uint4 kx[PER], vx[PER];
    int pages[PER];  // of the tile to be loaded next (-1: nothing to read)
    const auto find = [&](int j) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int t = begin + j * TILE + mine + u * STEP;
        pages[u] = ld_global_if(table + (t >> a.page_shift), t < end && (t >> a.page_shift) < a.max_blocks, -1);
      }
    };
    const auto load = [&](const uint8_t* p, int64_t page_stride, int64_t tok_stride, int j, uint4 (&x)[PER]) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int t = begin + j * TILE + mine + u * STEP;
        x[u] = ld_global_if(p + pages[u] * page_stride + (t & mask) * tok_stride,
                            pages[u] >= 0 && pages[u] < a.n_pages && sub * 16 < a.dim);
      }
    };
    const auto store = [&](uint32_t at, const uint4 (&x)[PER]) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int r = mine + u * STEP;
        uint32_t y[8];
        decode16(x[u], y);
        const uint32_t rowp = at + (sub / 4) * ATOM + r * 128;
        // the lanes of the second atom store their second chunk first: the two atoms' lanes meet in different banks
        const bool flip = sub >= 4;
        const int c0 = (sub % 4) * 2 + flip;
        st_shared_v4(rowp + ((c0 ^ (r & 7)) << 4), flip ? y[4] : y[0], flip ? y[5] : y[1], flip ? y[6] : y[2],
                     flip ? y[7] : y[3]);
        st_shared_v4(rowp + (((c0 ^ 1) ^ (r & 7)) << 4), flip ? y[0] : y[4], flip ? y[1] : y[5], flip ? y[2] : y[6],
                     flip ? y[3] : y[7]);
      }
    };
    // a lane of the first eight has a tile's group of 16 tokens: its page and, one tile ahead, its scales
    int group_page = -1, ks_byte = 0, vs_byte = 0;
    bool group_in = false;
    const auto find_group = [&](int j) {
      const int t = begin + j * TILE + ct * 16;
      group_page = ld_global_if(table + (t >> a.page_shift), ct < 8 && t < end && (t >> a.page_shift) < a.max_blocks, -1);
    };
    const auto find_scales = [&](int j) {  // of tile j, whose pages find_group has looked up; then the pages of the next
      group_in = group_page >= 0 && group_page < a.n_pages;
      ks_byte = ld_global_byte_if(a.ks + group_page * a.ks_page + head, group_in);
      vs_byte = ld_global_byte_if(a.vs + group_page * a.vs_page + head, group_in);
      find_group(j + 1);
    };
    if (n > 0) {
      find_group(0);
      find_scales(0);
      find(0);
      load(kp, a.k_page, row_k, 0, kx);
      load(vp, a.v_page, row_v, 0, vx);
    }
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      find(j + 1);
      ok = wait(ctl->k_empty[j & 1], (j >> 1) + 1);
      if (!ok) break;
      if (ct < 8) {
        ctl->ks[j & 3][ct] = group_in ? pow2i(ks_byte - 127) : 1.f;
        ctl->ve[j & 3][ct] = group_in ? static_cast<float>(vs_byte - 127) : 0.f;
      }
      find_scales(j + 1);
      store(k_at + (j & 1) * OPERAND, kx);
      fence_proxy_async();
      bd::mbar_arrive(bd::smem_u32(&ctl->k_full[j & 1]));
      if (j + 1 < n) load(kp, a.k_page, row_k, j + 1, kx);
      ok = wait(ctl->v_empty[j & 1], (j >> 1) + 1);
      if (!ok) break;
      store(v_at + (j & 1) * OPERAND, vx);
      fence_proxy_async();
      bd::mbar_arrive(bd::smem_u32(&ctl->v_full[j & 1]));
      if (j + 1 < n) load(vp, a.v_page, row_v, j + 1, vx);
    }
  } else {
    // ------------------------------------------------------------- softmax
    take_registers<184>();
    const int x = NM == 2 ? warp >> 2 : 0;  // half
    const int r = tid & 127, row = row0 + x * TILE + r, i = row / a.group;
    const bool live = row < rows;
    const int h = head * a.group + row - i * a.group;
    const int vis = live ? min(visible(a, sq, i), end) : 0;
    float coef = 0.f;
    if (n > 0) {
      // the row in f16 times a power of two, with the sign of the scale
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(sq.q0 + i) * a.q_tok + h * a.q_head;
      uint4 w[D / 8];
      float amax = 0.f;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        w[c] = make_uint4(0, 0, 0, 0);
        if (live && c * 8 < a.dim) w[c] = *reinterpret_cast<const uint4*>(q + c * 8);
        const uint32_t ww[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 f = T::to_float2(ww[u]);
          amax = bd::max3(amax, fabsf(f.x), fabsf(f.y));
        }
      }
      const int s = row_shift(amax);
      const float f = a.coef < 0.f ? -pow2i(s) : pow2i(s);
      coef = fabsf(a.coef) * pow2i(-s);
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const uint32_t ww[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
        uint32_t y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 v = T::to_float2(ww[u]);
          y[u] = f16x2(make_float2(v.x * f, v.y * f));
        }
        st_shared_v4(q_at + x * OPERAND + (c / 8) * ATOM + r * 128 + (((c % 8) ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
      }
      fence_proxy_async();
      bd::mbar_arrive(bd::smem_u32(&ctl->q_full));
    }

    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t o_at = tmem + lanes + O_COL + x * TILE;
    const bool any_live = __any_sync(~0u, live);
    float m = -INFINITY, M = -INFINITY, L = 0.f;
    bool ok = true;
    // One tile: the row's scores become weights, over themselves in tensor memory. CUT: some row of the warp does not see
    // all 128 tokens.
    const auto softmax = [&](auto cut, int slot, int j, int left) -> bool {
      constexpr bool CUT = decltype(cut)::value;
      const uint32_t s_at = tmem + lanes + slot * TILE;
      const float* ks = ctl->ks[j & 3];
      const float* ve = ctl->ve[j & 3];
      float v[TILE];
      __syncwarp();
      tmem_ld128(s_at, v);
      float s_top = -INFINITY, u_top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        if (CUT)
#pragma unroll
          for (int e = b * 16; e < b * 16 + 16; ++e)
            if (e >= left) v[e] = -INFINITY;
        float t = v[b * 16];
#pragma unroll
        for (int e = 1; e < 15; e += 2) t = bd::max3(t, v[b * 16 + e], v[b * 16 + e + 1]);
        t = fmaxf(t, v[b * 16 + 15]);
        const float s2 = CUT && t == -INFINITY ? t : t * (coef * ks[b]);
        s_top = fmaxf(s_top, s2);
        u_top = fmaxf(u_top, s2 + ve[b]);
      }
      const float m_new = fmaxf(m, s_top);
      L *= m_new == m ? 1.f : bd::ex2_approx(m - m_new);
      m = m_new;
      const bool grow = u_top > M + P_SLACK || (M == -INFINITY && u_top > M);
      if (__any_sync(~0u, grow)) {
        if (j > 0) {
          if (!wait(ctl->pv_done[x], j - 1)) return false;
          bd::tc_fence_after();
          const float f = grow ? bd::ex2_approx(M - u_top) : 1.f;
          __syncwarp();  // tensor-memory accesses take the whole warp at once
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            tmem_ld16(o_at + c * 16, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st16(o_at + c * 16, o);
          }
        }
        M = grow ? u_top : M;
      }
      __syncwarp();
      const float ms = m == -INFINITY ? 0.f : m, Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float f = coef * ks[c * 2 + b], ref = Ms - ve[c * 2 + b] - P_SHIFT;
          float2 sum = {0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const int col = c * 32 + b * 16 + e;
            const float2 y = bd::fma2(make_float2(v[col], v[col + 1]), make_float2(f, f), make_float2(-ref, -ref));
            float2 w = make_float2(bd::ex2_approx(y.x), bd::ex2_approx(y.y));
            if (CUT) {
              if (col >= left) w.x = 0.f;
              if (col + 1 >= left) w.y = 0.f;
            }
            sum = bd::add2(sum, w);
            p[b * 8 + e / 2] = f16x2(w);
          }
          L += (sum.x + sum.y) * bd::ex2_approx(ref - ms);
        }
        tmem_st16(s_at + c * 16, p);
      }
      bd::tmem_st_wait();
      return true;
    };

    for (int j = 0; j < n; ++j) {
      const int slot = NM == 1 ? j & 1 : x;
      ok = wait(ctl->s_full[slot], NM == 1 ? j >> 1 : j);
      if (!ok) break;
      bd::tc_fence_after();
      if (any_live) {
        const int left = vis - (begin + j * TILE);  // columns this row sees
        ok = __any_sync(~0u, left < TILE) ? softmax(std::true_type(), slot, j, left) : softmax(std::false_type(), slot, j, left);
        if (!ok) break;
      }
      bd::tc_fence_before();
      bd::mbar_arrive(bd::smem_u32(&ctl->p_full[slot]));
    }

    // The last tile's scores follow O's product of two tiles before it (NM == 1), so that is as far as O is known to be: a
    // parity wait must not skip a phase.
    if (NM == 1 && n > 1 && ok) ok = wait(ctl->pv_done[x], n - 2);
    if (n > 0 && ok) ok = wait(ctl->pv_done[x], n - 1);
    bd::tc_fence_after();
    const float ms = m == -INFINITY ? 0.f : m, Ms = M == -INFINITY ? 0.f : M;
    const float f = L == 0.f ? 0.f : bd::ex2_approx(Ms - P_SHIFT - ms) / L;
    const float lse2 = L == 0.f ? -INFINITY : ms + log2f(L);
    RowOut o = {nullptr, nullptr, nullptr};
    if (live) o = row_out(a, sq, seq, part, i, h, visible(a, sq, i));
    if (any_live) {
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float v[32];
        if (n > 0)
          bd::tmem_ld32(o_at + c * 32, v);
        else
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 32; e += 8)
          if (c * 32 + e < a.dim)
            store8<T>(o, c * 32 + e, make_float4(v[e] * f, v[e + 1] * f, v[e + 2] * f, v[e + 3] * f),
                      make_float4(v[e + 4] * f, v[e + 5] * f, v[e + 6] * f, v[e + 7] * f));
      }
      if (live) store_lse(o, lse2);
    }
  }

  __syncwarp();
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  if (warp == MMA_WARP) bd::tmem_dealloc(tmem, 512);
}

template <class T, int NM, int D>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  if (cudaError_t e = allow_smem(attn_tiles_kernel<T, NM, D>, smem_bytes<NM, D>(), ready); e != cudaSuccess) return e;
  const int tiles = (a.max_q * a.group + NM * TILE - 1) / (NM * TILE);
  const dim3 grid(tiles * a.n_kv, a.n_split, a.n_seq);
  attn_tiles_kernel<T, NM, D><<<grid, threads(NM), smem_bytes<NM, D>(), st>>>(a);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_type(const AttnArgs& a, cudaStream_t st) {
  const bool one = a.max_q * a.group <= TILE;
  if (a.dim <= 64) return one ? launch<T, 1, 64>(a, st) : launch<T, 2, 64>(a, st);
  return one ? launch<T, 1, 128>(a, st) : launch<T, 2, 128>(a, st);
}

}  // namespace

cudaError_t launch_attn_tiles(const AttnArgs& a, cudaStream_t st) {
  return a.f16 ? launch_type<F16>(a, st) : launch_type<Bf16>(a, st);
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
