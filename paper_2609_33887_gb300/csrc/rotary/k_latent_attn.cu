// bdrot_latent_attention: tcgen05 products of up to 64 rows (queries x heads)
// with tiles of 64 cached tokens, the tokens along the instruction's rows.
//
//   S^T [tokens, rows] = C Q^T     C the tile: 64 tokens x (latent, key part), in
//                                  128-byte columns as the TMA loads it
//   O^T [dims, rows] += C_l^T P    the same bytes, read with the token index
//                                  along K: a latent is loaded once for both
// Rows as columns of the accumulators keep O in half of tensor memory (512 dims
// x 64 rows are 4 x 64 columns), where rows as its rows would fill all of it,
// and cost a few rows no more than they fill columns.
// Tiles of 64 tokens, 73.7 KB of 512 + 64 elements, so that two of them fit next
// to 64 rows of queries and nearly three next to 16: the scores of a tile are
// under way before the weights of the one before it are. A tile's weights take
// the place of its key parts, which its scores have used up.
// Warps: one loads, one issues the scores' products and one the values', four or
// eight hold the softmax: a
// thread has one token and 8 or 16 rows, so maxima over tokens are taken across
// threads, and only when some score exceeds its row's reference by more than
// 2^15; sums stay with the threads until the end.
// Work: a unit is a request's 64 rows (or 32, 16) and the tiles that the last of
// them sees. Each CTA takes an equal share of all units' tiles, laid one behind
// another: the end of a unit, whole units, the beginning of another (a segment
// each). Only the device knows the lengths, so every CTA adds them up itself, and
// takes one unit whole where shares would not pay. Of a unit in several CTAs each
// leaves its part, which k_latent_join.cu joins. With more than a unit to each SM
// a CTA takes one (see make_plan); that is a kernel of its own, as both in one
// took 3 to 5 us longer, from the registers and the order of the code.
//
// 64 single tokens of 16 heads over 57 to 8189 tokens of 512 + 64 take 66 us with
// the join, one behind another: 3.5 us to the first load, 46 until half of the CTAs
// have their last tile (304 MB at 6.6 TB/s), 4 of CTAs that HBM serves later than
// others, 2.5 of results, 5.5 of the join, 4 to the next call's start. 32 x 5
// drafts of 128 heads over 300 to 4001 tokens 126 us, 760 TFLOP/s (0.40 of a
// library product's rate): about 2600 cycles a tile of 64 rows, of which products
// take 1920 (64 columns leave the instructions short of shared memory: M = 64, N
// = 64 takes 32 cycles, M = 128 48). The rest is the way round a ring of two
// tiles: values' products, 1500 cycles of load, scores, 600 of softmax.
#include <cfloat>

#include "rotary/latent.h"

namespace bdrot {
namespace {

using bdkv::Seq;

constexpr uint32_t CHUNK = TOKENS * 128, PAIR = 2 * CHUNK;  // bytes of 64 and of 128 elements of a tile
// A row's weights are 2^(score - reference). The reference is 2^8 below the largest score seen when it was set, and scores
// may exceed it by 2^15 before it is set again and O rescaled: weights of 2^15 at most, which f16 holds, with 11 bits down
// to 2^-22 of that largest score's.
constexpr float P_SHIFT = 8, P_MOST = 15;
constexpr float NO_REF = -FLT_MAX;  // no score has been seen; none that is finite is smaller

__device__ uint32_t g_status;  // bd::DEV_* bits

template <int N>
struct Ctl {
  uint64_t q_full, full[MAX_STAGES], empty[MAX_STAGES];
  uint64_t s_full[2], segment_done, s_drain, o_drain;    // (scores: by parity of the tile)
  uint64_t p_full[HANDOVERS], o_done[HANDOVERS];
  alignas(16) float ref[N];
  alignas(16) float factor[N];
  alignas(16) float scale[N];
  float part[4][N];  // of the warps of a token quarter: maxima, at the end sums
  int visible[N];
  uint64_t out[N];   // where a row goes (0: nowhere)
  int starts[MAX_SHARED_UNITS + 1];  // tiles of the requests before
  int first[MAX_SHARED_UNITS + 1], length[MAX_SHARED_UNITS];  // the requests' first queries and cached tokens
  int most, from, to;  // tiles of a unit, at most; the CTA's share of all units' tiles
  uint32_t tmem_base;
  int abort_flag;
};

// A tile comes in stages of one or two pairs of 64 columns of its latents, its key parts with the last: the warps that load
// and multiply spend some 400 cycles a stage on barriers whatever is in it (with a stage for each pair and one for the key
// parts, 64 rows took 2630 cycles a tile). Shared memory: the queries' columns, a ring of stages, and one of key parts (and
// weights) for as many tiles as those hold, the last maybe in part, so that a stage that is free says that its tile's key
// parts have a place.
struct Layout {
  int n_pairs, per_stage, per_tile;  // pairs of a tile and of a stage, stages of a tile
  int stages, tiles;
  size_t bytes;
};
template <int N>
Layout layout(int dim) {
  Layout l;
  l.n_pairs = (dim + 127) / 128;
  l.per_stage = pairs_per_stage(l.n_pairs);
  l.per_tile = (l.n_pairs + l.per_stage - 1) / l.per_stage;
  const size_t fixed = 1024 + sizeof(Ctl<N>) + (2 * l.n_pairs + 1) * N * 128, stage = l.per_stage * PAIR;
  const auto bytes = [&](int stages) { return fixed + stages * stage + (stages + l.per_tile - 1) / l.per_tile * CHUNK; };
  l.stages = std::min(MAX_STAGES, MAX_TILES * l.per_tile);
  while (bytes(l.stages) > 232448) --l.stages;  // (two tiles at least)
  l.tiles = (l.stages + l.per_tile - 1) / l.per_tile;
  l.bytes = bytes(l.stages);
  return l;
}
// (a power of two)
template <int N>
__host__ __device__ constexpr uint32_t tmem_columns(int n_pairs) {
  const int n = (2 + n_pairs) * N;
  return n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512;
}

// By predicate in the elected lane, with operands that are the same in all lanes: a branch, or a lane's own coordinates,
// costs hundreds of cycles a copy.
__device__ __forceinline__ void tma_load_3d(uint32_t issue, uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y,
                                            int z) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(issue)
      : "memory");
}
// The same of several columns of 64 elements at once: [64 elements, tokens, column, page].
__device__ __forceinline__ void tma_load_4d(uint32_t issue, uint32_t dst, const CUtensorMap* map, uint32_t bar, int y, int column,
                                            int page) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {0, %2, %3, %4}], [%5];\n\t}" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(y), "r"(column), "r"(page), "r"(bar), "r"(issue)
      : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t issue, uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
      "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
      "r"(bytes), "r"(issue)
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
// The 128 threads that have the same rows: a barrier, and one that says whether any of them has `some`.
__device__ __forceinline__ void group_sync(int g) { bd::named_barrier_sync(1 + g, 128); }
__device__ __forceinline__ bool group_any(int g, bool some) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(some)), "r"(1 + g), "r"(128)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
// 16 columns of this thread's lane, and back.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
template <int COLS>
__device__ __forceinline__ void tmem_load(uint32_t at, float (&v)[COLS]) {
  if constexpr (COLS == 16)
    tmem_ld16(at, v);
  else
    bd::tmem_ld32(at, v);
}
template <int COLS>
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[COLS]) {
  if constexpr (COLS == 16)
    tmem_st16(at, v);
  else
    bd::tmem_st32(at, v);
}
// An accumulator of 64 rows lies in the first 16 lanes of each warp's quarter: threads 0..15 get COLS columns of them,
// threads 16..31 of the same lanes the next COLS.
template <int COLS>
__device__ __forceinline__ void tmem_load_halves(uint32_t at, float (&v)[COLS]) {
  if constexpr (COLS == 16)
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16], 16;\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(at)
        : "memory");
  else
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8], 8;\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
        : "r"(at)
        : "memory");
}
// 16 bytes from global to shared memory, asynchronously; zeros where there is nothing to read.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// A row's reference for a largest score of `most`: scores so large that 8 is about a rounding of theirs go without the shift.
__device__ __forceinline__ float reference(float most) { return fabsf(most) < 1048576.f ? most - P_SHIFT : most; }

// v[c] combined over the 16 lanes of a half warp: column c % COLS is lane c's.
template <int COLS, class Op>
__device__ __forceinline__ float across_lanes(const float (&v)[COLS], int lane, Op op) {
  float w[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) w[c] = COLS == 16 ? v[c] : op(v[c], __shfl_xor_sync(~0u, v[c], 8));
  const auto step = [&](auto width) {
    constexpr int H = decltype(width)::value;
    const bool upper = lane & H;
#pragma unroll
    for (int u = 0; u < H; ++u) {
      const float other = __shfl_xor_sync(~0u, upper ? w[u] : w[u + H], H);
      w[u] = op(upper ? w[u + H] : w[u], other);
    }
  };
  if constexpr (COLS == 16) step(std::integral_constant<int, 8>());
  step(std::integral_constant<int, 4>());
  step(std::integral_constant<int, 2>());
  step(std::integral_constant<int, 1>());
  return w[0];
}

// N: rows of a CTA; SHARED: it takes its share of all units' tiles, else one unit.
template <int N, bool SHARED>
__global__ void __launch_bounds__(N == 64 ? 352 : 224, 1)
    latent_attn_kernel(const LatentArgs p, const int stages, const int tiles, const __grid_constant__ CUtensorMap latent_map,
                       const __grid_constant__ CUtensorMap rope_map) {
  constexpr int SOFT_WARPS = N == 64 ? 8 : 4, SOFT = SOFT_WARPS * 32, THREADS = SOFT + 96;
  constexpr int WIDE = N / (SOFT_WARPS / 4), COLS = WIDE / 2;  // rows of a softmax warp, and of a thread
  constexpr uint32_t Q_CHUNK = N * 128, O_COL = 2 * N;  // tensor memory: two tiles' scores, then O's dims by 128
  const bdkv::AttnArgs& a = p.a;
  extern __shared__ __align__(16) uint8_t raw[];
  const int n_pairs = (a.dim + 127) / 128, per_stage = pairs_per_stage(n_pairs);
  const uint32_t stage_bytes = per_stage * PAIR;
  const uint32_t base = (bd::smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t kv_at = base, rope_at = kv_at + stages * stage_bytes, q_at = rope_at + tiles * CHUNK;
  Ctl<N>* ctl = reinterpret_cast<Ctl<N>*>(raw + (q_at + (2 * n_pairs + 1) * Q_CHUNK - bd::smem_u32(raw)));
  const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(bd::warp_uniform(tid >> 5));

  // ------------------------------------------------------------------ work
  // A unit's rows and tiles; one with rows that see nothing counts as a tile, in which its zeros are written.
  const auto rows_end = [&](const Seq& sq, int tile) { return min(sq.q_len * a.group, tile * N + N); };
  const auto unit_sees = [&](const Seq& sq, int tile) { return bdkv::visible(a, sq, (rows_end(sq, tile) - 1) / a.group); };
  const auto unit_tiles = [&](const Seq& sq, int tile) {
    return tile * N >= sq.q_len * a.group ? 0 : max(1, (unit_sees(sq, tile) + TOKENS - 1) / TOKENS);
  };
  struct Segment {
    Seq sq;
    int seq, row0, begin, end, n;  // rows from row0 on; tokens; tiles
    bool whole, first;             // of its unit; of its CTA
  };
  const auto sequence = [&](int x) { return bdkv::make_seq(a, ctl->first[x], ctl->first[x + 1], ctl->length[x]); };
  int from = 0, to = 0;  // the CTA's share
  // the same in all lanes, and known to be: loops and products behind it then run from uniform registers
  const auto uniform = [](int x) { return static_cast<int>(bd::warp_uniform(static_cast<uint32_t>(x))); };
  Segment only;
  if constexpr (SHARED) {
    if (tid == 0) ctl->most = 0;
    for (int x = tid; x <= a.n_seq; x += THREADS) {
      ctl->first[x] = a.q_start[x];
      if (x < a.n_seq) ctl->length[x] = a.kv_lens[x];
    }
    __syncthreads();
    if (p.row_tiles <= 16) {
      for (int x = tid; x < a.n_seq; x += THREADS) {
        const Seq sq = sequence(x);
        int sum = 0, most = 0;
        for (int t = 0; t < p.row_tiles; ++t) {
          const int n = unit_tiles(sq, t);
          sum += n, most = max(most, n);
        }
        ctl->starts[x + 1] = sum;
        atomicMax(&ctl->most, most);
      }
    } else {
      for (int x = warp; x < a.n_seq; x += THREADS / 32) {
        const Seq sq = sequence(x);
        int sum = 0, most = 0;
        for (int t = lane; t < p.row_tiles; t += 32) {
          const int n = unit_tiles(sq, t);
          sum += n, most = max(most, n);
        }
        sum = __reduce_add_sync(~0u, sum), most = __reduce_max_sync(~0u, most);
        if (lane == 0) ctl->starts[x + 1] = sum, atomicMax(&ctl->most, most);
      }
    }
    __syncthreads();
    if (warp == 0) {
      constexpr int PER = MAX_SHARED_UNITS / 32;
      int v[PER], sum = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int x = lane * PER + i;
        sum += x < a.n_seq ? ctl->starts[x + 1] : 0;
        v[i] = sum;
      }
      int before = sum;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int other = __shfl_up_sync(~0u, before, d);
        if (lane >= d) before += other;
      }
      before -= sum;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane * PER + i < a.n_seq) ctl->starts[lane * PER + i + 1] = before + v[i];
      if (lane == 0) ctl->starts[0] = 0;
      __syncwarp();
      // The CTA's share (two tiles or more, where there are few). Parts cost their rows' results in fp32, written and
      // read, and the join's time: a CTA to each unit (there are no more units than CTAs) where the longest has but a few
      // tiles more than an equal share. With units of 64 rows: 150 of 2000 tokens 55 us, 86 in shares; 140 of 1000 to 2000
      // tokens 63 and 80, but 80 of them 57 and 53; 16 of 4000 tokens 92 and 37. Of 16 rows: 140 of 1000 to 1500 tokens
      // 49 us, 57 in shares; 60 of them 37 and 29. Of 32 rows: 140 of 1000 to 1500 tokens 51 and 62, 60 of them 40 and 35, 80 of
      // 1000 to 2000 50 and 49; but 140 of 1000 to 2000 61 and 71, and 100 of 800 to 1200 39 and 46, which this takes in shares.
      const int64_t total = ctl->starts[a.n_seq], ctas = min(static_cast<int64_t>(gridDim.x), (total + 1) / 2);
      const int64_t share = ctas > 0 ? total / ctas : 0;
      const bool whole = ctl->most <= share + share / 4 + (N == 64 ? 8 : 3);
      const int x = blockIdx.x / p.row_tiles, tile = blockIdx.x - x * p.row_tiles;
      if (whole && x < a.n_seq) {
        const Seq sq = sequence(x);
        int before = 0;
        for (int t = lane; t < tile; t += 32) before += unit_tiles(sq, t);
        from = ctl->starts[x] + __reduce_add_sync(~0u, before), to = from + unit_tiles(sq, tile);
      } else if (!whole && static_cast<int64_t>(blockIdx.x) < ctas) {
        from = static_cast<int>(blockIdx.x * total / ctas), to = static_cast<int>((blockIdx.x + 1) * total / ctas);
      }
      if (lane == 0) {
        ctl->from = from, ctl->to = to;
        if (blockIdx.x == 0) p.plan[a.n_seq * p.row_tiles] = make_int2(whole ? -1 : 0, 0);
      }
    }
    __syncthreads();
    from = uniform(ctl->from), to = uniform(ctl->to);
    if (from == to) return;
  } else {
    only.seq = blockIdx.y;
    only.sq = a.longest_first ? bdkv::ranked_seq<THREADS>(a, blockIdx.y, reinterpret_cast<int*>(raw), only.seq)
                              : bdkv::load_seq(a, only.seq);
    // the last rows first: under a causal mask they see the most
    const int tile = gridDim.x - 1 - blockIdx.x;
    to = unit_tiles(only.sq, tile);
    if (to == 0) return;
    only.row0 = tile * N, only.begin = 0, only.end = unit_sees(only.sq, tile), only.n = (only.end + TOKENS - 1) / TOKENS;
    only.whole = only.first = true;
  }
  from = uniform(from), to = uniform(to);
  // The segment that begins at tile `at` of the share, which `seq` (0 at first) keeps the request of; by whole warps.
  const auto segment = [&](int& at, int& seq) {
    Segment g = only;
    if constexpr (!SHARED) {
      at = to;
    } else {
      g.first = at == from;
      if (g.first) {
        int hi = a.n_seq - 1;  // the last request that begins at `at` or before
        while (seq < hi) {
          const int mid = (seq + hi + 1) / 2;
          if (ctl->starts[mid] <= at)
            seq = mid;
          else
            hi = mid - 1;
        }
      }
      while (ctl->starts[seq + 1] <= at) ++seq;
      g.seq = seq, g.sq = sequence(seq);
      int start = ctl->starts[seq], tile = 0, tiles = 0;
      for (int t0 = 0;; t0 += 32) {  // the unit
        const int mine = t0 + lane < p.row_tiles ? unit_tiles(g.sq, t0 + lane) : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int other = __shfl_up_sync(~0u, upto, d);
          if (lane >= d) upto += other;
        }
        const uint32_t past = __ballot_sync(~0u, start + upto > at);
        if (past != 0 || t0 + 32 >= p.row_tiles) {  // (it is there: the request ends behind `at`)
          const int l = past != 0 ? __ffs(past) - 1 : 31;
          tile = t0 + l, tiles = __shfl_sync(~0u, mine, l);
          start += __shfl_sync(~0u, upto, l) - tiles;
          break;
        }
        start += __shfl_sync(~0u, upto, 31);
      }
      const int stop = min(to, start + tiles);
      g.row0 = tile * N;
      g.begin = (at - start) * TOKENS, g.end = min(unit_sees(g.sq, tile), (stop - start) * TOKENS);
      g.n = g.end > g.begin ? (g.end - g.begin + TOKENS - 1) / TOKENS : 0;
      g.whole = at == start && stop == start + tiles;
      if (warp == 0 && lane == 0 && at == start) {  // for the join: a split unit's first part and last CTA
        const int64_t total = ctl->starts[a.n_seq], ctas = min(static_cast<int64_t>(gridDim.x), (total + 1) / 2);
        p.plan[seq * p.row_tiles + tile] =
            g.whole ? make_int2(-1, -1)
                    : make_int2(2 * blockIdx.x + !g.first, static_cast<int>(((start + tiles) * ctas + total - 1) / total) - 1);
      }
      at = uniform(stop);
    }
    g.seq = uniform(g.seq), g.row0 = uniform(g.row0), g.begin = uniform(g.begin), g.end = uniform(g.end), g.n = uniform(g.n);
    return g;
  };

  if (tid == 0) {
    bd::mbar_init(bd::smem_u32(&ctl->q_full), SOFT);
    for (int i = 0; i < stages; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->full[i]), 1);
      bd::mbar_init(bd::smem_u32(&ctl->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) bd::mbar_init(bd::smem_u32(&ctl->s_full[i]), 1);
    for (int i = 0; i < HANDOVERS; ++i) {
      bd::mbar_init(bd::smem_u32(&ctl->p_full[i]), SOFT_WARPS);
      bd::mbar_init(bd::smem_u32(&ctl->o_done[i]), 1);
    }
    bd::mbar_init(bd::smem_u32(&ctl->segment_done), 1);
    bd::mbar_init(bd::smem_u32(&ctl->s_drain), 1);
    bd::mbar_init(bd::smem_u32(&ctl->o_drain), 1);
    ctl->abort_flag = 0;
    bd::fence_mbar_init();
  }
  constexpr int LOAD_WARP = SOFT_WARPS, SCORE_WARP = SOFT_WARPS + 1, VALUE_WARP = SOFT_WARPS + 2;
  if (warp == VALUE_WARP) {
    bd::tmem_alloc(bd::smem_u32(&ctl->tmem_base), tmem_columns<N>(n_pairs));
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
    // Box b of a tile: a page's tokens, or 64 tokens of a larger page; lane b finds its page. What is not there (a column
    // behind the table, a page outside the cache, tokens that no row sees) is read from behind the cache's last page, as zeros.
    const int page_size = 1 << a.page_shift, step = min(page_size, TOKENS), boxes = TOKENS / step;
    const int outside = static_cast<int>(max(a.n_pages, static_cast<int64_t>(1)));
    if (lane == 0) {
      bd::prefetch_tmap(&latent_map);
      bd::prefetch_tmap(&rope_map);
    }
    int stage = 0, round = 0, tile = 0;  // of the next load: its places, and how often the stage's was used
    bool ok = true;
    const uint32_t issue = bd::elect_one();
    int pages[TOKENS / 16];  // of a tile's boxes
    const auto load = [&](const CUtensorMap* map, uint32_t dst, uint32_t bar, int x, int y) {
#pragma unroll
      for (int b = 0; b < TOKENS / 16; ++b)  // (more than one: whole pages)
        if (b < boxes) tma_load_3d(issue, dst + b * step * 128, map, bar, x, y, pages[b]);
    };
    for (int at = from, seq = 0; ok && at < to;) {
      const Segment g = segment(at, seq);
      const int32_t* table = a.table + g.seq * a.table_stride;
      const auto find = [&](int j) {  // the page as the table has it: a tile ahead, and not looked at until it is needed
        const int t = g.begin + j * TOKENS + lane * step, col = t >> a.page_shift;
        return lane < boxes && t < g.end && col < a.max_blocks ? table[col] : -1;
      };
      int found = find(0), following = find(1);
      for (int j = 0; ok && j < g.n; ++j) {
        const int y = static_cast<int>(bd::warp_uniform((g.begin + j * TOKENS) & (page_size - 1)));
        const int page = found >= 0 && found < a.n_pages ? found : outside;
        found = following;
        following = find(j + 2);
#pragma unroll
        for (int b = 0; b < TOKENS / 16; ++b) pages[b] = __shfl_sync(~0u, page, b);
        for (int s = 0; s < n_pairs; s += per_stage) {
          if (!(ok = wait(ctl->empty[stage], round + 1))) break;
          const bool last = s + per_stage >= n_pairs;
          const uint32_t bar = bd::warp_uniform(bd::smem_u32(&ctl->full[stage])), dst = bd::warp_uniform(kv_at + stage * stage_bytes);
          const int pairs = min(per_stage, n_pairs - s);
          // (columns behind the latents' last are read as zeros)
          expect_bytes(issue, bar, (p.columns ? stage_bytes : pairs * PAIR) + (last ? CHUNK : 0));
          if (p.columns)
            tma_load_4d(issue, dst, &latent_map, bar, y, 2 * s, pages[0]);
          else
            for (int c = 0; c < 2 * pairs; ++c) load(&latent_map, dst + c * CHUNK, bar, (2 * s + c) * 64, y);
          if (last) load(&rope_map, bd::warp_uniform(rope_at + tile * CHUNK), bar, 0, y);
          if (++stage == stages) stage = 0, ++round;
        }
        if (++tile == tiles) tile = 0;
      }
    }
    // nothing is on its way when the CTA ends (all of it has been waited for, unless a wait gave up)
    __syncwarp();
    for (int i = 0; i < stages; ++i) {
      const int loads = round + (i < stage);
      if (loads > 0) bd::mbar_drain(bd::smem_u32(&ctl->full[i]), (loads - 1) & 1);
    }
    __syncwarp();
  } else if (warp == SCORE_WARP) {
    // ------------------------------------------------------------- products
    // Two warps issue them: what one spends on barriers and descriptors between products, the other's fill. (One for both,
    // whichever was ready: 2960 cycles a tile of 64 rows, of which the products take 1920.)
    const uint32_t issue = bd::elect_one();
    const uint32_t idesc = bd::warp_uniform(bd::idesc_f16_f32(TOKENS, N) | (a.f16 ? 0u : (1u << 7) | (1u << 10)));
    const uint32_t q_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(q_at)));
    const uint32_t k_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(kv_at)));
    const uint32_t r_lo = bd::warp_uniform(static_cast<uint32_t>(bd::sw128_kmajor_desc(rope_at)));
    int stage = 0, round = 0, tile = 0, t = 0, segments = 0;  // (t: the CTA's tile)
    int done = 0, turn = 0;  // of the tile two before: its place, and how often the ring has been round
    bool ok = true;
    for (int at = from, seq = 0; ok && at < to;) {
      const Segment g = segment(at, seq);
      if (g.n > 0) ok = wait(ctl->q_full, segments++);
      for (int j = 0; ok && j < g.n; ++j, ++t) {
        // over the scores of two tiles before, which have become weights
        if (t >= 2) {
          if (!(ok = wait(ctl->p_full[done], turn))) break;
          if (++done == tiles) done = 0, ++turn;
        }
        const uint32_t s_at = bd::warp_uniform(tmem + (t & 1) * N);
        for (int s = 0; s < n_pairs; s += per_stage) {
          if (!(ok = wait(ctl->full[stage], round))) break;
          bd::tc_fence_after();
          for (int u = 0; u < per_stage && s + u < n_pairs; ++u) {
            const uint32_t kd = bd::warp_uniform(k_lo + ((stage * stage_bytes + u * PAIR) >> 4));
            const uint32_t qd = bd::warp_uniform(q_lo + (s + u) * (2 * Q_CHUNK >> 4));
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mma(issue, s_at, kd + (k / 4) * (CHUNK >> 4) + 2u * (k % 4), qd + (k / 4) * (Q_CHUNK >> 4) + 2u * (k % 4), DESC_HI,
                  DESC_HI, idesc, (s | u | k) != 0);
          }
          if (++stage == stages) stage = 0, ++round;
        }
        if (!ok) break;
        const uint32_t rd = bd::warp_uniform(r_lo + tile * (CHUNK >> 4)), qr = bd::warp_uniform(q_lo + n_pairs * (2 * Q_CHUNK >> 4));
#pragma unroll
        for (int k = 0; k < 4; ++k) mma(issue, s_at, rd + 2u * k, qr + 2u * k, DESC_HI, DESC_HI, idesc, 1);
        mma_commit(issue, bd::smem_u32(&ctl->s_full[t & 1]));
        if (++tile == tiles) tile = 0;
      }
    }
    mma_commit(issue, bd::smem_u32(&ctl->s_drain));  // all of its products have completed once it flips
    __syncwarp();
    bd::mbar_drain(bd::smem_u32(&ctl->s_drain), 0);
    __syncwarp();
  } else if (warp == VALUE_WARP) {
    const uint32_t issue = bd::elect_one();
    const uint32_t idesc = bd::warp_uniform(bd::idesc_f16_f32(128, N) | (a.f16 ? 0u : (1u << 7) | (1u << 10)) | A_MN_MAJOR | B_MN_MAJOR);
    const uint32_t v_lo = bd::warp_uniform(mn_low(kv_at, CHUNK)), p_lo = bd::warp_uniform(mn_low(rope_at, CHUNK));
    int stage = 0, tile = 0, turn = 0;  // (how often the ring has been round)
    bool ok = true;
    for (int at = from, seq = 0; ok && at < to;) {
      const Segment g = segment(at, seq);
      for (int j = 0; j < g.n; ++j) {
        if (!(ok = wait(ctl->p_full[tile], turn))) break;
        bd::tc_fence_after();
        const uint32_t pd = bd::warp_uniform(p_lo + tile * (CHUNK >> 4));
        for (int s = 0; s < n_pairs; s += per_stage) {
          for (int u = 0; u < per_stage && s + u < n_pairs; ++u) {
            const uint32_t vd = bd::warp_uniform(v_lo + ((stage * stage_bytes + u * PAIR) >> 4));
            const uint32_t od = bd::warp_uniform(tmem + O_COL + (s + u) * N);
#pragma unroll
            for (int k = 0; k < TOKENS / 16; ++k)
              mma(issue, od, vd + k * (2048u >> 4), pd + k * (2048u >> 4), DESC_HI, DESC_HI, idesc, (j | k) != 0);
          }
          mma_commit(issue, bd::smem_u32(&ctl->empty[stage]));
          if (++stage == stages) stage = 0;
        }
        mma_commit(issue, bd::smem_u32(&ctl->o_done[tile]));
        if (++tile == tiles) tile = 0, ++turn;
      }
      if (g.n > 0) mma_commit(issue, bd::smem_u32(&ctl->segment_done));
    }
    mma_commit(issue, bd::smem_u32(&ctl->o_drain));
    __syncwarp();
    bd::mbar_drain(bd::smem_u32(&ctl->o_drain), 0);
    __syncwarp();
  } else {
    // -------------------------------------------------------------- softmax
    const auto soft_sync = [] { bd::named_barrier_sync(3, SOFT); };
    // A wait that gives up (`ok`) ends no warp's loop: the barriers below count all of them.
    const int quarter = warp & 3, group = warp >> 2, col0 = group * WIDE + (lane >> 4) * COLS;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t s_at = tmem + lanes + group * WIDE, o_at = tmem + lanes + O_COL + group * WIDE;
    const int token = quarter * 16 + (lane & 15);
    // the weights of a token, its row of the second operand: the tile's rows contiguous
    const uint32_t w_at = rope_at + (token / 8) * 1024 + (token % 8) * 128;
    // A segment's queries: copies begun, once no product reads those of the segment before any more; and handed over.
    const auto begin_queries = [&](const Segment& g) {
      // a lane has up to three units of eight elements of every row; the key part's columns begin behind the padded latents'
      const int wide = a.dim + p.rope_dim, units = (2 * n_pairs + 1) * 8, rows = g.sq.q_len * a.group;
      int piece[3];
#pragma unroll
      for (int x = 0; x < 3; ++x) {
        const int u = lane + 32 * x;
        piece[x] = u < 16 * n_pairs ? (u * 8 < a.dim ? u * 8 : wide) : a.dim + (u - 16 * n_pairs) * 8;
      }
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(g.sq.q0) * a.q_tok;
      int i = (g.row0 + warp) / a.group, h = g.row0 + warp - i * a.group;
#pragma unroll 2
      for (int r = warp; r < N; r += SOFT_WARPS) {
        const uint16_t* src = q + i * a.q_tok + h * a.q_head;
        const uint32_t dst = q_at + r * 128;
#pragma unroll
        for (int x = 0; x < 3; ++x) {
          const int u = lane + 32 * x;
          const bool live = g.row0 + r < rows && piece[x] < wide;
          if (u < units) copy16(dst + (u / 8) * Q_CHUNK + (((u % 8) ^ (r & 7)) << 4), live ? src + piece[x] : q, live);
        }
        for (h += SOFT_WARPS; h >= a.group; h -= a.group) ++i;
      }
    };
    const auto end_queries = [&] {
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_proxy_async();
      bd::mbar_arrive(bd::smem_u32(&ctl->q_full));
    };
    bool ok = true;
    int stage = 0, tile = 0, turn = 0, t = 0, segments = 0;
    int at = from, seq = 0;
    Segment g = segment(at, seq), next = g;
    if (g.n > 0) begin_queries(g);
    bool handed = g.n == 0, more = true;  // whether the queries of the segment have been handed over
    while (more) {
      const int rows = g.sq.q_len * a.group;
      const int all_see = bdkv::visible(a, g.sq, g.row0 / a.group);  // its first row, and so all of them
      const int64_t part_row = static_cast<int64_t>(2 * blockIdx.x + !g.first) * N;
      if (tid < N) {
        const int row = g.row0 + tid, i = row / a.group, h = row - i * a.group;
        ctl->ref[tid] = NO_REF;
        ctl->visible[tid] = row < rows ? min(bdkv::visible(a, g.sq, i), g.end) : 0;
        ctl->out[tid] = row >= rows ? 0u
                        : g.whole   ? reinterpret_cast<uint64_t>(static_cast<uint16_t*>(a.out) +
                                                                 (static_cast<int64_t>(g.sq.q0) + i) * a.o_tok + h * a.o_head)
                                    : reinterpret_cast<uint64_t>(a.part_o + (part_row + tid) * a.dim);
      }
      soft_sync();
      more = at < to;
      if (more) next = segment(at, seq);
      if (!handed) end_queries();
      float2 L[COLS / 2];
#pragma unroll
      for (int c = 0; c < COLS / 2; ++c) L[c] = make_float2(0.f, 0.f);
      for (int j = 0; j < g.n; ++j, ++t) {
        const int t0 = g.begin + j * TOKENS;
        if (ok) ok = wait(ctl->s_full[t & 1], t >> 1);
        bd::tc_fence_after();
        float v[COLS];
        __syncwarp();
        tmem_load_halves<COLS>(s_at + (t & 1) * N, v);
#pragma unroll
        for (int c = 0; c < COLS; c += 2) {
          const float2 x = mul2(make_float2(v[c], v[c + 1]), make_float2(a.coef, a.coef));
          v[c] = x.x, v[c + 1] = x.y;
        }
        if (t0 + TOKENS > min(all_see, g.end)) {  // some row does not see all of the tile
#pragma unroll
          for (int c = 0; c < COLS; ++c)
            if (t0 + token >= ctl->visible[col0 + c]) v[c] = -INFINITY;
        }
        float2 x[COLS / 2];
        const auto subtract = [&] {
#pragma unroll
          for (int c = 0; c < COLS; c += 4) {
            const float4 r = *reinterpret_cast<const float4*>(&ctl->ref[col0 + c]);
            x[c / 2] = bd::add2(make_float2(v[c], v[c + 1]), make_float2(-r.x, -r.y));
            x[c / 2 + 1] = bd::add2(make_float2(v[c + 2], v[c + 3]), make_float2(-r.z, -r.w));
          }
        };
        subtract();
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < COLS / 2; ++c) top = bd::max3(top, x[c].x, x[c].y);
        if (group_any(group, top > P_MOST)) {
          const int col = col0 + (lane & (COLS - 1));
          const bool first = (lane & 15) < COLS;  // of the lanes that have this column
          const float most_here = across_lanes<COLS>(v, lane, [](float x, float y) { return fmaxf(x, y); });
          if (first) ctl->part[quarter][col] = most_here;
          group_sync(group);
          const float most = fmaxf(fmaxf(ctl->part[0][col], ctl->part[1][col]), fmaxf(ctl->part[2][col], ctl->part[3][col]));
          const float before = ctl->ref[col];
          group_sync(group);
          if (quarter == 0 && first) {
            const bool up = most - before > P_MOST;
            ctl->factor[col] = up ? bd::ex2_approx(before - reference(most)) : 1.f;
            if (up) ctl->ref[col] = reference(most);
          }
          group_sync(group);
          subtract();
#pragma unroll
          for (int c = 0; c < COLS; c += 2)
            L[c / 2] = mul2(L[c / 2], make_float2(ctl->factor[col0 + c], ctl->factor[col0 + c + 1]));
          if (j > 0) {
            // the tile before, in the place before
            if (ok) ok = tile > 0 ? wait(ctl->o_done[tile - 1], turn) : wait(ctl->o_done[tiles - 1], turn - 1);
            bd::tc_fence_after();
            for (int s = 0; s < n_pairs; ++s) {
              float o[WIDE];
              uint32_t y[WIDE];
              __syncwarp();
              tmem_load<WIDE>(o_at + s * N, o);
#pragma unroll
              for (int c = 0; c < WIDE; ++c) y[c] = __float_as_uint(o[c] * ctl->factor[group * WIDE + c]);
              tmem_store<WIDE>(o_at + s * N, y);
            }
            bd::tmem_st_wait();
          }
        }
        uint32_t w[COLS / 2];
#pragma unroll
        for (int c = 0; c < COLS / 2; ++c) {
          const float2 e = make_float2(bd::ex2_approx(x[c].x), bd::ex2_approx(x[c].y));
          L[c] = bd::add2(L[c], e);
          // The product takes one type for both operands, so weights get the latents': 11 bits in f16, 8 in bf16, each off by half
          // a step at most, as independent errors of a sum's terms. bf16 results, which are rounded to 8 bits anyway, are off by
          // 2.0e-3 in the 2-norm, 1.7e-3 with weights in fp32 (f16 2.1e-4 to 2.5e-4, 2.1e-4). A second product, of what the
          // rounding left, would bring that back for nearly half more of the products' time. The row's sum has them in fp32.
          w[c] = a.f16 ? F16::from_float2(e) : Bf16::from_float2(e);
        }
#pragma unroll
        for (int i = 0; i < COLS / 8; ++i)
          st_shared_v4(w_at + tile * CHUNK + (((col0 / 8 + i) ^ (token & 7)) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2],
                       w[4 * i + 3]);
        if (t0 + TOKENS > g.end) {
          // What a page holds behind the last token may be anything, and zero times it NaN: its latents become zeros.
          const int live = g.end - t0, units = (TOKENS - live) * 16;
          for (int s = 0; s < n_pairs; ++s) {
            int place = stage + s / per_stage;
            if (place >= stages) place -= stages;
            const uint32_t at = kv_at + place * stage_bytes + s % per_stage * PAIR;
            for (int x = tid; x < units; x += SOFT)
              st_shared_v4(at + (x % 16 / 8) * CHUNK + (live + x / 16) * 128 + ((x % 8) << 4), 0, 0, 0, 0);
          }
        }
        stage += (n_pairs + per_stage - 1) / per_stage;
        if (stage >= stages) stage -= stages;
        fence_proxy_async();
        bd::tc_fence_before();
        __syncwarp();
        if (lane == 0) bd::mbar_arrive(bd::smem_u32(&ctl->p_full[tile]));
        if (++tile == tiles) tile = 0, ++turn;
      }

      // all of the segment's scores are done: the next one's queries can come
      if (more && next.n > 0) begin_queries(next);

      // a row's sum: over the lanes, then over the four warps that have its tokens
      float sums[COLS];
#pragma unroll
      for (int c = 0; c < COLS; ++c) sums[c] = c & 1 ? L[c / 2].y : L[c / 2].x;
      const float sum_here = across_lanes<COLS>(sums, lane, [](float x, float y) { return x + y; });
      const int col = col0 + (lane & (COLS - 1));
      const bool first = (lane & 15) < COLS;
      if (first) ctl->part[quarter][col] = sum_here;
      group_sync(group);
      if (quarter == 0 && first) {
        const float sum = (ctl->part[0][col] + ctl->part[1][col]) + (ctl->part[2][col] + ctl->part[3][col]);
        // a whole row is 0 where it sees nothing, NaN where all of its scores are -inf (a part may well hold nothing)
        ctl->scale[col] = sum == 0.f ? (g.whole && ctl->visible[col] > 0 ? NAN : 0.f) : 1.f / sum;
        const int row = g.row0 + col;
        if (!g.whole) {  // a part's reference and sum: their log-sum-exp in one number would lose the sum of large scores
          reinterpret_cast<float2*>(a.part_l)[part_row + col] = make_float2(sum == 0.f ? -INFINITY : ctl->ref[col], sum);
        } else if (row < rows && a.lse != nullptr) {
          const int i = row / a.group, h = row - i * a.group;
          a.lse[(static_cast<int64_t>(g.sq.q0) + i) * a.group + h] =
              sum == 0.f ? -INFINITY : (ctl->ref[col] + log2f(sum)) / bd::LOG2E;
        }
      }
      group_sync(group);
      if (g.n > 0) {
        if (ok) ok = wait(ctl->segment_done, segments);
        ++segments;
      }
      bd::tc_fence_after();
      handed = true;
      if (more && next.n > 0) end_queries();
      for (int s = 0; s < n_pairs; ++s) {
        float o[WIDE];
        __syncwarp();
        if (g.n > 0)
          tmem_load<WIDE>(o_at + s * N, o);
        else
#pragma unroll
          for (int c = 0; c < WIDE; ++c) o[c] = 0.f;
        // Four lanes exchange until each has four dims next to each other, of a row in four: their stores are wider and fewer.
        const int d = s * 128 + quarter * 32 + (lane & ~3);
        const bool odd = lane & 1, upper = lane & 2;
        float2 two[WIDE / 2];
#pragma unroll
        for (int c = 0; c < WIDE; c += 2) {
          const float2 f = *reinterpret_cast<const float2*>(&ctl->scale[group * WIDE + c]);
          const float lo = o[c] * f.x, hi = o[c + 1] * f.y;
          const float other = __shfl_xor_sync(~0u, odd ? lo : hi, 1);
          two[c / 2] = odd ? make_float2(other, hi) : make_float2(lo, other);
        }
        if (g.whole) {
#pragma unroll
          for (int c = 0; c < WIDE; c += 4) {
            const uint32_t lo = a.f16 ? F16::from_float2(two[c / 2]) : Bf16::from_float2(two[c / 2]);
            const uint32_t hi = a.f16 ? F16::from_float2(two[c / 2 + 1]) : Bf16::from_float2(two[c / 2 + 1]);
            const uint32_t other = __shfl_xor_sync(~0u, upper ? lo : hi, 2);
            const uint64_t dst = ctl->out[group * WIDE + c + (lane & 3)];
            if (dst != 0 && d < a.dim)
              asm volatile("st.global.v2.b32 [%0], {%1, %2};" ::"l"(dst + d * 2), "r"(upper ? other : lo), "r"(upper ? hi : other)
                           : "memory");
          }
        } else {
#pragma unroll
          for (int c = 0; c < WIDE; c += 4) {
            const float2 lo = two[c / 2], hi = two[c / 2 + 1];
            const float2 give = upper ? lo : hi;
            const float2 other = make_float2(__shfl_xor_sync(~0u, give.x, 2), __shfl_xor_sync(~0u, give.y, 2));
            const uint64_t dst = ctl->out[group * WIDE + c + (lane & 3)];
            if (dst != 0 && d < a.dim)
              asm volatile("st.global.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(dst + d * 4), "f"(upper ? other.x : lo.x),
                           "f"(upper ? other.y : lo.y), "f"(upper ? hi.x : other.x), "f"(upper ? hi.y : other.y)
                           : "memory");
          }
        }
      }
      soft_sync();  // the rows have left
      g = next;
    }
  }

  __syncwarp();
  bd::tc_fence_before();
  __syncthreads();
  bd::tc_fence_after();
  if (warp == VALUE_WARP) bd::tmem_dealloc(tmem, tmem_columns<N>(n_pairs));
}

template <int N, bool SHARED>
cudaError_t launch(const LatentArgs& p, const CUtensorMap& latent, const CUtensorMap& rope, int sm_count, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // by device
  if (cudaError_t e = bdkv::allow_smem(latent_attn_kernel<N, SHARED>, 232448, ready); e != cudaSuccess) return e;
  const Layout l = layout<N>(p.a.dim);
  const dim3 grid = SHARED ? dim3(sm_count) : dim3(p.row_tiles, p.a.n_seq);
  latent_attn_kernel<N, SHARED><<<grid, N == 64 ? 352 : 224, l.bytes, st>>>(p, l.stages, l.tiles, latent, rope);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_latent_attn(const LatentArgs& p, const CUtensorMap& latent, const CUtensorMap& rope, int sm_count,
                               cudaStream_t st) {
  const auto run = p.shared ? (p.rows == 16 ? launch<16, true> : p.rows == 32 ? launch<32, true> : launch<64, true>)
                            : (p.rows == 16 ? launch<16, false> : p.rows == 32 ? launch<32, false> : launch<64, false>);
  return run(p, latent, rope, sm_count, st);
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
