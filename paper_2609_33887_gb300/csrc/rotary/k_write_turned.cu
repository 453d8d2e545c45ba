// bdrot_write: keys turned on their way into the 8-bit cache, and the queries of the same tokens turned by further CTAs
// of the same launch.
//
// A CTA takes a few rows (a chunk) and some heads, one head after another, and does every run that starts among them, as
// the cache library's write does (cache/k_write.cu: runs, scales, tokens that are not finite). A thread has one or
// two pieces of a row, 16 elements each: of keys, the eight pairs that are turned together, whose sines and cosines it
// keeps for all heads. Turned keys are rounded to their type before their magnitudes and codes are taken, so that scales
// and codes are those of rows turned before. The next head's rows are on their way while a head's scales are agreed on.
// 131072 tokens of 32 query heads and 2 x 8 of 128 take 477 us, 6.2 TB/s (0.91 of a copy): 158 us the keys and values alone in
// whole pages, where kv_write takes 152 (157 from 256 requests that begin inside pages) and turning first 84; in pages of 16,
// 32, 128 and 256 tokens 174, 172, 187 and 276 (377, 226, 205 and 258). Few warps are what bounds them: 512 threads to an SM,
// with 128 registers each that do not quite do (48 to 56 bytes a thread are spilled, 160 where several runs are done at
// once). 64 tokens 8.3 to 8.7 us (replayed from a graph), latency: slots, rows, positions and angles, the page's scale.
// (Threads that compute sines and cosines for each head, or read them from shared memory with a thread to eight elements: 823
// and 683 us for 131072 tokens of 32 + 2 x 8 heads.)
// Runs of pages of 16 and 32 tokens are the work of a few warps each, so several are done at once (one after another: 384 and
// 225 us). A page of 256 tokens, whose runs would be four pieces to a thread, takes two CTAs, each for half of its rows, which
// give each other their largest magnitudes (a cluster).
#include "cache/write_rows.cuh"
#include "rotary/rotary.cuh"

namespace bdrot {
namespace {

using bdkv::WRITE_THREADS;
// Threads for which a run's rows, of up to eight pieces each, are two pieces to a thread, and in how many CTAs.
constexpr int threads_for(int page_size) { return page_size <= 64 ? 256 : 512; }
constexpr int ctas_for(int page_size) { return page_size <= 128 ? 1 : 2; }
static_assert(WRITE_THREADS == ROTATE_THREADS, "CTAs of both kinds in one launch");

// A piece: 16 elements of a row, in two groups of eight.
struct Piece {
  uint4 a, b;
};
__device__ __forceinline__ uint32_t top_of(const Piece& x) {
  const uint32_t t = __vmaxu2(bdkv::top_of(x.a), bdkv::top_of(x.b));
  return max(t & 0xffffu, t >> 16);
}
template <class T>
__device__ __forceinline__ uint2 codes_of(uint4 x, float f) {
  using namespace bdkv;
  return make_uint2(e4m3x4(scaled(T::to_float2(x.x), f), scaled(T::to_float2(x.y), f)),
                    e4m3x4(scaled(T::to_float2(x.z), f), scaled(T::to_float2(x.w), f)));
}
// Codes held under one scale, under a larger one.
__device__ __forceinline__ uint32_t rescaled(uint32_t x, float g) {
  using namespace bdkv;
  uint32_t lo, hi;
  decode4(x, lo, hi);
  return e4m3x4(scaled(bdkv::F16::to_float2(lo), g), scaled(bdkv::F16::to_float2(hi), g));
}

template <class T, bool INTER, int THREADS, int CTAS, bool TEAMS>
__device__ __forceinline__ void write_turned(const bdkv::WriteArgs& a, const Turn& turn, int heads, uint32_t block) {
  using namespace bdkv;
  constexpr uint32_t INF = std::is_same<T, bdkv::Bf16>::value ? 0x7f80u : 0x7c00u;
  constexpr int WARPS = THREADS / 32, PAGE = CTAS * THREADS / 4;
  __shared__ int64_t sl[2 * PAGE + 64];   // slots, from page_size rows before the chunk to as many behind
  __shared__ uint32_t top[2][2][CTAS * WARPS];  // of the heads in turn: keys' and values' largest patterns, of all CTAs' warps
  __shared__ uint8_t bad[PAGE];                 // a run's rows with something that is not finite
  const int rank = CTAS == 1 ? 0 : static_cast<int>(bd::cluster_ctarank());
  const auto sync = [] {
    if constexpr (CTAS == 1)
      __syncthreads();
    else
      bd::cluster_sync_all();
  };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, page_size = TEAMS ? a.c.page_size : PAGE;
  const int groups = (a.c.n_heads + heads - 1) / heads;
  const int h0 = static_cast<int>(block % groups) * heads, h_end = min(h0 + heads, a.c.n_heads);
  const int64_t r0 = static_cast<int64_t>(block / groups) * a.chunk, first = r0 - page_size;
  for (int i = tid; i < 2 * page_size + a.chunk; i += THREADS) {
    const int64_t r = first + i;
    const int64_t s = r >= 0 && r < a.n_tokens ? a.slots[r] : -1;
    sl[i] = s < a.n_slots ? s : -1;
  }
  sync();
  uint64_t starts = 0;  // rows of the chunk that start a run
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int t = part * 32 + lane;
    const int64_t s = t < a.chunk ? sl[page_size + t] : -1;
    bool begins = s >= 0;
    if (begins) {
      const int off = static_cast<int>(s & (page_size - 1));
      int d = 1;  // to the row before that is stored at all
      while (d <= off && sl[page_size + t - d] < 0) ++d;
      begins = d > off || sl[page_size + t - d] != s - d;
    }
    starts |= static_cast<uint64_t>(__ballot_sync(~0u, begins)) << (part * 32);
  }

  // A run of a small page is a few warps' work (a team): several runs at once.
  const int units = a.c.head_dim / 16, rows = page_size / CTAS;
  const int size = TEAMS ? ((rows * units + 1) / 2 + 31) / 32 * 32 : THREADS;
  const int teams = TEAMS ? min(THREADS / size, PAGE / page_size) : 1, team = TEAMS ? tid / size : 0, local = tid - team * size;
  int t_of[2], u_of[2], e0[2], e1[2];  // a piece's row of the run and place in it; where keys' two groups begin
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    t_of[i] = (local + i * size) / units, u_of[i] = local + i * size - t_of[i] * units;
    t_of[i] = t_of[i] < rows ? t_of[i] + rank * rows : PAGE;  // (PAGE: of no run)
    const bool halves = !INTER && u_of[i] * 16 < turn.dim;
    e0[i] = halves ? u_of[i] * 8 : u_of[i] * 16, e1[i] = halves ? turn.dim / 2 + u_of[i] * 8 : u_of[i] * 16 + 8;
  }
  int buf = 0;
  while (starts != 0) {
    uint64_t mine = team < teams ? starts : 0;
    for (int i = 0; i < team; ++i) mine &= mine - 1;  // (of several runs, the team's)
    for (int i = 0; i < teams; ++i) starts &= starts - 1;
    const bool some = !TEAMS || mine != 0;
    const int at = some ? page_size + __ffsll(static_cast<long long>(mine)) - 1 : 0;
    const int64_t slot = some ? sl[at] : 0, page = slot >> a.shift, row = first + at;
    const int off = static_cast<int>(slot & (page_size - 1)), n = some ? page_size - off : 0;
    bool live[2];
    Piece k[2], v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) live[i] = t_of[i] < n && sl[at + t_of[i]] == slot + t_of[i];
    const auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        k[i].a = k[i].b = v[i].a = v[i].b = make_uint4(0, 0, 0, 0);
        if (!live[i]) continue;
        const uint16_t* p = a.k + (row + t_of[i]) * a.k_tok + h * a.k_head;
        const uint16_t* q = a.v + (row + t_of[i]) * a.v_tok + h * a.v_head + u_of[i] * 16;
        k[i].a = *reinterpret_cast<const uint4*>(p + e0[i]), k[i].b = *reinterpret_cast<const uint4*>(p + e1[i]);
        v[i].a = *reinterpret_cast<const uint4*>(q), v[i].b = *reinterpret_cast<const uint4*>(q + 8);
      }
    };
    load(h0);
    float2 cs[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (live[i] && u_of[i] * 16 < turn.dim) {
        const int position = turn.positions[row + t_of[i]];
#pragma unroll
        for (int x = 0; x < 8; x += 2) {
          const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(turn.turns + u_of[i] * 8 + x);
          cs[i][x] = cos_sin(turn, f.x, position);
          cs[i][x + 1] = cos_sin(turn, f.y, position);
        }
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) cs[i][x] = make_float2(1.f, 0.f);
      }
    for (int h = h0; h < h_end; ++h, buf ^= 1) {
      uint8_t* k_scale = a.c.k_scale + page * a.c.k_scale_stride + h;
      uint8_t* v_scale = a.c.v_scale + page * a.c.v_scale_stride + h;
      const int k_before = off != 0 ? *k_scale : 0, v_before = off != 0 ? *v_scale : 0;
      Piece x[2], y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = k[i], y[i] = v[i];
        if (u_of[i] * 16 < turn.dim) turn8<T, INTER>(x[i].a, x[i].b, cs[i]);
      }
      uint32_t k_top = max(top_of(x[0]), top_of(x[1])), v_top = max(top_of(y[0]), top_of(y[1])), k_most, v_most, any;
      const auto give = [&] {
        const uint32_t k_warp = __reduce_max_sync(~0u, k_top), v_warp = __reduce_max_sync(~0u, v_top);
        if (lane != 0) return;
        uint32_t* mine = &top[buf][0][rank * WARPS + warp];
        mine[0] = k_warp, mine[CTAS * WARPS] = v_warp;
        if constexpr (CTAS > 1) {
          const uint32_t other = bd::mapa_shared(bd::smem_u32(mine), rank ^ 1);
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(other), "r"(k_warp) : "memory");
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(other + CTAS * WARPS * 4), "r"(v_warp) : "memory");
        }
      };
      const auto take = [&] {
        k_most = v_most = any = 0;
#pragma unroll
        for (int i = 0; i < CTAS * WARPS; ++i) {
          const uint32_t k_warp = top[buf][0][i], v_warp = top[buf][1][i];
          if (TEAMS) any = max(any, max(k_warp, v_warp));
          if (!TEAMS || (i * 32 >= team * size && i * 32 < team * size + size))
            k_most = max(k_most, k_warp), v_most = max(v_most, v_warp);
        }
        if (!TEAMS) any = max(k_most, v_most);
      };
      give();
      if (h + 1 < h_end) load(h + 1);
      sync();
      take();
      const bool some_bad = any >= INF;
      if (some_bad) {  // such rows do not count for either tensor's scale: find them, and the largest of the others
        if (tid < PAGE) bad[tid] = 0;
        sync();
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (top_of(x[i]) >= INF || top_of(y[i]) >= INF) bad[team * page_size + t_of[i]] = 1;
        __syncthreads();
        k_top = v_top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (live[i] && !bad[team * page_size + t_of[i]]) k_top = max(k_top, top_of(x[i])), v_top = max(v_top, top_of(y[i]));
        give();
        sync();
        take();
      }
      const int k_e = max(scale_byte(T::to_float2(k_most).x), k_before), v_e = max(scale_byte(T::to_float2(v_most).x), v_before);
      const float k_f = pow2i(127 - k_e), v_f = pow2i(127 - v_e);
      uint8_t* k_codes = a.c.k + page * a.c.k_stride[0] + h * a.c.k_stride[2];
      uint8_t* v_codes = a.c.v + page * a.c.v_stride[0] + h * a.c.v_stride[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!live[i]) continue;
        uint2 ka = codes_of<T>(x[i].a, k_f), kb = codes_of<T>(x[i].b, k_f);
        uint2 va = codes_of<T>(y[i].a, v_f), vb = codes_of<T>(y[i].b, v_f);
        if (some_bad && bad[team * page_size + t_of[i]]) {
          ka.x = ka.y = kb.x = kb.y = 0x7f7f7f7fu;
          va.x = va.y = vb.x = vb.y = 0u;
        }
        uint8_t* p = k_codes + (off + t_of[i]) * a.c.k_stride[1];
        if (INTER) {
          *reinterpret_cast<uint4*>(p + u_of[i] * 16) = make_uint4(ka.x, ka.y, kb.x, kb.y);
        } else {
          *reinterpret_cast<uint2*>(p + e0[i]) = ka;
          *reinterpret_cast<uint2*>(p + e1[i]) = kb;
        }
        *reinterpret_cast<uint4*>(v_codes + (off + t_of[i]) * a.c.v_stride[1] + u_of[i] * 16) = make_uint4(va.x, va.y, vb.x, vb.y);
      }
      // the tokens that the page holds already
      const auto again = [&](uint8_t* codes, int64_t cell, int before, int e) {
        const float g = before - e < -126 ? 0.f : pow2i(before - e);
        for (int i = rank * size + local; i < off * units; i += CTAS * size) {
          uint4* p = reinterpret_cast<uint4*>(codes + i / units * cell + i % units * 16);
          const uint4 w = *p;
          *p = make_uint4(rescaled(w.x, g), rescaled(w.y, g), rescaled(w.z, g), rescaled(w.w, g));
        }
      };
      if (off != 0 && k_e > k_before) again(k_codes, a.c.k_stride[1], k_before, k_e);
      if (off != 0 && v_e > v_before) again(v_codes, a.c.v_stride[1], v_before, v_e);
      if (some && local == 0 && rank == 0) {  // (read by all before the barrier above)
        if (k_e != k_before) *k_scale = static_cast<uint8_t>(k_e);
        if (v_e != v_before) *v_scale = static_cast<uint8_t>(v_e);
      }
      if (some_bad) __syncthreads();  // `bad` is free again; `top` alternates
    }
  }
  if constexpr (CTAS > 1) bd::cluster_sync_all();  // (the other may still write here)
}

template <class T, int THREADS, int CTAS, bool TEAMS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS)
    write_turned_kernel(bdkv::WriteArgs a, Turn turn, int heads, uint32_t writes, RotateArgs q) {
  constexpr uint32_t PER = THREADS / ROTATE_THREADS;  // blocks of rows of queries
  if (blockIdx.x >= writes)
    rotate_rows<T, 4>(q, (blockIdx.x - writes) * PER + threadIdx.x / ROTATE_THREADS, threadIdx.x % ROTATE_THREADS);
  else if (turn.inter)
    write_turned<T, true, THREADS, CTAS, TEAMS>(a, turn, heads, blockIdx.x / CTAS);
  else
    write_turned<T, false, THREADS, CTAS, TEAMS>(a, turn, heads, blockIdx.x / CTAS);
}

}  // namespace

cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, const Turn& turn, const RotateArgs* q, int64_t q_blocks, int sm_count,
                         cudaStream_t st) {
  int64_t writes = 0;
  bdkv::WriteArgs a = bdkv::write_args(c, k, v, slot_map, n_tokens, sm_count, &writes);
  // rows of a CTA: 64, so that small pages make several runs, fewer while the CTAs would not fill the SMs twice
  a.chunk = 64;
  while (a.chunk > 1 && (n_tokens + a.chunk - 1) / a.chunk * c.n_heads < 2 * sm_count) a.chunk /= 2;
  const RotateArgs r = q != nullptr ? *q : RotateArgs{};
  const bool bf16 = k.dtype == BDKV_BF16;
  // heads of a CTA: as many as leave eight CTAs to each SM
  const int64_t chunks = (n_tokens + a.chunk - 1) / a.chunk;
  int heads = c.n_heads;
  while (heads > 1 && chunks * ((c.n_heads + heads - 1) / heads) < 8 * sm_count) heads = (heads + 1) / 2;
  const int threads = threads_for(c.page_size), per = threads / ROTATE_THREADS, ctas = ctas_for(c.page_size);
  writes = chunks * ((c.n_heads + heads - 1) / heads) * ctas;
  const int64_t rest = (q_blocks + per - 1) / per, grid = writes + (rest + ctas - 1) / ctas * ctas;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  const auto of = [&](auto bf16_kernel, auto f16_kernel) { return bf16 ? bf16_kernel : f16_kernel; };
  const auto kernel = c.page_size > 128  ? of(write_turned_kernel<Bf16, 512, 2, false>, write_turned_kernel<F16, 512, 2, false>)
                      : c.page_size > 64 ? of(write_turned_kernel<Bf16, 512, 1, false>, write_turned_kernel<F16, 512, 1, false>)
                      : c.page_size > 32 ? of(write_turned_kernel<Bf16, 256, 1, false>, write_turned_kernel<F16, 256, 1, false>)
                                         : of(write_turned_kernel<Bf16, 256, 1, true>, write_turned_kernel<F16, 256, 1, true>);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, turn, heads, static_cast<uint32_t>(writes), r);
}

}  // namespace bdrot
