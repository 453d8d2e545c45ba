// bdrot_latent_write: a latent and a turned key part of each token into the paged latent cache.
//
// A warp takes eight tokens (one of a few): their latents go through registers, so that a token with an element that is not
// finite is seen before anything is stored, and their key parts, four lanes each, are turned together. Bound by the bytes
// moved: 131072 tokens of 512 + 64 take 49 us, 6.2 TB/s (0.91 of a copy); 64 tokens 4.2 us, latency. (A token to a warp, with 4 of its 32 lanes busy turning: 72 us.)
#include "rotary/latent.h"

namespace bdrot {
namespace {

constexpr int THREADS = 256;

struct LatentWriteArgs {
  bdrot_latent c;
  const uint16_t* latent;
  const uint16_t* rope;
  int64_t latent_tok, rope_tok, n_tokens, n_slots;
  const int64_t* slots;
  int shift;
  Turn turn;  // dim 0: none
};

// The largest magnitude pattern of eight elements, in each half of a word.
__device__ __forceinline__ uint32_t top_of(uint4 x) {
  return __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}

// PER: tokens of a warp.
template <class T, int PER>
__global__ void __launch_bounds__(THREADS) latent_write_kernel(LatentWriteArgs a) {
  // the patterns of infinities and NaN are the ones from here on
  constexpr uint32_t INF = std::is_same<T, Bf16>::value ? 0x7f80u : 0x7c00u;
  constexpr int BATCH = PER < 4 ? PER : 4;  // tokens whose latents are loaded before any is looked at
  const int lane = threadIdx.x & 31;
  const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (THREADS / 32) + (threadIdx.x >> 5)) * PER;
  // a lane's piece of a key part, eight pairs: of token lane / units. (Rows are read whether or not they are stored: nothing
  // waits for a slot before its elements are on their way.)
  const int units = a.c.rope_dim / 16, half = a.c.rope_dim / 2, of = lane / units, unit = lane - of * units;
  const bool halves = a.turn.dim != 0 && !a.turn.inter;
  const int e0 = halves ? unit * 8 : unit * 16, e1 = halves ? half + unit * 8 : unit * 16 + 8;
  const int64_t my_row = row0 + of;
  const bool mine = of < PER && my_row < a.n_tokens;
  uint4 y[2];
  int position = 0;
  if (mine) {
    const uint16_t* r = a.rope + my_row * a.rope_tok;
    y[0] = *reinterpret_cast<const uint4*>(r + e0);
    y[1] = *reinterpret_cast<const uint4*>(r + e1);
    if (a.turn.dim != 0) position = a.turn.positions[my_row];
  }
  int64_t slot = lane < PER && row0 + lane < a.n_tokens ? a.slots[row0 + lane] : -1;  // lane u: token u's
  if (slot >= a.n_slots) slot = -1;
  uint32_t bad = 0;  // tokens
#pragma unroll
  for (int u0 = 0; u0 < PER; u0 += BATCH) {
    uint4 x[BATCH][2];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t row = row0 + u0 + u;
        const int e = (i * 32 + lane) * 8;
        x[u][i] = row < a.n_tokens && e < a.c.latent_dim
                      ? *reinterpret_cast<const uint4*>(a.latent + row * a.latent_tok + e)
                      : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const uint32_t t = __vmaxu2(top_of(x[u][0]), top_of(x[u][1]));
      const bool off_range = __any_sync(~0u, max(t & 0xffffu, t >> 16) >= INF);
      bad |= static_cast<uint32_t>(off_range) << (u0 + u);
      const int64_t to = __shfl_sync(~0u, slot, u0 + u);
      if (to < 0) continue;
      uint16_t* dst = static_cast<uint16_t*>(a.c.latent) + (to >> a.shift) * a.c.latent_stride[0] +
                      (to & (a.c.page_size - 1)) * a.c.latent_stride[1];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = (i * 32 + lane) * 8;
        if (e < a.c.latent_dim) *reinterpret_cast<uint4*>(dst + e) = off_range ? make_uint4(0, 0, 0, 0) : x[u][i];
      }
    }
  }
  const int64_t to = __shfl_sync(~0u, slot, of < PER ? of : 0);
  if (!mine || to < 0) return;
  if (a.turn.dim != 0) {
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(a.turn.turns + unit * 8 + i);
      cs[i] = cos_sin(a.turn, f.x, position);
      cs[i + 1] = cos_sin(a.turn, f.y, position);
    }
    if (a.turn.inter)
      turn8<T, true>(y[0], y[1], cs);
    else
      turn8<T, false>(y[0], y[1], cs);
  }
  if (bad >> of & 1) y[0] = y[1] = make_uint4(~0u, ~0u, ~0u, ~0u);  // NaN in both types
  uint16_t* r = static_cast<uint16_t*>(a.c.rope) + (to >> a.shift) * a.c.rope_stride[0] +
                (to & (a.c.page_size - 1)) * a.c.rope_stride[1];
  *reinterpret_cast<uint4*>(r + e0) = y[0];
  *reinterpret_cast<uint4*>(r + e1) = y[1];
}

template <class T>
void launch(const LatentWriteArgs& a, int sm_count, cudaStream_t st) {
  // eight tokens to a warp where that leaves a few CTAs to each SM
  const int64_t ctas = (a.n_tokens + THREADS / 32 - 1) / (THREADS / 32);
  if (ctas >= 16 * int64_t(sm_count))
    latent_write_kernel<T, 8><<<static_cast<unsigned>((ctas + 7) / 8), THREADS, 0, st>>>(a);
  else
    latent_write_kernel<T, 1><<<static_cast<unsigned>(ctas), THREADS, 0, st>>>(a);
}

}  // namespace

cudaError_t launch_latent_write(const bdrot_latent& c, const bdkv_rows& latent, const bdkv_rows& rope,
                                const int64_t* slot_map, int64_t n_tokens, const Turn* turn, int sm_count,
                                cudaStream_t st) {
  LatentWriteArgs a = {};
  a.c = c;
  a.latent = static_cast<const uint16_t*>(latent.data), a.latent_tok = latent.stride_token;
  a.rope = static_cast<const uint16_t*>(rope.data), a.rope_tok = rope.stride_token;
  a.n_tokens = n_tokens, a.n_slots = c.n_pages * c.page_size, a.slots = slot_map;
  while ((1 << a.shift) < c.page_size) ++a.shift;
  if (turn != nullptr) a.turn = *turn;
  if (c.dtype == BDKV_BF16)
    launch<Bf16>(a, sm_count, st);
  else
    launch<F16>(a, sm_count, st);
  return cudaGetLastError();
}

}  // namespace bdrot
