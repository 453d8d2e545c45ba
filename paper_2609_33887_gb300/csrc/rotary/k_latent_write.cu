// bdrot_latent_write: a latent and a turned key part of each token into the paged latent cache.
//
// A warp takes a token: its latent goes through registers, so that a token with an element that is not finite is seen
// before anything is stored. Bound by the bytes moved.
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

template <class T>
__global__ void __launch_bounds__(THREADS) latent_write_kernel(LatentWriteArgs a) {
  // the patterns of infinities and NaN are the ones from here on
  constexpr uint32_t INF = std::is_same<T, Bf16>::value ? 0x7f80u : 0x7c00u;
  const int lane = threadIdx.x & 31;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (THREADS / 32) + (threadIdx.x >> 5);
  if (row >= a.n_tokens) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || slot >= a.n_slots) return;
  const int64_t page = slot >> a.shift, off = slot & (a.c.page_size - 1);

  const uint16_t* src = a.latent + row * a.latent_tok;
  uint4 x[2];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = (i * 32 + lane) * 8;
    x[i] = e < a.c.latent_dim ? *reinterpret_cast<const uint4*>(src + e) : make_uint4(0, 0, 0, 0);
  }
  // the key part: eight pairs of a lane
  const int n_units = a.c.rope_dim / 16, half = a.c.rope_dim / 2;
  const bool halves = a.turn.dim != 0 && !a.turn.inter;
  const int e0 = halves ? lane * 8 : lane * 16, e1 = halves ? half + lane * 8 : lane * 16 + 8;
  uint4 y[2];
  if (lane < n_units) {
    const uint16_t* r = a.rope + row * a.rope_tok;
    y[0] = *reinterpret_cast<const uint4*>(r + e0);
    y[1] = *reinterpret_cast<const uint4*>(r + e1);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t t = __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                                __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
    most = max(most, max(t & 0xffffu, t >> 16));
  }
  const bool bad = __any_sync(~0u, most >= INF);
  uint16_t* dst = static_cast<uint16_t*>(a.c.latent) + page * a.c.latent_stride[0] + off * a.c.latent_stride[1];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = (i * 32 + lane) * 8;
    if (e < a.c.latent_dim) *reinterpret_cast<uint4*>(dst + e) = bad ? make_uint4(0, 0, 0, 0) : x[i];
  }
  if (lane >= n_units) return;
  if (a.turn.dim != 0) {
    const int position = a.turn.positions[row];
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(a.turn.turns + lane * 8 + i);
      cs[i] = cos_sin(a.turn, f.x, position);
      cs[i + 1] = cos_sin(a.turn, f.y, position);
    }
    if (a.turn.inter)
      turn8<T, true>(y[0], y[1], cs);
    else
      turn8<T, false>(y[0], y[1], cs);
  }
  if (bad) y[0] = y[1] = make_uint4(~0u, ~0u, ~0u, ~0u);  // NaN in both types
  uint16_t* r = static_cast<uint16_t*>(a.c.rope) + page * a.c.rope_stride[0] + off * a.c.rope_stride[1];
  *reinterpret_cast<uint4*>(r + e0) = y[0];
  *reinterpret_cast<uint4*>(r + e1) = y[1];
}

}  // namespace

cudaError_t launch_latent_write(const bdrot_latent& c, const bdkv_rows& latent, const bdkv_rows& rope,
                                const int64_t* slot_map, int64_t n_tokens, const Turn* turn, cudaStream_t st) {
  LatentWriteArgs a = {};
  a.c = c;
  a.latent = static_cast<const uint16_t*>(latent.data), a.latent_tok = latent.stride_token;
  a.rope = static_cast<const uint16_t*>(rope.data), a.rope_tok = rope.stride_token;
  a.n_tokens = n_tokens, a.n_slots = c.n_pages * c.page_size, a.slots = slot_map;
  while ((1 << a.shift) < c.page_size) ++a.shift;
  if (turn != nullptr) a.turn = *turn;
  const unsigned grid = static_cast<unsigned>((n_tokens + THREADS / 32 - 1) / (THREADS / 32));
  if (c.dtype == BDKV_BF16)
    latent_write_kernel<Bf16><<<grid, THREADS, 0, st>>>(a);
  else
    latent_write_kernel<F16><<<grid, THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace bdrot
