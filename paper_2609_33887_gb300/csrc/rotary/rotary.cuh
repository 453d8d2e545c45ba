// What the kernels of libbdrotary share: the rotation of pairs by positions.
#pragma once

#include "cache/cache.h"

namespace bdrot {

using bdkv::Bf16;
using bdkv::F16;

// A rotation as the kernels take it.
struct Turn {
  const unsigned long long* turns;  // fractions of a turn a position, times 2^64
  const int32_t* positions;
  int dim;
  bool inter, back;
  float scale, scale_low;      // the scale as two terms, so that it costs cosines no rounding
  float radians, radians_low;  // scale * 2 pi / 2^32, alike for sines
};

#ifdef __CUDACC__
// scale * (cos, sin) of position * turns. The product modulo 2^64 leaves the whole turns out without any error, at any
// position; of its upper 32 bits, two (after rounding) are the quadrant and the others an angle x of at most an eighth of a
// turn, whose sine and cosine are their power series: the terms left out are below 2^-29 and 2^-33.
__device__ __forceinline__ float2 cos_sin(const Turn& t, unsigned long long turns, int position) {
  const uint32_t at = static_cast<uint32_t>((turns * static_cast<unsigned long long>(static_cast<long long>(position))) >> 32);
  const uint32_t quadrant = (at + 0x20000000u) >> 30;
  const float r = static_cast<float>(static_cast<int32_t>(at - (quadrant << 30))), x = r * 1.4629180792671596e-9f;
  const float y = x * x, xs = fmaf(r, t.radians, r * t.radians_low);
  const float s = fmaf(xs * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), xs);
  const float p = fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -.5f);
  const float c = fmaf(y * t.scale, p, t.scale_low) + t.scale;
  const float a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;
  return make_float2((quadrant + 1) & 2 ? -a : a, quadrant & 2 ? -b : b);
}

// One element of a turned pair: the first with its second and -sin, the second with its first and sin. Written out, so that
// every kernel rounds alike.
__device__ __forceinline__ float turn_one(float own, float other, float c, float s) {
  return fmaf(own, c, __fmul_rn(other, s));
}
__device__ __forceinline__ float2 turn_pair(float2 x, float2 cs) {
  return make_float2(turn_one(x.x, x.y, cs.x, -cs.y), turn_one(x.y, x.x, cs.x, cs.y));
}

// Eight pairs of a row, in two words of four: with halves, firsts and seconds; interleaved, pairs 0..3 and 4..7.
template <class T, bool INTER>
__device__ __forceinline__ void turn8(uint4& x, uint4& y, const float2 (&cs)[8]) {
  uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = T::to_float2(u[i]), b = T::to_float2(v[i]);
    if (INTER) {
      u[i] = T::from_float2(turn_pair(a, cs[i]));
      v[i] = T::from_float2(turn_pair(b, cs[4 + i]));
    } else {
      const float2 x0 = turn_pair(make_float2(a.x, b.x), cs[2 * i]), x1 = turn_pair(make_float2(a.y, b.y), cs[2 * i + 1]);
      u[i] = T::from_float2(make_float2(x0.x, x1.x));
      v[i] = T::from_float2(make_float2(x0.y, x1.y));
    }
  }
  x = make_uint4(u[0], u[1], u[2], u[3]);
  y = make_uint4(v[0], v[1], v[2], v[3]);
}
#endif

constexpr int ROTATE_THREADS = 256;

// Rows to be turned. A block takes `ROTATE_THREADS / units` tokens and `per` heads of them.
struct RotateArgs {
  Turn turn;
  const uint16_t* x;
  uint16_t* out;
  int64_t x_tok, x_head, o_tok, o_head, n_tokens;
  int n_heads, units, per, groups;  // units: 16 elements of a row each; groups of heads
  bool in_place;
};
RotateArgs rotate_args(const bdkv_rows& x, const bdkv_rows& out, int n_heads, int head_dim, const Turn& turn,
                       int64_t n_tokens, int sm_count, int64_t* blocks);

#ifdef __CUDACC__
// A thread has eight pairs of its token, whose sines and cosines it computes once for all heads of its block.
template <class T, bool INTER, int AHEAD>
__device__ __forceinline__ void rotate_heads(const RotateArgs& a, int64_t token, int u, int h, int end) {
  const bool turned = u * 16 < a.turn.dim;
  if (!turned && a.in_place) return;
  const int e0 = INTER || !turned ? u * 16 : u * 8, e1 = INTER || !turned ? u * 16 + 8 : a.turn.dim / 2 + u * 8;
  float2 cs[8];
  if (turned) {
    const int position = a.turn.positions[token];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(a.turn.turns + u * 8 + i);
      cs[i] = cos_sin(a.turn, f.x, position);
      cs[i + 1] = cos_sin(a.turn, f.y, position);
    }
    if (a.turn.back)
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i].y = -cs[i].y;
  }
  const uint16_t* x = a.x + token * a.x_tok;
  uint16_t* o = a.out + token * a.o_tok;
  for (; h < end; h += AHEAD) {
    uint4 p[AHEAD], q[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (h + i >= end) break;
      p[i] = *reinterpret_cast<const uint4*>(x + (h + i) * a.x_head + e0);
      q[i] = *reinterpret_cast<const uint4*>(x + (h + i) * a.x_head + e1);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (h + i >= end) break;
      if (turned) turn8<T, INTER>(p[i], q[i], cs);
      *reinterpret_cast<uint4*>(o + (h + i) * a.o_head + e0) = p[i];
      *reinterpret_cast<uint4*>(o + (h + i) * a.o_head + e1) = q[i];
    }
  }
}

template <class T, int AHEAD>
__device__ __forceinline__ void rotate_rows(const RotateArgs& a, uint32_t block, int thread) {
  const int tokens = ROTATE_THREADS / a.units, local = thread / a.units, u = thread - local * a.units;
  const uint32_t at = block / a.groups, group = block - at * a.groups;
  const int64_t token = static_cast<int64_t>(at) * tokens + local;
  if (local >= tokens || token >= a.n_tokens) return;
  const int h = static_cast<int>(group) * a.per, end = min(h + a.per, a.n_heads);
  if (a.turn.inter)
    rotate_heads<T, true, AHEAD>(a, token, u, h, end);
  else
    rotate_heads<T, false, AHEAD>(a, token, u, h, end);
}
#endif

cudaError_t launch_rotate(const RotateArgs& a, int64_t blocks, bool f16, cudaStream_t st);
cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, const Turn& turn, const RotateArgs* q, int64_t q_blocks, int sm_count,
                         cudaStream_t st);

}  // namespace bdrot
