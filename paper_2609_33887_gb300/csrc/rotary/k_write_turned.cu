// bdrot_write: keys turned on their way into the 8-bit cache, and the queries of the same tokens turned by further CTAs
// of the same launch.
//
// The write is that of the cache library (cache/write_rows.cuh), whose key rows are turned as they are read and rounded
// to their type, so that its scales and codes are those of rows turned before. A thread reads the eight elements that
// its own are paired with as well (they are in L1 then: their own thread reads them at the same time).
#include "cache/write_rows.cuh"
#include "rotary/rotary.cuh"

namespace bdrot {
namespace {

using bdkv::WRITE_THREADS;
static_assert(WRITE_THREADS == ROTATE_THREADS, "CTAs of both kinds in one launch");

template <class T>
struct TurnedRows {
  Turn turn;
  __device__ __forceinline__ uint4 operator()(const uint16_t* p, int64_t row, int sub, int w) const {
    uint4 x = *reinterpret_cast<const uint4*>(p);
    const int e = sub * 8, half = turn.dim / 2;
    if (w != 0 || e >= turn.dim) return x;
    const int position = turn.positions[row];
    uint32_t u[4] = {x.x, x.y, x.z, x.w};
    if (turn.inter) {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(turn.turns + sub * 4 + i);
        const float2 s = cos_sin(turn, f.x, position), t = cos_sin(turn, f.y, position);
        u[i] = T::from_float2(turn_pair(T::to_float2(u[i]), s));
        u[i + 1] = T::from_float2(turn_pair(T::to_float2(u[i + 1]), t));
      }
    } else {
      const bool second = e >= half;
      const uint4 y = *reinterpret_cast<const uint4*>(second ? p - half : p + half);
      const uint32_t v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(turn.turns + (second ? e - half : e) + 2 * i);
        float2 s = cos_sin(turn, f.x, position), t = cos_sin(turn, f.y, position);
        if (!second) s.y = -s.y, t.y = -t.y;
        const float2 own = T::to_float2(u[i]), other = T::to_float2(v[i]);
        u[i] = T::from_float2(make_float2(turn_one(own.x, other.x, s.x, s.y), turn_one(own.y, other.y, t.x, t.y)));
      }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};

template <class T>
__global__ void __launch_bounds__(WRITE_THREADS, 3) write_turned_kernel(bdkv::WriteArgs a, Turn turn, int64_t writes, RotateArgs q) {
  if (blockIdx.x < writes)
    bdkv::write_rows<T>(a, TurnedRows<T>{turn}, blockIdx.x);
  else
    rotate_rows<T, 2>(q, blockIdx.x - static_cast<uint32_t>(writes));
}

}  // namespace

cudaError_t launch_write(const bdkv_cache& c, const bdkv_rows& k, const bdkv_rows& v, const int64_t* slot_map,
                         int64_t n_tokens, const Turn& turn, const RotateArgs* q, int64_t q_blocks, int sm_count,
                         cudaStream_t st) {
  int64_t writes = 0;
  const bdkv::WriteArgs a = bdkv::write_args(c, k, v, slot_map, n_tokens, sm_count, &writes);
  const int64_t grid = writes + q_blocks;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  const RotateArgs r = q != nullptr ? *q : RotateArgs{};
  if (k.dtype == BDKV_BF16)
    write_turned_kernel<Bf16><<<static_cast<unsigned>(grid), WRITE_THREADS, 0, st>>>(a, turn, writes, r);
  else
    write_turned_kernel<F16><<<static_cast<unsigned>(grid), WRITE_THREADS, 0, st>>>(a, turn, writes, r);
  return cudaGetLastError();
}

}  // namespace bdrot
