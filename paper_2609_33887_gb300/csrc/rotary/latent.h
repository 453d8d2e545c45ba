// Internal interface of the latent cache's kernels.
#pragma once

#include <cuda.h>

#include "rotary/rotary.cuh"
#include "bdrotary.h"

namespace bdrot {

cudaError_t launch_latent_write(const bdrot_latent& c, const bdkv_rows& latent, const bdkv_rows& rope,
                                const int64_t* slot_map, int64_t n_tokens, const Turn* turn, int sm_count,
                                cudaStream_t st);

// What the attention kernels read of one call: lengths, masks and outputs as the 8-bit cache's kernels have them (one
// key/value head, dim = latent_dim); latents and key parts come through the tensor maps.
struct LatentArgs {
  bdkv::AttnArgs a;  // part_o [2 CTAs, rows, dim], part_l [2 CTAs, rows, 2]: parts of units that begin (0) or end in a CTA
  int rope_dim;
  int rows;       // (queries x heads) of a unit: 16, 32 or 64
  int row_tiles;  // units of a request, at most
  bool shared;    // the units' tiles shared out equally (else a CTA to each unit)
  bool columns;   // the latents' map is [64 elements, token, column, page], its boxes a stage's columns of 64 tokens
  int2* plan;     // [n_seq, row_tiles], of units that have rows: the first part of a split one (-1: it is whole) and its last
                  // CTA; behind them -1 where no unit is split
};
constexpr int TOKENS = 64;           // cached tokens of a tile
constexpr int MAX_STAGES = 6, MAX_TILES = 3;  // in shared memory: of latents, and of key parts
// Barriers by which weights are handed over and values' products say that they have ended: one for each place of the ring, in
// turn. A wait knows a phase by its parity, so a barrier must not get two phases ahead of a warp that waits for it. The loads
// see to that: nothing of the next tile in a place comes before the values' products have read the last. (With two, by the
// tile's parity, scores and weights could overtake the warp that issues those products in a ring of three tiles.)
constexpr int HANDOVERS = MAX_TILES;
__host__ __device__ constexpr int pairs_per_stage(int n_pairs) { return n_pairs < 2 ? 1 : 2; }  // of columns of 64
constexpr int MAX_SHARED_UNITS = 256;  // units whose tiles are shared out, at most
cudaError_t launch_latent_attn(const LatentArgs& p, const CUtensorMap& latent, const CUtensorMap& rope, int sm_count,
                               cudaStream_t st);
cudaError_t launch_latent_join(const LatentArgs& p, int sm_count, cudaStream_t st);
cudaError_t latent_status(cudaStream_t st, uint32_t* bits);

}  // namespace bdrot
