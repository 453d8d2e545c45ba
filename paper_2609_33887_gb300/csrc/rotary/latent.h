// Internal interface of the latent cache's kernels.
#pragma once

#include <cuda.h>

#include "rotary/rotary.cuh"
#include "bdrotary.h"

namespace bdrot {

cudaError_t launch_latent_write(const bdrot_latent& c, const bdkv_rows& latent, const bdkv_rows& rope,
                                const int64_t* slot_map, int64_t n_tokens, const Turn* turn, int sm_count,
                                cudaStream_t st);

// What the attention kernels read of one call: lengths, masks, outputs and the split as the 8-bit cache's kernels have
// them (one key/value head, dim = latent_dim; part_l
// holds two floats a row and part, its reference and sum of weights); latents and key parts come through the tensor maps.
struct LatentArgs {
  bdkv::AttnArgs a;
  int rope_dim;
  int rows;  // (queries x heads) of a CTA: 16, 32 or 64
};
constexpr int TOKENS = 64;  // cached tokens of a tile
cudaError_t launch_latent_attn(const LatentArgs& p, const CUtensorMap& latent, const CUtensorMap& rope, cudaStream_t st);
cudaError_t launch_latent_join(const LatentArgs& p, cudaStream_t st);
cudaError_t latent_status(cudaStream_t st, uint32_t* bits);

}  // namespace bdrot
