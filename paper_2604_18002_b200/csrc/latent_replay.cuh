// Launch parameters shared by the kernels of ngc_latent_replay_attn and its gradient.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ngc_common.cuh"

namespace ngc {

constexpr int kLatNope = 128, kLatV = 128;    // channels of a head's own key part and of its value
constexpr int kLatTile = 128;                 // keys (and queries) per tile
constexpr int kNeverGone = 0x7fffffff;

struct LatentReplayParams {
  const int64_t* seq_off;
  const int32_t* lens;
  const __nv_bfloat16* q;       // [L][rows][H][128 + dr]
  const __nv_bfloat16* kv;      // [L][rows][H][256]
  const __nv_bfloat16* kr;      // [L][rows][dr]
  const int32_t* alive_pos;
  const int32_t* alive_count;
  const int32_t* total_before;
  int32_t* gone;                // [B][G][gone_cap] sequence length at the round that evicted each token; null: no rounds
  int4* tile_gone;              // [B][G][gone_cap / 128] of a tile of 128 tokens: smallest and largest of its first 64, of its others
  void* out;                    // [L][rows][H][128]
  float* lse;                   // [L][H][rows] or null
  const __nv_bfloat16* go;      // gradient of out
  float* delta;                 // [L][H][rows] sum over channels of out * go
  float* dkr_part;              // [L][H][rows][dr] each head's share of the gradient of kr
  __nv_bfloat16* gq;
  __nv_bfloat16* gkv;
  __nv_bfloat16* gkr;
  int32_t* dev_status;
  int64_t rows;
  int L, B, H, G, dr, lists, n_rounds, kt_max, max_len, gone_cap, out_bf16;
  float scale, scale_log2;
};

// First row and number of tokens of sequence b; 0 tokens (reported) where the length is none.
__device__ __forceinline__ int latent_seq(const LatentReplayParams& p, int b, int64_t& row0) {
  const int64_t lo = p.seq_off[b], hi = p.seq_off[b + 1];
  const int n = p.lens[b];
  row0 = lo;
  if (n < 0 || n > p.max_len || lo < 0 || hi > p.rows || n > hi - lo) {
    set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
    return 0;
  }
  return n;
}

int launch_latent_fwd(const LatentReplayParams& p, cudaStream_t stream);
int launch_latent_bwd(const LatentReplayParams& p, cudaStream_t stream);

}  // namespace ngc
