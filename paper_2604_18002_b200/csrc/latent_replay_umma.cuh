// Device pieces shared by the tensor-core kernels of the expanded form: tensor maps and the walk over tiles.
#pragma once

#include <cuda.h>

#include "kv_map.cuh"
#include "latent_replay.cuh"
#include "umma.cuh"

namespace ngc {

constexpr int kLatChunk = kLatTile * 128;      // 128 rows x 64 channels

// Token-major rows as a 3-D tensor (channel, head, row); box = 64 channels of one head x `box` rows.  Channels and rows that the
// tensor does not have read as zeros.
inline bool make_token_map(CUtensorMap* map, const void* base, int width, int heads, int64_t rows, int box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn || rows <= 0 || rows > 0x7fffffffLL) return false;
  cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)width * heads * 2};
  cuuint32_t size[3] = {64, 1, (cuuint32_t)box}, step[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, size, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Items of one or two blocks (A, B) of 128 queries of one head, the longest first, dealt out to the CTAs in turn; and for each the
// tiles of 128 keys that any of its queries sees.  Every warp of a CTA walks alike (all lanes together).
template <int BLOCKS> struct QueryWalk {
  int it, n_items;              // next item
  int l, b, h, q0, T, n;        // the current one; its key tiles are 0 .. n - 1
  int64_t row0;                 // first row of the sequence, within a layer
  const int2* tiles;            // of its list, or null
  int i, window;                // current tile, first tile of the window
  uint32_t live, plain_a, plain_b;             // of the window: tiles that a query sees; ones without a key that goes before query block A's (B's) last
  bool first;                   // the current tile is the item's first

  __device__ __forceinline__ QueryWalk(int items) : it(blockIdx.x), n_items(items), n(0), i(0), window(0), live(0), plain_a(0), plain_b(0) {}
  __device__ __forceinline__ bool has_b() const { return BLOCKS == 2 && q0 + kLatTile < T; }
  __device__ __forceinline__ bool for_a() const { return i * kLatTile <= q0; }
  __device__ __forceinline__ bool last_a() const { return i * kLatTile == q0; }
  __device__ __forceinline__ bool last() const { return i == n - 1; }
  __device__ __forceinline__ void load_window(const LatentReplayParams& p) {
    const int t = window + (threadIdx.x & 31);
    int2 g = make_int2(kNeverGone, kNeverGone);
    if (tiles && t < n) g = tiles[t];
    live = __ballot_sync(0xffffffffu, t < n && g.y > q0);
    plain_a = __ballot_sync(0xffffffffu, g.x > q0 + kLatTile - 1);
    plain_b = __ballot_sync(0xffffffffu, g.x > q0 + 2 * kLatTile - 1);
  }
  __device__ __forceinline__ bool next(const LatentReplayParams& p) {
    first = false;
    for (;;) {
      while (live == 0 && window + 32 < n) { window += 32; load_window(p); }
      if (live != 0) {
        const int k = __ffs(live) - 1;
        live &= live - 1;
        i = window + k;
        return true;
      }
      // the next item
      for (;;) {
        if (it >= n_items) return false;
        const int per = p.L * p.B * p.H, m = n_items / per - 1 - it / per, x = it % per;
        it += gridDim.x;
        h = x % p.H; b = x / p.H % p.B; l = x / p.H / p.B;
        q0 = m * BLOCKS * kLatTile;
        T = latent_seq(p, b, row0);
        if (q0 < T) break;
      }
      n = q0 / kLatTile + 1 + (has_b() ? 1 : 0);
      tiles = p.tile_gone ? p.tile_gone + ((int64_t)b * p.G + list_of(p.lists, l, 0, 1)) * (p.gone_cap / kLatTile) : nullptr;
      window = 0;
      load_window(p);
      first = true;
    }
  }
};

// Items of 128 keys of one head, the first (which most queries see) first; and for each the tiles of 64 queries from its own first
// key to the last query that sees one of them.
struct KeyWalk {
  static constexpr int kQ = 64;
  int it, n_items;
  int l, b, h, j0, T, i, n;     // current query tile, and the one behind the last
  int64_t row0;
  bool first;

  __device__ __forceinline__ KeyWalk(int items) : it(blockIdx.x), n_items(items), i(-1), n(0) {}
  __device__ __forceinline__ bool last() const { return i == n - 1; }
  __device__ __forceinline__ bool next(const LatentReplayParams& p) {
    first = false;
    if (++i < n) return true;
    for (;;) {
      if (it >= n_items) return false;
      const int per = p.L * p.B * p.H, x = it % per;
      j0 = it / per * kLatTile;
      it += gridDim.x;
      h = x % p.H; b = x / p.H % p.B; l = x / p.H / p.B;
      T = latent_seq(p, b, row0);
      if (j0 >= T) continue;
      int end = T;
      if (p.tile_gone) end = min(T, p.tile_gone[((int64_t)b * p.G + list_of(p.lists, l, 0, 1)) * (p.gone_cap / kLatTile) + j0 / kLatTile].y);
      i = j0 / kQ;
      n = (end + kQ - 1) / kQ;
      first = true;
      if (i < n) return true;                            // (a key sees to its own query at least)
    }
  }
};

}  // namespace ngc
