// Launch parameters and device helpers shared by the paths of ngc_tree_attn.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {

struct TreeAttnParams {
  const void* k;                // [L][Hkv][rows][d]
  const void* v;
  const int64_t* seq_off;       // contiguous caches only
  const int32_t* lens;
  const void* q;                // [L][B][Hq][N][d]
  const void* tree_k;           // [L][B][Hkv][N][d]
  const void* tree_v;
  const int32_t* parent;        // [B][N]
  const int32_t* n_nodes;       // [B] or null
  void* out;                    // [L][B][Hq][N][d]
  float* part_o;                // parts of split rows: sums, unnormalised ...
  float2* part_ml;              // ... and (maximum in log2 units, sum of weights)
                                //   FMA path: [n_layers][B][Hq][N][n_split]; tensor cores: [CTA][2][block_rows]
  int2* plan;                   // tensor cores, cut units: per CTA, the unit that begins in it and goes on, the CTA it ends in or -1
  int32_t* dev_status;
  int64_t rows;
  int L, B, Hq, Hkv, d, g, N;
  int layer_begin, n_layers, n_split, row_blocks, out_bf16;
  int even, cut, cluster, grid, n_units, block_rows, tiles_m;    // tensor cores
  float scale_log2;             // scale * log2(e)
  const int32_t* page_table;    // [B][G][pages_cap] or null
  int page, pages_cap, lists, G;
  int lens_lists;
};

constexpr int kTreeMaxNodes = NGC_TREE_MAX_NODES;
constexpr int kTreeWords = kTreeMaxNodes / 32;

// Row capacity of sequence b.
__device__ __forceinline__ int64_t tree_capacity(const TreeAttnParams& p, int b) {
  return p.page_table ? (int64_t)p.pages_cap * p.page : p.seq_off[b + 1] - p.seq_off[b];
}

// Ancestor-or-self sets of a tree as bit masks, by pointer doubling: in every round a node takes over the set of the
// node its jump link points at and jumps as far again, so a tree of depth D needs ceil(log2 D) rounds.  Called by all
// NT threads of the CTA; `anc` [n][kTreeWords] and `jump` [n] are shared memory.  Returns (to every thread) false for
// a node count or a link that is none; nothing may be read from anc then.
template <int NT>
__device__ __forceinline__ bool tree_masks(const int32_t* parent, int n, int N, uint32_t (*anc)[kTreeWords], int* jump) {
  constexpr int kPer = (kTreeMaxNodes + NT - 1) / NT;         // nodes per thread
  const int tid = threadIdx.x;
  bool bad = n < 0 || n > N;
  if (bad) n = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = tid + e * NT;
    if (i < n) {
      const int pa = parent[i];
      const bool wrong = i == 0 ? pa != -1 : (pa < 0 || pa >= i);
      bad = bad || wrong;
      jump[i] = wrong ? -1 : pa;
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) anc[i][w] = (i >> 5) == w ? 1u << (i & 31) : 0u;
    }
  }
  if (__syncthreads_or(bad)) return false;
  for (;;) {
    uint32_t m[kPer][kTreeWords];
    int nj[kPer];
    bool more = false;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = tid + e * NT;
      nj[e] = -1;
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) m[e][w] = 0;
      if (i < n && jump[i] >= 0) {
        const int j = jump[i];
        nj[e] = jump[j];
        more = true;
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) m[e][w] = anc[j][w];
      }
    }
    if (!__syncthreads_or(more)) return true;                  // (also: every read of this round is done)
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = tid + e * NT;
      if (i < n) {
        jump[i] = nj[e];
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) anc[i][w] |= m[e][w];
      }
    }
    __syncthreads();
  }
}

// (m, l) of a row that is not computed (a node beyond the tree, a refused sequence): the combine kernel leaves it alone.
#define kNoPart make_float2(0.f, -1.f)

// Four consecutive output channels from element idx on.
__device__ __forceinline__ void tree_store_out4(const TreeAttnParams& p, int64_t idx, float4 v) {
  if (p.out_bf16)
    *reinterpret_cast<uint2*>((__nv_bfloat16*)p.out + idx) = make_uint2(ptx::pack_bf16x2(v.x, v.y), ptx::pack_bf16x2(v.z, v.w));
  else
    *reinterpret_cast<float4*>((float*)p.out + idx) = v;
}

// Tensor-core path (bf16 caches, tree_attn_umma.cu): M tiles of 128 query rows per CTA for KV heads of `rows` rows, and the
// keys of a tile.
__host__ __device__ constexpr int tree_umma_tiles(int rows) { return rows <= 128 ? 1 : 2; }
__host__ __device__ constexpr int tree_umma_keys(int tiles) { return tiles == 1 ? 64 : 128; }
// What beginning another unit costs a CTA, in tiles: the row sums leave, Q changes.
__host__ __device__ constexpr int tree_unit_cost(int tiles_m) { return tiles_m == 1 ? 9 : 5; }
constexpr int kTreeMaxCluster = 8;
int launch_tree_umma(const TreeAttnParams& p, cudaStream_t stream);

// Even split of `total` tiles, beginnings of units counted in: how many of `grid` CTAs take part (each gets so many tiles at
// least that joining its part costs less than it saves: one sequence of 16384 tokens under one node, 64-key tiles: 25 us, 35 us
// with three), the first tile of CTA c, and the CTA that has tile g.
__host__ __device__ constexpr int tree_min_tiles(int tiles_m) { return tiles_m == 1 ? 8 : 3; }
__host__ __device__ inline int tree_even_ctas(int total, int grid, int tiles_m) {
  const int most = total / tree_min_tiles(tiles_m);
  return most < 1 ? 1 : (most < grid ? most : grid);
}
struct TreeEven {
  uint32_t per, more;           // tiles per CTA; the first `more` CTAs have one more
  __device__ __forceinline__ TreeEven(int total, int ctas) : per((uint32_t)total / (uint32_t)ctas), more((uint32_t)total % (uint32_t)ctas) {}
  __device__ __forceinline__ int first(uint32_t c) const { return (int)(c * per + min(c, more)); }
  __device__ __forceinline__ int owner(uint32_t g) const {
    const uint32_t split = more * (per + 1);
    return (int)(g < split ? g / (per + 1) : more + (g - split) / per);
  }
};

}  // namespace ngc
