// ngc_tree_attn: attention for a tree of drafted tokens over the pruned cache.
//
// The query rows of one KV head are the N nodes of each of its g query heads; in the layout
// [Hq][N][d] they are g * N consecutive rows, so a work item is a block of those rows, all of which
// see the alive cache rows and, of the tree, their ancestors.  Keys are numbered through: cache rows
// first, then the nodes; a row's mask only matters in the node part, where it is a bit of the node's
// ancestor set.
//
// bf16 caches run on the tensor cores (tree_attn_umma.cu); fp32 caches on the FMA path (this file): tiles of 32 keys as
// fp32 in shared memory, the next one on its way by 16-byte asynchronous copies; four query rows per group of lanes, online
// softmax with the row statistics spread over the group.  Blocks of 64 rows use 16 lanes per group (4 rows x 2 keys of S, 4
// rows x 8 channels of O per thread at d = 128: 32 multiply-adds per 8 shared-memory wavefronts), blocks of at most 16 rows
// 32 lanes (twice the threads per row: those calls wait for memory, not for arithmetic).  One pass over K and V; with few
// items the key axis is split and a second kernel joins the parts.  32 sequences of 4096 tokens, 8 nodes, 4 heads, d = 128:
// 154 us (539 MB: 3.5 TB/s; shared memory feeds the multiply-adds); 4 sequences of 300 to 512 tokens: 14 us, all latency; one of
// 8192 / 32768 tokens, one node: 51 / 78 us, most of it the join, which takes the parts of a row one after the other.
#include <cuda_bf16.h>

#include "ngc_plan.h"
#include "tree_attn.cuh"

namespace ngc {
namespace {

constexpr int kKeyTile = 32;                    // keys per tile, and the split granularity
constexpr int kSms = 148;
// Tensor cores: what a second kernel costs, in tiles; up to a unit per SM, no call with so few tiles per unit cuts units.
constexpr int join_tiles(int tiles_m) { return tiles_m == 1 ? 23 : 5; }
constexpr int kClusterJoin = 3;                 // tensor cores: what joining in a cluster costs, in tiles
constexpr int kSplitMin = 2;                    // tiles a split has at least

__device__ __forceinline__ bool finite4(float4 x) {
  return isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w);
}
// 16-byte asynchronous copy that writes zeros instead when `live` is false (nothing is read then).
__device__ __forceinline__ void copy16_or_zero(void* dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(live ? 16 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void load_n(const float* p, float (&x)[N]) {
  if constexpr (N == 2) {
    const float2 t = *reinterpret_cast<const float2*>(p);
    x[0] = t.x; x[1] = t.y;
  } else {
    const float4 t = *reinterpret_cast<const float4*>(p);
    x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
  }
}

template <int D, int RB> struct Fma {
  static constexpr int kLanes = RB == 16 ? 32 : 16;          // per group of 4 rows
  static constexpr int kThreads = RB / 4 * kLanes;
  static constexpr int kStages = RB == 16 ? 1 : 2;           // small blocks: more CTAs per SM hide the loads better
  static constexpr int kKeys = kKeyTile / kLanes;            // keys of a tile per lane: tx + kLanes * u
  static constexpr int kVec = D / kLanes < 4 ? D / kLanes : 4, kVecs = D / kLanes / kVec;   // channels per lane: kVecs runs of kVec
  struct Smem {
    float q[RB][D + 4], k[kStages][kKeyTile][D + 4], v[kStages][kKeyTile][D];
    float p[kKeyTile][RB + 4];
    uint32_t anc[kTreeMaxNodes][kTreeWords];
    int jump[kTreeMaxNodes];
    int odd[2];                                 // the tile's V rows hold an infinity or a NaN in its node part
  };
};

template <int D, int RB>
__global__ void __launch_bounds__(Fma<D, RB>::kThreads) tree_fma_kernel(TreeAttnParams p) {
  using F = Fma<D, RB>;
  constexpr int NT = F::kThreads, ST = F::kStages, NL = F::kLanes, KL = F::kKeys, VW = F::kVec, VN = F::kVecs;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  typename F::Smem& sm = *reinterpret_cast<typename F::Smem*>(smem_raw);
  const int tid = threadIdx.x, tx = tid % NL, ty = tid / NL;

  int item = blockIdx.x;
  const int split = item % p.n_split; item /= p.n_split;
  const int rb = item % p.row_blocks; item /= p.row_blocks;
  const int h = item % p.Hkv; item /= p.Hkv;
  const int b = item % p.B;
  const int lr = item / p.B, l = p.layer_begin + lr;

  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int n = p.n_nodes ? p.n_nodes[b] : p.N;
  const int rows = p.g * p.N, r0 = rb * RB;
  const int64_t part0 = (((int64_t)lr * p.B + b) * p.Hq + (int64_t)h * p.g) * p.N;     // parts of the KV head's first row
  const int len = p.lens[len_index(p.lens_lists, p.L, p.Hkv, b, l, h)];
  const bool len_ok = len >= 0 && len <= tree_capacity(p, b), n_ok = n >= 0 && n <= p.N;
  const int keys = len_ok && n_ok ? len + n : 0;
  const int nt = (keys + kKeyTile - 1) / kKeyTile, tps = (nt + p.n_split - 1) / p.n_split;
  const int tile_lo = min(nt, split * tps), tile_hi = min(nt, tile_lo + tps);
  const int plane = l * p.Hkv + h;
  const int64_t strip = ((int64_t)l * p.B + b) * p.Hkv + h;
  const float* const kc = (const float*)p.k + ((int64_t)plane * p.rows + p.seq_off[b]) * D;
  const float* const vc = (const float*)p.v + ((int64_t)plane * p.rows + p.seq_off[b]) * D;
  const float* const kt = (const float*)p.tree_k + strip * p.N * D;
  const float* const vt = (const float*)p.tree_v + strip * p.N * D;
  const int64_t row0 = (((int64_t)l * p.B + b) * p.Hq + (int64_t)h * p.g) * p.N;       // first query row of the KV head

  auto fetch = [&](int t) {                                        // dead keys: zeros, so that weight 0 x value is 0
    const int s = t % ST;
    for (int i = tid; i < kKeyTile * (D / 4); i += NT) {
      const int jj = i / (D / 4), c = 4 * (i % (D / 4)), j = t * kKeyTile + jj;
      const bool live = j < keys;
      const int64_t at = (int64_t)(j < len ? j : j - len) * D + c;
      copy16_or_zero(&sm.k[s][jj][c], live ? (j < len ? kc : kt) + at : kt, live);
      copy16_or_zero(&sm.v[s][jj][c], live ? (j < len ? vc : vt) + at : vt, live);
    }
    ptx::cp_async_commit();
  };
  for (int i = tid; i < RB * (D / 4); i += NT) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    const bool live = r0 + r < rows;
    copy16_or_zero(&sm.q[r][c], (const float*)p.q + (row0 + (live ? r0 + r : 0)) * D + c, live);
  }
  if (ST == 2 && tile_lo < tile_hi) fetch(tile_lo);
  const bool tree_ok = tree_masks<NT>(p.parent + (int64_t)b * p.N, n, p.N, sm.anc, sm.jump);
  if (!tree_ok || !len_ok) {
    ptx::cp_async_wait_all();
    if (tid == 0) set_dev_status(p.dev_status, tree_ok ? NGC_DEV_BAD_COUNTS : NGC_DEV_BAD_TREE);
    if (p.n_split > 1)
      for (int r = r0 + tid; r < min(rows, r0 + RB); r += NT) p.part_ml[(part0 + r) * p.n_split + split] = kNoPart;
    return;
  }
  int node[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int r = r0 + 4 * ty + e;
    node[e] = r < rows && r % p.N < n ? r % p.N : -1;              // -1: a row that is not there, and not written
  }
  float m[4], lsum[4], acc[4][VN][VW];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = -INFINITY; lsum[e] = 0.f;
#pragma unroll
    for (int cv = 0; cv < VN; ++cv)
#pragma unroll
      for (int c = 0; c < VW; ++c) acc[e][cv][c] = 0.f;
  }
  if (tid < 2) sm.odd[tid] = 0;
  const bool works = r0 + 4 * (ty & ~(32 / NL - 1)) < rows;         // a warp without rows only helps to fetch

  for (int t = tile_lo; t < tile_hi; ++t) {
    const int j0 = t * kKeyTile, s = t % ST;
    if (ST == 1) fetch(t);
    if (ST == 2 && t + 1 < tile_hi) {
      fetch(t + 1);
      ptx::cp_async_wait_group<1>();
    } else {
      ptx::cp_async_wait_all();
    }
    __syncthreads();
    if (j0 + kKeyTile > len) {
      for (int i = tid; i < kKeyTile * (D / 4); i += NT) {
        const int jj = i / (D / 4);
        if (j0 + jj >= len && !finite4(*reinterpret_cast<const float4*>(&sm.v[s][jj][4 * (i % (D / 4))]))) sm.odd[s] = 1;
      }
      __syncthreads();
    }
    if (!works) {
      __syncthreads();
      continue;
    }
    // S: rows 4 ty + e, keys tx + NL u
    float z[4][KL];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int u = 0; u < KL; ++u) z[e][u] = 0.f;
#pragma unroll 8
    for (int c = 0; c < D; c += 4) {
      float4 kx[KL];
#pragma unroll
      for (int u = 0; u < KL; ++u) kx[u] = *reinterpret_cast<const float4*>(&sm.k[s][tx + NL * u][c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 x = *reinterpret_cast<const float4*>(&sm.q[4 * ty + e][c]);
#pragma unroll
        for (int u = 0; u < KL; ++u)
          z[e][u] = fmaf(x.x, kx[u].x, fmaf(x.y, kx[u].y, fmaf(x.z, kx[u].z, fmaf(x.w, kx[u].w, z[e][u]))));
      }
    }
    uint32_t vis = 0;                                              // bit KL e + u: row 4 ty + e sees key tx + NL u
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < KL; ++u) {
        const int j = j0 + tx + NL * u, i = j - len;
        const bool see = j < len || (j < keys && node[e] >= 0 && ((sm.anc[node[e]][i >> 5] >> (i & 31)) & 1u));
        vis |= (uint32_t)see << (KL * e + u);
        z[e][u] = see ? z[e][u] * p.scale_log2 : -INFINITY;
        mx = fmaxf(mx, z[e][u]);
      }
#pragma unroll
      for (int o = NL / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m[e], mx), m_eff = m_new == -INFINITY ? 0.f : m_new;    // nothing visible yet: weights 0
      const float alpha = exp2f(m[e] - m_eff);
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < KL; ++u) {
        const float w = exp2f(z[e][u] - m_eff);
        sm.p[tx + NL * u][4 * ty + e] = w;
        sum += w;
      }
      lsum[e] = lsum[e] * alpha + sum;                             // this lane's share; joined at the end
      m[e] = m_new;
#pragma unroll
      for (int cv = 0; cv < VN; ++cv)
#pragma unroll
        for (int c = 0; c < VW; ++c) acc[e][cv][c] *= alpha;
    }
    __syncwarp();                                                  // P of a row group stays within its lanes
    if (!sm.odd[s]) {
#pragma unroll 4
      for (int jj = 0; jj < kKeyTile; ++jj) {
        float w[4];
        load_n(&sm.p[jj][4 * ty], w);
#pragma unroll
        for (int cv = 0; cv < VN; ++cv) {
          float x[VW];
          load_n(&sm.v[s][jj][VW * (NL * cv + tx)], x);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < VW; ++c) acc[e][cv][c] = fmaf(w[e], x[c], acc[e][cv][c]);
        }
      }
    } else {
      // a node's V row holds an infinity or a NaN: it must not reach the rows that do not see the node (0 x inf)
      for (int jj = 0; jj < kKeyTile; ++jj) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t of = __shfl_sync(0xffffffffu, vis, (tid & 31 & ~(NL - 1)) + jj % NL);
          if (!(of >> (KL * e + jj / NL) & 1u)) continue;
          const float w = sm.p[jj][4 * ty + e];
#pragma unroll
          for (int cv = 0; cv < VN; ++cv)
#pragma unroll
            for (int c = 0; c < VW; ++c) acc[e][cv][c] = fmaf(w, sm.v[s][jj][VW * (NL * cv + tx) + c], acc[e][cv][c]);
        }
      }
    }
    __syncthreads();                                               // the stage may be overwritten
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int o = NL / 2; o > 0; o >>= 1) lsum[e] += __shfl_xor_sync(0xffffffffu, lsum[e], o);
    const int r = r0 + 4 * ty + e;
    const int64_t pit = (part0 + r) * p.n_split + split;
    if (node[e] < 0) {
      if (p.n_split > 1 && r < rows && tx == 0) p.part_ml[pit] = kNoPart;
      continue;
    }
    const bool whole = p.n_split == 1;
    const float inv = whole ? 1.f / lsum[e] : 1.f;                 // (a sum of 0: every score is -inf, the row is NaN)
    if (!whole && tx == 0) p.part_ml[pit] = make_float2(m[e], lsum[e]);
    float* const to = whole ? (float*)p.out + (row0 + r) * D : p.part_o + pit * D;
#pragma unroll
    for (int cv = 0; cv < VN; ++cv) {
      float* const at = to + VW * (NL * cv + tx);
      if constexpr (VW == 2) *reinterpret_cast<float2*>(at) = make_float2(acc[e][cv][0] * inv, acc[e][cv][1] * inv);
      else *reinterpret_cast<float4*>(at) = make_float4(acc[e][cv][0] * inv, acc[e][cv][1] * inv, acc[e][cv][2] * inv, acc[e][cv][3] * inv);
    }
  }
}

// Joins the splits of a query row: d / 4 threads per row, four channels each.
__global__ void __launch_bounds__(128) tree_combine_kernel(TreeAttnParams p) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int per_row = p.d / 4;
  const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / per_row;      // (lr, b, hq, node)
  const int c = 4 * (int)(((int64_t)blockIdx.x * blockDim.x + threadIdx.x) % per_row);
  const int64_t per_layer = (int64_t)p.B * p.Hq * p.N;
  if (row >= p.n_layers * per_layer) return;
  if (p.part_ml[row * p.n_split].y < 0.f) return;                  // kNoPart
  float mg = -INFINITY;
  for (int s = 0; s < p.n_split; ++s) mg = fmaxf(mg, p.part_ml[row * p.n_split + s].x);
  float ls = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < p.n_split; ++s) {
    const float2 ml = p.part_ml[row * p.n_split + s];
    if (ml.x == -INFINITY && ml.y == 0.f) continue;                // nothing visible in this part; a NaN sum stays one
    const float f = exp2f(ml.x - mg);
    const float4 x = *reinterpret_cast<const float4*>(p.part_o + (row * p.n_split + s) * p.d + c);
    o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
    ls = fmaf(ml.y, f, ls);
  }
  const float inv = 1.f / ls;
  tree_store_out4(p, ((int64_t)p.layer_begin * per_layer + row) * p.d + c, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
}

template <int D, int RB> cudaError_t launch_fma_rows(const TreeAttnParams& p, unsigned grid, cudaStream_t stream) {
  using F = Fma<D, RB>;
  return launch_pdl(tree_fma_kernel<D, RB>, dim3(grid), dim3(F::kThreads), sizeof(typename F::Smem), stream, p);
}
template <int D> cudaError_t launch_fma(const TreeAttnParams& p, unsigned grid, cudaStream_t stream) {
  return p.block_rows == 16 ? launch_fma_rows<D, 16>(p, grid, stream) : launch_fma_rows<D, 64>(p, grid, stream);
}
template <int D> cudaError_t opt_in_fma() {
  cudaError_t e = cudaFuncSetAttribute(tree_fma_kernel<D, 16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(typename Fma<D, 16>::Smem));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(tree_fma_kernel<D, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(typename Fma<D, 64>::Smem));
  return e;
}

// How a call over `layers` layers is laid out.
struct TreePlan {
  int block_rows, blocks;       // query rows per item, blocks per KV head
  int n_split;                  // FMA path: token splits
  int tiles_m;                  // tensor cores: M tiles per CTA
  int even, cut, grid, n_units; // tensor cores: tiles dealt to `grid` CTAs, units cut where that falls; or
  int cluster;                  //   a unit per cluster of so many CTAs
};
TreePlan tree_plan(const ngc_cache* c, int layers, int N) {
  const int rows = c->Hq / c->Hkv * N;
  TreePlan pl = {};
  pl.n_split = 1;
  if (c->dtype == NGC_BF16) {
    const int tiles = tree_umma_tiles(rows), keys = tree_umma_keys(tiles);
    pl.blocks = (rows + 128 * tiles - 1) / (128 * tiles);
    pl.block_rows = pl.blocks > 1 ? 128 * tiles : rows;
    const int64_t units = (int64_t)layers * c->B * c->Hkv * pl.blocks;
    const int64_t longest = ((int64_t)c->max_len + keys - 1) / keys + (N + keys - 1) / keys;
    pl.n_units = (int)(units > 0x7fffffffLL ? 0x7fffffffLL : units);
    pl.tiles_m = tiles;
    // Clusters: so many CTAs per unit as make its tiles and the join shortest, as long as all clusters run at once: 14 of
    // eight CTAs, 32 of four, 74 of two (16 of eight: 18.7 us instead of 11.0 us for 14, units of 1024 tokens).  One sequence of
    // 512 / 1024 / 2048 tokens, 2 KV heads: 9.3 / 9.5 / 11.0 us; a CTA per unit 12.0 us, cut units 12.7 / 14.3 us.
    pl.cluster = 1;
    int64_t alone = longest;
    for (int c = 2; c <= kTreeMaxCluster; c *= 2)
      if (units <= (c == 8 ? 14 : c == 4 ? 32 : 74) && (longest + c - 1) / c + kClusterJoin < (pl.cluster > 1 ? alone + kClusterJoin : alone)) {
        pl.cluster = c;
        alone = (longest + c - 1) / c;
      }
    // Cutting units costs a second kernel and the parts' way through memory, in all join_tiles() tiles, and saves what a CTA's
    // share of a unit takes beyond an equal share of all (lengths taken to be three quarters of the longest on average).  64
    // sequences of 4096 tokens: 50 us uncut, 61 us cut; 32 of 1024 to 8192: 43 us cut, 53 us in clusters of two; one of 131072:
    // 55 us cut, 149 us in clusters of eight.
    pl.even = units > kSms || 4 * (alone - join_tiles(tiles)) * kSms > 3 * units * longest;
    pl.cut = pl.even && units < 2 * kSms;
    if (pl.even) {
      pl.cluster = 1;
      // More units than SMs fill all SMs, however short they are: beginning one costs a CTA more than the least it gets.  (150 sequences
      // of 64 tokens, one node and KV head: 15.9 us; 26.3 us on the 37 CTAs that a share of their 300 tiles would give.)
      const int64_t most = units > kSms ? kSms : units * longest / tree_min_tiles(tiles);
      pl.grid = (int)(most < kSms ? most : kSms);
    } else {
      pl.grid = pl.n_units * pl.cluster;
    }
    return pl;
  }
  pl.block_rows = rows <= 16 ? 16 : 64;         // small blocks keep the arithmetic near the rows there are
  pl.blocks = (rows + pl.block_rows - 1) / pl.block_rows;
  const int64_t items = (int64_t)layers * c->B * c->Hkv * pl.blocks;
  int64_t ns = kSms * (pl.block_rows == 16 ? 4 : 2) / items;      // one round of the CTAs that fit
  const int64_t by_len = ((int64_t)c->max_len + N + kSplitMin * kKeyTile - 1) / (kSplitMin * kKeyTile);
  if (ns > by_len) ns = by_len;
  if (ns > kSms) ns = kSms;
  pl.n_split = ns < 1 ? 1 : (int)ns;
  return pl;
}

// Whether the line of tiles of a call on the tensor cores can be counted in 32 bits: each unit has its beginning, its tree's tiles and
// the cache tile that it shares with nobody; all other cache tiles are full.
bool tree_line_fits(const ngc_cache* c, const TreePlan& pl, int layers, int N) {
  if (c->dtype != NGC_BF16) return true;
  const int keys = tree_umma_keys(pl.tiles_m);
  const double strips = (double)layers * c->Hkv * pl.blocks;
  return strips * ((double)c->B * (tree_unit_cost(pl.tiles_m) + 1 + (N + keys - 1) / keys) + (double)c->rows / keys) < 2147483647.0;
}

// Scratch of one call: the parts' sums, their (m, l), the plan.
struct TreeScratch { size_t ml, plan, bytes; };
TreeScratch tree_scratch(const ngc_cache* c, const TreePlan& pl, int layers, int N) {
  if (pl.n_split <= 1 && !pl.cut) return {0, 0, 0};
  const size_t parts = pl.cut ? (size_t)pl.grid * 2 * pl.block_rows : (size_t)layers * c->B * c->Hq * N * pl.n_split;
  TreeScratch s;
  s.ml = align256(parts * c->d * 4);
  s.plan = s.ml + align256(parts * 8);
  s.bytes = s.plan + (pl.cut ? align256((size_t)pl.grid * 8) : 0);
  return s;
}

int tree_impl(const ngc_cache* c, const PagedView& pv, const void* q, const void* tree_k, const void* tree_v, const int32_t* parent,
              const int32_t* n_nodes, int N, int layer_begin, int layer_end, float scale, void* out, int out_dtype,
              void* ws, size_t ws_bytes, int32_t* dev_status, cudaStream_t stream) {
  if (!q || !tree_k || !tree_v || !parent || !out || N < 1 || layer_begin < 0 || layer_end > c->L || layer_begin >= layer_end)
    return NGC_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 2.0e38f) return NGC_ERR_INVALID_ARG;      // (times log2 e it is still finite)
  if ((((uintptr_t)q | (uintptr_t)tree_k | (uintptr_t)tree_v | (uintptr_t)out | (uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0)
    return NGC_ERR_INVALID_ARG;      // rows are moved as 16-byte vectors
  if (out_dtype != NGC_F32 && !(out_dtype == NGC_BF16 && c->dtype == NGC_BF16)) return NGC_ERR_INVALID_ARG;
  if (N > kTreeMaxNodes) return NGC_ERR_UNSUPPORTED;
  if (pv.table && (c->dtype != NGC_BF16 || c->d != 128)) return NGC_ERR_UNSUPPORTED;

  TreeAttnParams p;
  p.k = c->k; p.v = c->v; p.seq_off = c->seq_off; p.lens = c->lens;
  p.q = q; p.tree_k = tree_k; p.tree_v = tree_v; p.parent = parent; p.n_nodes = n_nodes; p.out = out;
  p.part_o = nullptr; p.part_ml = nullptr; p.dev_status = dev_status; p.rows = c->rows;
  p.L = c->L; p.B = c->B; p.Hq = c->Hq; p.Hkv = c->Hkv; p.d = c->d; p.g = c->Hq / c->Hkv; p.N = N;
  p.layer_begin = layer_begin; p.n_layers = layer_end - layer_begin;
  p.out_bf16 = out_dtype == NGC_BF16; p.scale_log2 = scale * 1.4426950408889634f;
  p.page_table = pv.table; p.page = pv.page; p.pages_cap = pv.pages_cap; p.lists = pv.lists;
  p.G = lists_G(pv.lists, c->L, c->Hkv); p.lens_lists = c->lens_lists;
  const TreePlan plan = tree_plan(c, p.n_layers, N);
  if (!tree_line_fits(c, plan, p.n_layers, N)) return NGC_ERR_UNSUPPORTED;
  p.row_blocks = plan.blocks; p.n_split = plan.n_split; p.block_rows = plan.block_rows;
  p.tiles_m = plan.tiles_m;
  p.even = plan.even; p.cut = plan.cut; p.cluster = plan.cluster; p.grid = plan.grid; p.n_units = plan.n_units; p.plan = nullptr;
  const TreeScratch need = tree_scratch(c, plan, p.n_layers, N);
  if (need.bytes > 0) {
    if (!ws || ws_bytes < need.bytes || ((uintptr_t)ws & 255)) return NGC_ERR_WORKSPACE;
    p.part_o = (float*)ws;
    p.part_ml = (float2*)((char*)ws + need.ml);
    p.plan = (int2*)((char*)ws + need.plan);
  }
  const int64_t items = (int64_t)p.n_layers * c->B * c->Hkv * p.row_blocks * p.n_split;
  const int64_t out_threads = (int64_t)p.n_layers * c->B * c->Hq * N * (c->d / 4);
  if (items > 0x7fffffffLL || out_threads / 128 > 0x7ffffff0LL) return NGC_ERR_UNSUPPORTED;

  if (c->dtype == NGC_BF16) {
    return launch_tree_umma(p, stream);
  } else {
    static PerDeviceOnce attr_once;
    const int rc = attr_once.run([] {
      cudaError_t e = opt_in_fma<64>();
      return e == cudaSuccess ? opt_in_fma<128>() : e;
    });
    if (rc != NGC_OK) return rc;
    NGC_CUDA_TRY(c->d == 64 ? launch_fma<64>(p, (unsigned)items, stream) : launch_fma<128>(p, (unsigned)items, stream));
  }
  if (p.n_split > 1)
    NGC_CUDA_TRY(launch_pdl(tree_combine_kernel, dim3((unsigned)((out_threads + 127) / 128)), dim3(128), 0, stream, p));
  return NGC_OK;
}

}  // namespace

// Workspace that serves a call over any layer range, and one that gives a smaller max_len (which may cut its units where
// this one does not).
size_t tree_workspace_bytes(const ngc_cache* c, int N) {
  if (N < 1 || N > kTreeMaxNodes) return 0;
  size_t worst = 0;
  for (int layers = 1; layers <= c->L; ++layers) {
    TreePlan pl = tree_plan(c, layers, N);
    if (c->dtype == NGC_BF16) {
      const int keys = tree_umma_keys(pl.tiles_m);
      const int64_t longest = ((int64_t)c->max_len + keys - 1) / keys + (N + keys - 1) / keys;
      pl.cut = pl.n_units < 2 * kSms && (pl.n_units > kSms || longest > join_tiles(pl.tiles_m));
      pl.grid = kSms;
    }
    const size_t bytes = tree_scratch(c, pl, layers, N).bytes;
    if (bytes > worst) worst = bytes;
  }
  return worst;
}

}  // namespace ngc

extern "C" int ngc_tree_attn_launches(const ngc_cache* c, int layers, int N) {
  using namespace ngc;
  if (!valid_cache(c) || layers < 1 || N < 1 || N > kTreeMaxNodes) return 0;
  const TreePlan pl = tree_plan(c, layers, N);
  if (!tree_line_fits(c, pl, layers, N)) return 0;
  return pl.n_split > 1 || pl.cut ? 2 : 1;
}

extern "C" int ngc_tree_attn(const ngc_cache* c, const void* q, const void* tree_k, const void* tree_v, const int32_t* parent,
                             const int32_t* n_nodes, int N, int layer_begin, int layer_end, float scale, void* out, int out_dtype,
                             void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_tree_attn");
  using namespace ngc;
  if (!valid_cache(c)) return NGC_ERR_INVALID_ARG;
  const PagedView none = {nullptr, 0, 0, NGC_LISTS_SHARED};
  return tree_impl(c, none, q, tree_k, tree_v, parent, n_nodes, N, layer_begin, layer_end, scale, out, out_dtype, ws, ws_bytes,
                   dev_status, (cudaStream_t)stream);
}

extern "C" int ngc_tree_attn_paged(const ngc_paged_cache* pc, const void* q, const void* tree_k, const void* tree_v,
                                   const int32_t* parent, const int32_t* n_nodes, int N, int layer_begin, int layer_end, float scale,
                                   void* out, int out_dtype, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_tree_attn_paged");
  using namespace ngc;
  ngc_cache c;
  if (!paged_as_cache(pc, &c)) return NGC_ERR_INVALID_ARG;
  const PagedView pv = {pc->page_table, pc->page, pc->pages_cap, pc->lists};
  return tree_impl(&c, pv, q, tree_k, tree_v, parent, n_nodes, N, layer_begin, layer_end, scale, out, out_dtype, ws, ws_bytes,
                   dev_status, (cudaStream_t)stream);
}
