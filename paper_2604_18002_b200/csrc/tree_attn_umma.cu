// ngc_tree_attn on the 5th-generation tensor cores (bf16 caches).
//
// A unit of work is a block of up to MT x 128 query rows of one KV head (rows = node of a head, heads of the group
// one after the other) with all of its key tiles: the cache rows, then the nodes of the tree.  The 128 rows of an M
// tile are the 128 lanes of tensor memory.
//
//   up to 128 rows   MT = 1, tiles of 64 keys, five stages of K and V.  Two softmax groups take turns at the tiles, each with
//                    an O of its own and two S buffers, so that S is there four tiles ahead of P V; their sums meet at the
//                    end of a unit;
//   more rows        MT = 2, tiles of 128 keys, two stages: K and V tiles serve both M tiles, whose softmax and products
//                    alternate on the tensor pipe.  (With 64 keys S = Q K^T waits for shared memory: Q is read again for
//                    every 64 keys.)
//
//   producer warps   one for Q (once per unit) and K, one for V, by tiled TMA (128-byte swizzle), K and V each in a ring
//                    of its own (K is free as soon as S is computed, V only after P V).  Issuing a load takes a warp
//                    some 150 cycles, so a whole tile of a contiguous cache is ONE load (the groups of 64 channels are a
//                    dimension of the tensor map); pages are a load per 64 channels, the tree's rows come in
//                    16-row boxes.  Page-table entries are fetched 32 at a time, a batch ahead;
//   MMA thread       S = Q K^T into tensor memory, O += P V with P read from tensor memory;
//   mask warp        the ancestor sets of the next unit's tree, by pointer doubling;
//   softmax warps    (two groups of four) one thread per row: mask (in tree tiles, its node's ancestors; in the cache's last tile a common
//                    one), online softmax in the log2 domain, P as bf16 over the S it came from, 64 keys at a time.  The
//                    maximum used only moves when the true one has grown by more than a factor 2^8, so O in tensor
//                    memory is rarely rescaled.
//
// The roles only meet at mbarriers, also from one unit to the next: loads and scores of the next unit run under the
// end of the current one.
//
// Work is dealt out by tiles: the tiles of all units form one line (with a gap before each unit that stands for the cost
// of beginning it) that is cut into a piece per CTA.  With many units a piece ends at the next unit's
// beginning.  With few (fewer than two per CTA) the pieces are equal, so that rollouts of any lengths keep all SMs busy to the
// end: a CTA then has at most two unfinished units, the one it begins in and the one it ends in; their sums go to its two
// slots of the workspace and a second kernel joins the parts of every unit that was cut.  Where
// that does not pay (few short units), a cluster of up to 8 CTAs takes a unit, each an equal part of its tiles, and joins the
// parts through distributed shared memory.
//
// What bounds it: up to 128 rows, DRAM in the steady state and some 12 us around it (64 sequences of 2048 / 4096 tokens, 142 /
// 276 MB: 31.7 / 50.6 us, the difference at 7.1 TB/s; of 8192, cut: 102 us, the difference at 5.2 TB/s), and the longest unit where
// lengths differ (1024 to 4096 tokens, 173 MB: 47 us); few sequences see what a tile takes its CTA, some 800 cycles.
// (One softmax group and S one tile ahead: 1450 cycles.  Two CTAs per SM of two stages and one group each: 2 to 10 % slower
// from 320 sequences on but for short ragged ones, 81 and 84 us for 512 of 200 to 500 tokens.)  More rows: the chain
// S -> softmax -> P -> O of a tile (3100 cycles per 128 keys and 256 rows, 2550 of them without any softmax arithmetic; the products
// alone are 2048 cycles of the tensor pipe), the beginnings of units, and M tiles without rows: 131072
// tokens under 64 nodes, 12 heads (384 rows: three of four M tiles), two layers in 129 us, 800 TFLOP/s, for the first 60 ms of a row of
// calls and 152 to 156 us, 670 TFLOP/s, from then on (1000 W, 1650 of 1965 MHz).
//
// bf16 P: one rounding per weight (2^-8), as in the decode and replay calls; the row sum takes the weights
// before it.  0 x V must be 0 whatever a dead V row holds: rows of the last 16-row box beyond the live ones are
// zeroed in shared memory before the product, and a tree tile's V rows are searched for infinities and NaN,
// which are taken out of the product and added to exactly the rows that see their node.
//
// Every wait is bounded; a wait that runs out raises the CTA's abort flag, all roles leave, copies and MMAs
// in flight are drained (bounded), tensor memory is freed and NGC_DEV_TIMEOUT is reported.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>

#include "kv_map.cuh"
#include "tree_attn.cuh"
#include "umma.cuh"

namespace ngc {
namespace {

namespace cg = cooperative_groups;

constexpr float kLazyRescale = 8.f;             // log2 units the row maximum may grow before O is rescaled

template <int D, int MT> struct Cfg {
  static constexpr int kKeys = tree_umma_keys(MT);         // keys per tile
  static constexpr int kBufs = MT == 1 ? 2 : 1;            // S buffers per M tile
  static constexpr int kSplit = MT == 1 ? 2 : 1;           // softmax groups that take turns at an M tile's key tiles
  static constexpr int kAhead = kBufs * kSplit;            // tiles whose S an M tile has room for
  static constexpr int kHalves = kKeys / 64;               // P is handed over 64 keys at a time
  static constexpr int kGroups = MT * kSplit;              // softmax groups: 128 threads, S buffers and O of their own
  static constexpr int kStages = (MT == 1 ? 5 : 2) * (128 / D);                 // of K and of V
  static constexpr int kThreads = (4 * kGroups + 4) * 32;
  static constexpr int kMmaWarp = 4 * kGroups, kMaskWarp = kMmaWarp + 1, kProducerWarp = kMmaWarp + 2;      // K and Q; V in the warp behind
  static constexpr int kBox = kKeys * 128;                 // a tile's 64 channels
  static constexpr int kTile = kKeys * D * 2;              // K or V tile
  static constexpr int kQBytes = 128 * D * 2;              // Q of an M tile
  static constexpr int kSmem = MT * kQBytes + 2 * kStages * kTile + 1024;
  static constexpr int kUnitCost = tree_unit_cost(MT);
  static_assert(kUnitCost >= tree_min_tiles(MT));          // a unit is enough for a CTA
  static_assert(128 * MT * D * 4 <= 2 * kStages * kTile);  // a part of a cluster lies over the rings
  static constexpr uint32_t kOCol = 128 * kGroups;         // S[group][buf] at 128 group + 64 buf, O[group] behind
  static constexpr uint32_t kCols = 512;                   // of tensor memory: all
};

// Tensor maps of a launch.  K and V: whole tiles (contiguous caches, all channels in one box) or pages; the tree's K and V
// (16 rows, a plane per strip); Q (128 rows).
struct KvMaps { CUtensorMap cache, tree; };
struct Maps { KvMaps k, v; CUtensorMap q; };

// A unit and where it begins on the line.
struct Found { int u, base, places; };

template <int D, int MT> struct Shared {
  using C = Cfg<D, MT>;
  uint64_t k_full[C::kStages], k_empty[C::kStages], v_full[C::kStages], v_empty[C::kStages];
  uint64_t s_full[C::kGroups][C::kBufs], p_full[C::kGroups][C::kBufs][C::kHalves], o_done[C::kGroups][C::kBufs];
  uint64_t sums_full, sums_empty;               // two groups per M tile: the rows' (maximum, sum) in `sums`; O has been read
  float2 sums[C::kSplit][128];
  uint64_t q_full, q_empty, masks_full[2], masks_empty[2], fixed[3], drain;
  // by piece & 1: ancestor-or-self sets of the nodes, and whether the links are none
  alignas(16) uint32_t anc[2][kTreeMaxNodes][kTreeWords];
  int refused[2], jump[kTreeMaxNodes];
  uint32_t odd[4][kTreeWords];                  // by piece & 3: nodes whose V row holds an infinity or a NaN
  uint32_t tmem;
  int abort;
  float2 ml[128 * MT];                          // clusters: (maximum, sum) of this CTA's part of the rows
  int warp_sum[C::kThreads / 32], chunk[C::kThreads], total;         // places of the line before each thread's units
  Found found[2];
};

// What every role needs to know about the piece of a unit that is being worked on.
struct Piece {
  int b, h, l, lr, rb, n, len, lo, n_tiles, n_ct;      // tiles [lo, lo + n_tiles) of the unit; the first n_ct are the cache's
  int plane, strip;                                    // of the cache; of the tree's K and V
  bool first, last;                                    // holds the unit's first / last tile
};
// This CTA's share of the line: from place `at` of unit `u` on, n_left places in all; `seq` pieces so far.  A unit's
// first kUnitCost places hold no tile.
struct Walk { int u, at, n_left, seq; };

// Decodes unit u.
__device__ __forceinline__ void unit_of(const TreeAttnParams& p, uint32_t u, Piece& w) {
  if (p.row_blocks > 1) { w.rb = u % (uint32_t)p.row_blocks; u /= (uint32_t)p.row_blocks; } else { w.rb = 0; }
  w.h = u % (uint32_t)p.Hkv; u /= (uint32_t)p.Hkv;
  w.lr = p.n_layers > 1 ? u / (uint32_t)p.B : 0;
  w.b = u - w.lr * p.B;
  w.l = p.layer_begin + w.lr;
  w.plane = w.l * p.Hkv + w.h;
  w.strip = (w.l * p.B + w.b) * p.Hkv + w.h;
}
// Its node count and length, loaded at once.  False if they cannot be worked with (links are checked later).
__device__ __forceinline__ bool load_counts(const TreeAttnParams& p, Piece& w) {
  const int n = p.n_nodes ? p.n_nodes[w.b] : p.N;
  const int len = p.lens[p.lens_lists ? len_index(p.lens_lists, p.L, p.Hkv, w.b, w.l, w.h) : w.b];
  const int64_t cap = p.page_table ? (int64_t)p.pages_cap * p.page : p.seq_off[w.b + 1] - p.seq_off[w.b];
  w.n = n;
  w.len = len;
  return (n >= 0) & (n <= p.N) & (len >= 0) & (len <= cap);
}
// Key tiles of a unit with these counts.
template <int KT> __device__ __forceinline__ int unit_tiles(int n, int len) {
  return n > 0 ? (int)((uint32_t)(len + KT - 1) / KT + (uint32_t)(n + KT - 1) / KT) : 0;
}

// The next piece of the walk; false at its end.  (A unit per cluster: also a piece without tiles.)
template <int KT, int kUnitCost> __device__ __forceinline__ bool next_piece(const TreeAttnParams& p, Walk& k, Piece& w) {
  while (k.n_left > 0) {
    unit_of(p, (uint32_t)k.u, w);
    const bool fits = load_counts(p, w);
    const int nt = fits ? unit_tiles<KT>(w.n, w.len) : 0;
    if (!p.even) {                              // a unit per cluster
      const int rank = (int)(blockIdx.x % (uint32_t)p.cluster);
      if (!fits && threadIdx.x == 0) set_dev_status(p.dev_status, w.n < 0 || w.n > p.N ? NGC_DEV_BAD_TREE : NGC_DEV_BAD_COUNTS);
      w.lo = nt * rank / p.cluster;
      w.n_tiles = nt * (rank + 1) / p.cluster - w.lo;
      k.n_left = 0;
    } else {
      const int places = nt > 0 ? min(nt + kUnitCost - k.at, k.n_left) : 0;
      w.lo = max(0, k.at - kUnitCost);
      w.n_tiles = max(0, k.at + places - kUnitCost) - w.lo;
      k.n_left -= places;
    }
    ++k.u;
    k.at = 0;
    if (w.n_tiles > 0 || !p.even) {
      w.n_ct = (int)((uint32_t)(w.len + KT - 1) / KT);
      w.first = w.lo == 0;
      w.last = w.lo + w.n_tiles == nt;
      ++k.seq;
      return true;
    }
  }
  return false;
}

// Places of unit u on the line.
template <int KT, int kUnitCost> __device__ __forceinline__ int unit_places(const TreeAttnParams& p, int u, bool reports) {
  Piece w;
  unit_of(p, (uint32_t)u, w);
  const bool fits = load_counts(p, w);
  // counts that cannot be worked with have no tiles
  if (reports && !fits) set_dev_status(p.dev_status, w.n < 0 || w.n > p.N ? NGC_DEV_BAD_TREE : NGC_DEV_BAD_COUNTS);
  const int t = fits ? unit_tiles<KT>(w.n, w.len) : 0;
  return t > 0 ? t + kUnitCost : 0;
}
// The unit that place g lies in (whole warp): first the thread whose units it lies in, then 32 of them at a time.
template <int KT, int kUnitCost>
__device__ __forceinline__ Found find_unit(const TreeAttnParams& p, const int* chunk, int threads, int per, int g) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = threads;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chunk[mid] <= g) lo = mid; else hi = mid;
  }
  int run = chunk[lo];
  for (int u0 = lo * per;; u0 += 32) {
    const int mine = u0 + lane < min(p.n_units, lo * per + per) ? unit_places<KT, kUnitCost>(p, u0 + lane, false) : 0;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, run + incl > g);
    if (over || u0 + 32 >= lo * per + per) {
      const int at = over ? __ffs(over) - 1 : 31;
      return {u0 + at, __shfl_sync(0xffffffffu, run + incl - mine, at), __shfl_sync(0xffffffffu, mine, at)};
    }
    run += __shfl_sync(0xffffffffu, incl, 31);
  }
}

// Page-table entries in order, 32 at a time in the lanes of a producer warp, the next batch on its way.  An entry that is
// none is reported and read as page 0.
struct PageWalk {
  const int32_t* table;
  int cap, len, at, cur, next;                  // len: pages in use
  int32_t* dev_status;
  __device__ __forceinline__ int fetch(int first) const {
    const int j = first + (int)(threadIdx.x & 31);
    if (j >= len) return 0;
    const int pg = table[j];
    if (pg >= 0 && pg < cap) return pg;
    set_dev_status(dev_status, NGC_DEV_BAD_PAGE);
    return 0;
  }
  __device__ __forceinline__ void start(const int32_t* t, int pages_cap, int pages, int first, int32_t* status) {
    table = t; cap = pages_cap; len = pages; at = first; dev_status = status;
    cur = fetch(at);
    next = fetch(at + 32);
  }
  // entry j (not before the last one asked for); every lane gets it
  __device__ __forceinline__ int get(int j) {
    while (j >= at + 32) {
      at += 32;
      cur = next;
      next = fetch(at + 32);
    }
    return __shfl_sync(0xffffffffu, cur, j - at);
  }
};

// Issues the loads of K or V tile t (whole warp; one lane issues).  The cache's last tile or page is fetched whole: its dead
// rows, and rows that are not loaded and keep old bytes, are masked and P V stops before them.
template <int D, int KT>
__device__ __forceinline__ void load_tile(const TreeAttnParams& p, const KvMaps& maps, PageWalk& pages, const Piece& w, int base, int t,
                                          uint8_t* dst, uint64_t* bar) {
  constexpr int kBox = KT * 128;
  if (t >= w.n_ct) {
    const int row0 = (t - w.n_ct) * KT, n16 = (min(KT, w.n - row0) + 15) >> 4;
    if (umma::elect_one()) {
      ptx::mbar_expect_tx(bar, (uint32_t)n16 * 16 * D * 2);
      for (int r = 0; r < 16 * n16; r += 16)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) ptx::tma_load_3d(dst + c * kBox + r * 128, &maps.tree, 64 * c, row0 + r, w.strip, bar);
    }
    __syncwarp();
    return;
  }
  if (!p.page_table) {
    int y = base + t * KT;                      // (beyond the plane's last row the tile is filled with zeros)
    if (!NGC_IN_BOUNDS(p.dev_status, y >= 0 && y < p.rows)) y = 0;
    if (umma::elect_one()) {
      ptx::mbar_expect_tx(bar, (uint32_t)KT * D * 2);
      ptx::tma_load_4d(dst, &maps.cache, 0, y, 0, w.plane, bar);
    }
    __syncwarp();
    return;
  }
  const int live = min(KT, w.len - t * KT), n_pages = (live + p.page - 1) / p.page;
  if (umma::elect_one()) ptx::mbar_expect_tx(bar, (uint32_t)(n_pages * p.page) * D * 2);
  __syncwarp();
  for (int i = 0; i < n_pages; ++i) {
    int y = base + pages.get(t * KT / p.page + i) * p.page;
    if (!NGC_IN_BOUNDS(p.dev_status, y >= 0 && y + p.page <= p.rows)) y = 0;
    if (umma::elect_one()) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) ptx::tma_load_3d(dst + c * kBox + i * p.page * 128, &maps.cache, 64 * c, y, w.plane, bar);
    }
    __syncwarp();
  }
}

// max that keeps a NaN
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 32 consecutive bytes, a whole sector, at once
__device__ __forceinline__ void store_sector(float* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// 32 channels of an output row from element idx on, scaled.
__device__ __forceinline__ void tree_store_row32(const TreeAttnParams& p, int64_t idx, const uint32_t* o, float inv) {
#pragma unroll
  for (int c = 0; c < 32; c += 4)
    tree_store_out4(p, idx + c, make_float4(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv,
                                            __uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv));
}

__device__ __forceinline__ uint32_t odd_half(uint32_t x) { return (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u; }
// Bits of x (two bf16) that belong to infinities or NaN.
__device__ __forceinline__ uint32_t odd_bits(uint32_t x) { return odd_half(x) | odd_half(x >> 16) << 16; }

// (m, l) of a row of a part that has no tiles.
#define kNoTiles make_float2(-INFINITY, -2.f)

// Four channels of a row of a CTA's part, in shared memory (over the rings); rows are rotated so that neither the rows of a
// warp nor the channels of a row meet in a bank.
template <int D> __device__ __forceinline__ uint4* cluster_part(uint8_t* base, int row, int quad) {
  return reinterpret_cast<uint4*>(base) + row * (D / 4) + (quad ^ (row & (D / 4 - 1)));
}

// Joins the parts of a unit that the CTAs of a cluster have in their shared memory: rows dealt out to the CTAs and their
// warps, four channels per lane (with d = 64: two rows per warp).
template <int D, int MT, typename Sh>
__device__ __forceinline__ void cluster_join(const TreeAttnParams& p, Sh& sh, uint8_t* parts) {
  constexpr int kLanes = D / 4;
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  cluster.sync();
  Piece w;
  unit_of(p, blockIdx.x / (uint32_t)p.cluster, w);
  const int r0 = w.rb * MT * 128, rows = min(128 * MT, p.g * p.N - r0), quad = threadIdx.x % kLanes;
  const int64_t row0 = (((int64_t)w.l * p.B + w.b) * p.Hq + (int64_t)w.h * p.g) * p.N + r0;
  for (int r = rank + ctas * (threadIdx.x / kLanes); r < rows; r += ctas * (blockDim.x / kLanes)) {
    float2 ml[kTreeMaxCluster];
    float mg = -INFINITY;
    bool none = false, some = false;
#pragma unroll
    for (int i = 0; i < kTreeMaxCluster; ++i) {
      ml[i] = i < ctas ? *cluster.map_shared_rank(&sh.ml[r], i) : kNoTiles;
      none = none || ml[i].y == -1.f;           // kNoPart
      some = some || ml[i].y != -2.f;
      mg = fmaxf(mg, ml[i].x);
    }
    if (none || !some) continue;
    float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kTreeMaxCluster; ++i) {
      if (ml[i].y == -2.f || (ml[i].x == -INFINITY && ml[i].y == 0.f)) continue;       // nothing visible in this part
      const float f = exp2f(ml[i].x - mg);
      const uint4 x = *cluster.map_shared_rank(cluster_part<D>(parts, r, quad), i);
      l = fmaf(ml[i].y, f, l);
      o[0] = fmaf(__uint_as_float(x.x), f, o[0]); o[1] = fmaf(__uint_as_float(x.y), f, o[1]);
      o[2] = fmaf(__uint_as_float(x.z), f, o[2]); o[3] = fmaf(__uint_as_float(x.w), f, o[3]);
    }
    const float inv = 1.f / l;
    tree_store_out4(p, (row0 + r) * D + 4 * quad, make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv));
  }
  cluster.sync();                               // nobody leaves while its part may still be read
}

template <int D, int MT>
__global__ void __launch_bounds__(Cfg<D, MT>::kThreads, 1)
tree_umma_kernel(const __grid_constant__ Maps maps, TreeAttnParams p) {
  using C = Cfg<D, MT>;
  constexpr int ST = C::kStages, NT = C::kThreads, KT = C::kKeys, NB = C::kBufs, NH = C::kHalves, SP = C::kSplit;
  extern __shared__ uint8_t smem_dyn[];
  __shared__ Shared<D, MT> sh;
  uint8_t* sQ = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);     // [MT][128 rows]
  uint8_t* sK = sQ + MT * C::kQBytes;                                            // [ST]
  uint8_t* sV = sK + ST * C::kTile;                                              // [ST]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rows = p.g * p.N;

  if (tid == 0) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      ptx::mbar_init(&sh.k_full[s], 1); ptx::mbar_init(&sh.v_full[s], 1);
      ptx::mbar_init(&sh.k_empty[s], 1); ptx::mbar_init(&sh.v_empty[s], 1);
    }
#pragma unroll
    for (int m = 0; m < C::kGroups; ++m)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        ptx::mbar_init(&sh.s_full[m][i], 1);
        ptx::mbar_init(&sh.o_done[m][i], 1);
#pragma unroll
        for (int e = 0; e < NH; ++e) ptx::mbar_init(&sh.p_full[m][i][e], 128);
      }
    ptx::mbar_init(&sh.q_full, 1);
    ptx::mbar_init(&sh.q_empty, 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&sh.masks_full[i], 32); ptx::mbar_init(&sh.masks_empty[i], 128 * C::kGroups); }
#pragma unroll
    for (int i = 0; i < 3; ++i) ptx::mbar_init(&sh.fixed[i], 128);
    ptx::mbar_init(&sh.sums_full, 128 * C::kGroups);
    ptx::mbar_init(&sh.sums_empty, 128 * C::kGroups);
    ptx::mbar_init(&sh.drain, 1);
    ptx::fence_barrier_init();
    sh.abort = 0;
    ptx::prefetch_tensormap(&maps.k.cache);
    ptx::prefetch_tensormap(&maps.v.cache);
    ptx::prefetch_tensormap(&maps.q);
  }
  if (warp == C::kMmaWarp) umma::tmem_alloc(&sh.tmem, C::kCols);
  ptx::grid_dep_wait();
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  ptx::grid_dep_launch();                       // from here on this CTA holds its tensor memory
  const uint32_t tmem = sh.tmem;

  if (p.cluster > 1)
    for (int i = tid; i < 128 * MT; i += NT) sh.ml[i] = kNoTiles;
  Walk walk = {(int)(blockIdx.x / (uint32_t)p.cluster), 0, 0x7fffffff, 0};
  if (p.even) {
    const int per = (p.n_units + NT - 1) / NT, u0 = min(p.n_units, tid * per), u1 = min(p.n_units, u0 + per);
    int sum = 0;
#pragma unroll 2
    for (int i = u0; i < u1; ++i) sum += unit_places<KT, C::kUnitCost>(p, i, blockIdx.x == 0);
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) sh.warp_sum[warp] = incl;
    __syncthreads();
    int before = incl - sum;
    for (int i = 0; i < warp; ++i) before += sh.warp_sum[i];
    sh.chunk[tid] = before;
    if (tid == NT - 1) sh.total = before + sum;
    __syncthreads();
    const int total = sh.total, ctas = tree_even_ctas(total, gridDim.x, MT);
    const TreeEven even(total, ctas);
    const int g0 = even.first(blockIdx.x), g1 = even.first(blockIdx.x + 1);
    const bool busy = (int)blockIdx.x < ctas && total > 0;
    // the units in which this CTA's piece begins and ends (of whole units: in which the next piece begins)
    if (busy && warp < 2) {
      const int g = warp == 0 ? g0 : p.cut ? g1 - 1 : min(g1, total - 1);
      const Found f = find_unit<KT, C::kUnitCost>(p, sh.chunk, NT, per, g);
      if (lane == 0) sh.found[warp] = f;
    }
    __syncthreads();
    const Found a = sh.found[0], z = sh.found[1];
    if (!busy) {
      walk.n_left = 0;
    } else if (p.cut) {
      walk = {a.u, g0 - a.base, g1 - g0, 0};
      // for the kernel that joins the parts: the unit that begins here and goes on elsewhere (at most the last one), and
      // the CTA that it ends in
      const int tile0 = z.base + C::kUnitCost, end = z.base + z.places;
      if (tid == 0) p.plan[blockIdx.x] = make_int2(z.u, tile0 >= g0 && tile0 < g1 && end > g1 ? even.owner(end - 1) : -1);
    } else {
      // units that begin at a place of the piece, to their ends
      const bool here = a.base == g0;
      const int begin = here ? g0 : a.base + a.places, end = g1 >= total ? total : z.base == g1 ? g1 : z.base + z.places;
      walk = {here ? a.u : a.u + 1, 0, max(0, end - begin), 0};
    }
    if (!busy && p.cut && tid == 0) p.plan[blockIdx.x] = make_int2(0, -1);
  }

  // Every role takes the same walk.  Ring positions and barrier phases follow from running counters over its pieces: tiles
  // -> K/V stage; per M tile, tiles -> S buffer and P / O phases.
  Piece w;
  int kv = 0;
  if (warp >= C::kProducerWarp) {
    // ------------------------------------------------------------------ producers
    const bool is_v = warp != C::kProducerWarp;
    uint8_t* ring = is_v ? sV : sK;
    uint64_t* full = is_v ? sh.v_full : sh.k_full;
    uint64_t* empty = is_v ? sh.v_empty : sh.k_empty;
    const KvMaps& map = is_v ? maps.v : maps.k;
    int n_q = 0;
    bool ok = true, more = next_piece<KT, C::kUnitCost>(p, walk, w);
    for (Piece next; ok && more && w.n_tiles > 0; w = next) {
      const int base = (int)(p.page_table ? (int64_t)w.b * p.pages_cap * p.page : p.seq_off[w.b]);
      PageWalk pages;
      if (p.page_table)
        pages.start(p.page_table + ((int64_t)w.b * p.G + list_of(p.lists, w.l, w.h, p.Hkv)) * p.pages_cap, p.pages_cap,
                    (w.len + p.page - 1) / p.page, min(w.lo * KT, w.len) / p.page, p.dev_status);
      for (int i = 0; ok && i < w.n_tiles; ++i) {
        const int s = kv % ST;
        ok = kv < ST || umma::warp_wait(&empty[s], (kv / ST - 1) & 1, &sh.abort, p.dev_status);
        if (!ok) break;
        load_tile<D, KT>(p, map, pages, w, base, w.lo + i, ring + s * C::kTile, &full[s]);
        ++kv;
        if (i == 0 && is_v) more = next_piece<KT, C::kUnitCost>(p, walk, next);      // (found out while this piece runs)
        if (is_v || i > 0) continue;
        // Q behind the first K tile: its buffer is free once the last S of the piece before is done, the ring earlier
        const int r0 = w.rb * MT * 128, tiles_m = min(MT, (rows - r0 + 127) >> 7);
        const int64_t row0 = (((int64_t)w.l * p.B + w.b) * p.Hq + (int64_t)w.h * p.g) * p.N;
        ok = n_q == 0 || umma::warp_wait(&sh.q_empty, (n_q - 1) & 1, &sh.abort, p.dev_status);
        if (!ok) break;
        if (umma::elect_one()) {
          ptx::mbar_expect_tx(&sh.q_full, (uint32_t)(tiles_m * C::kQBytes));
          // rows beyond the KV head's belong to the next head (zeros past the end): they only feed rows that are never written
          for (int m = 0; m < tiles_m; ++m)
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
              ptx::tma_load_2d(sQ + m * C::kQBytes + c * (128 * 128), &maps.q, 64 * c, (int)(row0 + r0 + 128 * m), &sh.q_full);
        }
        __syncwarp();
        ++n_q;
        more = next_piece<KT, C::kUnitCost>(p, walk, next);
      }
    }
    if (!ok) {                                  // giving up: no copy may be in flight when the CTA ends
      if (!is_v && n_q > 0) ptx::mbar_wait_bounded(&sh.q_full, (n_q - 1) & 1);
      for (int j = max(0, kv - ST); j < kv; ++j) ptx::mbar_wait_bounded(&full[j % ST], (j / ST) & 1);
    }
  } else if (warp == C::kMaskWarp) {
    // ------------------------------------------------------------------ ancestor sets, four nodes per lane
    while (next_piece<KT, C::kUnitCost>(p, walk, w) && w.n_tiles > 0) {        // (a piece ahead of the others)
      const int slot = walk.seq & 1, use = (walk.seq - 1) >> 1;
      int link[kTreeWords];
#pragma unroll
      for (int x = 0; x < kTreeWords; ++x) link[x] = lane + 32 * x < w.n ? p.parent[(int64_t)w.b * p.N + lane + 32 * x] : -1;
      // (all softmax threads have taken the sets of two pieces ago, hence left the piece before that one)
      if (use > 0 && !umma::warp_wait(&sh.masks_empty[slot], (use - 1) & 1, &sh.abort, p.dev_status)) break;
      bool wrong = false;
#pragma unroll
      for (int x = 0; x < kTreeWords; ++x) {
        const int i = lane + 32 * x;
        const bool bad = i < w.n && (i == 0 ? link[x] != -1 : (link[x] < 0 || link[x] >= i));
        wrong = wrong || bad;
        sh.jump[i] = bad ? -1 : link[x];
#pragma unroll
        for (int y = 0; y < kTreeWords; ++y) sh.anc[slot][i][y] = y == x ? 1u << lane : 0u;
      }
      wrong = __any_sync(0xffffffffu, wrong);
      if (lane == 0) sh.refused[slot] = wrong;
      if (lane < kTreeWords) sh.odd[walk.seq & 3][lane] = 0;
      // in every round a node takes over the set of the node that its jump points at and jumps as far again
      for (bool more = true; more;) {
        more = false;
        uint4 got[kTreeWords];
        int far[kTreeWords];
        __syncwarp();
#pragma unroll
        for (int x = 0; x < kTreeWords; ++x) {
          const int j = sh.jump[lane + 32 * x];
          far[x] = j >= 0 ? sh.jump[j] : -1;
          got[x] = j >= 0 ? *reinterpret_cast<const uint4*>(sh.anc[slot][j]) : make_uint4(0, 0, 0, 0);
          more = more || j >= 0;
        }
        __syncwarp();
#pragma unroll
        for (int x = 0; x < kTreeWords; ++x) {
          uint4* at = reinterpret_cast<uint4*>(sh.anc[slot][lane + 32 * x]);
          const uint4 own = *at;
          sh.jump[lane + 32 * x] = far[x];
          *at = make_uint4(own.x | got[x].x, own.y | got[x].y, own.z | got[x].z, own.w | got[x].w);
        }
        more = __any_sync(0xffffffffu, more);
      }
      ptx::mbar_arrive(&sh.masks_full[slot]);
    }
  } else if (warp == C::kMmaWarp) {
    // ------------------------------------------------------------------ MMA issue
    // One thread does it all: a wait of the whole warp takes about 150 cycles even if it is over, and the tensor pipe runs dry
    // meanwhile (64 sequences of 2048 tokens: 28.5 us, 34 us with the warp at it).
    if (umma::elect_one()) {
      // Operand descriptors differ only in their low word (start address / 16, of which 14 bits: in a cluster, shared-memory
      // addresses hold the CTA's rank above them).
      const uint64_t desc_hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
      const uint32_t q_base = ((ptx::smem_u32(sQ) >> 4) & 0x3fff) | (1u << 16);
      const uint32_t k_base = (ptx::smem_u32(sK) >> 4) & 0x3fff, v_base = (ptx::smem_u32(sV) >> 4) & 0x3fff;
      const uint32_t v_lbo = (uint32_t)(C::kBox >> 4) << 16;                     // V: the next 64 channels are one box on
      int n_q = 0, done[C::kGroups];            // tiles per softmax group so far
      int k_at = 0, k_ph = 0, v_at = 0, v_ph = 0;           // stages of the next K and V tile, and their barriers' phases
#pragma unroll
      for (int g = 0; g < C::kGroups; ++g) done[g] = 0;
      auto wait = [&](uint64_t* bar, int phase) { return umma::wait_or_abort(bar, phase, &sh.abort, p.dev_status); };
      bool ok = true, more = next_piece<KT, C::kUnitCost>(p, walk, w);
      for (Piece next; ok && more && w.n_tiles > 0; w = next) {
        const int tiles_m = min(MT, (rows - w.rb * MT * 128 + 127) >> 7);        // M tiles that have a row
        auto steps_of = [&](int i) {            // 16-key steps of tile i that hold a live key
          const int t = w.lo + i;
          return min(KT / 16, (int)((t < w.n_ct ? w.len - t * KT : w.n - (t - w.n_ct) * KT) + 15) >> 4);
        };
        // softmax group of tile i of M tile m, and the tile's place in the group's order
        auto group_of = [&](int m, int i) { return SP == 2 ? i & 1 : m; };
        auto place_of = [&](int m, int i) { return SP == 2 ? (i & 1 ? done[C::kGroups - 1] : done[0]) + (i >> 1) : done[m] + i; };
        // S of tile i, from the next K stage
        auto issue_s = [&](int m, int i) {
          const int grp = group_of(m, i), buf = place_of(m, i) % NB;
          const uint32_t k_lo = (k_base + (uint32_t)(k_at * C::kTile >> 4)) | (1u << 16);
          const uint32_t q_lo = q_base + (uint32_t)((m * C::kQBytes) >> 4);
          const uint32_t idesc = umma::instr_desc(128, 0, false) | ((uint32_t)steps_of(i) * 2) << 17;    // N = 16 per step
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t a = desc_hi | (uint64_t)(q_lo + (uint32_t)(((ks >> 2) * (128 * 128) + (ks & 3) * 32) >> 4));
            const uint64_t bd = desc_hi | (uint64_t)(k_lo + (uint32_t)(((ks >> 2) * C::kBox + (ks & 3) * 32) >> 4));
            umma::mma_bf16(tmem + (uint32_t)(128 * grp + 64 * buf), a, bd, idesc, ks > 0);
          }
          umma::commit(&sh.s_full[grp][buf]);
          if (m + 1 == tiles_m) {
            umma::commit(&sh.k_empty[k_at]);
            if (i + 1 == w.n_tiles) umma::commit(&sh.q_empty);
          }
        };
        auto k_used = [&]() { if (++k_at == ST) { k_at = 0; k_ph ^= 1; } };
        // S into all buffers.  (P of the tile that used one before was consumed by a product issued before, and the pipe runs
        // them in issue order.)
        ok = wait(&sh.q_full, n_q & 1);
        ++n_q;
        for (int i = 0; ok && i < min(C::kAhead, w.n_tiles); ++i) {
          ok = wait(&sh.k_full[k_at], k_ph);
          if (!ok) break;
          for (int m = 0; m < tiles_m; ++m) issue_s(m, i);
          k_used();
        }
        more = next_piece<KT, C::kUnitCost>(p, walk, next);
        for (int i = 0; ok && i < w.n_tiles; ++i) {
          const bool s_next = i + C::kAhead < w.n_tiles;     // S of the tile that follows in this one's buffer
          const int steps = steps_of(i);
          if (MT == 2 && s_next) {
            ok = wait(&sh.k_full[k_at], k_ph);
            if (!ok) break;
          }
          ok = wait(&sh.v_full[v_at], v_ph);
          const uint32_t v_lo = (v_base + (uint32_t)(v_at * C::kTile >> 4)) | v_lbo;
          for (int m = 0; ok && m < tiles_m; ++m) {
            const int grp = group_of(m, i), place = place_of(m, i), buf = place % NB;
            const uint32_t o_tmem = tmem + C::kOCol + (uint32_t)(D * grp), p_tmem = tmem + (uint32_t)(128 * grp + 64 * buf);
#pragma unroll
            for (int e = 0; e < NH; ++e) {
              ok = ok && wait(&sh.p_full[grp][buf][e], (place / NB) & 1);
              if (!ok) break;
              umma::fence_after_sync();         // P was written with tcgen05.st by the softmax threads
#pragma unroll
              for (int kk = 4 * e; kk < 4 * e + 4; ++kk)
                if (kk < steps)
                  umma::mma_bf16_a_tmem(o_tmem, p_tmem + 8 * kk, desc_hi | (uint64_t)(v_lo + (uint32_t)((kk * 2048) >> 4)),
                                        umma::instr_desc(128, D, true), (i >= SP || kk > 0) ? 1u : 0u);
            }
            if (!ok) break;
            umma::commit(&sh.o_done[grp][buf]);
            if (m + 1 == tiles_m) umma::commit(&sh.v_empty[v_at]);
            if (!s_next) continue;
            if (MT == 1) ok = wait(&sh.k_full[k_at], k_ph);
            if (ok) issue_s(m, i + C::kAhead);
          }
          if (s_next) k_used();
          if (++v_at == ST) { v_at = 0; v_ph ^= 1; }
        }
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) done[g] += SP == 2 ? (w.n_tiles + 1 - g) / 2 : g < tiles_m ? w.n_tiles : 0;
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax: one thread per query row
    const int grp = warp >> 2, m = SP == 2 ? 0 : grp, turn = SP == 2 ? grp : 0;
    const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t o_addr = tmem + lane_base + C::kOCol + (uint32_t)(D * grp);
    int tc = 0, fixes[3] = {0, 0, 0};           // tiles of this group so far; uses of sh.fixed
    bool ok = true, more = next_piece<KT, C::kUnitCost>(p, walk, w);
    while (ok && more) {
      if (w.n_tiles <= 0) break;                // (a unit per cluster: no tile of it is this CTA's)
      const int r0 = w.rb * MT * 128, seq = walk.seq, slot = seq & 3;
      Piece next;
      more = next_piece<KT, C::kUnitCost>(p, walk, next);
      const int r = r0 + 128 * m + 32 * (warp & 3) + lane;
      const int node = (int)((uint32_t)r % (uint32_t)p.N);
      const bool live_row = r < rows && node < w.n;
      ok = umma::warp_wait(&sh.masks_full[seq & 1], ((seq - 1) >> 1) & 1, &sh.abort, p.dev_status);
      const uint4 set = live_row ? *reinterpret_cast<const uint4*>(sh.anc[seq & 1][node]) : make_uint4(0, 0, 0, 0);
      const uint32_t aw[kTreeWords] = {set.x, set.y, set.z, set.w};
      const bool refused = sh.refused[seq & 1] != 0;
      ptx::mbar_arrive(&sh.masks_empty[seq & 1]);
      const bool in_tail = w.len % KT != 0 && w.lo < w.n_ct && w.lo + w.n_tiles >= w.n_ct;
      const bool in_tree0 = w.lo <= w.n_ct && w.lo + w.n_tiles > w.n_ct, in_tree1 = w.lo <= w.n_ct + 1 && w.lo + w.n_tiles > w.n_ct + 1;
      if (r0 + 128 * m < rows) {
        const bool live_warp = r0 + 128 * m + 32 * (warp & 3) < rows;
        float m_use = -INFINITY, l_run = 0.f;
        for (int i = turn; ok && i < w.n_tiles; i += SP) {
          const int t = w.lo + i, place = tc + i / SP, buf = place % NB;
          const bool in_tree = t >= w.n_ct;
          const int live = in_tree ? w.n - (t - w.n_ct) * KT : w.len - t * KT;
          const bool masked = in_tree || live < KT;
          const int f = in_tree ? 1 + t - w.n_ct : 0;
          auto wait_s = [&] { return umma::warp_wait(&sh.s_full[grp][buf], (place / NB) & 1, &sh.abort, p.dev_status); };
          // A V stage's barrier may be asked for this tile once the stage's last tile was loaded, or its phase would be mistaken.
          // S runs kAhead tiles ahead of P V; it is there once P V of the tile kAhead before was issued: as many stages or more.
          // (MT = 2: S of the tile before, which is behind us, says the same, and the rows are mended under S of this one.  But
          // not of a piece's first tile: its S says that the second group has left the last wait for `fixed` of the piece before,
          // which an arrival at the same barrier would make it miss.)
          const bool s_first = MT == 1 || i == 0;
          if (s_first) ok = wait_s();
          if (!ok) break;
          if (masked && m == 0) {
            // V rows that must not meet a zero weight: by the tile's group, or the first M tile's
            const int s = (kv + i) % ST;
            ok = umma::warp_wait(&sh.v_full[s], ((kv + i) / ST) & 1, &sh.abort, p.dev_status);
            if (!ok) break;
            const int n_rows = min(KT, ((live + 15) >> 4) << 4);
            for (int e = tid & 127; e < n_rows * (D / 8); e += 128) {
              const int rr = e / (D / 8), c = e % (D / 8);               // (the swizzle permutes pieces within a row only)
              uint4* at = reinterpret_cast<uint4*>(sV + s * C::kTile + (c >> 3) * C::kBox + rr * 128 + (c & 7) * 16);
              if (rr >= live) {
                *at = make_uint4(0, 0, 0, 0);
              } else if (in_tree) {
                const uint4 x = *at;
                const uint4 o = make_uint4(odd_bits(x.x), odd_bits(x.y), odd_bits(x.z), odd_bits(x.w));
                if (o.x | o.y | o.z | o.w) {
                  *at = make_uint4(x.x & ~o.x, x.y & ~o.y, x.z & ~o.z, x.w & ~o.w);
                  const int j = (t - w.n_ct) * KT + rr;
                  atomicOr(&sh.odd[slot][j >> 5], 1u << (j & 31));
                }
              }
            }
            ptx::fence_proxy_async();
            ptx::mbar_arrive(&sh.fixed[f]);
          }
          if (!s_first) ok = wait_s();
          // (behind S of this tile every earlier use of the barrier is over, and the first group cannot come to its next use
          // before this group's P of the tile)
          if (ok && masked && m != 0)
            ok = umma::warp_wait(&sh.fixed[f], (f == 0 ? fixes[0] : f == 1 ? fixes[1] : fixes[2]) & 1, &sh.abort, p.dev_status);
          if (!ok) break;
          umma::fence_after_sync();
          if (!live_warp) {                     // rows that are not there: whatever P holds for them goes nowhere
#pragma unroll
            for (int e = 0; e < NH; ++e) ptx::mbar_arrive(&sh.p_full[grp][buf][e]);
            continue;
          }
          // 64 scores of the row at a time.  Of a 128-key tile the second half is read for the maximum, then the first half,
          // which stays in registers for its exponentials; the second half is read again behind them (a read costs about
          // 50 cycles; 128 scores in registers do not fit).
          uint32_t zr[2][32];
          const uint32_t s_addr = tmem + lane_base + (uint32_t)(128 * grp + 64 * buf);
          auto read_half = [&](int e) {
            umma::tmem_ld32(s_addr + 64 * e, zr[0]);
            umma::tmem_ld32(s_addr + 64 * e + 32, zr[1]);
            umma::tmem_ld_wait();
            if (masked) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                uint32_t see;
                if (!in_tree) see = live >= 64 * e + 32 * c + 32 ? 0xffffffffu : live > 64 * e + 32 * c ? (1u << (live - 64 * e - 32 * c)) - 1u : 0u;
                else if (KT == 128) see = e == 0 ? aw[c] : aw[2 + c];
                else see = t == w.n_ct ? aw[c] : aw[2 + c];
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (!(see >> j & 1u)) zr[c][j] = 0xff800000u;          // -inf
              }
            }
          };
          float mxc[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = NH - 1; e >= 0; --e) {
            read_half(e);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int j = 0; j < 32; j += 8) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  mxc[x] = max3_nan(mxc[x], __uint_as_float(zr[c][j + 2 * x]), __uint_as_float(zr[c][j + 2 * x + 1]));
              }
          }
          const float mx = max3_nan(max3_nan(mxc[0], mxc[1], mxc[2]), mxc[3], mxc[3]) * p.scale_log2;
          if (!(mx < INFINITY)) {               // a score of infinity or NaN: the row is NaN (also if it is all there is so far)
            l_run = __int_as_float(0x7fffffff);
            if (m_use == -INFINITY) m_use = 0.f;
          }
          const bool grow = mx > m_use + kLazyRescale;                    // also the first visible key (m_use = -inf)
          const bool rescale = grow && m_use != -INFINITY && i >= SP;       // O already holds something for this row
          if (__any_sync(0xffffffffu, rescale)) {
            // P V of the tile before is complete (with one S buffer: S of this tile came behind it)
            if (NB == 2) {
              ok = umma::warp_wait(&sh.o_done[grp][(place - 1) % NB], ((place - 1) / NB) & 1, &sh.abort, p.dev_status);
              if (!ok) break;
              umma::fence_after_sync();
            }
            const float alpha = rescale ? ptx::ex2_approx(m_use - mx) : 1.f;
            l_run *= alpha;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 16) {
              uint32_t o[16];
              umma::tmem_ld16(o_addr + c0, o);
              umma::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
              umma::tmem_st8(o_addr + c0, o);
              umma::tmem_st8(o_addr + c0 + 8, o + 8);
            }
            umma::tmem_st_wait();
          }
          if (grow) m_use = mx;
          const float m_eff = m_use == -INFINITY ? 0.f : m_use;           // nothing visible yet: every exponential is 0
          const uint64_t sc2 = umma::pack2(p.scale_log2, p.scale_log2), nm2 = umma::pack2(-m_eff, -m_eff);
          uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
          for (int e = 0; e < NH; ++e) {
            if (e > 0) read_half(e);
            uint32_t pk[32];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                float x0, x1;
                umma::unpack2(umma::fma2(umma::pack2(__uint_as_float(zr[c][j]), __uint_as_float(zr[c][j + 1])), sc2, nm2), x0, x1);
                const float p0 = ptx::ex2_approx(x0), p1 = ptx::ex2_approx(x1);
                acc2[(j >> 1) & 3] = umma::add2(acc2[(j >> 1) & 3], umma::pack2(p0, p1));
                pk[16 * c + (j >> 1)] = ptx::pack_bf16x2(p0, p1);
              }
            umma::tmem_st32(s_addr + 32 * e, pk);                         // P over the S columns it came from, packed to half
            umma::tmem_st_wait();
            umma::fence_before_sync();
            ptx::mbar_arrive(&sh.p_full[grp][buf][e]);
          }
          float s0, s1;
          umma::unpack2(umma::add2(umma::add2(acc2[0], acc2[1]), umma::add2(acc2[2], acc2[3])), s0, s1);
          l_run += s0 + s1;
        }
        // ---- the row's sums leave
        const int mine = (w.n_tiles - turn + SP - 1) / SP, last = tc + mine - 1;
        // (sh.odd is complete once `fixed` is.  Of two M tiles, the second's group asked in the tile, and must not ask again: the
        // first group may have used the barrier for the next piece by now.  Two groups of one M tile leave a piece together.)
        const bool ask = SP == 2 || m == 0;
        ok = ok && (mine == 0 || umma::warp_wait(&sh.o_done[grp][last % NB], (last / NB) & 1, &sh.abort, p.dev_status)) &&
             (!ask || !in_tree0 || umma::warp_wait(&sh.fixed[1], fixes[1] & 1, &sh.abort, p.dev_status)) &&
             (!ask || !in_tree1 || umma::warp_wait(&sh.fixed[2], fixes[2] & 1, &sh.abort, p.dev_status));
        if (!ok) break;
        umma::fence_after_sync();
        // two groups: their sums meet, and each takes half of the channels from here on
        float f0 = 1.f, f1 = 0.f;
        if constexpr (SP == 2) {
          sh.sums[turn][tid & 127] = make_float2(m_use, l_run);
          umma::fence_before_sync();
          ptx::mbar_arrive(&sh.sums_full);
          ok = umma::warp_wait(&sh.sums_full, (seq - 1) & 1, &sh.abort, p.dev_status);
          if (!ok) break;
          umma::fence_after_sync();
          const float2 a = sh.sums[0][tid & 127], b = sh.sums[SP - 1][tid & 127];
          m_use = fmaxf(a.x, b.x);
          const float m_eff = m_use == -INFINITY ? 0.f : m_use;
          f0 = exp2f(a.x - m_eff);
          f1 = exp2f(b.x - m_eff);
          l_run = a.y * f0 + b.y * f1;
        }
        const bool whole = w.first && w.last;
        const int64_t pit = ((int64_t)blockIdx.x * 2 + (w.first ? 1 : 0)) * p.block_rows + (r - r0);     // in this CTA's slots
        if (refused && tid == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_TREE);
        const float2 ml = live_row && !refused ? make_float2(m_use, l_run) : kNoPart;
        if (turn == 0 && p.cluster > 1) sh.ml[r - r0] = ml;
        else if (turn == 0 && !whole && r < rows) p.part_ml[pit] = ml;
        if (live_warp && !refused) {
          uint32_t odd[kTreeWords];
#pragma unroll
          for (int x = 0; x < kTreeWords; ++x) odd[x] = in_tree0 || in_tree1 ? sh.odd[slot][x] & aw[x] : 0u;
          const float inv = 1.f / l_run;        // (a sum of 0: every score is -inf, the row is NaN)
          const int64_t out_row = (((int64_t)w.l * p.B + w.b) * p.Hq + (int64_t)w.h * p.g) * p.N + r;
          const __nv_bfloat16* tv = (const __nv_bfloat16*)p.tree_v + (int64_t)w.strip * p.N * D;
#pragma unroll 1
          for (int c0 = turn * (D / SP); c0 < (turn + 1) * (D / SP); c0 += 32) {
            uint32_t o[32];
            __syncwarp();
            if constexpr (SP == 1) {
              umma::tmem_ld32(o_addr + c0, o);
              umma::tmem_ld_wait();
            } else {
              const uint32_t from = tmem + lane_base + C::kOCol + c0;
              uint32_t o1[32];
              umma::tmem_ld32(from, o);
              if (w.n_tiles > 1) umma::tmem_ld32(from + D, o1);
              umma::tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                const float x = __uint_as_float(o[c]) * f0;
                o[c] = __float_as_uint(w.n_tiles > 1 ? fmaf(__uint_as_float(o1[c]), f1, x) : x);
              }
            }
            if (odd[0] | odd[1] | odd[2] | odd[3]) {
              for (int j = 0; j < w.n; ++j) {
                const uint32_t word = j < 64 ? (j < 32 ? odd[0] : odd[1]) : (j < 96 ? odd[2] : odd[3]);
                if (!(word >> (j & 31) & 1u)) continue;
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                  const float v = __bfloat162float(tv[(int64_t)j * D + c0 + c]);
                  if (!isfinite(v)) o[c] = __float_as_uint(__uint_as_float(o[c]) + v);
                }
              }
            }
            if (!live_row) {
              // nothing to write
            } else if (p.cluster > 1) {         // (every product of this CTA has been taken: the rings are free)
#pragma unroll
              for (int c = 0; c < 32; c += 4)
                *cluster_part<D>(sK, r - r0, (c0 + c) / 4) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
            } else if (!whole) {
#pragma unroll
              for (int c = 0; c < 32; c += 8) store_sector(p.part_o + pit * D + c0 + c, o + c);
            } else {
              tree_store_row32(p, out_row * D + c0, o, inv);
            }
          }
        }
        umma::fence_before_sync();              // O may be overwritten once the next P of this thread is out ...
        if constexpr (SP == 2) {                // ... which has to wait for both readers
          ptx::mbar_arrive(&sh.sums_empty);
          ok = umma::warp_wait(&sh.sums_empty, (seq - 1) & 1, &sh.abort, p.dev_status);
        }
        tc += mine;
      }
      kv += w.n_tiles;
      fixes[0] += in_tail;
      fixes[1] += in_tree0;
      fixes[2] += in_tree1;
      w = next;
    }
  }
  __syncthreads();
  // ---- teardown: every role has left its loops; every MMA has completed before tensor memory is released
  if (warp == C::kMmaWarp) {
    if (umma::elect_one()) umma::commit(&sh.drain);
    __syncwarp();
    ptx::mbar_wait_bounded(&sh.drain, 0);
  }
  umma::fence_before_sync();
  __syncthreads();
  if (warp == C::kMmaWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, C::kCols);
  }
  if (p.cluster > 1) cluster_join<D, MT>(p, sh, sK);
}

// Joins the parts of the units that were cut.  blockIdx.x: the CTA of the main kernel that the unit began in, if one did;
// 16 lanes per query row, D / 16 channels per lane.  The lanes fetch the parts' (m, l) together, then four parts' sums
// are on their way at a time.
constexpr int kJoinRows = 16;                   // rows per CTA
template <int D> __global__ void __launch_bounds__(16 * kJoinRows) tree_join_kernel(TreeAttnParams p) {
  constexpr int kPer = D / 16, kAhead = 4;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int c0 = blockIdx.x, lane = threadIdx.x & 15, rr = blockIdx.y * kJoinRows + (threadIdx.x >> 4);
  const int2 cut = p.plan[c0];                  // (unit, CTA that it ends in)
  const int c1 = cut.y;
  if (c1 < 0) return;
  const int r = (int)((uint32_t)cut.x % (uint32_t)p.row_blocks) * p.block_rows + rr;
  const bool live_row = rr < p.block_rows && r < p.g * p.N;
  // part of CTA x: the unit begins in c0 (its second slot) and goes on through the others (their first)
  auto slot = [&](int x) { return ((int64_t)x * 2 + (x == c0 ? 1 : 0)) * p.block_rows + (live_row ? rr : 0); };
  float mg = -INFINITY, ls = 0.f, o[kPer];
  bool none = !live_row;
#pragma unroll
  for (int c = 0; c < kPer; ++c) o[c] = 0.f;
  for (int x0 = c0; x0 <= c1; x0 += 16) {
    const int n = min(16, c1 - x0 + 1);
    const float2 ml = lane < n ? p.part_ml[slot(x0 + lane)] : make_float2(-INFINITY, 0.f);
    const float l_first = __shfl_sync(0xffffffffu, ml.y, 0, 16);
    if (x0 == c0 && l_first < 0.f) none = true;                                    // kNoPart (then all parts are)
    float m_new = ml.x;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) m_new = fmaxf(m_new, __shfl_xor_sync(0xffffffffu, m_new, d));
    m_new = fmaxf(mg, m_new);
    const float m_eff = m_new == -INFINITY ? 0.f : m_new;                          // nothing visible so far: weights 0
    const float old = exp2f(mg - m_eff), f = exp2f(ml.x - m_eff);
    float l = ml.x == -INFINITY ? 0.f : ml.y * f;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    ls = ls * old + l;
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] *= old;
    mg = m_new;
    for (int i0 = 0; i0 < n; i0 += kAhead) {
      float4 y[kAhead][kPer / 4];
      float w[kAhead];
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        w[e] = __shfl_sync(0xffffffffu, f, (i0 + e) & 15, 16);
        // (a part in which the row saw nothing holds no sums)
        const float m_part = __shfl_sync(0xffffffffu, ml.x, (i0 + e) & 15, 16);
        const bool live = !none && i0 + e < n && m_part != -INFINITY;
        const float4* from = reinterpret_cast<const float4*>(p.part_o + slot(live ? x0 + i0 + e : c0) * D + kPer * lane);
#pragma unroll
        for (int c = 0; c < kPer / 4; ++c) y[e][c] = live ? from[c] : make_float4(0.f, 0.f, 0.f, 0.f);
        if (!live) w[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < kAhead; ++e)
#pragma unroll
        for (int c = 0; c < kPer / 4; ++c) {
          o[4 * c] = fmaf(y[e][c].x, w[e], o[4 * c]); o[4 * c + 1] = fmaf(y[e][c].y, w[e], o[4 * c + 1]);
          o[4 * c + 2] = fmaf(y[e][c].z, w[e], o[4 * c + 2]); o[4 * c + 3] = fmaf(y[e][c].w, w[e], o[4 * c + 3]);
        }
    }
  }
  if (none) return;
  uint32_t item = (uint32_t)cut.x / (uint32_t)p.row_blocks;
  const int h = item % (uint32_t)p.Hkv;
  item /= (uint32_t)p.Hkv;
  const int b = item % (uint32_t)p.B, l = p.layer_begin + (int)(item / (uint32_t)p.B);
  const float inv = 1.f / ls;
  const int64_t to = ((((int64_t)l * p.B + b) * p.Hq + (int64_t)h * p.g) * p.N + r) * D + kPer * lane;
#pragma unroll
  for (int c = 0; c < kPer; c += 4) tree_store_out4(p, to + c, make_float4(o[c] * inv, o[c + 1] * inv, o[c + 2] * inv, o[c + 3] * inv));
}

template <int D, int MT> cudaError_t opt_in() {
  return cudaFuncSetAttribute(tree_umma_kernel<D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, MT>::kSmem);
}
template <int D, int MT> cudaError_t launch(const Maps& maps, const TreeAttnParams& p, cudaStream_t stream) {
  using C = Cfg<D, MT>;
  return launch_pdl_cluster(tree_umma_kernel<D, MT>, dim3(p.grid), dim3(C::kThreads), (unsigned)p.cluster, C::kSmem, stream, maps, p);
}
template <int D> cudaError_t launch_d(const Maps& maps, const TreeAttnParams& p, cudaStream_t stream) {
  return p.tiles_m == 1 ? launch<D, 1>(maps, p, stream) : launch<D, 2>(maps, p, stream);
}
template <int D> cudaError_t opt_in_d() {
  const cudaError_t e = opt_in<D, 1>();
  return e == cudaSuccess ? opt_in<D, 2>() : e;
}

}  // namespace

int launch_tree_umma(const TreeAttnParams& p, cudaStream_t stream) {
  const int planes = p.L * p.Hkv;
  const int64_t strips = (int64_t)p.L * p.B * p.Hkv, q_rows = (int64_t)p.L * p.B * p.Hq * p.N;
  if (p.rows > 0x7fffffffLL || strips > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;      // TMA coordinates are 32-bit
  Maps maps;
  bool ok = make_rows_map(&maps.q, p.q, q_rows, 128, p.d);
  auto kv_maps = [&](KvMaps* m, const void* cache, const void* tree) {
    ok = ok && make_kv_map(&m->tree, tree, p.N, (int)strips, 16, p.d);
    if (p.rows == 0) m->cache = m->tree;         // a cache without rows: never read
    else ok = ok && (p.page_table ? make_kv_map(&m->cache, cache, p.rows, planes, p.page, p.d)
                                  : make_strip_map(&m->cache, cache, p.rows, planes, tree_umma_keys(p.tiles_m), p.d));
  };
  kv_maps(&maps.k, p.k, p.tree_k);
  kv_maps(&maps.v, p.v, p.tree_v);
  if (!ok) return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce attr_once;
  const int rc = attr_once.run([] {
    cudaError_t e = opt_in_d<64>();
    return e == cudaSuccess ? opt_in_d<128>() : e;
  });
  if (rc != NGC_OK) return rc;
  NGC_CUDA_TRY(p.d == 64 ? launch_d<64>(maps, p, stream) : launch_d<128>(maps, p, stream));
  if (p.cut) {
    const dim3 grid((unsigned)p.grid, (unsigned)((p.block_rows + kJoinRows - 1) / kJoinRows)), block(16 * kJoinRows);
    NGC_CUDA_TRY(p.d == 64 ? launch_pdl(tree_join_kernel<64>, grid, block, 0, stream, p)
                           : launch_pdl(tree_join_kernel<128>, grid, block, 0, stream, p));
  }
  return NGC_OK;
}

}  // namespace ngc
