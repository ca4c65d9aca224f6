// ngc_tree_attn on the 5th-generation tensor cores (bf16 caches).
//
// A work item is up to MT x 128 query rows of one KV head (rows = node of a head, heads of the group one
// after the other) over a range of key tiles; the 128 rows of an M tile are the 128 lanes of tensor memory.
// Key tiles of 64: the cache rows, then the nodes of the tree.  K and V come by tiled TMA, 128-byte swizzled,
// each in a ring of its own (K is free as soon as S is computed, V only after the P V product).
//
//   producer thread      Q once, then K and V of every tile: whole tiles or pages, the partly filled last
//                        tile of the cache and the tree tiles in 16-row boxes;
//   MMA threads (MT)     S = Q K^T (M = 128, N = 64) into a double-buffered S in tensor memory, O += P V with P
//                        read from tensor memory; S of the next tile is issued before P V of the current one;
//   softmax warps (4 MT) one thread per row: mask (only in tree tiles, a bit of the node's ancestor set, and in
//                        the cache's last tile), online softmax in the log2 domain, P as bf16 over the S it came
//                        from.  The maximum used only moves when the true one has grown by more than a factor
//                        2^8, so O in tensor memory is rarely rescaled.
//
// bf16 P: one rounding per weight (2^-8), as in the decode and replay calls; the row sum takes the weights
// before it.  0 x V must be 0 whatever a dead V row holds: rows of the last 16-row box beyond the live ones are
// zeroed in shared memory before the product, and a tree tile's V rows are searched for infinities and NaN,
// which are taken out of the product and added to exactly the rows that see their node.
//
// Every wait is bounded; a wait that runs out raises the CTA's abort flag, all roles leave, copies and MMAs
// in flight are drained (bounded), tensor memory is freed and NGC_DEV_TIMEOUT is reported.
#include <cuda.h>
#include <cuda_bf16.h>

#include "kv_map.cuh"
#include "tree_attn.cuh"
#include "umma.cuh"

namespace ngc {
namespace {

constexpr int kKeys = 64;                       // keys per tile
constexpr int kBox = kKeys * 128;               // 64 keys x 64 channels
constexpr float kLazyRescale = 8.f;             // log2 units the row maximum may grow before O is rescaled

template <int D, int MT> struct Cfg {
  static constexpr int kStages = MT == 1 ? 2 : 4;          // of K and of V; one M tile: two CTAs share an SM
  static constexpr int kCtas = MT == 1 ? 2 : 1;
  static constexpr int kThreads = (4 * MT + MT + 1) * 32;
  static constexpr int kMmaWarp = 4 * MT, kProducerWarp = 5 * MT;
  static constexpr int kTile = kKeys * D * 2;              // K or V tile
  static constexpr int kQBytes = 128 * D * 2;              // Q of an M tile
  static constexpr int kSmem = MT * kQBytes + 2 * kStages * kTile + 1024;
  static constexpr uint32_t kOCol = 128 * MT;              // S[m][buf] at (2 m + buf) * 64, O[m] behind
  static constexpr uint32_t kCols = MT == 1 ? 256 : 512;
};

// Tensor maps of a launch: K and V by tiles (64 rows, or one page) and by 16 rows; the tree's K and V (16 rows, a plane
// per strip); Q (128 rows).
struct Maps { CUtensorMap k, v, k16, v16, tk, tv, q; };

template <int MT, int ST> struct Shared {
  uint64_t k_full[ST], k_empty[ST], v_full[ST], v_empty[ST], s_full[MT][2], p_full[MT][2], o_done[MT][2];
  uint64_t q_full, fixed[3], drain[MT];
  uint32_t anc[kTreeMaxNodes][kTreeWords];
  int jump[kTreeMaxNodes];
  uint32_t odd[kTreeWords];                     // nodes whose V row holds an infinity or a NaN
  uint32_t tmem;
  int abort;
};

template <int D>
__device__ __forceinline__ void load_box(uint8_t* dst, const CUtensorMap* map, int y, int z, uint64_t* bar) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) ptx::tma_load_3d(dst + c * kBox, map, 64 * c, y, z, bar);
}

// Issues the loads of K (or V) tile t into dst.
template <int D>
__device__ __forceinline__ void load_tile(const TreeAttnParams& p, const CUtensorMap* whole, const CUtensorMap* part, const CUtensorMap* tree,
                                          const int32_t* table, int t, int n_ct, int len, int n, int row0, int plane, int strip,
                                          uint8_t* dst, uint64_t* bar) {
  const int live = t < n_ct ? len - t * kKeys : n - (t - n_ct) * kKeys;      // may exceed a tile
  if (t >= n_ct || live < kKeys) {
    const int boxes = min(4, (live + 15) >> 4);
    ptx::mbar_expect_tx(bar, (uint32_t)boxes * 16 * D * 2);
    for (int r = 0; r < boxes; ++r) {
      if (t >= n_ct) {
        load_box<D>(dst + r * 2048, tree, (t - n_ct) * kKeys + 16 * r, strip, bar);
        continue;
      }
      const int at = t * kKeys + 16 * r;
      int y = row0 + at;
      if (table) {
        int pg = table[at / p.page];
        if (pg < 0 || pg >= p.pages_cap) { set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE); pg = 0; }
        y = row0 + pg * p.page + at % p.page;
      }
      if (!NGC_IN_BOUNDS(p.dev_status, y >= 0 && y < p.rows)) y = 0;
      load_box<D>(dst + r * 2048, part, y, plane, bar);
    }
    return;
  }
  ptx::mbar_expect_tx(bar, (uint32_t)kKeys * D * 2);
  const int n_sub = table ? kKeys / p.page : 1;
  for (int u = 0; u < n_sub; ++u) {
    int y = row0 + t * kKeys;
    if (table) {
      int pg = table[t * n_sub + u];
      if (pg < 0 || pg >= p.pages_cap) { set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE); pg = 0; }
      y = row0 + pg * p.page;
    }
    if (!NGC_IN_BOUNDS(p.dev_status, y >= 0 && y + kKeys / n_sub <= p.rows)) y = 0;
    load_box<D>(dst + u * (kBox / n_sub), whole, y, plane, bar);
  }
}

__device__ __forceinline__ uint32_t odd_half(uint32_t x) { return (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u; }
// Bits of x (two bf16) that belong to infinities or NaN.
__device__ __forceinline__ uint32_t odd_bits(uint32_t x) { return odd_half(x) | odd_half(x >> 16) << 16; }

template <int D, int MT>
__global__ void __launch_bounds__(Cfg<D, MT>::kThreads, Cfg<D, MT>::kCtas)
tree_umma_kernel(const __grid_constant__ Maps maps, TreeAttnParams p) {
  using C = Cfg<D, MT>;
  constexpr int ST = C::kStages, NT = C::kThreads;
  extern __shared__ uint8_t smem_dyn[];
  __shared__ Shared<MT, ST> sh;
  uint8_t* sQ = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);     // [MT][128 rows]
  uint8_t* sK = sQ + MT * C::kQBytes;                                            // [ST]
  uint8_t* sV = sK + ST * C::kTile;                                              // [ST]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  int item = blockIdx.x;
  const int split = item % p.n_split; item /= p.n_split;
  const int rb = item % p.row_blocks; item /= p.row_blocks;
  const int h = item % p.Hkv; item /= p.Hkv;
  const int b = item % p.B;
  const int lr = item / p.B, l = p.layer_begin + lr;
  const int rows = p.g * p.N, r0 = rb * MT * 128;
  const int live_warps = min(4 * MT, (rows - r0 + 31) >> 5);     // softmax warps that have a row
  const int tiles_m = (live_warps + 3) >> 2;                     // M tiles that have one

  if (tid == 0) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      ptx::mbar_init(&sh.k_full[s], 1); ptx::mbar_init(&sh.v_full[s], 1);
      ptx::mbar_init(&sh.k_empty[s], tiles_m); ptx::mbar_init(&sh.v_empty[s], tiles_m);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ptx::mbar_init(&sh.s_full[m][i], 1);
        ptx::mbar_init(&sh.p_full[m][i], max(1, 32 * min(4, live_warps - 4 * m)));
        ptx::mbar_init(&sh.o_done[m][i], 1);
      }
      ptx::mbar_init(&sh.drain[m], 1);
    }
    ptx::mbar_init(&sh.q_full, 1);
#pragma unroll
    for (int i = 0; i < 3; ++i) ptx::mbar_init(&sh.fixed[i], 32 * min(4, live_warps));
    ptx::fence_barrier_init();
    sh.abort = 0;
    ptx::prefetch_tensormap(&maps.k);
    ptx::prefetch_tensormap(&maps.v);
    ptx::prefetch_tensormap(&maps.q);
  }
  if (tid < kTreeWords) sh.odd[tid] = 0;
  if (warp == C::kMmaWarp) umma::tmem_alloc(&sh.tmem, C::kCols);
  ptx::grid_dep_wait();
  umma::fence_before_sync();
  const int n = p.n_nodes ? p.n_nodes[b] : p.N;
  const int len = p.lens[len_index(p.lens_lists, p.L, p.Hkv, b, l, h)];
  const bool tree_ok = tree_masks<NT>(p.parent + (int64_t)b * p.N, n, p.N, sh.anc, sh.jump);   // (a barrier of the whole CTA inside)
  umma::fence_after_sync();
  ptx::grid_dep_launch();                       // from here on this CTA holds its tensor memory
  const uint32_t tmem = sh.tmem;
  const int64_t row0 = (((int64_t)l * p.B + b) * p.Hq + (int64_t)h * p.g) * p.N;       // first query row of the KV head
  const int64_t part0 = (((int64_t)lr * p.B + b) * p.Hq + (int64_t)h * p.g) * p.N;

  const bool ok_item = tree_ok && len >= 0 && len <= tree_capacity(p, b);
  const int n_ct = ok_item ? (len + kKeys - 1) / kKeys : 0, n_tt = ok_item ? (n + kKeys - 1) / kKeys : 0;
  const int nt = n_ct + n_tt, tps = (nt + p.n_split - 1) / p.n_split;
  const int tile_lo = min(nt, split * tps), n_tiles = min(nt, tile_lo + tps) - tile_lo;
  if (!ok_item && tid == 0) set_dev_status(p.dev_status, tree_ok ? NGC_DEV_BAD_COUNTS : NGC_DEV_BAD_TREE);

  if (n_tiles == 0) {
    // a refused sequence, an empty tree, or a split that got no tile
    if (p.n_split > 1)
      for (int r = r0 + tid; r < min(rows, r0 + MT * 128); r += NT)
        p.part_ml[(part0 + r) * p.n_split + split] = ok_item && r % p.N < n ? make_float2(-INFINITY, 0.f) : kNoPart;
  } else if (warp == C::kProducerWarp) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      const int32_t* table = p.page_table ? p.page_table + ((int64_t)b * p.G + list_of(p.lists, l, h, p.Hkv)) * p.pages_cap : nullptr;
      const int base = (int)(p.page_table ? (int64_t)b * p.pages_cap * p.page : p.seq_off[b]);
      const int plane = l * p.Hkv + h, strip = (l * p.B + b) * p.Hkv + h;
      ptx::mbar_expect_tx(&sh.q_full, (uint32_t)(tiles_m * C::kQBytes));
      // rows beyond the KV head's belong to the next head (zeros past the end): they only feed rows that are never written
      for (int m = 0; m < tiles_m; ++m)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
          ptx::tma_load_2d(sQ + m * C::kQBytes + c * (128 * 128), &maps.q, 64 * c, (int)(row0 + r0 + 128 * m), &sh.q_full);
      int issued = 0;
      for (; issued < n_tiles; ++issued) {
        const int s = issued % ST, t = tile_lo + issued;
        const uint32_t ph = ((issued / ST) - 1) & 1;
        if (issued >= ST && !umma::wait_or_abort(&sh.k_empty[s], ph, &sh.abort, p.dev_status)) break;
        load_tile<D>(p, &maps.k, &maps.k16, &maps.tk, table, t, n_ct, len, n, base, plane, strip, sK + s * C::kTile, &sh.k_full[s]);
        if (issued >= ST && !umma::wait_or_abort(&sh.v_empty[s], ph, &sh.abort, p.dev_status)) {
          ptx::mbar_wait_bounded(&sh.k_full[s], (issued / ST) & 1);
          break;
        }
        load_tile<D>(p, &maps.v, &maps.v16, &maps.tv, table, t, n_ct, len, n, base, plane, strip, sV + s * C::kTile, &sh.v_full[s]);
      }
      // no copy is in flight when the CTA ends
      ptx::mbar_wait_bounded(&sh.q_full, 0);
      for (int i = max(0, issued - ST); i < issued; ++i) {
        ptx::mbar_wait_bounded(&sh.k_full[i % ST], (i / ST) & 1);
        ptx::mbar_wait_bounded(&sh.v_full[i % ST], (i / ST) & 1);
      }
    }
    __syncwarp();
  } else if (warp >= C::kMmaWarp) {
    // ------------------------------------------------------------------ MMA issue: one thread per M tile
    const int m = warp - C::kMmaWarp;
    if (lane == 0 && m < tiles_m) {
      constexpr uint32_t idesc_s = umma::instr_desc(128, kKeys, false);
      constexpr uint32_t idesc_o = umma::instr_desc(128, D, true);
      // operand descriptors differ only in their low word (start address / 16)
      const uint64_t desc_hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
      const uint32_t q_lo = ((ptx::smem_u32(sQ) + m * C::kQBytes) >> 4) | (1u << 16);
      const uint32_t v_lbo = (uint32_t)(kBox >> 4) << 16;                        // V: the next 64 channels are one box on
      const uint32_t o_tmem = tmem + C::kOCol + (uint32_t)(D * m);
      auto issue_s = [&](int i) {
        const int s = i % ST;
        const uint32_t k_lo = ((ptx::smem_u32(sK) + s * C::kTile) >> 4) | (1u << 16);
        const uint32_t d = tmem + (uint32_t)((2 * m + (i & 1)) * kKeys);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint64_t a = desc_hi | (uint64_t)(q_lo + (uint32_t)(((ks >> 2) * (128 * 128) + (ks & 3) * 32) >> 4));
          const uint64_t bd = desc_hi | (uint64_t)(k_lo + (uint32_t)(((ks >> 2) * kBox + (ks & 3) * 32) >> 4));
          umma::mma_bf16(d, a, bd, idesc_s, ks > 0);
        }
        umma::commit(&sh.s_full[m][i & 1]);
        umma::commit(&sh.k_empty[s]);
      };
      bool ok = umma::wait_or_abort(&sh.q_full, 0, &sh.abort, p.dev_status) &&
                umma::wait_or_abort(&sh.k_full[0], 0, &sh.abort, p.dev_status);
      if (ok) issue_s(0);
      for (int i = 0; ok && i < n_tiles; ++i) {
        const int s = i % ST, t = tile_lo + i;
        if (i + 1 < n_tiles) {
          // its S buffer held S and P of two tiles ago: that P V product was issued before, and they run in issue order
          ok = umma::wait_or_abort(&sh.k_full[(i + 1) % ST], ((i + 1) / ST) & 1, &sh.abort, p.dev_status);
          if (!ok) break;
          issue_s(i + 1);
        }
        ok = umma::wait_or_abort(&sh.v_full[s], (i / ST) & 1, &sh.abort, p.dev_status) &&
             umma::wait_or_abort(&sh.p_full[m][i & 1], (i >> 1) & 1, &sh.abort, p.dev_status);
        if (!ok) break;
        umma::fence_after_sync();                         // P was written with tcgen05.st by the softmax threads
        const int live = t < n_ct ? len - t * kKeys : n - (t - n_ct) * kKeys;
        const int steps = min(4, (live + 15) >> 4);       // 16 keys each; V rows beyond were not loaded
        const uint32_t v_lo = ((ptx::smem_u32(sV) + s * C::kTile) >> 4) | v_lbo;
        const uint32_t p_tmem = tmem + (uint32_t)((2 * m + (i & 1)) * kKeys);
        for (int kk = 0; kk < steps; ++kk)
          umma::mma_bf16_a_tmem(o_tmem, p_tmem + 8 * kk, desc_hi | (uint64_t)(v_lo + (uint32_t)((kk * 2048) >> 4)), idesc_o,
                                (i > 0 || kk > 0) ? 1u : 0u);
        umma::commit(&sh.o_done[m][i & 1]);
        umma::commit(&sh.v_empty[s]);
      }
      // everything issued has completed before tensor memory is released
      umma::commit(&sh.drain[m]);
      ptx::mbar_wait_bounded(&sh.drain[m], 0);
    }
    __syncwarp();
  } else if (warp < live_warps) {
    // ------------------------------------------------------------------ softmax: one thread per query row
    const int m = warp >> 2;
    const int r = r0 + 128 * m + 32 * (warp & 3) + lane;
    const int node = r % p.N;
    const bool live_row = r < rows && node < n;
    uint32_t aw[kTreeWords];
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) aw[w] = live_row ? sh.anc[node][w] : 0u;
    const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t o_addr = tmem + lane_base + C::kOCol + (uint32_t)(D * m);
    float m_use = -INFINITY, l_run = 0.f;
    bool ok = true;
    for (int i = 0; i < n_tiles; ++i) {
      const int t = tile_lo + i;
      const bool in_tree = t >= n_ct;
      const int live = in_tree ? n - (t - n_ct) * kKeys : len - t * kKeys;
      if (in_tree || live < kKeys) {
        // V rows that must not meet a zero weight: by the warps of the first M tile, the others wait for them
        uint64_t* fixed = &sh.fixed[in_tree ? 1 + t - n_ct : 0];
        if (m == 0) {
          const int s = i % ST;
          if (!umma::warp_wait(&sh.v_full[s], (i / ST) & 1, &sh.abort, p.dev_status)) { ok = false; break; }
          const int n_rows = min(kKeys, ((live + 15) >> 4) << 4), step = 32 * min(4, live_warps);
          for (int e = tid; e < n_rows * (D / 8); e += step) {
            const int rr = e / (D / 8), c = e % (D / 8);               // (the swizzle permutes pieces within a row only)
            uint4* at = reinterpret_cast<uint4*>(sV + s * C::kTile + (c >> 3) * kBox + rr * 128 + (c & 7) * 16);
            if (rr >= live) {
              *at = make_uint4(0, 0, 0, 0);
            } else if (in_tree) {
              const uint4 x = *at;
              const uint4 o = make_uint4(odd_bits(x.x), odd_bits(x.y), odd_bits(x.z), odd_bits(x.w));
              if (o.x | o.y | o.z | o.w) {
                *at = make_uint4(x.x & ~o.x, x.y & ~o.y, x.z & ~o.z, x.w & ~o.w);
                const int j = (t - n_ct) * kKeys + rr;
                atomicOr(&sh.odd[j >> 5], 1u << (j & 31));
              }
            }
          }
          ptx::fence_proxy_async();
          ptx::mbar_arrive(fixed);
        } else if (!umma::warp_wait(fixed, 0, &sh.abort, p.dev_status)) {
          ok = false;
          break;
        }
      }
      if (!umma::warp_wait(&sh.s_full[m][i & 1], (i >> 1) & 1, &sh.abort, p.dev_status)) { ok = false; break; }
      umma::fence_after_sync();
      uint32_t zr[2][32];
      const uint32_t s_addr = tmem + lane_base + (uint32_t)((2 * m + (i & 1)) * kKeys);
      umma::tmem_ld32(s_addr, zr[0]);
      umma::tmem_ld32(s_addr + 32, zr[1]);
      umma::tmem_ld_wait();
      if (in_tree || live < kKeys) {
        uint32_t see[2];
        if (in_tree) {
          see[0] = t == n_ct ? aw[0] : aw[2];
          see[1] = t == n_ct ? aw[1] : aw[3];
        } else {
          see[0] = live >= 32 ? 0xffffffffu : (1u << live) - 1u;
          see[1] = live > 32 ? (1u << (live - 32)) - 1u : 0u;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (!(see[half] >> j & 1u)) zr[half][j] = 0xff800000u;       // -inf
      }
      float mxc[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            mxc[c] = umma::max3(mxc[c], __uint_as_float(zr[half][j + 2 * c]), __uint_as_float(zr[half][j + 2 * c + 1]));
        }
      const float mx = fmaxf(fmaxf(mxc[0], mxc[1]), fmaxf(mxc[2], mxc[3])) * p.scale_log2;
      const bool grow = mx > m_use + kLazyRescale;                        // also the first visible key (m_use = -inf)
      const bool rescale = grow && m_use != -INFINITY && i > 0;           // O already holds something for this row
      if (__any_sync(0xffffffffu, rescale)) {
        if (!umma::warp_wait(&sh.o_done[m][(i - 1) & 1], ((i - 1) >> 1) & 1, &sh.abort, p.dev_status)) { ok = false; break; }
        umma::fence_after_sync();
        const float alpha = rescale ? ptx::ex2_approx(m_use - mx) : 1.f;
        l_run *= alpha;
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          uint32_t o[32];
          umma::tmem_ld32(o_addr + c0, o);
          umma::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
          umma::tmem_st32(o_addr + c0, o);
        }
        umma::tmem_st_wait();
      }
      if (grow) m_use = mx;
      const float m_eff = m_use == -INFINITY ? 0.f : m_use;               // nothing visible yet: every exponential is 0
      const uint64_t sc2 = umma::pack2(p.scale_log2, p.scale_log2), nm2 = umma::pack2(-m_eff, -m_eff);
      uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
      uint32_t pk[32];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          float x0, x1;
          umma::unpack2(umma::fma2(umma::pack2(__uint_as_float(zr[half][j]), __uint_as_float(zr[half][j + 1])), sc2, nm2), x0, x1);
          const float p0 = ptx::ex2_approx(x0), p1 = ptx::ex2_approx(x1);
          acc2[(j >> 1) & 3] = umma::add2(acc2[(j >> 1) & 3], umma::pack2(p0, p1));
          pk[16 * half + (j >> 1)] = ptx::pack_bf16x2(p0, p1);
        }
      {
        float s0, s1;
        umma::unpack2(umma::add2(umma::add2(acc2[0], acc2[1]), umma::add2(acc2[2], acc2[3])), s0, s1);
        l_run += s0 + s1;
      }
      umma::tmem_st32(s_addr, pk);                                        // P over the first 32 columns of its S
      umma::tmem_st_wait();
      umma::fence_before_sync();
      ptx::mbar_arrive(&sh.p_full[m][i & 1]);
    }
    if (ok) ok = umma::warp_wait(&sh.o_done[m][(n_tiles - 1) & 1], ((n_tiles - 1) >> 1) & 1, &sh.abort, p.dev_status);
    uint32_t odd[kTreeWords] = {0u, 0u, 0u, 0u};
    for (int t = max(tile_lo, n_ct); ok && t < tile_lo + n_tiles; ++t)
      ok = umma::warp_wait(&sh.fixed[1 + t - n_ct], 0, &sh.abort, p.dev_status);
    if (ok && tile_lo + n_tiles > n_ct) {
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) odd[w] = sh.odd[w] & aw[w];
    }
    if (ok) {
      umma::fence_after_sync();
      const float inv = l_run == 0.f ? 0.f : 1.f / l_run;                 // a NaN stays one
      const int64_t pit = (part0 + r) * p.n_split + split;
      if (p.n_split > 1 && r < rows) p.part_ml[pit] = live_row ? make_float2(m_use, l_run) : kNoPart;
      const __nv_bfloat16* tv = (const __nv_bfloat16*)p.tree_v + (((int64_t)l * p.B + b) * p.Hkv + h) * p.N * D;
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        __syncwarp();
        umma::tmem_ld32(o_addr + c0, o);
        umma::tmem_ld_wait();
        if (odd[0] | odd[1] | odd[2] | odd[3]) {
          for (int j = 0; j < n; ++j) {
            if (!(odd[j >> 5] >> (j & 31) & 1u)) continue;
#pragma unroll
            for (int c = 0; c < 32; ++c) {
              const float v = __bfloat162float(tv[(int64_t)j * D + c0 + c]);
              if (!isfinite(v)) o[c] = __float_as_uint(__uint_as_float(o[c]) + v);
            }
          }
        }
        if (!live_row) {
          // nothing to write
        } else if (p.n_split > 1) {
#pragma unroll
          for (int c = 0; c < 32; c += 4)
            *reinterpret_cast<uint4*>(p.part_o + pit * D + c0 + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
        } else if (p.out_bf16) {
#pragma unroll
          for (int c = 0; c < 32; c += 8)
            *reinterpret_cast<uint4*>((__nv_bfloat16*)p.out + (row0 + r) * D + c0 + c) =
                make_uint4(ptx::pack_bf16x2(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv),
                           ptx::pack_bf16x2(__uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv),
                           ptx::pack_bf16x2(__uint_as_float(o[c + 4]) * inv, __uint_as_float(o[c + 5]) * inv),
                           ptx::pack_bf16x2(__uint_as_float(o[c + 6]) * inv, __uint_as_float(o[c + 7]) * inv));
        } else {
#pragma unroll
          for (int c = 0; c < 32; c += 4)
            *reinterpret_cast<float4*>((float*)p.out + (row0 + r) * D + c0 + c) =
                make_float4(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv,
                            __uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
        }
      }
    }
  }
  // ---- teardown: every role has left its loops; nothing of this CTA is in flight any more
  umma::fence_before_sync();
  __syncthreads();
  if (warp == C::kMmaWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, C::kCols);
  }
}

template <int D, int MT> cudaError_t opt_in() {
  return cudaFuncSetAttribute(tree_umma_kernel<D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, MT>::kSmem);
}
template <int D, int MT> cudaError_t launch(const Maps& maps, const TreeAttnParams& p, unsigned grid, cudaStream_t stream) {
  return launch_pdl(tree_umma_kernel<D, MT>, dim3(grid), dim3(Cfg<D, MT>::kThreads), Cfg<D, MT>::kSmem, stream, maps, p);
}

}  // namespace

int launch_tree_umma(const TreeAttnParams& p, unsigned grid, cudaStream_t stream) {
  const int planes = p.L * p.Hkv;
  const int64_t strips = (int64_t)p.L * p.B * p.Hkv, q_rows = (int64_t)p.L * p.B * p.Hq * p.N;
  if (p.rows > 0x7fffffffLL || strips > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;      // TMA coordinates are 32-bit
  Maps maps;
  bool ok = make_kv_map(&maps.tk, p.tree_k, p.N, (int)strips, 16, p.d) && make_kv_map(&maps.tv, p.tree_v, p.N, (int)strips, 16, p.d) &&
            make_rows_map(&maps.q, p.q, q_rows, 128, p.d);
  if (ok && p.rows > 0) {
    const int box = p.page_table ? p.page : kKeys;
    ok = make_kv_map(&maps.k, p.k, p.rows, planes, box, p.d) && make_kv_map(&maps.v, p.v, p.rows, planes, box, p.d) &&
         make_kv_map(&maps.k16, p.k, p.rows, planes, 16, p.d) && make_kv_map(&maps.v16, p.v, p.rows, planes, 16, p.d);
  } else {
    maps.k = maps.k16 = maps.tk;                 // a cache without rows: never read
    maps.v = maps.v16 = maps.tv;
  }
  if (!ok) return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce attr_once;
  const int rc = attr_once.run([] {
    cudaError_t e = opt_in<64, 1>();
    if (e == cudaSuccess) e = opt_in<64, 2>();
    if (e == cudaSuccess) e = opt_in<128, 1>();
    if (e == cudaSuccess) e = opt_in<128, 2>();
    return e;
  });
  if (rc != NGC_OK) return rc;
  const bool one = tree_umma_tiles(p.g * p.N) == 1;
  if (p.d == 64) NGC_CUDA_TRY(one ? (launch<64, 1>(maps, p, grid, stream)) : (launch<64, 2>(maps, p, grid, stream)));
  else NGC_CUDA_TRY(one ? (launch<128, 1>(maps, p, grid, stream)) : (launch<128, 2>(maps, p, grid, stream)));
  return NGC_OK;
}

}  // namespace ngc
