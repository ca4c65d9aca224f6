// ngc_latent_decode: absorbed latent attention of one token per sequence over a pool of pages, on the 5th-generation
// tensor cores.
//
// All heads share the rows (c_j | r_j), so both products are tall: with X the rows of a tile of 64 tokens and Q the heads'
// queries, scores are S^T = X Q^T and the sums O^T += C^T P^T, C the latent part of the same rows.  Tokens, then latent
// channels are the M dimension of the tensor core (64 and 128 rows per product), the heads its N (16, 32 or 64 per CTA):
// few heads cost few columns, where heads as M would cost 128 rows for 16 heads.  One copy of a tile in shared memory serves
// as K-major A operand of the first product and as MN-major A operand of the second.  Every row is read from HBM once, which
// bounds the call up to some 100 heads; the products of 128 heads take as long (36 + 16 steps per tile and 64 heads).
//
// Work is dealt out by tiles: the tiles of all (layer, sequence) units in one line, cut into equal pieces, one per CTA (per
// group of heads).  A unit that lies in several pieces leaves unnormalised sums, maxima and weights per piece in the
// workspace, and a second kernel joins them.  Roles of a CTA, which meet at mbarriers only:
//   producers (2 warps)   the tile's rows by TMA, a box of 64 channels per page, into a ring of stages; a warp per page of a tile
//   mender (1 warp)       rows behind a unit's last token: zeros (they may hold anything; a NaN times a zero weight is NaN)
//   queries (1 thread)    the heads' queries of the next unit, when the last unit's scores are done
//   scores (1 thread)     S^T of the next tile, pair of 128 channels by pair as they come; it runs under the softmax of this one
//   sums (1 thread)       O^T; a pair of channels whose products are done makes room for the next tile but one's
//   softmax (4 or 8 warps) 16 tokens each.  A thread holds two tokens of four heads; weights go to shared memory
//                         by transposing matrix stores, as the K-major B operand.  The maximum that the exponentials refer to
//                         moves only when a score exceeds it by 2^8 (exact in bf16 and fp32), which is one vote per tile.
// Every wait is bounded; one that runs out makes all roles leave and is reported.
//
// 64 sequences of 1024 to 4096 tokens, 16 heads of 512 + 64 channels, one layer: 49 us with the second kernel, 3.9 TB/s; beginning,
// first tile and joining are most of the 13 us that a call of one sequence takes.  24 sequences of 2048 to 8192, 128 heads, two
// layers: 123 us, 555 TFLOP/s: the queries of 64 heads leave shared memory room for two tiles.  A tile holds its place for some 5500 cycles:
// 1700 until its first rows are there, 1400 until the last, 1850 of softmax and its hand-overs, 800 of sums; with every row in L2 the
// call takes 108 us.
#include <cuda.h>
#include <cuda_bf16.h>

#include "kv_map.cuh"
#include "latent_pool.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace ngc {
namespace {

constexpr int kTile = 64;                      // tokens per tile
constexpr int kBox = kTile * 128;              // 64 tokens x 64 channels
constexpr int kPair = 2 * kBox;                // 128 channels of the latent part: what arrives, is used and makes room together
constexpr int kMaxPairs = 9, kMaxStages = 4;  // in shared memory, at most
// Warps: softmax, four for 16 heads, else eight (a warp reaches a quarter of tensor memory's lanes; 16 for 64 heads: 147 -> 157 us
// for 24 sequences of two layers, 128 heads), then one each for the scores, the first and
// the second page of a tile, the mender, the queries, the sums (scores and sums issued by one thread as they came: 1 to 2 % slower).
__host__ __device__ constexpr int softmax_warps(int nh) { return nh < 32 ? 4 : 8; }
__host__ __device__ constexpr int cta_threads(int nh) { return (softmax_warps(nh) + 6) * 32; }
constexpr int kSmemLimit = 227 * 1024;
constexpr int kStaticReserve = 2048;           // barriers and exchange buffers (static shared memory)
constexpr float kLazy = 8.f;
constexpr int kMaxCtas = 148;                  // one per SM

struct LatentDecodeParams {
  const int32_t* table;
  const int32_t* lens;
  void* out;
  float* part_o;                // [piece][2][H padded to the groups][dc] sums, unnormalised
  float2* part_ml;              // [piece][2][H padded] (maximum in log2 units, sum of weights)
  int2* plan;                   // [piece] the unit that begins in the piece and goes on behind it, the piece it ends in; or -1
  int32_t* dev_status;
  int B, H, G, dc, dr, page, cap, n_pages, lists, layer_begin, n_layers, out_bf16;
  int stages, pieces, groups, heads_pad;
  float scale_log2;
};

struct Maps { CUtensorMap rows, ql, qr; };

template <int NH> struct Shared {
  uint64_t full[kMaxPairs], empty[kMaxPairs], raw[kMaxPairs], r_full[kMaxStages], r_empty[kMaxStages];
  uint64_t s_full[2], s_free[2], p_full, o_done, q_full, q_empty, drain;
  uint32_t tmem;
  int abort;
  int u0, t0, len0, g0, n_tiles, total;        // where this CTA's piece begins, how many tiles it has, tiles of the call
  int warp_sum[cta_threads(NH) / 32];
  float ex[4][NH];                             // per warp: column maxima, later sums of weights
  float m[NH], alpha[NH];                      // the maximum that the exponentials refer to (log2 units), and what its last move costs
};

__device__ __forceinline__ int unit_len(const LatentDecodeParams& p, int u) {
  const int n = p.lens[(int64_t)(u % p.B) * p.G + list_of(p.lists, p.layer_begin + u / p.B, 0, 1)];
  return n < 0 || n > p.cap * p.page ? -1 : n;
}

// The pieces: how many there are (a tile each at least), which tile of the line piece i begins at, and which piece has tile g.
__device__ __forceinline__ int pieces_used(int total, int pieces) { return max(1, min(pieces, total)); }
__device__ __forceinline__ int piece_first(int total, int pieces, int i) { return (int)((int64_t)total * i / pieces); }
__device__ __forceinline__ int piece_of(int total, int pieces, int g) {
  int i = (int)(((int64_t)g * pieces) / total);
  while (i + 1 < pieces && piece_first(total, pieces, i + 1) <= g) ++i;
  while (i > 0 && piece_first(total, pieces, i) > g) --i;
  return i;
}

// Position in a ring: the slot to fill or use next, and the parity of its use.
struct Ring {
  int n, slot, phase;
  bool first;                   // no slot has been used twice
  __device__ __forceinline__ explicit Ring(int slots) : n(slots), slot(0), phase(0), first(true) {}
  __device__ __forceinline__ bool fresh() const { return first; }
  __device__ __forceinline__ void next() { if (++slot == n) { slot = 0; phase ^= 1; first = false; } }
};

// The parts of units that make up a piece, in order.
struct Walk {
  int u, t, left, first;        // next unit, its next tile, tiles left in the piece; length of the piece's first unit
  int unit, t_begin, t_end, n, len;            // the current part: tiles t_begin .. t_end of the n of unit
  template <int NH> __device__ __forceinline__ explicit Walk(const Shared<NH>& sh) : u(sh.u0), t(sh.t0), left(sh.n_tiles), first(sh.len0) {}
  __device__ __forceinline__ bool next(const LatentDecodeParams& p) {
    if (left <= 0) return false;
    do {
      if (u >= p.n_layers * p.B) return false;           // (the lengths changed under the call)
      len = first > 0 ? first : unit_len(p, u);
      first = 0;
      n = len > 0 ? (len + kTile - 1) / kTile : 0;
      unit = u++;
    } while (n == 0);           // (left > 0: a unit with tiles follows)
    t_begin = t;
    t_end = min(n, t + left);
    left -= t_end - t_begin;
    t = 0;
    return true;
  }
};

// 16 lanes x 8 columns per matrix fragment: register 4 j + {0, 1}: row lane / 4, columns 8 j + 2 (lane % 4) + {0, 1}; 4 j + {2, 3}: row + 8.
__device__ __forceinline__ void ld_frags(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr));
}

__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}

// Barrier of the softmax warps; true to all where `mine` is true to one.
template <int N> __device__ __forceinline__ bool softmax_any(bool mine) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(r) : "r"((uint32_t)mine), "n"(N) : "memory");
  return r != 0;
}
template <int N> __device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(N) : "memory"); }

template <int NH, int DC>
__global__ void __launch_bounds__(cta_threads(NH), 1) latent_decode_kernel(const __grid_constant__ Maps maps, LatentDecodeParams p) {
  constexpr int kSoft = softmax_warps(NH), kThreads = cta_threads(NH);
  constexpr int kScoreWarp = kSoft, kProducerWarp = kSoft + 1, kMenderWarp = kSoft + 3, kQueryWarp = kSoft + 4, kSumWarp = kSoft + 5;
  extern __shared__ uint8_t smem_dyn[];
  __shared__ Shared<NH> sh;
  uint8_t* sQ = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);     // [chunks][NH rows x 128 B]
  constexpr int kChunks = DC / 64 + 1, kM = DC / 128;                            // 64-channel chunks of a row (the last: rotary part, then zeros), pairs
  constexpr int kStage = kChunks * kBox;
  uint8_t* sP = sQ + kChunks * NH * 128;                                         // [NH rows x 64 tokens]
  uint8_t* sK = sP + NH * 128;                                                   // [stages][chunks][64 tokens x 128 B]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int piece = blockIdx.x / p.groups, hg = blockIdx.x % p.groups;
  constexpr uint32_t kCols = NH == 64 ? 512 : (NH == 32 ? 256 : 128);            // O^T: 4 x NH, S^T: 2 x NH
  const int U = p.n_layers * p.B;

  if (warp == 0) {
    if (lane < p.stages * kM) { ptx::mbar_init(&sh.full[lane], kTile / p.page); ptx::mbar_init(&sh.empty[lane], 1); ptx::mbar_init(&sh.raw[lane], kTile / p.page); }
    if (lane < p.stages) { ptx::mbar_init(&sh.r_full[lane], kTile / p.page); ptx::mbar_init(&sh.r_empty[lane], 1); }
    if (lane == 31) {
      ptx::mbar_init(&sh.s_full[0], 1); ptx::mbar_init(&sh.s_full[1], 1);
      ptx::mbar_init(&sh.s_free[0], kSoft); ptx::mbar_init(&sh.s_free[1], kSoft);
      ptx::mbar_init(&sh.p_full, kSoft);
      ptx::mbar_init(&sh.o_done, 1);
      ptx::mbar_init(&sh.q_full, 1); ptx::mbar_init(&sh.q_empty, 1); ptx::mbar_init(&sh.drain, 2);
      sh.abort = 0; sh.u0 = 0; sh.t0 = 0; sh.len0 = 0;
    }
    ptx::fence_barrier_init();
  } else if (warp == kProducerWarp && lane == 0) {
    ptx::prefetch_tensormap(&maps.rows); ptx::prefetch_tensormap(&maps.ql); ptx::prefetch_tensormap(&maps.qr);
  }
  if (warp == kScoreWarp) umma::tmem_alloc(&sh.tmem, kCols);
  ptx::grid_dep_wait();
  // ---- the line of tiles, and where this piece begins: every thread sums a run of units
  {
    const int per = (U + kThreads - 1) / kThreads, u_lo = min(tid * per, U), u_hi = min(u_lo + per, U);
    int mine = 0, len = 0;
    for (int u = u_lo; u < u_hi; ++u) {
      len = unit_len(p, u);
      if (len < 0) set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
      mine += (max(len, 0) + kTile - 1) / kTile;
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) sh.warp_sum[warp] = incl;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) { const int v = sh.warp_sum[w]; if (w < warp) before += v; total += v; }
    const int used = pieces_used(total, p.pieces);
    const int g0 = piece < used ? piece_first(total, used, piece) : 0, g1 = piece < used ? piece_first(total, used, piece + 1) : 0;
    int at = before + incl - mine;                       // first tile of this thread's run
    if (g0 < g1 && g0 >= at && g0 < at + mine) {
      for (int u = u_lo; u < u_hi; ++u) {
        if (per > 1) len = unit_len(p, u);
        const int n = (max(len, 0) + kTile - 1) / kTile;
        if (g0 < at + n) { sh.u0 = u; sh.t0 = g0 - at; sh.len0 = len; break; }
        at += n;
      }
    }
    if (tid == 0) {
      sh.n_tiles = g1 - g0; sh.total = total; sh.g0 = g0;
      if (hg == 0) p.plan[piece] = make_int2(-1, -1);
    }
  }
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const int n_tiles = sh.n_tiles;
  const uint32_t s_tmem = tmem + 4 * NH;
  ptx::grid_dep_launch();                                // (all CTAs are resident: the second kernel's can wait beside them)

  if (warp == kProducerWarp || warp == kProducerWarp + 1) {
    // ------------------------------------------------------------------ rows of the tiles: a warp per page of a tile
    const int k = warp - kProducerWarp, per = kTile / p.page;
    if (k < per) {
      uint32_t raw_last = 0, raw_phase = 0;              // bit s: pair s was last filled through raw / parity of raw's next use
      Ring at(p.stages);
      int issued = 0, done = 0;                          // pairs and rotary parts loaded
      bool ok = true;
      Walk w(sh);
      while (ok && w.next(p)) {
        const int l = p.layer_begin + w.unit / p.B, b = w.unit % p.B;
        const int32_t* row = p.table + ((int64_t)b * p.G + list_of(p.lists, l, 0, 1)) * p.cap;
        const int n_pages = (w.len + p.page - 1) / p.page;
        int have = 0, pages = 0;                         // lane j holds the page of tile have - 32 + j
        for (int i = w.t_begin; ok && i < w.t_end; ++i) {
          if (i >= have) {
            const int j = (i + lane) * per + k;
            pages = j < n_pages ? row[j] : 0;
            if ((uint32_t)pages >= (uint32_t)p.n_pages) {
              if (i + lane < w.t_end) set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE);
              pages = 0;
            }
            have = i + 32;
          }
          const int n = min(kTile, w.len - i * kTile);
          const bool tail = n < kTile;                   // the mender hands it on
          const bool mine = k * p.page < n;              // (a short last tile may have no second page)
          int y = (l * p.n_pages + __shfl_sync(0xffffffffu, pages, i - (have - 32))) * p.page;
          if (!NGC_IN_BOUNDS(p.dev_status, y >= 0 && y / p.page < (p.layer_begin + p.n_layers) * p.n_pages)) y = 0;
          const uint32_t bytes = (uint32_t)(p.page * 128);
#pragma unroll
          for (int m = 0; m < kM; ++m) {
            const int slot = at.slot * kM + m;
            ok = ok && (at.fresh() || umma::warp_wait(&sh.empty[slot], at.phase ^ 1, &sh.abort, p.dev_status));
            if (!ok) break;
            if (umma::elect_one()) {
              uint64_t* bar = tail ? &sh.raw[slot] : &sh.full[slot];
              uint8_t* dst = sK + at.slot * kStage + m * kPair + k * (kBox / 2);
              if (mine) {
                ptx::mbar_expect_tx(bar, 2 * bytes);
                ptx::tma_load_2d(dst, &maps.rows, 128 * m, y, bar);
                ptx::tma_load_2d(dst + kBox, &maps.rows, 128 * m + 64, y, bar);
              } else {
                ptx::mbar_arrive(bar);
              }
            }
            __syncwarp();
            raw_last = tail ? raw_last | 1u << slot : raw_last & ~(1u << slot);
            if (tail) raw_phase ^= 1u << slot;
            ++issued;
          }
          ok = ok && (at.fresh() || umma::warp_wait(&sh.r_empty[at.slot], at.phase ^ 1, &sh.abort, p.dev_status));
          if (!ok) break;
          if (umma::elect_one()) {
            if (mine) {
              ptx::mbar_expect_tx(&sh.r_full[at.slot], bytes);
              ptx::tma_load_2d(sK + at.slot * kStage + kM * kPair + k * (kBox / 2), &maps.rows, DC, y, &sh.r_full[at.slot]);
            } else {
              ptx::mbar_arrive(&sh.r_full[at.slot]);
            }
          }
          __syncwarp();
          at.next();
          ++done;
        }
      }
      // nothing is in flight when the CTA ends: the last use of every barrier
      for (int x = max(0, issued - p.stages * kM); x < issued; ++x) {
        const int use = x / (p.stages * kM), slot = x - use * p.stages * kM;
        if (raw_last >> slot & 1) ptx::mbar_wait_bounded(&sh.raw[slot], ((raw_phase >> slot) & 1) ^ 1);
        else ptx::mbar_wait_bounded(&sh.full[slot], use & 1);
      }
      for (int x = max(0, done - p.stages); x < done; ++x) ptx::mbar_wait_bounded(&sh.r_full[x % p.stages], (x / p.stages) & 1);
    }
    __syncwarp();
  } else if (warp == kMenderWarp) {
    // ------------------------------------------------------------------ rows behind the last token
    int t = 0;
    uint32_t raw_phase = 0;
    bool ok = true;
    Walk w(sh);
    while (ok && w.next(p)) {
      t += w.t_end - w.t_begin;
      const int n = w.len - (w.n - 1) * kTile;
      if (w.t_end < w.n || n == kTile) continue;
      for (int m = 0; m < kM && ok; ++m) {
        const int s = (t - 1) % p.stages * kM + m;
        ok = umma::warp_wait(&sh.raw[s], (raw_phase >> s) & 1, &sh.abort, p.dev_status);
        if (!ok) break;
        raw_phase ^= 1u << s;
        uint8_t* dst = sK + (t - 1) % p.stages * kStage + m * kPair;
        for (int c = 0; c < 2; ++c)
          for (int x = n * 8 + lane; x < kTile * 8; x += 32) *reinterpret_cast<uint4*>(dst + c * kBox + x * 16) = make_uint4(0, 0, 0, 0);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane < kTile / p.page) ptx::mbar_arrive(&sh.full[s]);
      }
    }
  } else if (warp == kQueryWarp) {
    // ------------------------------------------------------------------ queries of the units
    int k = 0;
    Walk w(sh);
    for (; w.next(p); ++k) {
      if (k > 0 && !umma::warp_wait(&sh.q_empty, (k - 1) & 1, &sh.abort, p.dev_status)) break;
      const int z = (p.layer_begin + w.unit / p.B) * p.B + w.unit % p.B;
      if (umma::elect_one()) {
        ptx::mbar_expect_tx(&sh.q_full, (uint32_t)(kChunks * NH * 128));
#pragma unroll
        for (int c = 0; c < DC / 64; ++c) ptx::tma_load_3d(sQ + c * NH * 128, &maps.ql, 64 * c, hg * NH, z, &sh.q_full);
        ptx::tma_load_3d(sQ + DC / 64 * NH * 128, &maps.qr, 0, hg * NH, z, &sh.q_full);
      }
      __syncwarp();
    }
    if (k > 0) ptx::mbar_wait_bounded(&sh.q_full, (k - 1) & 1);
    __syncwarp();
  } else if (warp == kScoreWarp) {
    // ------------------------------------------------------------------ scores
    // One elected thread issues them: the compiler keeps descriptors in uniform registers then (with `lane == 0` a product took 90
    // cycles to issue and the CTA 4500 per tile), and nothing is spent on meeting the warp again.
    if (n_tiles > 0 && umma::elect_one()) {
      constexpr uint32_t idesc = umma::instr_desc(64, NH, false);
      const uint64_t hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
      const uint32_t k_lo = (ptx::smem_u32(sK) >> 4) | 1u << 16, q_lo = (ptx::smem_u32(sQ) >> 4) | 1u << 16;
      const int steps_r = p.dr / 16;
      auto wait = [&](uint64_t* bar, uint32_t parity) { return umma::wait_quick(bar, parity, &sh.abort, p.dev_status); };
      Walk w(sh);
      Ring at(p.stages);
      int t = 0, n_q = 0;                                // tiles, units begun
      bool ok = true;
      while (ok && w.next(p)) {
        ok = wait(&sh.q_full, n_q++ & 1);
        for (int i = w.t_begin; ok && i < w.t_end; ++i, ++t) {
          ok = t < 2 || wait(&sh.s_free[t & 1], ((t >> 1) - 1) & 1);
          const uint32_t d = s_tmem + (uint32_t)((t & 1) * NH), a_lo = k_lo + at.slot * (kStage >> 4);
#pragma unroll
          for (int m = 0; m <= kM; ++m) {                // pairs of channels as they come, the rotary part last
            ok = ok && wait(m < kM ? &sh.full[at.slot * kM + m] : &sh.r_full[at.slot], at.phase);
            if (!ok) break;
            umma::fence_after_sync();
#pragma unroll
            for (int k = 0; k < (m < kM ? 8 : 4); ++k)
              if (m < kM || k < steps_r)
                umma::mma_bf16(d, hi | (a_lo + ((m * kPair + (k >> 2) * kBox + (k & 3) * 32) >> 4)),
                               hi | (q_lo + (((2 * m + (k >> 2)) * NH * 128 + (k & 3) * 32) >> 4)), idesc, (m > 0 || k > 0) ? 1u : 0u);
          }
          if (!ok) break;
          umma::commit(&sh.s_full[t & 1]);
          umma::commit(&sh.r_empty[at.slot]);
          if (i + 1 == w.t_end) umma::commit(&sh.q_empty);
          at.next();
        }
      }
      umma::commit(&sh.drain);                           // everything issued has completed before tensor memory is released
      ptx::mbar_wait_bounded(&sh.drain, 0);
    }
    __syncwarp();
  } else if (warp == kSumWarp) {
    // ------------------------------------------------------------------ sums
    if (n_tiles > 0 && umma::elect_one()) {
      constexpr uint32_t idesc = umma::instr_desc(128, NH, false, true);
      const uint64_t hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
      const uint32_t k_lo = (ptx::smem_u32(sK) >> 4) | (uint32_t)(kBox >> 4) << 16, p_lo = (ptx::smem_u32(sP) >> 4) | 1u << 16;
      Walk w(sh);
      Ring at(p.stages);
      int t = 0;
      bool ok = true;
      while (ok && w.next(p))
        for (int i = w.t_begin; ok && i < w.t_end; ++i, ++t) {
          ok = umma::wait_quick(&sh.p_full, t & 1, &sh.abort, p.dev_status);
          if (!ok) break;
          umma::fence_after_sync();
          const uint32_t a_lo = k_lo + at.slot * (kStage >> 4);
          const bool fresh = i == w.t_begin;
#pragma unroll
          for (int m = 0; m < kM; ++m) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              umma::mma_bf16(tmem + (uint32_t)(m * NH), hi | (a_lo + ((m * kPair + kk * 2048) >> 4)), hi | (p_lo + 2 * kk), idesc,
                             (!fresh || kk > 0) ? 1u : 0u);
            umma::commit(&sh.empty[at.slot * kM + m]);
          }
          umma::commit(&sh.o_done);
          at.next();
        }
      umma::commit(&sh.drain);
      ptx::mbar_wait_bounded(&sh.drain, 0);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax
    const int nh = min(NH, p.H - hg * NH);               // heads of this CTA
    for (int u = piece; u < U; u += p.pieces)            // empty sequences
      if (unit_len(p, u) == 0) {
        const int64_t o = (((int64_t)p.layer_begin * p.B + u) * p.H + hg * NH) * DC;
        for (int x = tid; x < nh * DC; x += kSoft * 32)
          if (p.out_bf16) ((__nv_bfloat16*)p.out)[o + x] = __float2bfloat16(0.f); else ((float*)p.out)[o + x] = 0.f;
      }
    constexpr int kBlocks = NH / 4 / kSoft;              // of 16 heads per warp
    const int quad = warp & 3, col0 = 16 * kBlocks * (warp >> 2);        // 16 tokens
    const uint32_t lane_base = (uint32_t)(32 * quad) << 16;
    const int row_lo = 16 * quad + (lane >> 2);          // tokens row_lo and row_lo + 8 of the tile, heads col0 + 8 j + 2 (lane % 4) + {0, 1}
    // matrix stores: lane i gives the address of row i % 8 of matrix i / 8: heads col0 + 8 (i / 16) + i % 8, token octet 2 quad + (i / 8) % 2
    const int st_head = col0 + 8 * (lane >> 4) + (lane & 7), st_piece = 2 * quad + ((lane >> 3) & 1);
    const uint32_t st_addr = ptx::smem_u32(sP) + st_head * 128 + ((st_piece ^ (st_head & 7)) << 4);
    constexpr int NC = 4 * kBlocks;                      // columns per thread
    const int col = col0 + 2 * (lane & 3);               // columns col + 8 j + {0, 1}
    int t = 0;
    bool gone = false, ok = true;                        // ok: this warp's waits have ended well; the four leave together, at a vote
    Walk w(sh);
    while (!gone && w.next(p)) {
      float m[NC], l[NC];
#pragma unroll
      for (int j = 0; j < NC; ++j) { m[j] = -INFINITY; l[j] = 0.f; }
      for (int i = w.t_begin; i < w.t_end; ++i, ++t) {
        ok = umma::warp_wait(&sh.s_full[t & 1], (t >> 1) & 1, &sh.abort, p.dev_status) && ok;
        umma::fence_after_sync();
        uint32_t z[8 * kBlocks];
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) ld_frags(s_tmem + lane_base + (uint32_t)((t & 1) * NH + col0 + 16 * k), z + 8 * k);
        umma::tmem_ld_wait();
        umma::fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.s_free[t & 1]);
        const int n = w.len - i * kTile;
        if (n < kTile) {
#pragma unroll
          for (int j = 0; j < 8 * kBlocks; ++j)
            if (row_lo + ((j & 2) ? 8 : 0) >= n) z[j] = 0xff800000u;
        }
        bool grow = false;
#pragma unroll
        for (int j = 0; j < 8 * kBlocks; ++j) {
          const int c = (j >> 2) * 2 + (j & 1);
          grow = grow || __uint_as_float(z[j]) * p.scale_log2 > m[c] + kLazy;
        }
        if (softmax_any<kSoft * 32>(grow || !ok || i == w.t_begin)) {
          if (i > w.t_begin) ok = umma::warp_wait(&sh.o_done, (t - 1) & 1, &sh.abort, p.dev_status) && ok;
          if (softmax_any<kSoft * 32>(!ok)) { gone = true; break; }
          // new maxima: columns over this warp's 16 tokens, then over the warps
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const int j = (c >> 1) * 4 + (c & 1);
            float x = fmaxf(__uint_as_float(z[j]), __uint_as_float(z[j + 2]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            if (lane < 4) sh.ex[quad][col + 8 * (c >> 1) + (c & 1)] = x;
          }
          softmax_sync<kSoft * 32>();
          if (tid < NH) {
            const float x = fmaxf(fmaxf(sh.ex[0][tid], sh.ex[1][tid]), fmaxf(sh.ex[2][tid], sh.ex[3][tid])) * p.scale_log2;
            const float was = i == w.t_begin ? -INFINITY : sh.m[tid], now = fmaxf(was, x);
            sh.m[tid] = now;
            sh.alpha[tid] = now == -INFINITY ? 1.f : ptx::ex2_approx(was - now);
          }
          softmax_sync<kSoft * 32>();
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            m[c] = sh.m[col + 8 * (c >> 1) + (c & 1)];
            l[c] *= sh.alpha[col + 8 * (c >> 1) + (c & 1)];
          }
          if (i > w.t_begin) {                           // the sums so far follow
            umma::fence_after_sync();
#pragma unroll 1
            for (int mt = warp >> 2; mt < DC / 128; mt += kSoft / 4)
#pragma unroll 1
              for (int c0 = 0; c0 < NH; c0 += 16) {
                uint32_t o[16];
                const uint32_t a = tmem + lane_base + (uint32_t)(mt * NH + c0);
                umma::tmem_ld16(a, o);
                umma::tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * sh.alpha[c0 + c]);
                umma::tmem_st8(a, o);
                umma::tmem_st8(a + 8, o + 8);
              }
            umma::tmem_st_wait();
          }
        }
        // weights: rounded to bf16 for the second product, summed before that
        float m_eff[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) m_eff[c] = m[c] == -INFINITY ? 0.f : m[c];
        uint32_t pk[4 * kBlocks];
#pragma unroll
        for (int k = 0; k < 4 * kBlocks; ++k) {          // column group k / 2, token octet k % 2
          const float p0 = ptx::ex2_approx(fmaf(__uint_as_float(z[2 * k]), p.scale_log2, -m_eff[2 * (k >> 1)]));
          const float p1 = ptx::ex2_approx(fmaf(__uint_as_float(z[2 * k + 1]), p.scale_log2, -m_eff[2 * (k >> 1) + 1]));
          l[2 * (k >> 1)] += p0;
          l[2 * (k >> 1) + 1] += p1;
          pk[k] = ptx::pack_bf16x2(p0, p1);
        }
        if (t > 0) ok = umma::warp_wait(&sh.o_done, (t - 1) & 1, &sh.abort, p.dev_status) && ok;     // the weights' buffer is free again
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
          stmatrix_x4_trans(st_addr + k * 16 * 128, pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
        ptx::fence_proxy_async();
        umma::fence_before_sync();
        __syncwarp();                                    // (one arrival per warp: they are taken one by one)
        if (lane == 0) ptx::mbar_arrive(&sh.p_full);
      }
      if (gone) break;
      // ---- end of the part: sums of weights over all tokens, then the rows leave
      ok = umma::warp_wait(&sh.o_done, (t - 1) & 1, &sh.abort, p.dev_status) && ok;
      if (softmax_any<kSoft * 32>(!ok)) break;
      umma::fence_after_sync();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[c] += __shfl_xor_sync(0xffffffffu, l[c], o);
        if (lane < 4) sh.ex[quad][col + 8 * (c >> 1) + (c & 1)] = l[c];
      }
      softmax_sync<kSoft * 32>();
      const bool whole = w.t_begin == 0 && w.t_end == w.n;
      const int64_t slot = ((int64_t)piece * 2 + (w.t_begin > 0 ? 0 : 1)) * p.heads_pad + hg * NH;
      if (tid < NH) {
        const float sum = sh.ex[0][tid] + sh.ex[1][tid] + sh.ex[2][tid] + sh.ex[3][tid];
        if (whole) sh.alpha[tid] = 1.f / sum;
        else p.part_ml[slot + tid] = make_float2(sh.m[tid], sum);
      }
      softmax_sync<kSoft * 32>();
      const int64_t out_row = ((int64_t)p.layer_begin * p.B + w.unit) * p.H + hg * NH;
#pragma unroll 1
      for (int mt = warp >> 2; mt < DC / 128; mt += kSoft / 4) {
        const int d = 128 * mt + 32 * quad + lane;       // this thread's channel
#pragma unroll 1
        for (int c0 = 0; c0 < nh; c0 += 16) {
          uint32_t o[16];
          umma::tmem_ld16(tmem + lane_base + (uint32_t)(mt * NH + c0), o);
          umma::tmem_ld_wait();
          if (!whole) {
#pragma unroll
            for (int c = 0; c < 16; ++c)
              if (c0 + c < nh) p.part_o[(slot + c0 + c) * DC + d] = __uint_as_float(o[c]);
          } else if (!p.out_bf16) {
#pragma unroll
            for (int c = 0; c < 16; ++c)
              if (c0 + c < nh) ((float*)p.out)[(out_row + c0 + c) * DC + d] = __uint_as_float(o[c]) * sh.alpha[c0 + c];
          } else {
            // two heads at a time: even lanes take the first head's channels d, d + 1, odd lanes the second's d - 1, d
#pragma unroll
            for (int c = 0; c < 16; c += 2) {
              const float v0 = __uint_as_float(o[c]) * sh.alpha[c0 + c], v1 = __uint_as_float(o[c + 1]) * sh.alpha[c0 + c + 1];
              const float far = __shfl_xor_sync(0xffffffffu, (lane & 1) ? v0 : v1, 1);
              const int h = c0 + c + (lane & 1);
              if (h < nh)
                *reinterpret_cast<uint32_t*>((__nv_bfloat16*)p.out + (out_row + h) * DC + (d & ~1)) =
                    (lane & 1) ? ptx::pack_bf16x2(far, v1) : ptx::pack_bf16x2(v0, far);
            }
          }
        }
      }
      if (tid == 0 && hg == 0 && w.t_begin == 0 && !whole) {
        const int used = pieces_used(sh.total, p.pieces), at = sh.g0 + t - (w.t_end - w.t_begin);      // first tile of the unit
        p.plan[piece] = make_int2(w.unit, piece_of(sh.total, used, at + w.n - 1));
      }
      umma::fence_before_sync();                         // (the next unit's first sums overwrite O once its weights are published)
    }
  }
  // ---- every role has left its loops; nothing of this CTA is in flight any more
  umma::fence_before_sync();
  __syncthreads();
  if (warp == kScoreWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, kCols);
  }
}

// Joins the parts of units that lie in several pieces.  Bound by latency, plan -> maxima and sums of the parts -> result, so the CTAs are
// small enough to be resident all at once with up to 32 heads (with more up to 3552 on 148 SMs that hold 2368).  The first p.pieces x H / 4 take a unit in few parts each, the one that begins in their piece,
// and four heads of it: a warp works out the weights of one head's parts, then a thread sums four channels of all four.  The others take
// the heads of units in many parts, 128 channels at a time, a quarter of the parts to each warp (one sequence of 8192 tokens, 128 parts: the
// call takes 25 us, 82 where a thread adds up all of them).  Many are 8 or more: with 6, 16 sequences of 128 heads take 51 us instead of 45,
// with 12, 16 sequences of 16 heads 37 instead of 33.
constexpr int kJoin = 4, kManyParts = 8, kAhead = 4, kJoinExtra = 8 * kMaxCtas;
__device__ __forceinline__ int64_t part_of(const LatentDecodeParams& p, int i0, int i, int h) {
  return ((int64_t)(i0 + i) * 2 + (i == 0 ? 1 : 0)) * p.heads_pad + h;
}
// One warp: what part i of head h counts, for all of the unit's n parts.
__device__ __forceinline__ void join_weights(const LatentDecodeParams& p, int i0, int n, int h, float* weight) {
  constexpr int kRounds = (kMaxCtas + 31) / 32;
  const int lane = threadIdx.x & 31;
  float2 ml[kRounds];
  float m = -INFINITY, total = 0.f;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    ml[k] = 32 * k + lane < n ? p.part_ml[part_of(p, i0, 32 * k + lane, h)] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, ml[k].x);
  }
  m = warp_max(m);
  if (m == -INFINITY) m = 0.f;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    ml[k].x = ptx::ex2_approx(ml[k].x - m);
    total += ml[k].y * ml[k].x;
  }
  const float inv = 1.f / warp_sum(total);
#pragma unroll
  for (int k = 0; k < kRounds; ++k)
    if (32 * k + lane < n) weight[32 * k + lane] = ml[k].x * inv;
}
__device__ __forceinline__ void join_store(const LatentDecodeParams& p, int unit, int h, int c, const float4& o) {
  const int64_t at = (((int64_t)p.layer_begin * p.B + unit) * p.H + h) * p.dc + c;
  if (p.out_bf16)
    *reinterpret_cast<uint2*>((__nv_bfloat16*)p.out + at) = make_uint2(ptx::pack_bf16x2(o.x, o.y), ptx::pack_bf16x2(o.z, o.w));
  else
    *reinterpret_cast<float4*>((float*)p.out + at) = o;
}
__device__ __forceinline__ void add_part(float4& o, const float4& v, float f) { o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f; }

__global__ void __launch_bounds__(128) latent_join_kernel(LatentDecodeParams p) {
  __shared__ float weight[kJoin][kMaxCtas];
  __shared__ float4 sums[4][32];
  __shared__ int3 units[kMaxCtas / (kManyParts - 1) + 1];                // unit, first piece, parts
  __shared__ int n_units;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, few = p.pieces * ((p.H + kJoin - 1) / kJoin);
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  if ((int)blockIdx.x < few) {
    const int i0 = blockIdx.x % p.pieces, h0 = kJoin * (blockIdx.x / p.pieces), c = 4 * threadIdx.x;
    const int2 plan = p.plan[i0];
    const int n = plan.y - i0 + 1;
    if (plan.x < 0 || n >= kManyParts) return;
    if (h0 + warp < p.H) join_weights(p, i0, n, h0 + warp, weight[warp]);
    __syncthreads();
    if (c >= p.dc) return;
    float4 o[kJoin];
#pragma unroll
    for (int k = 0; k < kJoin; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int k = 0; k < kJoin; ++k)
        if (h0 + k < p.H) add_part(o[k], *reinterpret_cast<const float4*>(p.part_o + part_of(p, i0, i, h0 + k) * p.dc + c), weight[k][i]);
#pragma unroll
    for (int k = 0; k < kJoin; ++k)
      if (h0 + k < p.H) join_store(p, plan.x, h0 + k, c, o[k]);
    return;
  }
  if (warp == 0) {
    int at = 0;
    for (int k = 0; k < p.pieces; k += 32) {
      const int2 plan = k + lane < p.pieces ? p.plan[k + lane] : make_int2(-1, -1);
      const bool many = plan.x >= 0 && plan.y - (k + lane) + 1 >= kManyParts;
      const uint32_t all = __ballot_sync(0xffffffffu, many);
      if (many) units[at + __popc(all & ((1u << lane) - 1))] = make_int3(plan.x, k + lane, plan.y - (k + lane) + 1);
      at += __popc(all);
    }
    if (lane == 0) n_units = at;
  }
  __syncthreads();
  const int slices = p.dc / 128;
  for (int item = blockIdx.x - few; item < n_units * p.H * slices; item += gridDim.x - few) {
    const int c = 128 * (item % slices) + 4 * lane, h = item / slices % p.H, i0 = units[item / slices / p.H].y, n = units[item / slices / p.H].z;
    float4 v[kAhead], o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto part = [&](int i) { return *reinterpret_cast<const float4*>(p.part_o + part_of(p, i0, i, h) * p.dc + c); };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)                     // (asked for along with the maxima)
      if (warp + 4 * k < n) v[k] = part(warp + 4 * k);
    join_weights(p, i0, n, h, weight[warp]);
    __syncwarp();
    for (int i = warp; i < n; i += 4 * kAhead)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i + 4 * k < n) add_part(o, v[k], weight[warp][i + 4 * k]);
        if (i + 4 * (k + kAhead) < n) v[k] = part(i + 4 * (k + kAhead));
      }
    sums[warp][lane] = o;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < 4; ++w) add_part(o, sums[w][lane], 1.f);
      join_store(p, units[item / slices / p.H].x, h, c, o);
    }
    __syncthreads();                                     // (before the next item's weights and sums)
  }
}

// bf16 rows of `d` channels, `mid` x `outer` of them, as a 3-D tensor; box = 64 channels x `box` rows of the middle axis.
// Channels and rows of a box that the tensor does not have read as zeros.
bool make_box_map(CUtensorMap* map, const void* base, int d, int64_t mid, int64_t outer, int box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)mid, (cuuint64_t)outer};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)mid * d * 2};
  cuuint32_t size[3] = {64, (cuuint32_t)box, 1}, step[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, size, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Heads per CTA: as many columns of the products as the heads need, 64 at most.
int heads_per_cta(int H) { return H <= 16 ? 16 : (H <= 32 ? 32 : 64); }

struct Space { int nh, groups, pieces; size_t ml, plan, all; };
Space space_of(const ngc_latent_pool* c, int H) {
  Space w;
  w.nh = heads_per_cta(H);
  w.groups = (H + w.nh - 1) / w.nh;
  w.pieces = kMaxCtas / w.groups;
  const size_t rows = (size_t)w.pieces * 2 * w.groups * w.nh;
  w.ml = align256(rows * c->d_latent * 4);
  w.plan = w.ml + align256(rows * 8);
  w.all = w.plan + align256((size_t)w.pieces * 8);
  return w;
}

template <int NH, int DC> int launch(const Maps& maps, LatentDecodeParams& p, cudaStream_t stream) {
  constexpr int kChunks = DC / 64 + 1, kFree = kSmemLimit - kStaticReserve - 1024 - kChunks * NH * 128 - NH * 128;
  p.stages = kFree / (kChunks * kBox);
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  if (p.stages * (DC / 128) > kMaxPairs) p.stages = kMaxPairs / (DC / 128);
  static_assert(sizeof(Shared<NH>) <= kStaticReserve, "static shared memory");
  static PerDeviceOnce once;
  const int rc = once.run([] {
    return cudaFuncSetAttribute(latent_decode_kernel<NH, DC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit - kStaticReserve);
  });
  if (rc != NGC_OK) return rc;
  // (all of it, however little the ring takes: two CTAs of an SM would fight for its tensor memory)
  NGC_CUDA_TRY(launch_pdl(latent_decode_kernel<NH, DC>, dim3(p.pieces * p.groups), dim3(cta_threads(NH)), kSmemLimit - kStaticReserve, stream, maps, p));
  NGC_CUDA_TRY(launch_pdl(latent_join_kernel, dim3(p.pieces * ((p.H + kJoin - 1) / kJoin) + kJoinExtra), dim3(128), 0, stream, p));
  return launch_status();
}

template <int NH> int launch_heads(const Maps& maps, LatentDecodeParams& p, cudaStream_t stream) {
  switch (p.dc) {
    case 128: return launch<NH, 128>(maps, p, stream);
    case 256: return launch<NH, 256>(maps, p, stream);
    case 384: return launch<NH, 384>(maps, p, stream);
    default: return launch<NH, 512>(maps, p, stream);
  }
}

}  // namespace
}  // namespace ngc

extern "C" size_t ngc_latent_decode_workspace_bytes(const ngc_latent_pool* c, int H) {
  return c && c->d_latent > 0 && H > 0 ? ngc::space_of(c, H).all : 0;
}

extern "C" int ngc_latent_decode(const ngc_latent_pool* c, const void* q_latent, const void* q_rope, int H, int layer_begin, int layer_end,
                                 float scale, void* out, int out_dtype, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_latent_decode");
  if (!valid_latent_pool(c) || !q_latent || !q_rope || !out || layer_begin < 0 || layer_begin >= layer_end || layer_end > c->L || H < 1 ||
      !(scale > 0.f && scale <= 2e38f) || (out_dtype != NGC_F32 && out_dtype != NGC_BF16) || !aligned16(c->rows) || !aligned16(q_latent) ||
      !aligned16(q_rope) || !aligned16(out))
    return NGC_ERR_INVALID_ARG;
  if (c->dtype != NGC_BF16 || !built_latent_dims(c->d_latent, c->d_rope) || H > 128 || (int64_t)c->L * c->B > 0x7fffffffLL ||
      (int64_t)(layer_end - layer_begin) * c->B * (((int64_t)c->pages_cap * c->page + kTile - 1) / kTile) > 0x7fffffffLL)
    return NGC_ERR_UNSUPPORTED;
  const Space w = space_of(c, H);
  if (!ws || ws_bytes < w.all || ((uintptr_t)ws & 255)) return NGC_ERR_WORKSPACE;
  LatentDecodeParams p;
  p.table = c->page_table; p.lens = c->lens; p.out = out; p.dev_status = dev_status;
  p.part_o = (float*)ws; p.part_ml = (float2*)((uint8_t*)ws + w.ml); p.plan = (int2*)((uint8_t*)ws + w.plan);
  p.B = c->B; p.H = H; p.G = lists_G(c->lists, c->L, 1); p.dc = c->d_latent; p.dr = c->d_rope; p.page = c->page; p.cap = c->pages_cap;
  p.n_pages = c->n_pages; p.lists = c->lists; p.layer_begin = layer_begin; p.n_layers = layer_end - layer_begin;
  p.out_bf16 = out_dtype == NGC_BF16; p.stages = 0; p.pieces = w.pieces; p.groups = w.groups;
  p.heads_pad = w.groups * w.nh; p.scale_log2 = scale * 1.4426950408889634f;
  Maps maps;
  const int64_t LB = (int64_t)c->L * c->B;
  if (!make_rows_map(&maps.rows, c->rows, (int64_t)c->L * c->n_pages * c->page, c->page, c->d_latent + c->d_rope) ||
      !make_box_map(&maps.ql, q_latent, c->d_latent, H, LB, w.nh) || !make_box_map(&maps.qr, q_rope, c->d_rope, H, LB, w.nh))
    return NGC_ERR_UNSUPPORTED;
  return w.nh == 16 ? launch_heads<16>(maps, p, stream) : w.nh == 32 ? launch_heads<32>(maps, p, stream) : launch_heads<64>(maps, p, stream);
}
