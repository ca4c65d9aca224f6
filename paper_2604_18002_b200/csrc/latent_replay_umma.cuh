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

// Deals the items of a call out to its CTAs: blocks of `size` tokens of every (sequence, head, layer), level by level (all first
// blocks, all second ones, ...; or from the last level down), so that the long ones come first; and in turn from the first CTA to the
// last and back, so that who gets a longer one gets a shorter one next.  Only blocks that exist are counted.  All lanes of a warp
// together.
struct Deal {
  int size, pass, m, before, count;            // level, items before it, sequences that have it
  int at, seen;                                // the 32 sequences that the last item came from, sequences of the level before them
  bool down;
  __device__ __forceinline__ Deal(const LatentReplayParams& p, int block, bool from_last)
      : size(block), pass(0), m(0), before(0), count(0), at(0), seen(0), down(from_last) {
    if (down) {
      int longest = 0;
      int64_t row0;
      for (int b = threadIdx.x & 31; b < p.B; b += 32) longest = max(longest, latent_seq(p, b, row0));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
      m = (longest + size - 1) / size - 1;
    }
    count = m >= 0 ? sequences(p) : 0;
  }
  static __device__ __forceinline__ int length(const LatentReplayParams& p, int b) {
    int64_t row0;
    return b < p.B ? latent_seq(p, b, row0) : 0;
  }
  __device__ __forceinline__ int sequences(const LatentReplayParams& p) const {
    int n = 0;
#pragma unroll 1                                         // (unrolled: rollouts of 8192 tokens forward 289 -> 295 to 299 us, the other roles' code moves)
    for (int b0 = 0; b0 < p.B; b0 += 32) n += __popc(__ballot_sync(0xffffffffu, length(p, b0 + (threadIdx.x & 31)) > (int64_t)m * size));
    return n;
  }
  // The next item of this CTA: block m of a sequence.  Sequences come in order within a level and layer, so the search goes on where
  // the last one ended (from the first sequence on for every item: 8192 of 32 tokens 57 instead of 5.2 ms forward, 115 instead of 7.5 back).
  __device__ __forceinline__ bool next(const LatentReplayParams& p, int& l, int& b, int& h) {
    const int k = pass * (int)gridDim.x + ((pass & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x), per = p.L * p.H;
    while (count > 0 && k - before >= count * per) {
      before += count * per;
      m += down ? -1 : 1;
      count = m >= 0 ? sequences(p) : 0;
      at = seen = 0;
    }
    if (count == 0) return false;                        // (levels only end behind the last one)
    ++pass;
    int x = k - before;
    h = x % p.H;
    x /= p.H;
    l = x / count;
    x %= count;
    if (x < seen) at = seen = 0;                         // (the next layer)
    for (;; at += 32) {
      const uint32_t has = __ballot_sync(0xffffffffu, length(p, at + (threadIdx.x & 31)) > (int64_t)m * size);
      const int n = __popc(has);
      if (x - seen < n) { b = at + (int)__fns(has, 0, x - seen + 1); return true; }
      seen += n;
    }
  }
};

// An item's description, made by the planner warp (which also loads what stays in shared memory throughout the item) some items
// ahead, so that no other role meets the chain of reads behind it.
constexpr int kPlans = 4, kPlanWindows = 8;
struct ReplayPlan {
  int valid, l, b, h, x0, T, n;                // first token of the item's block; query walks: key tiles, key walks: query tiles
  uint32_t lower[kPlanWindows], upper[kPlanWindows], plain_a[kPlanWindows], plain_b[kPlanWindows];       // query walks: see there, of the first 256 tiles
  int64_t row0;                                // first row of the sequence, within a layer
};
struct PlanRing {
  uint64_t full[kPlans], empty[kPlans];
  ReplayPlan plan[kPlans];
  static constexpr int kReaders = 11;          // producer, mender, MMA, eight softmax warps
  __device__ __forceinline__ void init(int i) { ptx::mbar_init(&full[i], 1); ptx::mbar_init(&empty[i], kReaders); }
};
// What every walk needs of a launch.
struct WalkEnv {
  const LatentReplayParams& p;
  PlanRing* ring;
  int* abort;
  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) const { return umma::warp_wait(bar, parity, abort, p.dev_status); }
  __device__ __forceinline__ bool wait_alone(uint64_t* bar, uint32_t parity) const { return umma::wait_quick(bar, parity, abort, p.dev_status); }
  // Plan of item k: wait for it, and give it back (by a warp, or by one thread that stands for its warp).
  template <bool ALONE> __device__ __forceinline__ bool obtain(int k) const {
    uint64_t* bar = &ring->full[k % kPlans];
    return ALONE ? wait_alone(bar, (k / kPlans) & 1) : wait(bar, (k / kPlans) & 1);
  }
  template <bool ALONE> __device__ __forceinline__ void release(int k) const {
    if (!ALONE) __syncwarp();
    if (ALONE || (threadIdx.x & 31) == 0) ptx::mbar_arrive(&ring->empty[k % kPlans]);
  }
  __device__ __forceinline__ const int4* tiles(int l, int b) const {
    return p.tile_gone ? p.tile_gone + ((int64_t)b * p.G + list_of(p.lists, l, 0, 1)) * (p.gone_cap / kLatTile) : nullptr;
  }
};

// Items of one or two blocks (A, B) of 128 queries of one head; and for each the tiles of 128 keys that any of its queries sees.
template <int BLOCKS> struct QueryWalk {
  int k;                        // items so far
  int l, b, h, q0, T, n;        // the current item; its key tiles are 0 .. n - 1
  int64_t row0;
  const int4* tiles;            // of its list, or null
  int i, window;                // current tile, first tile of the window
  uint32_t live, lower, upper;                 // of the window: tiles still to come that a query sees; of those, whether it sees the first 64 keys, the others
  uint32_t plain_a, plain_b;                   // ones without a key that goes before query block A's (B's) last
  bool first;                   // the current tile is the item's first

  __device__ __forceinline__ QueryWalk() : k(0), n(0), i(0), window(0), live(0), lower(0), upper(0), plain_a(0), plain_b(0) {}
  __device__ __forceinline__ bool has_b() const { return BLOCKS == 2 && q0 + kLatTile < T; }
  __device__ __forceinline__ bool for_a() const { return i * kLatTile <= q0; }
  __device__ __forceinline__ bool last_a() const { return i * kLatTile == q0; }
  __device__ __forceinline__ bool last() const { return i == n - 1; }
  // Masks of the window: by all lanes, or (ALONE) by one thread.
  template <bool ALONE> __device__ __forceinline__ void load_window() {
    auto look = [&](int t, bool& lo, bool& up, bool& pa, bool& pb) {
      int4 g = make_int4(kNeverGone, kNeverGone, kNeverGone, kNeverGone);
      if (tiles && t < n) g = tiles[t];
      lo = t < n && g.y > q0;
      up = t < n && g.w > q0 && t * kLatTile + 64 < T;
      pa = min(g.x, g.z) > q0 + kLatTile - 1;
      pb = min(g.x, g.z) > q0 + 2 * kLatTile - 1;
    };
    bool lo, up, pa, pb;
    if (ALONE) {
      lower = upper = plain_a = plain_b = 0;
      for (int t = window; t < min(window + 32, n); ++t) {
        look(t, lo, up, pa, pb);
        lower |= (uint32_t)lo << (t - window); upper |= (uint32_t)up << (t - window);
        plain_a |= (uint32_t)pa << (t - window); plain_b |= (uint32_t)pb << (t - window);
      }
    } else {
      look(window + (threadIdx.x & 31), lo, up, pa, pb);
      lower = __ballot_sync(0xffffffffu, lo); upper = __ballot_sync(0xffffffffu, up);
      plain_a = __ballot_sync(0xffffffffu, pa); plain_b = __ballot_sync(0xffffffffu, pb);
    }
    live = lower | upper;
  }
  // The planner's part.
  __device__ __forceinline__ bool plan(const WalkEnv& e, Deal& deal) {
    if (!deal.next(e.p, l, b, h)) return false;
    q0 = deal.m * BLOCKS * kLatTile;
    T = latent_seq(e.p, b, row0);
    n = q0 / kLatTile + 1 + (has_b() ? 1 : 0);
    tiles = e.tiles(l, b);
    return true;
  }
  __device__ __forceinline__ void publish(ReplayPlan& r) {
    const bool one = (threadIdx.x & 31) == 0;
    if (one) { r.l = l; r.b = b; r.h = h; r.x0 = q0; r.T = T; r.n = n; r.row0 = row0; }
    for (int w = 0; w < kPlanWindows && 32 * w < n; ++w) {
      window = 32 * w;
      load_window<false>();
      if (one) { r.lower[w] = lower; r.upper[w] = upper; r.plain_a[w] = plain_a; r.plain_b[w] = plain_b; }
    }
  }
  // The other roles', by all lanes of a warp or by one thread alone.  (An item's plan is held until its last tile has been passed.)
  template <bool ALONE = false> __device__ __forceinline__ bool next(const WalkEnv& e) {
    first = false;
    if (live == 0) advance<ALONE>(e);
    if (live == 0) {
      if (k > 0) e.release<ALONE>(k - 1);
      if (!e.obtain<ALONE>(k)) return false;
      const ReplayPlan& r = e.ring->plan[k % kPlans];
      ++k;
      if (!r.valid) return false;
      l = r.l; b = r.b; h = r.h; q0 = r.x0; T = r.T; n = r.n; row0 = r.row0; take(r, 0);
      tiles = e.tiles(l, b);
      window = 0;
      first = true;
      if (live == 0) advance<ALONE>(e);                  // (a query sees its own key: one tile is live)
    }
    const int at = __ffs(live) - 1;
    live &= live - 1;
    i = window + at;
    return true;
  }
  __device__ __forceinline__ void take(const ReplayPlan& r, int w) {
    lower = r.lower[w]; upper = r.upper[w]; plain_a = r.plain_a[w]; plain_b = r.plain_b[w];
    live = lower | upper;
  }
  // Which halves of the current tile are seen: bit 0 the first 64 keys, bit 1 the others.
  __device__ __forceinline__ int halves() const { return (lower >> (i - window) & 1) | (upper >> (i - window) & 1) << 1; }
  template <bool ALONE> __device__ __forceinline__ void advance(const WalkEnv& e) {
    while (live == 0 && window + 32 < n) {
      window += 32;
      if (window < 32 * kPlanWindows) {
        const ReplayPlan& r = e.ring->plan[(k - 1) % kPlans];
        take(r, window / 32);
      } else {
        load_window<ALONE>();
      }
    }
  }
};

// The same by tiles of 64 keys, one block of queries per item.
struct HalfWalk {
  QueryWalk<1> w;
  int k0, pending;              // first key; halves of w's tile still to come
  bool fresh, first, last;      // fresh: no tile of the item has been taken

  __device__ __forceinline__ HalfWalk() : pending(0), fresh(false) {}
  __device__ __forceinline__ bool plan(const WalkEnv& e, Deal& deal) { return w.plan(e, deal); }
  __device__ __forceinline__ void publish(ReplayPlan& r) { w.publish(r); }
  template <bool ALONE = false> __device__ __forceinline__ bool next(const WalkEnv& e) {
    if (pending == 0) {
      if (!w.next<ALONE>(e)) return false;
      pending = w.halves();
      fresh = fresh || w.first;
    }
    const bool up = !(pending & 1);
    pending &= pending - 1;
    k0 = w.i * kLatTile + (up ? 64 : 0);
    first = fresh;
    fresh = false;
    last = w.last() && pending == 0;
    return true;
  }
};

// Items of 128 keys of one head; and for each the tiles of 64 queries from its own first key to the last query that sees one of
// them.
struct KeyWalk {
  static constexpr int kQ = 64;
  int k;
  int l, b, h, j0, T, i, n;     // current query tile, and the one behind the last
  int64_t row0;
  bool first;

  __device__ __forceinline__ KeyWalk() : k(0), i(-1), n(0) {}
  __device__ __forceinline__ bool last() const { return i == n - 1; }
  __device__ __forceinline__ bool plan(const WalkEnv& e, Deal& deal) {
    if (!deal.next(e.p, l, b, h)) return false;
    j0 = deal.m * kLatTile;
    T = latent_seq(e.p, b, row0);
    const int4* tiles = e.tiles(l, b);
    const int end = tiles ? min(T, max(tiles[j0 / kLatTile].y, tiles[j0 / kLatTile].w)) : T;
    n = (end + kQ - 1) / kQ;                             // (a key sees to its own query at least: one tile or more)
    return true;
  }
  __device__ __forceinline__ void publish(ReplayPlan& r) const {
    if ((threadIdx.x & 31) == 0) { r.l = l; r.b = b; r.h = h; r.x0 = j0; r.T = T; r.n = n; r.row0 = row0; }
  }
  template <bool ALONE = false> __device__ __forceinline__ bool next(const WalkEnv& e) {
    first = false;
    if (++i < n) return true;
    if (k > 0) e.release<ALONE>(k - 1);
    if (!e.obtain<ALONE>(k)) return false;
    const ReplayPlan& r = e.ring->plan[k % kPlans];
    ++k;
    if (!r.valid) return false;
    l = r.l; b = r.b; h = r.h; j0 = r.x0; T = r.T; n = r.n; row0 = r.row0;
    i = j0 / kQ;
    first = true;
    return true;
  }
};

// The planner warp: plans item after item and calls load(walk, number of the item) for each; false ends it.
template <typename Walk, typename Load> __device__ __forceinline__ void run_planner(const WalkEnv& e, int block, bool from_last, Load&& load) {
  Deal deal(e.p, block, from_last);
  Walk w;
  for (int k = 0;; ++k) {
    const int slot = k % kPlans;
    const bool valid = w.plan(e, deal);
    if (k >= kPlans && !e.wait(&e.ring->empty[slot], (k / kPlans - 1) & 1)) return;
    if (valid) w.publish(e.ring->plan[slot]);
    if ((threadIdx.x & 31) == 0) {
      e.ring->plan[slot].valid = valid;
      ptx::mbar_arrive(&e.ring->full[slot]);
    }
    __syncwarp();
    if (!valid || !load(w, k)) return;
  }
}

}  // namespace ngc
