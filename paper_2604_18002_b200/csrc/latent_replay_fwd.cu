// The forward pass of ngc_latent_replay_attn on the 5th-generation tensor cores.
//
// An item is 256 queries of one head, two blocks of 128 (the lanes of tensor memory) that share the tiles of 128 keys they see:
// S = Q K^T over 128 + d_rope channels (the rotary chunk of K is the same for all heads), O += P V with P read from tensor memory.
// What a query sees is one number per key (the sequence length when it was evicted), so tiles that no query of an item sees are
// passed over, halves of 64 keys of the others too (rollouts 330 -> 311 us), and most need no look at single keys.  Roles, which meet at mbarriers only:
//   producer warp     K and V chunks of 128 rows x 64 channels by TMA into a ring of eight 16 KB slots, K of tile i + 1 before V of
//                     tile i: K makes room as soon as both blocks' scores are done
//   planner warp      what the other roles need to know of the items, up to two ahead, and the queries of the next item when the
//                     last scores of this one are done, block by block
//   mender warp       values behind a sequence's end: zeros (they belong to others; a NaN times a zero weight is NaN)
//   MMA thread        P V of block A, S of its next tile, P V of block B, S of its next tile: one block's softmax runs under
//                     the other's products
//   softmax warps     4 per block, a query per thread: mask, online softmax in the log2 domain, P as bf16 over its S.  The maximum used
//                     moves only when the true one has grown by more than 2^8, so O is rarely rescaled
// 128-key tiles because a product of 128 x 64 waits for shared memory (Q is read again for every tile).
// Bound by the tensor pipe: causal, 8192 tokens of 16 heads, batch 2: 588 us, 1169 TFLOP/s; rollouts of 6500 to 8192 tokens with a round
// every 1024: 287 to 304 us, some 710 TFLOP/s of visible pairs, the rest are products of half and whole tiles that a round cuts through.
#include <cuda.h>
#include <cuda_bf16.h>

#include <type_traits>

#include "latent_replay_umma.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

constexpr int kSlots = 8;
constexpr int kMmaWarp = 8, kProducerWarp = 9, kMenderWarp = 10, kPlannerWarp = 11;
constexpr int kThreads = 12 * 32;
constexpr int kQBlock = 3 * kLatChunk;         // 128 queries, 192 channels
constexpr int kSmemBytes = 2 * kQBlock + kSlots * kLatChunk + 1024;
constexpr uint32_t kTmemCols = 512;            // S (P over its first half) of block A, B at 0, 128; O at 256, 384
constexpr float kLazy = 8.f;

struct Maps { CUtensorMap q, kv, kr; };

struct Shared {
  uint64_t k_full[2], k_empty[2], v_full[2], v_raw[2], v_empty[2];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_done[2], drain;
  uint32_t tmem;
  int abort;
  PlanRing ring;
};

// ROUNDS: whether keys go at all.  Without, no tile is looked at for them or done by halves: the causal pass of 8192 tokens, 16 heads,
// batch 2 takes 588 us against 672 as one kernel for both; rollouts of the same length with a round every 1024 tokens take 292.
//
// The softmax's warps take over registers that the others can do without (8 x 32 x 208 + 4 x 32 x 88 are the 384 x 168 of the launch):
// 616 -> 588 us, 316 -> 292.  With rounds the MMA warp's thread needs more of them for the plans (104 and 200: 292 us, 88 and 208: 301).
template <bool ROUNDS>
__global__ void __launch_bounds__(kThreads, 1) latent_fwd_kernel(const __grid_constant__ Maps maps, LatentReplayParams p) {
  extern __shared__ uint8_t smem_dyn[];
  __shared__ Shared sh;
  uint8_t* sQ = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);     // [2 blocks][3 chunks]
  uint8_t* ring = sQ + 2 * kQBlock;                                              // [8 slots]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (warp == 0) {
    if (lane < 2) {
      ptx::mbar_init(&sh.k_full[lane], 1); ptx::mbar_init(&sh.k_empty[lane], 1);
      ptx::mbar_init(&sh.v_full[lane], 1); ptx::mbar_init(&sh.v_raw[lane], 1); ptx::mbar_init(&sh.v_empty[lane], 1);
      ptx::mbar_init(&sh.q_full[lane], 1); ptx::mbar_init(&sh.q_empty[lane], 1);
      ptx::mbar_init(&sh.s_full[lane], 1); ptx::mbar_init(&sh.p_full[lane], 4); ptx::mbar_init(&sh.o_done[lane], 1);
    }
    if (lane < kPlans) sh.ring.init(lane);
    if (lane == 2) { ptx::mbar_init(&sh.drain, 1); sh.abort = 0; }
    ptx::fence_barrier_init();
  } else if (warp == kProducerWarp && lane == 0) {
    ptx::prefetch_tensormap(&maps.q); ptx::prefetch_tensormap(&maps.kv); ptx::prefetch_tensormap(&maps.kr);
  }
  if (warp == kMmaWarp) umma::tmem_alloc(&sh.tmem, kTmemCols);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tmem = sh.tmem;
  ptx::grid_dep_wait();
  const WalkEnv env{p, &sh.ring, &sh.abort};
  auto wait = [&](uint64_t* bar, uint32_t parity) { return env.wait(bar, parity); };

  if (warp >= kMmaWarp) {
    ptx::fewer_registers<ROUNDS ? 104 : 88>();
    if (warp == kProducerWarp) {
      // ------------------------------------------------------------------ keys and values
      // Tile t (over all items) has its keys in slots 5 t .. 5 t + 2 and its values in 5 t + 3, 5 t + 4 (mod 8): keys of tile t fit
      // when the values of t - 2 are used up, values of t when the keys of t - 1 are.
      QueryWalk<2> w, v;                                   // v: the tile before
      int t = 0, tv = 0, n_raw[2] = {0, 0};
      uint32_t v_through = 0;                              // bit b: the last values of parity b went through raw
      bool ok = true, more = w.next(env);
      auto values = [&]() {                                // of tile tv
        if (tv > 0) ok = wait(&sh.k_empty[(tv - 1) & 1], ((tv - 1) >> 1) & 1);
        if (!ok) return;
        const int64_t y = (int64_t)v.l * p.rows + v.row0 + v.i * kLatTile;
        const bool tail = (v.i + 1) * kLatTile > v.T;
        if (umma::elect_one()) {
          uint64_t* bar = tail ? &sh.v_raw[tv & 1] : &sh.v_full[tv & 1];
          ptx::mbar_expect_tx(bar, 2 * kLatChunk);
          for (int c = 0; c < 2; ++c)
            ptx::tma_load_3d(ring + ((5 * tv + 3 + c) & 7) * kLatChunk, &maps.kv, kLatNope + 64 * c, v.h, (int)y, bar);
        }
        __syncwarp();
        v_through = tail ? v_through | 1u << (tv & 1) : v_through & ~(1u << (tv & 1));
        n_raw[0] += tail && !(tv & 1); n_raw[1] += tail && (tv & 1);
        ++tv;
      };
      while (ok && more) {
        if (t > 1) ok = wait(&sh.v_empty[t & 1], ((t >> 1) - 1) & 1);
        if (!ok) break;
        const int64_t y = (int64_t)w.l * p.rows + w.row0 + w.i * kLatTile;
        if (umma::elect_one()) {
          ptx::mbar_expect_tx(&sh.k_full[t & 1], 3 * kLatChunk);
          for (int c = 0; c < 2; ++c) ptx::tma_load_3d(ring + ((5 * t + c) & 7) * kLatChunk, &maps.kv, 64 * c, w.h, (int)y, &sh.k_full[t & 1]);
          ptx::tma_load_2d(ring + ((5 * t + 2) & 7) * kLatChunk, &maps.kr, 0, (int)y, &sh.k_full[t & 1]);
        }
        __syncwarp();
        ++t;
        if (t > 1) values();                               // of the tile before
        v = w;
        more = ok && w.next(env);
      }
      if (ok && t > tv) values();
      // nothing is in flight when the CTA ends
      for (int x = max(0, t - 2); x < t; ++x) ptx::mbar_wait_bounded(&sh.k_full[x & 1], (x >> 1) & 1);
      for (int x = max(0, tv - 2); x < tv; ++x) {
        if (v_through >> (x & 1) & 1) ptx::mbar_wait_bounded(&sh.v_raw[x & 1], (n_raw[x & 1] - 1) & 1);
        else ptx::mbar_wait_bounded(&sh.v_full[x & 1], (x >> 1) & 1);
      }
      __syncwarp();
    } else if (warp == kMenderWarp) {
      // ------------------------------------------------------------------ values behind a sequence's end
      QueryWalk<2> w;
      uint32_t phase = 0;
      for (int t = 0; w.next(env); ++t) {
        if ((w.i + 1) * kLatTile <= w.T) continue;
        if (!wait(&sh.v_raw[t & 1], (phase >> (t & 1)) & 1)) break;
        phase ^= 1u << (t & 1);
        const int n = w.T - w.i * kLatTile;                // rows that are tokens
        for (int c = 0; c < 2; ++c) {
          uint8_t* chunk = ring + ((5 * t + 3 + c) & 7) * kLatChunk;
          for (int x = n * 8 + lane; x < kLatTile * 8; x += 32) *reinterpret_cast<uint4*>(chunk + x * 16) = make_uint4(0, 0, 0, 0);
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.v_full[t & 1]);
      }
    } else if (warp == kPlannerWarp) {
      // ------------------------------------------------------------------ plans and queries of the items
      int na = 0, nb = 0;                                  // blocks loaded
      run_planner<QueryWalk<2>>(env, 2 * kLatTile, true, [&](const QueryWalk<2>& w, int) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          int& n = x ? nb : na;
          if (x && !w.has_b()) break;
          if (n > 0 && !wait(&sh.q_empty[x], (n - 1) & 1)) return false;
          if (umma::elect_one()) {
            const int y = (int)((int64_t)w.l * p.rows + w.row0 + w.q0 + x * kLatTile);
            ptx::mbar_expect_tx(&sh.q_full[x], kQBlock);
            for (int c = 0; c < 3; ++c) ptx::tma_load_3d(sQ + x * kQBlock + c * kLatChunk, &maps.q, 64 * c, w.h, y, &sh.q_full[x]);
          }
          __syncwarp();
          ++n;
        }
        return true;
      });
      if (na > 0) ptx::mbar_wait_bounded(&sh.q_full[0], (na - 1) & 1);
      if (nb > 0) ptx::mbar_wait_bounded(&sh.q_full[1], (nb - 1) & 1);
      __syncwarp();
    } else if (warp == kMmaWarp) {
      // ------------------------------------------------------------------ products
      constexpr uint32_t idesc_s = umma::instr_desc(kLatTile, kLatTile, false);
      constexpr uint32_t idesc_s64 = umma::instr_desc(kLatTile, 64, false);
      constexpr uint32_t idesc_o = umma::instr_desc(kLatTile, kLatV, true), idesc_half = umma::instr_desc(kLatTile, 64, true);
      const uint64_t hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
      const uint32_t q_lo = (ptx::smem_u32(sQ) >> 4) | 1u << 16, ring_lo = ptx::smem_u32(ring) >> 4;
      const int steps_r = p.dr / 16;
      // One thread does it all: what a whole warp takes to wait, elect and meet again adds up (the gradient's kernel for keys: 723
      // -> 671 us for rollouts of 8192 tokens).
      if (umma::elect_one()) {
        struct { bool a, b, first, last_a, last_b; int halves; } cur = {false, false, false, false, false, 3};
        QueryWalk<2> nxt;
        uint32_t q_phase = 0, p_phase = 0;                   // bit x: parity of block x's next queries, next weights
        bool ok = true, have = false, more = nxt.next<true>(env);
        for (int t = -1; ok && (have || more); ++t) {
#pragma unroll 1
          for (int x = 0; x < 2; ++x) {
            if (have && (x ? cur.b : cur.a)) {
              // O += P V of block x for tile t
              ok = env.wait_alone(&sh.v_full[t & 1], (t >> 1) & 1) && env.wait_alone(&sh.p_full[x], (p_phase >> x) & 1);
              if (!ok) break;
              p_phase ^= 1u << x;
              umma::fence_after_sync();
              const int s0 = (5 * t + 3) & 7;
              const uint32_t pa = tmem + 128u * x, d = tmem + 256u + 128u * x, v0 = ring_lo + s0 * (kLatChunk >> 4);
              {
                if (s0 < 7) {
                  const uint32_t b = v0 | (uint32_t)(kLatChunk >> 4) << 16;
#pragma unroll
                  for (int k = 0; k < 8; ++k)
                    if (!ROUNDS || (cur.halves >> (k >> 2) & 1))
                      umma::mma_bf16_a_tmem(d, pa + 8 * k, hi | (b + ((k * 2048) >> 4)), idesc_o, (!cur.first || k > (ROUNDS && cur.halves == 2 ? 4 : 0)) ? 1u : 0u);
                } else {                                     // the two chunks lie at the ring's two ends
#pragma unroll 1
                  for (int k = cur.halves == 2 ? 4 : 0; k < (cur.halves == 1 ? 4 : 8); ++k) {
                    const uint32_t add = (!cur.first || k > (ROUNDS && cur.halves == 2 ? 4 : 0)) ? 1u : 0u;
                    umma::mma_bf16_a_tmem(d, pa + 8 * k, hi | ((v0 | 1u << 16) + ((k * 2048) >> 4)), idesc_half, add);
                    umma::mma_bf16_a_tmem(d + 64, pa + 8 * k, hi | ((ring_lo | 1u << 16) + ((k * 2048) >> 4)), idesc_half, add);
                  }
                }
                if (x ? cur.last_b : cur.last_a) umma::commit(&sh.o_done[x]);
                if (x || !cur.b) umma::commit(&sh.v_empty[t & 1]);
              }
            }
            if (more && (x ? nxt.has_b() : nxt.for_a())) {
              // scores of block x for tile t + 1
              const int tn = t + 1;
              if (nxt.first) {
                ok = env.wait_alone(&sh.q_full[x], (q_phase >> x) & 1);
                q_phase ^= 1u << x;
              }
              ok = ok && env.wait_alone(&sh.k_full[tn & 1], (tn >> 1) & 1);
              if (!ok) break;
              umma::fence_after_sync();
              const bool last = x ? nxt.last() : nxt.last_a(), k_done = x || !nxt.has_b();
              const uint32_t k0 = ring_lo + ((5 * tn) & 7) * (kLatChunk >> 4), k1 = ring_lo + ((5 * tn + 1) & 7) * (kLatChunk >> 4),
                             k2 = ring_lo + ((5 * tn + 2) & 7) * (kLatChunk >> 4);
              // (of a tile of which only one half is seen, only that half's 64 keys and columns)
              const int halves = ROUNDS ? nxt.halves() : 3;
              const uint32_t a = q_lo + x * (kQBlock >> 4), d = tmem + 128u * x + (halves == 2 ? 64u : 0u), up = halves == 2 ? kLatChunk >> 5 : 0u,
                             idesc = halves == 3 ? idesc_s : idesc_s64;
              {
#pragma unroll
                for (int c = 0; c < 3; ++c) {
                  const uint32_t b = ((c == 0 ? k0 : c == 1 ? k1 : k2) + up) | 1u << 16;
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    if (c < 2 || k < steps_r) umma::mma_bf16(d, hi | (a + ((c * kLatChunk + k * 32) >> 4)), hi | (b + 2 * k), idesc, (c > 0 || k > 0) ? 1u : 0u);
                }
                umma::commit(&sh.s_full[x]);
                if (last) umma::commit(&sh.q_empty[x]);
                if (k_done) umma::commit(&sh.k_empty[tn & 1]);
              }
            }
          }
          have = more;
          if (more) {
            cur.a = nxt.for_a(); cur.b = nxt.has_b(); cur.first = nxt.first; cur.last_a = nxt.last_a(); cur.last_b = nxt.last(); cur.halves = ROUNDS ? nxt.halves() : 3;
            more = nxt.next<true>(env);
          }
        }
        umma::commit(&sh.drain);                             // everything issued has completed before tensor memory is released
      }
      __syncwarp();
      ptx::mbar_wait_bounded(&sh.drain, 0);
      __syncwarp();
    }
  } else {
    ptx::more_registers<ROUNDS ? 200 : 208>();
    // ------------------------------------------------------------------ softmax: a query per thread
    const int x = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t s_addr = tmem + lane_base + 128u * x, o_addr = tmem + lane_base + 256u + 128u * x;
    QueryWalk<2> w;
    int n_s = 0, n_o = 0;                                // score tiles and items of this block so far
    float m_use = -INFINITY, l_run = 0.f;
    bool begun = false;                                  // this block has had a tile of the item
    while (w.next(env)) {
      if (w.first) { m_use = -INFINITY; l_run = 0.f; begun = false; }
      if (x ? !w.has_b() : !w.for_a()) continue;
      const bool plain = !ROUNDS || ((x ? w.plain_b : w.plain_a) >> (w.i - w.window) & 1);
      int g[4];                                          // (asked for before the wait: the answer takes as long)
      if (!plain) {
        const int32_t* gone = p.gone + ((int64_t)w.b * p.G + list_of(p.lists, w.l, 0, 1)) * p.gone_cap + w.i * kLatTile + lane;
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = gone[32 * k];
      }
      if (!wait(&sh.s_full[x], n_s & 1)) break;
      ++n_s;
      umma::fence_after_sync();
      const int t_q = w.q0 + x * kLatTile + row;
      // NK blocks of 32 columns from block k0 on
      auto softmax = [&](auto blocks, auto begin) {
        constexpr int NK = decltype(blocks)::value, k0 = decltype(begin)::value;
        uint32_t z[NK][32];
#pragma unroll
        for (int k = 0; k < NK; ++k) umma::tmem_ld32(s_addr + 32 * (k0 + k), z[k]);
        umma::tmem_ld_wait();
        const int j0 = w.i * kLatTile + 32 * k0, q_lo = w.q0 + x * kLatTile;
        if (j0 + 32 * NK - 1 > q_lo) {                    // the tile on the diagonal: keys behind the query
#pragma unroll
          for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j0 + 32 * k + j > t_q) z[k][j] = 0xff800000u;
        }
        if (!plain) {
          // keys that have gone: the same for all queries of the block where no round falls between its first and last
#pragma unroll
          for (int k = 0; k < NK; ++k) {
            const uint32_t seen = __ballot_sync(0xffffffffu, g[k0 + k] > q_lo + kLatTile - 1);
            if (seen == __ballot_sync(0xffffffffu, g[k0 + k] > q_lo)) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(seen >> j & 1)) z[k][j] = 0xff800000u;
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (__shfl_sync(0xffffffffu, g[k0 + k], j) <= t_q) z[k][j] = 0xff800000u;
            }
          }
        }
        float mxc[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int j = 0; j < 32; j += 8)
#pragma unroll
            for (int c = 0; c < 4; ++c) mxc[c] = umma::max3(mxc[c], __uint_as_float(z[k][j + 2 * c]), __uint_as_float(z[k][j + 2 * c + 1]));
        const float mx = fmaxf(fmaxf(mxc[0], mxc[1]), fmaxf(mxc[2], mxc[3])) * p.scale_log2;
        const bool grow = mx > m_use + kLazy;              // also the first key that is seen (m_use = -inf)
        const bool rescale = grow && m_use != -INFINITY && begun;
        if (__any_sync(0xffffffffu, rescale)) {            // (the scores came behind the sums of the tile before: those are complete)
          const float alpha = rescale ? ptx::ex2_approx(m_use - mx) : 1.f;
          l_run *= alpha;
#pragma unroll 1
          for (int c0 = 0; c0 < kLatV; c0 += 16) {
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
        begun = true;
        if (grow) m_use = mx;
        const float m_eff = m_use == -INFINITY ? 0.f : m_use;
        const uint64_t sc2 = umma::pack2(p.scale_log2, p.scale_log2), nm2 = umma::pack2(-m_eff, -m_eff);
        uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int half = 0; half < NK / 2; ++half) {
          uint32_t pk[32];
#pragma unroll
          for (int j = 0; j < 64; j += 2) {
            const int k = 2 * half + (j >> 5), e = j & 31;
            float x0, x1;
            umma::unpack2(umma::fma2(umma::pack2(__uint_as_float(z[k][e]), __uint_as_float(z[k][e + 1])), sc2, nm2), x0, x1);
            const float p0 = ptx::ex2_approx(x0), p1 = ptx::ex2_approx(x1);
            acc2[(j >> 1) & 3] = umma::add2(acc2[(j >> 1) & 3], umma::pack2(p0, p1));
            pk[j >> 1] = ptx::pack_bf16x2(p0, p1);
          }
          umma::tmem_st32(s_addr + 32 * half + 16 * k0, pk);         // P over the scores that are in registers
        }
        {
          float s0, s1;
          umma::unpack2(umma::add2(umma::add2(acc2[0], acc2[1]), umma::add2(acc2[2], acc2[3])), s0, s1);
          l_run += s0 + s1;
        }
      };
      const int halves = ROUNDS ? w.halves() : 3;
      if (!ROUNDS || halves == 3) softmax(std::integral_constant<int, 4>{}, std::integral_constant<int, 0>{});
      else if (halves == 1) softmax(std::integral_constant<int, 2>{}, std::integral_constant<int, 0>{});
      else softmax(std::integral_constant<int, 2>{}, std::integral_constant<int, 2>{});
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();                                      // (one arrival per warp: they are taken one by one)
      if (lane == 0) ptx::mbar_arrive(&sh.p_full[x]);
      if (!(x ? w.last() : w.last_a())) continue;
      // ---- the block's last tile: its rows leave
      if (!wait(&sh.o_done[x], n_o & 1)) break;
      ++n_o;
      umma::fence_after_sync();
      const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
      const int64_t out_row = (((int64_t)w.l * p.rows + w.row0 + t_q) * p.H + w.h) * kLatV;
#pragma unroll
      for (int c0 = 0; c0 < kLatV; c0 += 32) {
        uint32_t o[32];
        umma::tmem_ld32(o_addr + c0, o);
        umma::tmem_ld_wait();
        if (t_q < w.T) {
          if (p.out_bf16) {
#pragma unroll
            for (int c = 0; c < 32; c += 8)
              *reinterpret_cast<uint4*>((__nv_bfloat16*)p.out + out_row + c0 + c) =
                  make_uint4(ptx::pack_bf16x2(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv),
                             ptx::pack_bf16x2(__uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv),
                             ptx::pack_bf16x2(__uint_as_float(o[c + 4]) * inv, __uint_as_float(o[c + 5]) * inv),
                             ptx::pack_bf16x2(__uint_as_float(o[c + 6]) * inv, __uint_as_float(o[c + 7]) * inv));
          } else {
#pragma unroll
            for (int c = 0; c < 32; c += 4)
              *reinterpret_cast<float4*>((float*)p.out + out_row + c0 + c) =
                  make_float4(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv, __uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
          }
        }
      }
      if (p.lse && t_q < w.T)
        p.lse[((int64_t)w.l * p.H + w.h) * p.rows + w.row0 + t_q] = l_run > 0.f ? (m_use + log2f(l_run)) * 0.6931471805599453f : (l_run == 0.f ? -INFINITY : l_run);
      umma::fence_before_sync();                         // (the next item's first sums overwrite O once this thread has published its weights)
    }
  }
  // ---- every role has left its loops; nothing of this CTA is in flight any more
  umma::fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

int launch_latent_fwd(const LatentReplayParams& p, cudaStream_t stream) {
  const int64_t blocks = ((int64_t)p.max_len + 2 * kLatTile - 1) / (2 * kLatTile), items = blocks * p.L * p.B * p.H;
  if (items > 0x7fff0000LL) return NGC_ERR_UNSUPPORTED;
  Maps maps;
  const int64_t rows = (int64_t)p.L * p.rows;
  if (!make_token_map(&maps.q, p.q, kLatNope + p.dr, p.H, rows, kLatTile) || !make_token_map(&maps.kv, p.kv, kLatNope + kLatV, p.H, rows, kLatTile) ||
      !make_rows_map(&maps.kr, p.kr, rows, kLatTile, p.dr))
    return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce once;
  static int sms[kMaxDevices] = {0};
  int dev = -1;
  const int rc = once.run([] {
    int cur = -1;
    cudaError_t e = cudaGetDevice(&cur);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms[cur], cudaDevAttrMultiProcessorCount, cur);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(latent_fwd_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(latent_fwd_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    return e;
  }, &dev);
  if (rc != NGC_OK) return rc;
  const int grid = (int)(items < sms[dev] ? items : sms[dev]);
  NGC_CUDA_TRY(launch_pdl(p.tile_gone ? latent_fwd_kernel<true> : latent_fwd_kernel<false>, dim3(grid), dim3(kThreads), kSmemBytes, stream, maps, p));
  return launch_status();
}

}  // namespace ngc
