// The gradient of ngc_latent_replay_attn on the 5th-generation tensor cores.
//
// With the forward pass's lse and D = sum over channels of out * grad_out, P = exp(z - lse) and dz = P (dP - D), dP = dO V^T
// (the scale of z is applied to the finished sums).  Two kernels, each of which computes S and dP again, so that every sum lies in one
// CTA's tensor memory: no atomics, the same bits in every run.
//   queries   an item is 128 queries of a head; over its tiles of 64 keys: S = Q K^T, dP = dO V^T, dQ += dZ K.  Q and dO are copied to
//             tensor memory once per item and are A operands there, so the products read shared memory for keys and values alone, and
//             four tiles of K and three of V fit (tiles of 128 keys left room for two: rollouts of 8192 tokens 1126 -> 1151 us).
//             Tiles of 64 keys that no query of the item sees are passed over
//   keys      an item is 128 keys of a head; over the tiles of 64 queries that see them: S^T = K Q^T, dP^T = V dO^T,
//             dV += P^T dO, dK += dZ^T Q.  Keys are the lanes of tensor memory, so what a query sees is one range of columns per
//             thread.  64 queries because dV, dK (320 columns), S^T, dP^T and the bf16 P^T, dZ^T fill tensor memory
// P and dZ are A operands in tensor memory, in columns of their own: the scores of the next tile are computed while the softmax
// warps work on this one.  The head's share of the rotary keys' gradient goes to the workspace in fp32; a last kernel sums the heads
// in order.  Roles as in the forward pass: producers by TMA, a mender (rows behind a sequence's end are zeroed where they are
// summed over), one thread that issues all products, eight softmax warps (two per quarter of the lanes, half of the columns each; 16 warps
// changed nothing: 1016 -> 1012 us for the queries', 1028 for the keys').
//
// Bound by the tensor pipe and the hand-overs around it: causal, 4096 tokens of 16 heads, batch 2, the keys' kernel takes 342 us with the
// tensor pipe 73 % busy (a product of 128 x 64 reads its A operand, keys or values, from shared memory again for every tile, and dV,
// dK, S and dP leave tensor memory no room for it), the queries' 275 us with 57 % (S and dP have one buffer: dQ, Q and dO fill the
// rest).  8192 tokens: 2180 us, 820 TFLOP/s of the five products that the gradient needs; seven are computed.
#include <cuda.h>
#include <cuda_bf16.h>

#include "latent_replay_umma.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

constexpr int kMmaWarp = 8, kProducerWarp = 9, kMenderWarp = 10, kPlannerWarp = 11;
constexpr int kThreads = 12 * 32;
constexpr uint32_t kTmemCols = 512;
constexpr int kQBytes = 3 * kLatChunk, kVBytes = 2 * kLatChunk;          // 128 rows of 192 and of 128 channels

struct Maps { CUtensorMap q, kv, kr, go; };

// The row of 128 (or fewer) fp32 sums of this thread as bf16, `n` of them from column taddr on, times `f`.
__device__ __forceinline__ void store_bf16(uint32_t taddr, int n, float f, __nv_bfloat16* dst, bool mine) {
#pragma unroll 1
  for (int c0 = 0; c0 < n; c0 += 16) {
    uint32_t o[16];
    umma::tmem_ld16(taddr + c0, o);
    umma::tmem_ld_wait();
    if (!mine) continue;
#pragma unroll
    for (int c = 0; c < 16; c += 8)
      *reinterpret_cast<uint4*>(dst + c0 + c) =
          make_uint4(ptx::pack_bf16x2(__uint_as_float(o[c]) * f, __uint_as_float(o[c + 1]) * f),
                     ptx::pack_bf16x2(__uint_as_float(o[c + 2]) * f, __uint_as_float(o[c + 3]) * f),
                     ptx::pack_bf16x2(__uint_as_float(o[c + 4]) * f, __uint_as_float(o[c + 5]) * f),
                     ptx::pack_bf16x2(__uint_as_float(o[c + 6]) * f, __uint_as_float(o[c + 7]) * f));
  }
}

// ------------------------------------------------------------------------------------------------------------ queries

constexpr int kKTile = 64;                     // keys per tile
constexpr int kKChunk = kKTile * 128;          // 64 keys x 64 channels
constexpr int kStagesK = 4, kStagesV = 3;      // tiles of keys (3 chunks; in use until dQ has them) and of values (2 chunks; until dP)
constexpr int kSmemQ = kQBytes + kVBytes + kStagesK * 3 * kKChunk + kStagesV * 2 * kKChunk + 1024;

struct SharedQ {
  uint64_t k_full[kStagesK], k_raw[kStagesK], k_empty[kStagesK], v_empty[kStagesV];
  uint64_t sp_full, sp_free, z_full, z_empty, q_full, q_empty, a_full, dq_done, drain;
  uint32_t tmem;
  int abort;
  PlanRing ring;
};

__global__ void __launch_bounds__(kThreads, 1) latent_grad_q_kernel(const __grid_constant__ Maps maps, LatentReplayParams p) {
  extern __shared__ uint8_t smem_dyn[];
  __shared__ SharedQ sh;
  uint8_t* sQ = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
  uint8_t* sG = sQ + kQBytes;
  uint8_t* sK = sG + kVBytes;
  uint8_t* sV = sK + kStagesK * 3 * kKChunk;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 0) {
    if (lane < kStagesK) { ptx::mbar_init(&sh.k_full[lane], 2); ptx::mbar_init(&sh.k_raw[lane], 1); ptx::mbar_init(&sh.k_empty[lane], 1); }
    if (lane < kStagesV) ptx::mbar_init(&sh.v_empty[lane], 1);
    if (lane < kPlans) sh.ring.init(lane);
    if (lane == 31) {
      ptx::mbar_init(&sh.sp_full, 1); ptx::mbar_init(&sh.sp_free, 8); ptx::mbar_init(&sh.z_full, 8); ptx::mbar_init(&sh.z_empty, 1);
      ptx::mbar_init(&sh.q_full, 1); ptx::mbar_init(&sh.q_empty, 8); ptx::mbar_init(&sh.a_full, 8);
      ptx::mbar_init(&sh.dq_done, 1); ptx::mbar_init(&sh.drain, 1);
      sh.abort = 0;
    }
    ptx::fence_barrier_init();
  } else if (warp == kProducerWarp && lane == 0) {
    ptx::prefetch_tensormap(&maps.q); ptx::prefetch_tensormap(&maps.kv); ptx::prefetch_tensormap(&maps.kr); ptx::prefetch_tensormap(&maps.go);
  }
  if (warp == kMmaWarp) umma::tmem_alloc(&sh.tmem, kTmemCols);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tmem = sh.tmem;
  constexpr uint32_t kO = 0, kQa = 192, kGa = 288, kS = 352, kP = 416, kZ = 480;         // columns of dQ, Q, dO, S, dP, dZ
  ptx::grid_dep_wait();
  const WalkEnv env{p, &sh.ring, &sh.abort};
  auto wait = [&](uint64_t* bar, uint32_t parity) { return env.wait(bar, parity); };

  if (warp == kProducerWarp) {
    HalfWalk w;
    int tk = 0, sk = 0, sv = 0, pk = 0, pv = 0;          // tiles loaded, stages, parities of their uses
    bool given_up = false;
    uint32_t through_raw = 0, raw_phase = 0;
    while (w.next(env)) {
      const int y = (int)((int64_t)w.w.l * p.rows + w.w.row0 + w.k0), h = w.w.h;
      const bool tail = w.k0 + kKTile > w.w.T;
      if (tk >= kStagesK && !wait(&sh.k_empty[sk], pk ^ 1)) break;
      if (umma::elect_one()) {
        uint64_t* bar = tail ? &sh.k_raw[sk] : &sh.k_full[sk];           // (k_full: one arrival for K, one for V)
        uint8_t* dst = sK + sk * 3 * kKChunk;
        ptx::mbar_expect_tx(bar, 3 * kKChunk);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(dst + c * kKChunk, &maps.kv, 64 * c, h, y, bar);
        ptx::tma_load_2d(dst + 2 * kKChunk, &maps.kr, 0, y, bar);
      }
      __syncwarp();
      through_raw = tail ? through_raw | 1u << sk : through_raw & ~(1u << sk);
      if (tail) raw_phase ^= 1u << sk;
      if (tk >= kStagesV && !wait(&sh.v_empty[sv], pv ^ 1)) { given_up = true; break; }
      if (umma::elect_one()) {
        ptx::mbar_expect_tx(&sh.k_full[sk], 2 * kKChunk);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(sV + (2 * sv + c) * kKChunk, &maps.kv, kLatNope + 64 * c, h, y, &sh.k_full[sk]);
      }
      __syncwarp();
      ++tk;
      if (++sk == kStagesK) { sk = 0; pk ^= 1; }
      if (++sv == kStagesV) { sv = 0; pv ^= 1; }
    }
    // nothing is in flight when the CTA ends (a tile given up half way: its keys, which have a second or so to come)
    for (int x = max(0, tk - kStagesK); x < tk; ++x) {
      const int s = x % kStagesK;
      if (through_raw >> s & 1) ptx::mbar_wait_bounded(&sh.k_raw[s], ((raw_phase >> s) & 1) ^ 1);
      ptx::mbar_wait_bounded(&sh.k_full[s], (x / kStagesK) & 1);
    }
    if (given_up) ptx::mbar_wait_bounded(through_raw >> sk & 1 ? &sh.k_raw[sk] : &sh.k_full[sk], through_raw >> sk & 1 ? ((raw_phase >> sk) & 1) ^ 1 : pk);
    __syncwarp();
  } else if (warp == kMenderWarp) {
    // keys behind the sequence's end: dQ sums over them
    HalfWalk w;
    uint32_t phase = 0;
    for (int t = 0; w.next(env); ++t) {
      const int s = t % kStagesK, n = w.w.T - w.k0;
      if (n >= kKTile) continue;
      if (!wait(&sh.k_raw[s], (phase >> s) & 1)) break;
      phase ^= 1u << s;
      for (int c = 0; c < 3; ++c)
        for (int x = n * 8 + lane; x < kKTile * 8; x += 32)
          *reinterpret_cast<uint4*>(sK + (3 * s + c) * kKChunk + x * 16) = make_uint4(0, 0, 0, 0);
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.k_full[s]);
    }
  } else if (warp == kPlannerWarp) {
    int n = 0;
    run_planner<HalfWalk>(env, kLatTile, true, [&](const HalfWalk& x, int k) {
      const QueryWalk<1>& w = x.w;
      if (k > 0 && !wait(&sh.q_empty, (k - 1) & 1)) return false;
      if (umma::elect_one()) {
        const int y = (int)((int64_t)w.l * p.rows + w.row0 + w.q0);
        ptx::mbar_expect_tx(&sh.q_full, kQBytes + kVBytes);
        for (int c = 0; c < 3; ++c) ptx::tma_load_3d(sQ + c * kLatChunk, &maps.q, 64 * c, w.h, y, &sh.q_full);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(sG + c * kLatChunk, &maps.go, 64 * c, w.h, y, &sh.q_full);
      }
      __syncwarp();
      ++n;
      return true;
    });
    if (n > 0) ptx::mbar_wait_bounded(&sh.q_full, (n - 1) & 1);
    __syncwarp();
  } else if (warp == kMmaWarp) {
    constexpr uint32_t idesc = umma::instr_desc(kLatTile, kKTile, false), idesc_q = umma::instr_desc(kLatTile, 192, true);
    const uint64_t hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
    const uint32_t v_lo = (ptx::smem_u32(sV) >> 4) | 1u << 16,
                   k_lo = ptx::smem_u32(sK) >> 4;
    const int steps_r = p.dr / 16;
    // One thread issues everything: scores of the next tile before the sums of this one; at an item's end the other way round, since
    // the next queries are still on their way.
    if (umma::elect_one()) {
      HalfWalk nxt;
      uint32_t flags = 0;                                // two bits for each of the tiles between scores and sums: first, last of an item
      int n_q = 0, ts = 0, tz = 0, sk = 0, pk = 0, sv = 0, sz = 0;       // query blocks begun, tiles whose scores, whose sums are issued; stages
      bool more = nxt.next<true>(env), fresh = true;     // fresh: nxt's scores are not issued yet
      while (more || tz < ts) {
        if (more && !(nxt.first && tz < ts)) {
          if (nxt.first && !env.wait_alone(&sh.a_full, n_q++ & 1)) break;
          if (!env.wait_alone(&sh.k_full[sk], pk) || (ts > 0 && !env.wait_alone(&sh.sp_free, (ts - 1) & 1))) break;
          umma::fence_after_sync();
          const uint32_t b = (k_lo + sk * (3 * kKChunk >> 4)) | 1u << 16, v = v_lo + sv * (2 * kKChunk >> 4);
#pragma unroll
          for (int k = 0; k < 12; ++k)
            if (k < 8 || k - 8 < steps_r)
              umma::mma_bf16_a_tmem(tmem + kS, tmem + kQa + 8 * k, hi | (b + (((k >> 2) * kKChunk + (k & 3) * 32) >> 4)), idesc, k > 0 ? 1u : 0u);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            umma::mma_bf16_a_tmem(tmem + kP, tmem + kGa + 8 * k, hi | (v + (((k >> 2) * kKChunk + (k & 3) * 32) >> 4)), idesc, k > 0 ? 1u : 0u);
          umma::commit(&sh.sp_full);
          umma::commit(&sh.v_empty[sv]);
          flags |= (uint32_t)((nxt.first ? 1 : 0) | (nxt.last ? 2 : 0)) << (2 * (ts & 1));
          ++ts;
          if (++sk == kStagesK) { sk = 0; pk ^= 1; }
          if (++sv == kStagesV) sv = 0;
          fresh = false;
        }
        if (tz + 1 < ts || (tz < ts && (!more || fresh))) {              // sums of the tile before, or of the last
          const int z = tz & 1;
          if (!env.wait_alone(&sh.z_full, z)) break;
          umma::fence_after_sync();
          const bool first = flags >> (2 * z) & 1, last = flags >> (2 * z) & 2;
          flags &= ~(3u << (2 * z));
          const uint32_t b = (k_lo + sz * (3 * kKChunk >> 4)) | (uint32_t)(kKChunk >> 4) << 16;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma::mma_bf16_a_tmem(tmem + kO, tmem + kZ + 8 * k, hi | (b + ((k * 2048) >> 4)), idesc_q, (!first || k > 0) ? 1u : 0u);
          umma::commit(&sh.k_empty[sz]);
          umma::commit(&sh.z_empty);
          if (last) umma::commit(&sh.dq_done);
          ++tz;
          if (++sz == kStagesK) sz = 0;
        }
        if (!fresh) {                                    // (while the products run: the thread's own instructions take long)
          more = more && nxt.next<true>(env);
          fresh = true;
        }
      }
      umma::commit(&sh.drain);
    }
    __syncwarp();
    ptx::mbar_wait_bounded(&sh.drain, 0);
    __syncwarp();
  } else {
    const int half = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    HalfWalk x;
    const QueryWalk<1>& w = x.w;
    float lse2 = 0.f, delta = 0.f;
    int n_items_done = 0;
    for (int t = 0; x.next(env); ++t) {
      const int t_q = w.q0 + row;
      const bool mine = t_q < w.T;
      if (x.first) {
        const int64_t at = ((int64_t)w.l * p.H + w.h) * p.rows + w.row0 + t_q;
        lse2 = mine ? p.lse[at] * 1.4426950408889634f : 0.f;
        delta = mine ? p.delta[at] : 0.f;
        // this query's channels from shared into tensor memory (the item before is done with its own: its last scores are here);
        // the products then read shared memory for keys and values alone
        if (!wait(&sh.q_full, n_items_done & 1)) break;
        auto copy = [&](const uint8_t* src, int piece0, int pieces, uint32_t dst) {      // 16-byte pieces of a row of 128-byte chunks
          for (int c = 0; c < pieces; c += 2) {
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int q = piece0 + c + e;
              *reinterpret_cast<uint4*>(v + 4 * e) = *reinterpret_cast<const uint4*>(src + (q >> 3) * kLatChunk + row * 128 + (((q & 7) ^ (row & 7)) << 4));
            }
            umma::tmem_st8(lanes + dst + 4 * (piece0 + c), v);
          }
        };
        copy(sQ, 12 * half, 12, kQa);
        copy(sG, 8 * half, 8, kGa);
        umma::tmem_st_wait();
        umma::fence_before_sync();
        __syncwarp();
        if (lane == 0) { ptx::mbar_arrive(&sh.a_full); ptx::mbar_arrive(&sh.q_empty); }
      }
      const int j0 = x.k0 + 32 * half;
      const bool plain = !w.tiles || (w.plain_a >> (w.i - w.window) & 1);
      // (asked for before the wait: the answer takes as long)
      const int g = plain ? 0 : p.gone[((int64_t)w.b * p.G + list_of(p.lists, w.l, 0, 1)) * p.gone_cap + j0 + lane];
      if (!wait(&sh.sp_full, t & 1)) break;
      umma::fence_after_sync();
      uint32_t z[32], d[32];
      umma::tmem_ld32(lanes + kS + 32 * half, z);
      umma::tmem_ld32(lanes + kP + 32 * half, d);
      umma::tmem_ld_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.sp_free);
      uint32_t seen = 0xffffffffu;                       // bit j: this query sees key j0 + j
      const int behind = t_q - j0;                       // keys behind the query do not count
      if (behind < 31) seen = behind < 0 ? 0u : (2u << behind) - 1u;
      if (!plain) {
        const uint32_t lo = __ballot_sync(0xffffffffu, g > w.q0 + kLatTile - 1);
        if (lo == __ballot_sync(0xffffffffu, g > w.q0)) {
          seen &= lo;
        } else {
          uint32_t m = 0;
#pragma unroll
          for (int j = 0; j < 32; ++j) m |= __shfl_sync(0xffffffffu, g, j) > t_q ? 1u << j : 0u;
          seen &= m;
        }
      }
      uint32_t pk[16];
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        float e[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float pr = ptx::ex2_approx(fmaf(__uint_as_float(z[j + c]), p.scale_log2, -lse2));
          e[c] = (seen >> (j + c) & 1) ? pr * (__uint_as_float(d[j + c]) - delta) : 0.f;
        }
        pk[j >> 1] = ptx::pack_bf16x2(e[0], e[1]);
      }
      if (t > 0 && !wait(&sh.z_empty, (t - 1) & 1)) break;
      umma::tmem_st8(lanes + kZ + 16 * half, pk);
      umma::tmem_st8(lanes + kZ + 16 * half + 8, pk + 8);
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.z_full);
      if (!x.last) continue;
      if (!wait(&sh.dq_done, n_items_done++ & 1)) break;
      umma::fence_after_sync();
      __nv_bfloat16* dst = p.gq + (((int64_t)w.l * p.rows + w.row0 + t_q) * p.H + w.h) * (kLatNope + p.dr);
      // the first half of the warps: channels 0 .. 95, the others the rest
      if (half == 0) store_bf16(lanes + kO, 96, p.scale, dst, mine);
      else store_bf16(lanes + kO + 96, 32 + p.dr, p.scale, dst + 96, mine);
      umma::fence_before_sync();
    }
  }
  umma::fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, kTmemCols);
  }
}

// --------------------------------------------------------------------------------------------------------------- keys

constexpr int kQTile = KeyWalk::kQ;
constexpr int kQChunk = kQTile * 128;          // 64 queries x 64 channels
constexpr int kStageBytes = 5 * kQChunk;           // Q: 3 chunks, dO: 2
constexpr int kStages = 3;
constexpr int kSmemK = kQBytes + kVBytes + kStages * kStageBytes + 1024;

struct SharedK {
  uint64_t full[kStages], raw[kStages], empty[kStages], kv_full, kv_empty, sp_full, sp_free, z_full, z_empty, done, drain;
  uint32_t tmem;
  int abort;
  PlanRing ring;
  float2 rows[8][2][32];                       // per warp, two buffers: (lse in log2 units, D) of its columns' queries
};

__global__ void __launch_bounds__(kThreads, 1) latent_grad_kv_kernel(const __grid_constant__ Maps maps, LatentReplayParams p) {
  extern __shared__ uint8_t smem_dyn[];
  __shared__ SharedK sh;
  uint8_t* sK = (uint8_t*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
  uint8_t* sV = sK + kQBytes;
  uint8_t* stage = sV + kVBytes;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 0) {
    if (lane < kStages) { ptx::mbar_init(&sh.full[lane], 1); ptx::mbar_init(&sh.raw[lane], 1); ptx::mbar_init(&sh.empty[lane], 1); }
    if (lane < kPlans) sh.ring.init(lane);
    if (lane == 31) {
      ptx::mbar_init(&sh.kv_full, 1); ptx::mbar_init(&sh.kv_empty, 1); ptx::mbar_init(&sh.sp_full, 1); ptx::mbar_init(&sh.sp_free, 8);
      ptx::mbar_init(&sh.z_full, 8); ptx::mbar_init(&sh.z_empty, 1); ptx::mbar_init(&sh.done, 1); ptx::mbar_init(&sh.drain, 1);
      sh.abort = 0;
    }
    ptx::fence_barrier_init();
  } else if (warp == kProducerWarp && lane == 0) {
    ptx::prefetch_tensormap(&maps.q); ptx::prefetch_tensormap(&maps.kv); ptx::prefetch_tensormap(&maps.kr); ptx::prefetch_tensormap(&maps.go);
  }
  if (warp == kMmaWarp) umma::tmem_alloc(&sh.tmem, kTmemCols);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tmem = sh.tmem;
  constexpr uint32_t kDv = 0, kDk = 128, kS = 320, kDp = 384, kP = 448, kZ = 480;        // columns
  ptx::grid_dep_wait();
  const WalkEnv env{p, &sh.ring, &sh.abort};
  auto wait = [&](uint64_t* bar, uint32_t parity) { return env.wait(bar, parity); };

  if (warp == kProducerWarp) {
    KeyWalk w;
    int t = 0, s = 0, phase = 0;
    uint32_t through_raw = 0, raw_phase = 0;
    while (w.next(env)) {
      if (t >= kStages && !wait(&sh.empty[s], phase ^ 1)) break;
      const bool tail = (w.i + 1) * kQTile > w.T;
      const int y = (int)((int64_t)w.l * p.rows + w.row0 + w.i * kQTile);
      if (umma::elect_one()) {
        uint64_t* bar = tail ? &sh.raw[s] : &sh.full[s];
        uint8_t* dst = stage + s * kStageBytes;
        ptx::mbar_expect_tx(bar, kStageBytes);
        for (int c = 0; c < 3; ++c) ptx::tma_load_3d(dst + c * kQChunk, &maps.q, 64 * c, w.h, y, bar);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(dst + (3 + c) * kQChunk, &maps.go, 64 * c, w.h, y, bar);
      }
      __syncwarp();
      through_raw = tail ? through_raw | 1u << s : through_raw & ~(1u << s);
      if (tail) raw_phase ^= 1u << s;
      ++t;
      if (++s == kStages) { s = 0; phase ^= 1; }
    }
    for (int x = max(0, t - kStages); x < t; ++x) {     // nothing is in flight when the CTA ends
      const int k = x % kStages;
      if (through_raw >> k & 1) ptx::mbar_wait_bounded(&sh.raw[k], ((raw_phase >> k) & 1) ^ 1);
      else ptx::mbar_wait_bounded(&sh.full[k], (x / kStages) & 1);
    }
    __syncwarp();
  } else if (warp == kMenderWarp) {
    // queries behind the sequence's end: dV and dK sum over them
    KeyWalk w;
    uint32_t raw_phase = 0;
    for (int t = 0; w.next(env); ++t) {
      if ((w.i + 1) * kQTile <= w.T) continue;
      const int s = t % kStages, n = w.T - w.i * kQTile;
      if (!wait(&sh.raw[s], (raw_phase >> s) & 1)) break;
      raw_phase ^= 1u << s;
      for (int c = 0; c < 5; ++c)
        for (int x = n * 8 + lane; x < kQTile * 8; x += 32)
          *reinterpret_cast<uint4*>(stage + s * kStageBytes + c * kQChunk + x * 16) = make_uint4(0, 0, 0, 0);
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.full[s]);
    }
  } else if (warp == kPlannerWarp) {
    int n = 0;
    run_planner<KeyWalk>(env, kLatTile, false, [&](const KeyWalk& w, int k) {
      if (k > 0 && !wait(&sh.kv_empty, (k - 1) & 1)) return false;
      if (umma::elect_one()) {
        const int y = (int)((int64_t)w.l * p.rows + w.row0 + w.j0);
        ptx::mbar_expect_tx(&sh.kv_full, kQBytes + kVBytes);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(sK + c * kLatChunk, &maps.kv, 64 * c, w.h, y, &sh.kv_full);
        ptx::tma_load_2d(sK + 2 * kLatChunk, &maps.kr, 0, y, &sh.kv_full);
        for (int c = 0; c < 2; ++c) ptx::tma_load_3d(sV + c * kLatChunk, &maps.kv, kLatNope + 64 * c, w.h, y, &sh.kv_full);
      }
      __syncwarp();
      ++n;
      return true;
    });
    if (n > 0) ptx::mbar_wait_bounded(&sh.kv_full, (n - 1) & 1);
    __syncwarp();
  } else if (warp == kMmaWarp) {
    constexpr uint32_t idesc = umma::instr_desc(kLatTile, kQTile, false), idesc_v = umma::instr_desc(kLatTile, kLatV, true),
                       idesc_k = umma::instr_desc(kLatTile, 192, true);
    const uint64_t hi = (uint64_t)umma::smem_desc_sw128(0, 0, 1024) & 0xffffffff00000000ull;
    const uint32_t k_lo = (ptx::smem_u32(sK) >> 4) | 1u << 16, v_lo = (ptx::smem_u32(sV) >> 4) | 1u << 16, st_lo = ptx::smem_u32(stage) >> 4;
    const int steps_r = p.dr / 16;
    if (umma::elect_one()) {
      KeyWalk nxt;
      umma::Patience patience;
      uint32_t flags = 0;                                // of the two tiles between scores and sums: first, last of an item
      int n_k = 0, ts = 0, tz = 0, s_nxt = 0, ph_nxt = 0, s_cur = 0;
      bool more = nxt.next<true>(env);
      while (more || tz < ts) {
        bool moved = false;
        if (more && ts <= tz + 1 && ptx::mbar_test_wait(&sh.full[s_nxt], ph_nxt) && (ts == 0 || ptx::mbar_test_wait(&sh.sp_free, (ts - 1) & 1)) &&
            (!nxt.first || ptx::mbar_test_wait(&sh.kv_full, n_k & 1))) {
          umma::fence_after_sync();
          const uint32_t b = (st_lo + s_nxt * (kStageBytes >> 4)) | 1u << 16;
#pragma unroll
          for (int k = 0; k < 12; ++k)
            if (k < 8 || k - 8 < steps_r)
              umma::mma_bf16(tmem + kS, hi | (k_lo + (((k >> 2) * kLatChunk + (k & 3) * 32) >> 4)), hi | (b + (((k >> 2) * kQChunk + (k & 3) * 32) >> 4)),
                             idesc, k > 0 ? 1u : 0u);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            umma::mma_bf16(tmem + kDp, hi | (v_lo + (((k >> 2) * kLatChunk + (k & 3) * 32) >> 4)),
                           hi | (b + (((3 + (k >> 2)) * kQChunk + (k & 3) * 32) >> 4)), idesc, k > 0 ? 1u : 0u);
          umma::commit(&sh.sp_full);
          if (nxt.last()) umma::commit(&sh.kv_empty);
          n_k += nxt.first;
          if (++s_nxt == kStages) { s_nxt = 0; ph_nxt ^= 1; }
          flags |= (uint32_t)((nxt.first ? 1 : 0) | (nxt.last() ? 2 : 0)) << (2 * (ts & 1));
          ++ts;
          moved = true;
          more = nxt.next<true>(env);
        }
        if (tz < ts && ptx::mbar_test_wait(&sh.z_full, tz & 1)) {
          umma::fence_after_sync();
          const bool first = flags >> (2 * (tz & 1)) & 1, last = flags >> (2 * (tz & 1)) & 2;
          flags &= ~(3u << (2 * (tz & 1)));
          const uint32_t b = (st_lo + s_cur * (kStageBytes >> 4)) | (uint32_t)(kQChunk >> 4) << 16;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma::mma_bf16_a_tmem(tmem + kDv, tmem + kP + 8 * k, hi | (b + ((3 * kQChunk + k * 2048) >> 4)), idesc_v, (!first || k > 0) ? 1u : 0u);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma::mma_bf16_a_tmem(tmem + kDk, tmem + kZ + 8 * k, hi | (b + ((k * 2048) >> 4)), idesc_k, (!first || k > 0) ? 1u : 0u);
          umma::commit(&sh.empty[s_cur]);
          umma::commit(&sh.z_empty);
          if (last) umma::commit(&sh.done);
          if (++s_cur == kStages) s_cur = 0;
          ++tz;
          moved = true;
        }
        if (moved) patience.moved();
        else if (!patience.more(&sh.abort, p.dev_status)) break;
      }
      umma::commit(&sh.drain);
    }
    __syncwarp();
    ptx::mbar_wait_bounded(&sh.drain, 0);
    __syncwarp();
  } else {
    const int half = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    KeyWalk w;
    int lo = 0, hi = 0, n_done = 0;                      // queries that see this thread's key: lo .. hi - 1
    const float* lse = nullptr;
    const float* delta = nullptr;
    float2 ahead = make_float2(0.f, 0.f);
    for (int t = 0; w.next(env); ++t) {
      const int j = w.j0 + row;
      if (w.first) {
        lo = j;
        hi = j < w.T ? w.T : 0;
        if (p.gone && j < w.T) hi = min(hi, p.gone[((int64_t)w.b * p.G + list_of(p.lists, w.l, 0, 1)) * p.gone_cap + j]);
        const int64_t at = ((int64_t)w.l * p.H + w.h) * p.rows + w.row0;
        lse = p.lse + at;
        delta = p.delta + at;
      }
      const int t0 = w.i * kQTile + 32 * half;
      auto row_of = [&](int t_q) { return t_q < w.T ? make_float2(lse[t_q] * 1.4426950408889634f, delta[t_q]) : make_float2(0.f, 0.f); };
      if (w.first) ahead = row_of(t0 + lane);
      sh.rows[warp][t & 1][lane] = ahead;
      __syncwarp();
      if (!w.last()) ahead = row_of(t0 + kQTile + lane);     // the next tile's, a tile early
      if (!wait(&sh.sp_full, t & 1)) break;
      umma::fence_after_sync();
      uint32_t z[32], d[32];
      umma::tmem_ld32(lanes + kS + 32 * half, z);
      umma::tmem_ld32(lanes + kDp + 32 * half, d);
      umma::tmem_ld_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.sp_free);
      const int c_lo = max(lo - t0, 0);
      const uint32_t width = (uint32_t)max(hi - t0 - c_lo, 0);
      uint32_t pp[16], pz[16];
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        const float4 r = *reinterpret_cast<const float4*>(&sh.rows[warp][t & 1][c]);
        float e0 = ptx::ex2_approx(fmaf(__uint_as_float(z[c]), p.scale_log2, -r.x)), e1 = ptx::ex2_approx(fmaf(__uint_as_float(z[c + 1]), p.scale_log2, -r.z));
        const bool s0 = (uint32_t)(c - c_lo) < width, s1 = (uint32_t)(c + 1 - c_lo) < width;
        e0 = s0 ? e0 : 0.f;
        e1 = s1 ? e1 : 0.f;
        pp[c >> 1] = ptx::pack_bf16x2(e0, e1);
        pz[c >> 1] = ptx::pack_bf16x2(s0 ? e0 * (__uint_as_float(d[c]) - r.y) : 0.f, s1 ? e1 * (__uint_as_float(d[c + 1]) - r.w) : 0.f);
      }
      if (t > 0 && !wait(&sh.z_empty, (t - 1) & 1)) break;
      umma::tmem_st8(lanes + kP + 16 * half, pp);
      umma::tmem_st8(lanes + kP + 16 * half + 8, pp + 8);
      umma::tmem_st8(lanes + kZ + 16 * half, pz);
      umma::tmem_st8(lanes + kZ + 16 * half + 8, pz + 8);
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.z_full);
      if (!w.last()) continue;
      if (!wait(&sh.done, n_done++ & 1)) break;
      umma::fence_after_sync();
      const bool mine = j < w.T;
      __nv_bfloat16* dst = p.gkv + (((int64_t)w.l * p.rows + w.row0 + j) * p.H + w.h) * (kLatNope + kLatV);
      if (half == 0) {
        store_bf16(lanes + kDk, kLatNope, p.scale, dst, mine);
      } else {
        store_bf16(lanes + kDv, kLatV, 1.f, dst + kLatNope, mine);
        float* part = p.dkr_part + (((int64_t)w.l * p.H + w.h) * p.rows + w.row0 + j) * p.dr;
#pragma unroll 1
        for (int c0 = 0; c0 < p.dr; c0 += 16) {
          uint32_t o[16];
          umma::tmem_ld16(lanes + kDk + kLatNope + c0, o);
          umma::tmem_ld_wait();
          if (mine) {
#pragma unroll
            for (int c = 0; c < 16; c += 4)
              *reinterpret_cast<float4*>(part + c0 + c) = make_float4(__uint_as_float(o[c]) * p.scale, __uint_as_float(o[c + 1]) * p.scale,
                                                                      __uint_as_float(o[c + 2]) * p.scale, __uint_as_float(o[c + 3]) * p.scale);
          }
        }
      }
      umma::fence_before_sync();
    }
  }
  umma::fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    umma::fence_after_sync();
    umma::tmem_dealloc(tmem, kTmemCols);
  }
}

// ------------------------------------------------------------------------------------------- the heads' shares of the rotary keys

// Four channels of a token per thread, heads in order.  Bound by HBM: 60 MB in 12 us for 14.7 thousand tokens of 16 heads (5 TB/s).
__global__ void __launch_bounds__(256) latent_grad_rope_kernel(LatentReplayParams p) {
  const int b = blockIdx.y % p.B, l = blockIdx.y / p.B, per = p.dr / 4;
  int64_t row0;
  ptx::grid_dep_wait();
  const int T = latent_seq(p, b, row0);
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = x / per;
  const int c = 4 * (int)(x % per);
  if (t >= T) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  const float* part = p.dkr_part + ((int64_t)l * p.H * p.rows + row0 + t) * p.dr + c;
#pragma unroll 4
  for (int h = 0; h < p.H; ++h) {
    const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)h * p.rows * p.dr);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  *reinterpret_cast<uint2*>(p.gkr + ((int64_t)l * p.rows + row0 + t) * p.dr + c) = make_uint2(ptx::pack_bf16x2(s.x, s.y), ptx::pack_bf16x2(s.z, s.w));
}

}  // namespace

int launch_latent_bwd(const LatentReplayParams& p, cudaStream_t stream) {
  const int64_t items = ((int64_t)p.max_len + kLatTile - 1) / kLatTile * p.L * p.B * p.H;
  if (items > 0x7fff0000LL) return NGC_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)p.L * p.rows;
  Maps mq, mk;
  if (!make_token_map(&mq.q, p.q, kLatNope + p.dr, p.H, rows, kLatTile) || !make_token_map(&mq.kv, p.kv, kLatNope + kLatV, p.H, rows, kLatTile) ||
      !make_rows_map(&mq.kr, p.kr, rows, kLatTile, p.dr) || !make_token_map(&mq.go, p.go, kLatV, p.H, rows, kLatTile))
    return NGC_ERR_UNSUPPORTED;
  mk = mq;                                       // what is loaded once per item in boxes of 128 rows, tiles of 64
  if (!make_token_map(&mq.kv, p.kv, kLatNope + kLatV, p.H, rows, kKTile) || !make_rows_map(&mq.kr, p.kr, rows, kKTile, p.dr) ||
      !make_token_map(&mk.q, p.q, kLatNope + p.dr, p.H, rows, kQTile) || !make_token_map(&mk.go, p.go, kLatV, p.H, rows, kQTile))
    return NGC_ERR_UNSUPPORTED;
  static PerDeviceOnce once;
  static int sms[kMaxDevices] = {0};
  int dev = -1;
  const int rc = once.run([] {
    int cur = -1;
    cudaError_t e = cudaGetDevice(&cur);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms[cur], cudaDevAttrMultiProcessorCount, cur);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(latent_grad_q_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemQ);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(latent_grad_kv_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemK);
    return e;
  }, &dev);
  if (rc != NGC_OK) return rc;
  const int grid = (int)(items < sms[dev] ? items : sms[dev]);
  NGC_CUDA_TRY(launch_pdl(latent_grad_kv_kernel, dim3(grid), dim3(kThreads), kSmemK, stream, mk, p));
  NGC_CUDA_TRY(launch_pdl(latent_grad_q_kernel, dim3(grid), dim3(kThreads), kSmemQ, stream, mq, p));
  const dim3 g((unsigned)(((int64_t)p.max_len * (p.dr / 4) + 255) / 256), p.L * p.B);
  NGC_CUDA_TRY(launch_pdl(latent_grad_rope_kernel, g, dim3(256), 0, stream, p));
  return launch_status();
}

}  // namespace ngc
