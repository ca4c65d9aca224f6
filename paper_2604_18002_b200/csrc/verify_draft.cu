// ngc_verify_draft: multi-round speculative sampling over a drafted tree.
//
// A cluster of up to 8 CTAs per sequence; every CTA owns a slice of the vocabulary, every warp a contiguous range of
// the slice.  All CTAs take the same walk from the same numbers, so only sums over the vocabulary are exchanged: each
// warp writes its own into the shared memory of all CTAs, one cluster barrier later everyone adds them in one order.
//
// The children of the current node are a ballot over the parents that the lanes of each warp hold.  What a test needs of
// the big rows, p(x) and q(x) at the parent, is fetched for all nodes at once before the walk: the walk itself reads shared
// memory only.  With draft rows, k rejections at a node leave w = max(p - c q, 0): the max of nested subtractions of
// non-negative multiples of q is the subtraction of their sum, so one number c stands for the whole residual and nothing is
// stored.  The sum after a rejection is also the one that the final draw needs; a vocabulary row is read again only if a
// second child is rejected.
//
// All decisions and sums are in fp64 (fp32 inputs are exact in it); multiplications and subtractions are kept apart (no
// fused multiply-add), so that the arithmetic is the one written down.  The final draw is an inverse CDF: the sums
// per CTA and per warp lead to a range of 1 / 64 of a large vocabulary, which the CTA that owns it scans.
//
// What bounds it: a rejection is a pass over two rows that waits for the one before.  One sequence, 131072 tokens: 9.3 us
// with none (launch, tree, one pass, draw), then 1.8 us each.  64 sequences: 15 us with none (a row each, 34 MB), 31 us
// with up to five, whose rows come from L2 after the first time.  Without draft rows there is one pass, the last: 48
// sequences of 50001 tokens and 33 nodes take 9.9 us (19.5 us when tried tokens were a list that every thread searched for
// every token).
#include <cooperative_groups.h>

#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

namespace cg = cooperative_groups;

enum { kModeDraft = 0, kModePoint = 1, kModeGreedy = 2 };
constexpr int kVerifyThreads = 256, kVerifyWarps = kVerifyThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kWords = NGC_TREE_MAX_NODES / 32;
constexpr int kUnroll = 4;                           // 16-byte loads a lane has in flight per row

struct VerifyParams {
  const int32_t* tokens;
  const int32_t* parent;
  const int32_t* n_nodes;
  const float* target;
  const float* draft;
  const float* uniforms;
  int32_t* path;
  int32_t* n_path;
  int32_t* next_token;
  int32_t* dev_status;
  int N, vocab;
};

struct VerifyShared {
  int parent[NGC_TREE_MAX_NODES], token[NGC_TREE_MAX_NODES], path[NGC_TREE_MAX_NODES];
  float u[NGC_TREE_MAX_NODES], p[NGC_TREE_MAX_NODES], q[NGC_TREE_MAX_NODES];     // p, q: of the node's token, at its parent
  double scan[kVerifyWarps];
  float warp_max[kVerifyWarps];
  int warp_arg[kVerifyWarps];
  // what the CTAs tell one another; two of each, so that one cluster barrier per exchange is enough
  double sums[2][kMaxCluster][kVerifyWarps];            // of all CTAs' warps, written by them
  float cta_max[2];
  int cta_arg[2];
  int last;
};

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// What is left of the current node's row after the rejections so far.
template <int MODE> struct Residual {
  const float* p;
  const float* q;
  const int* token;                                  // of the nodes
  double c;                                          // with draft rows
  uint32_t tried[kWords];                            // without: children whose token has no mass left
  // of a token that has not been tried
  __device__ __forceinline__ double of(float pv, float qv) const {
    if constexpr (MODE != kModeDraft) return (double)max_nan(pv, 0.f);
    const double w = (double)pv;
    const double rest = __dsub_rn(w, __dmul_rn(c, (double)qv));
    return rest < 0.0 ? 0.0 : rest;                  // a NaN stays one
  }
  __device__ __forceinline__ bool with_q() const { return MODE == kModeDraft && c != 0.0; }
  // f(token) for all tried ones
  template <typename F> __device__ __forceinline__ void for_tried(F f) const {
    if constexpr (MODE == kModePoint) {
#pragma unroll
      for (int k = 0; k < kWords; ++k)
        for (uint32_t bits = tried[k]; bits; bits &= bits - 1) f(token[32 * k + __ffs(bits) - 1]);
    }
  }
  // the same as far as tokens [lo, hi) are concerned: hardly any of them has been tried (whole warp)
  __device__ __forceinline__ Residual within(int lo, int hi) const {
    Residual r = *this;
    if constexpr (MODE == kModePoint) {
#pragma unroll
      for (int k = 0; k < kWords; ++k)
        if (tried[k]) {
          const int x = tried[k] >> (threadIdx.x & 31) & 1u ? token[32 * k + (threadIdx.x & 31)] : -1;
          r.tried[k] = __ballot_sync(0xffffffffu, x >= lo && x < hi);
        }
    }
    return r;
  }
  __device__ __forceinline__ double at(int x) const {
    float pv = p[x];
    for_tried([&](int y) { if (x == y) pv = 0.f; });
    return of(pv, with_q() ? q[x] : 0.f);
  }
};

// Four tokens of a row from x0 on, with `fill` in place of those outside [lo, hi).  One load where `vec` says that x0 is
// 16-byte aligned and all four are asked for.
__device__ __forceinline__ float4 load4(const float* row, int x0, int lo, int hi, bool vec, float fill) {
  if (vec && x0 >= lo && x0 + 4 <= hi) return *reinterpret_cast<const float4*>(row + x0);
  float4 v;
  v.x = x0 >= lo && x0 < hi ? row[x0] : fill;
  v.y = x0 + 1 >= lo && x0 + 1 < hi ? row[x0 + 1] : fill;
  v.z = x0 + 2 >= lo && x0 + 2 < hi ? row[x0 + 2] : fill;
  v.w = x0 + 3 >= lo && x0 + 3 < hi ? row[x0 + 3] : fill;
  return v;
}
// Places of a row that are 16-byte aligned: x with (x + phase) % 4 == 0.
__device__ __forceinline__ int row_phase(const float* row) { return (int)((uintptr_t)row >> 2) & 3; }

// Sum over this warp's range.
template <int MODE> __device__ __forceinline__ double range_sum(const Residual<MODE>& all, int lo, int hi) {
  const Residual<MODE> w = all.within(lo, hi);
  const int lane = threadIdx.x & 31, phase = row_phase(w.p);
  const bool with_q = w.with_q(), q_vec = with_q && row_phase(w.q) == phase;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int x0 = ((lo + phase) & ~3) - phase + 4 * lane; x0 < hi; x0 += 128 * kUnroll) {
    float4 pv[kUnroll], qv[kUnroll];
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      pv[e] = load4(w.p, x0 + 128 * e, lo, hi, true, 0.f);
      qv[e] = with_q ? load4(w.q, x0 + 128 * e, lo, hi, q_vec, 0.f) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    w.for_tried([&](int y) {
#pragma unroll
      for (int e = 0; e < kUnroll; ++e) {
        const int c = y - (x0 + 128 * e);
        if (c == 0) pv[e].x = 0.f;
        if (c == 1) pv[e].y = 0.f;
        if (c == 2) pv[e].z = 0.f;
        if (c == 3) pv[e].w = 0.f;
      }
    });
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      s[0] += w.of(pv[e].x, qv[e].x);
      s[1] += w.of(pv[e].y, qv[e].y);
      s[2] += w.of(pv[e].z, qv[e].z);
      s[3] += w.of(pv[e].w, qv[e].w);
    }
  }
  return warp_sum((s[0] + s[1]) + (s[2] + s[3]));
}

template <int MODE, int kCtasSm>
__global__ void __launch_bounds__(kVerifyThreads, kCtasSm) verify_draft_kernel(VerifyParams p) {
  __shared__ VerifyShared sh;
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int b = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  cluster.barrier_arrive();                          // (shared memory of a CTA may be written from outside once it runs)
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  // the tree, and of the big rows what the tests need: two rounds of loads for all nodes at once
  int n = p.N, pa = 0, x = 0;
  if (p.n_nodes) n = p.n_nodes[b];
  if (tid < p.N) {
    pa = p.parent[(int64_t)b * p.N + tid];
    x = p.tokens[(int64_t)b * p.N + tid];
    if (MODE != kModeGreedy) sh.u[tid] = p.uniforms[(int64_t)b * p.N + tid];
  }
  bool bad = n < 0 || n > p.N;
  if (bad) n = 0;
  const int64_t row0 = (int64_t)b * p.N * p.vocab;
  if (tid < n) {
    if (tid == 0) bad = pa != -1;
    else bad = pa < 0 || pa >= tid || x < 0 || x >= p.vocab;
    sh.parent[tid] = pa;
    sh.token[tid] = x;
    if (MODE != kModeGreedy && tid > 0 && !bad) {
      const float px = p.target[row0 + (int64_t)pa * p.vocab + x];
      const float qx = MODE == kModeDraft ? p.draft[row0 + (int64_t)pa * p.vocab + x] : 0.f;
      // NaN: one of the two is no probability, which counts if the child is tested
      sh.p[tid] = px < INFINITY && qx >= 0.f && qx < INFINITY ? px : NAN;
      if (MODE == kModeDraft) sh.q[tid] = qx;
    }
  }
  int status = __syncthreads_or(bad) ? NGC_DEV_BAD_TREE : NGC_DEV_OK;
  cluster.barrier_wait();

  // slices of the CTAs, ranges of the warps
  const int per_cta = (p.vocab + ctas - 1) / ctas, cta_lo = min(p.vocab, rank * per_cta), cta_hi = min(p.vocab, cta_lo + per_cta);
  const int per_warp = (per_cta + kVerifyWarps - 1) / kVerifyWarps;
  const int lo = min(cta_hi, cta_lo + warp * per_warp), hi = min(cta_hi, lo + per_warp);
  int exchange = 0;

  // sum of a residual over the vocabulary: the same value in every thread of the cluster; every CTA has all warps' sums
  auto vocab_sum = [&](const Residual<MODE>& w) {
    const double s = range_sum(w, lo, hi);
    if (lane < ctas) cluster.map_shared_rank(&sh, lane)->sums[exchange & 1][rank][warp] = s;
    cluster.sync();
    double t = 0.0;
    for (int i = lane; i < ctas * kVerifyWarps; i += 32) t += sh.sums[exchange & 1][i / kVerifyWarps][i % kVerifyWarps];
    ++exchange;
    return warp_sum(t);
  };
  // argmax of a row (the smallest index of equal values), or -1 if the row holds a NaN
  auto better = [](float v, int a, float& best, int& arg) {
    if (v > best || (v == best && a < arg)) { best = v; arg = a; }
  };
  auto warp_best = [&](float& best, int& arg) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float v = __shfl_xor_sync(0xffffffffu, best, o);
      const int a = __shfl_xor_sync(0xffffffffu, arg, o);
      better(v, a, best, arg);
    }
  };
  auto row_argmax = [&](const float* row) {
    float best = -INFINITY;
    int arg = 0x7fffffff;
    bool nan = false;
    const int phase = row_phase(row);
    for (int x0 = ((lo + phase) & ~3) - phase + 4 * lane; x0 < hi; x0 += 128 * kUnroll) {
      float4 v[kUnroll];
#pragma unroll
      for (int e = 0; e < kUnroll; ++e) v[e] = load4(row, x0 + 128 * e, lo, hi, true, -INFINITY);
#pragma unroll
      for (int e = 0; e < kUnroll; ++e) {
        const float at[4] = {v[e].x, v[e].y, v[e].z, v[e].w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int x = x0 + 128 * e + c;
          nan = nan || at[c] != at[c];
          if (x >= lo && x < hi) better(at[c], x, best, arg);
        }
      }
    }
    warp_best(best, arg);
    nan = __syncthreads_or(nan);
    if (lane == 0) { sh.warp_max[warp] = best; sh.warp_arg[warp] = arg; }
    __syncthreads();
    if (warp == 0) {
      best = lane < kVerifyWarps ? sh.warp_max[lane] : -INFINITY;
      arg = lane < kVerifyWarps ? sh.warp_arg[lane] : 0x7fffffff;
      warp_best(best, arg);
      if (lane == 0) { sh.cta_max[exchange & 1] = best; sh.cta_arg[exchange & 1] = nan ? -1 : arg; }
    }
    cluster.sync();
    best = lane < ctas ? cluster.map_shared_rank(sh.cta_max, lane)[exchange & 1] : -INFINITY;
    arg = lane < ctas ? cluster.map_shared_rank(sh.cta_arg, lane)[exchange & 1] : 0x7fffffff;
    ++exchange;
    nan = __any_sync(0xffffffffu, arg < 0);
    warp_best(best, arg);
    return nan ? -1 : arg;
  };

  int n_path = 0, next = -1;
  bool draws = false;                                // this CTA holds the token of the final draw
  if (status == NGC_DEV_OK && n > 0) {
    double mass = 1.0;
    bool summed = false;                             // mass is the sum of w as it stands, its shares are in shared memory
    Residual<MODE> w = {p.target + row0, MODE == kModeDraft ? p.draft + row0 : nullptr, sh.token, 0.0, {}};
    // parents and tokens of the nodes, spread over the lanes: children and tokens are found by ballots
    int par[kWords], tok[kWords];
    uint32_t kids[kWords];                           // children of the current node that have not been tested
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      par[k] = lane + 32 * k < n ? sh.parent[lane + 32 * k] : -2;
      tok[k] = MODE == kModePoint && lane + 32 * k < n ? sh.token[lane + 32 * k] : -1;
      kids[k] = 32 * k < n ? __ballot_sync(0xffffffffu, par[k] == 0) : 0u;
    }
    int best = MODE == kModeGreedy ? row_argmax(w.p) : 0;
    if (tid == 0) sh.path[0] = 0;
    n_path = 1;
    while (status == NGC_DEV_OK && best >= 0) {
      int i = 0;
#pragma unroll
      for (int k = 0; k < kWords; ++k)
        if (i == 0 && kids[k]) {
          i = 32 * k + __ffs(kids[k]) - 1;
          kids[k] &= kids[k] - 1;
        }
      if (i == 0) break;
      const int x = sh.token[i];
      bool ok;
      if (MODE == kModeGreedy) {
        ok = x == best;
      } else {
        uint32_t again = 0;                          // children with the same token that were tried before
        if constexpr (MODE == kModePoint) {
#pragma unroll
          for (int k = 0; k < kWords; ++k)
            if (w.tried[k]) again |= __ballot_sync(0xffffffffu, tok[k] == x) & w.tried[k];
        }
        if (!(sh.p[i] >= 0.f)) {                     // (marked above; nothing else would notice in a row that is not summed)
          status = NGC_DEV_BAD_PROBS;
          break;
        }
        const double wx = again ? 0.0 : w.of(sh.p[i], MODE == kModeDraft ? sh.q[i] : 0.f), u = (double)sh.u[i];
        ok = MODE == kModeDraft ? __dmul_rn(__dmul_rn(u, (double)sh.q[i]), mass) < wx : __dmul_rn(u, mass) < wx;
        if (!ok && MODE == kModeDraft) {
          const double c = w.c;
          w.c = __dadd_rn(c, mass);
          const double rest = vocab_sum(w);
          summed = rest > 0.0;
          if (!isfinite(rest)) status = NGC_DEV_BAD_PROBS;
          else if (rest > 0.0) mass = rest;
          else w.c = c;
        } else if (!ok) {
          const double rest = __dsub_rn(mass, wx);
          if (rest > 0.0) {
            mass = rest;
#pragma unroll
            for (int k = 0; k < kWords; ++k) w.tried[k] |= i >> 5 == k ? 1u << (i & 31) : 0u;
          }
        }
      }
      if (ok) {
        if (tid == 0) sh.path[n_path] = i;
        ++n_path;
        w.p = p.target + row0 + (int64_t)i * p.vocab;
        if (MODE == kModeDraft) w.q = p.draft + row0 + (int64_t)i * p.vocab;
        w.c = 0.0;
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
          w.tried[k] = 0;
          kids[k] = 32 * k < n ? __ballot_sync(0xffffffffu, par[k] == i) : 0u;
        }
        mass = 1.0;
        summed = false;
        if (MODE == kModeGreedy) best = row_argmax(w.p);
      }
    }
    if (MODE == kModeGreedy) {
      next = best;
      draws = rank == 0;
      if (best < 0) status = NGC_DEV_BAD_PROBS;
    } else if (status == NGC_DEV_OK) {
      const double total = summed ? mass : vocab_sum(w);
      if (!isfinite(total) || !(total > 0.0)) {
        status = NGC_DEV_BAD_PROBS;
      } else {
        // the CTA and the warp range that the target falls into; rounding may leave it at the very end: then the last
        // token with mass
        double t = __dmul_rn((double)sh.u[0], total), before = 0.0;
        const int slot = (exchange - 1) & 1;         // of the sums of w as it stands
        double share = 0.0;                          // lane i: CTA i
        if (lane < ctas)
          for (int i = 0; i < kVerifyWarps; ++i) share += sh.sums[slot][lane][i];
        int own = -1, last = 0;
        double last_before = 0.0;
        for (int i = 0; i < ctas; ++i) {
          const double s = __shfl_sync(0xffffffffu, share, i);
          if (s > 0.0) { last = i; last_before = before; }
          if (own < 0 && before + s > t) own = i;
          if (own < 0) before += s;
        }
        if (own < 0) { own = last; before = last_before; t = INFINITY; }
        draws = rank == own;
        if (draws) {
          int range = -1;
          last = 0;
          const double shares = lane < kVerifyWarps ? sh.sums[slot][rank][lane] : 0.0;
          for (int i = 0; i < kVerifyWarps; ++i) {
            const double s = __shfl_sync(0xffffffffu, shares, i);
            if (s > 0.0) { last = i; last_before = before; }
            if (range < 0 && before + s > t) range = i;
            if (range < 0) before += s;
          }
          if (range < 0) { range = last; before = last_before; t = INFINITY; }
          // the whole CTA scans the range: a run of consecutive tokens per thread
          const int r_lo = min(cta_hi, cta_lo + range * per_warp), r_hi = min(cta_hi, r_lo + per_warp);
          const int run = (per_warp + kVerifyThreads - 1) / kVerifyThreads;
          const int x0 = min(r_hi, r_lo + tid * run), x1 = min(r_hi, x0 + run);
          const Residual<MODE> part = w.within(r_lo, r_hi);
          double s = 0.0;
          int tail = -1;
          for (int x = x0; x < x1; ++x) {
            const double wx = part.at(x);
            s += wx;
            if (wx > 0.0) tail = x;
          }
          double c = s;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += y;
          }
          if (tid == 0) { sh.last = -1; sh.warp_arg[0] = 0x7fffffff; }
          if (lane == 31) sh.scan[warp] = c;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < kVerifyWarps; ++i) before += i < warp ? sh.scan[i] : 0.0;
          // (rounding may begin a run beyond the target already: a token without mass is passed over all the same)
          double upto = before + (c - s);
          int hit = -1;
          if (upto + s > t)
            for (int x = x0; x < x1 && hit < 0; ++x) {
              const double wx = part.at(x);
              upto += wx;
              if (wx > 0.0 && upto > t) hit = x;
            }
          if (hit >= 0) atomicMin(&sh.warp_arg[0], hit);
          if (tail >= 0) atomicMax(&sh.last, tail);
          __syncthreads();
          next = sh.warp_arg[0] != 0x7fffffff ? sh.warp_arg[0] : sh.last;
        }
      }
    }
  }
  if (status != NGC_DEV_OK || n == 0) {
    if (tid == 0 && status != NGC_DEV_OK) set_dev_status(p.dev_status, status);
    n_path = 0;
    next = -1;
    draws = rank == 0;
  }
  __syncthreads();
  if (rank == 0) {
    for (int i = tid; i < p.N; i += kVerifyThreads) p.path[(int64_t)b * p.N + i] = i < n_path ? sh.path[i] : -1;
    if (tid == 0) p.n_path[b] = n_path;
  }
  if (draws && tid == 0) p.next_token[b] = next;
  cluster.sync();                                    // nobody leaves while its sums may still be read
}

}  // namespace
}  // namespace ngc

extern "C" int ngc_verify_draft(const int32_t* tokens, const int32_t* parent, const int32_t* n_nodes, const float* target_probs,
                                const float* draft_probs, const float* uniforms, int B, int N, int vocab, int greedy,
                                int32_t* path, int32_t* n_path, int32_t* next_token, int32_t* dev_status, ngc_stream stream) {
  NGC_API_RANGE("ngc_verify_draft");
  using namespace ngc;
  if (!tokens || !parent || !target_probs || !path || !n_path || !next_token || (!greedy && !uniforms) || B < 1 || N < 1 || vocab < 1)
    return NGC_ERR_INVALID_ARG;
  if (N > NGC_TREE_MAX_NODES || vocab > 1 << 30) return NGC_ERR_UNSUPPORTED;      // (indices a round ahead stay in 32 bits)
  const VerifyParams p = {tokens, parent, n_nodes, target_probs, draft_probs, uniforms, path, n_path, next_token, dev_status, N, vocab};
  // CTAs per sequence: a slice of at least 2048 tokens each, at most 8, and no more than one round of CTAs in all (four fit
  // an SM): a sequence that rejects many children takes many passes, which others should not queue behind.  256 threads each:
  // with 512 a sequence that rejects nothing takes longer (37 sequences: 21.4 instead of 14.4 us).
  int cluster = vocab / 2048;
  if (cluster > 4 * 148 / B) cluster = 4 * 148 / B;
  if (cluster > kMaxCluster) cluster = kMaxCluster;
  if (cluster < 1) cluster = 1;
  if ((int64_t)B * cluster > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(B * cluster)), block(kVerifyThreads);
  // With draft rows a thread has use for more registers than four CTAs per SM leave it (4 rejections, 131072 tokens, one
  // sequence: 18.5 us with 64 registers, 16.5 us with 80); where three per SM do not hold all CTAs at once, four are
  // better (64 sequences without a rejection: 21.2 us with three, 15.3 us with four).
  const bool three = (int64_t)B * cluster <= 3 * 148;
  auto kernel = greedy ? verify_draft_kernel<kModeGreedy, 4> : !draft_probs ? verify_draft_kernel<kModePoint, 4>
              : three  ? verify_draft_kernel<kModeDraft, 3> : verify_draft_kernel<kModeDraft, 4>;
  NGC_CUDA_TRY(launch_pdl_cluster(kernel, grid, block, (unsigned)cluster, 0, (cudaStream_t)stream, p));
  return NGC_OK;
}
