// ngc_verify_draft: multi-round speculative sampling over a drafted tree.
//
// A cluster of up to 8 CTAs per sequence; every CTA owns a slice of the vocabulary, every warp a contiguous range of
// the slice.  All CTAs take the same walk from the same numbers, so only sums over the vocabulary are exchanged (one
// number per CTA through distributed shared memory, added in rank order).
//
// Nodes are numbered with parents before children, so one ascending sweep over the nodes visits the children of
// the current node in index order.  What a test needs of the big rows, p(x) and q(x) at the parent, is fetched for
// all nodes at once before the walk: the walk itself reads shared memory only.  With draft rows, k rejections at
// a node leave w = max(p - c q, 0): the max of nested subtractions of non-negative multiples of q is the subtraction
// of their sum, so one number c stands for the whole residual and nothing is stored.  The sum after a rejection
// is also the one that the final draw needs; a vocabulary row is read again only if a second child is rejected.
//
// All decisions and sums are in fp64 (fp32 inputs are exact in it); multiplications and subtractions are kept apart (no
// fused multiply-add), so that the arithmetic is the one written down.  The final draw is an inverse CDF: the sums
// per CTA and per warp lead to a range of 1 / 64 or 1 / 128 of the vocabulary (8 CTAs of 8 or 16 warps), which the CTA
// that owns it scans.
#include <cooperative_groups.h>

#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

namespace cg = cooperative_groups;

enum { kModeDraft = 0, kModePoint = 1, kModeGreedy = 2 };
constexpr int kMaxWarps = 16;                        // per CTA
constexpr int kMaxCluster = 8;
constexpr int kUnroll = 8;                           // loads a lane has in flight per row

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
  int parent[NGC_TREE_MAX_NODES], token[NGC_TREE_MAX_NODES], path[NGC_TREE_MAX_NODES], tried[NGC_TREE_MAX_NODES];
  float u[NGC_TREE_MAX_NODES], p[NGC_TREE_MAX_NODES], q[NGC_TREE_MAX_NODES];     // p, q: of the node's token, at its parent
  double warp_sum[kMaxWarps];
  float warp_max[kMaxWarps];
  int warp_arg[kMaxWarps];
  // what the other CTAs read; two of each, so that one cluster barrier per exchange is enough
  double cta_sum[2];
  float cta_max[2];
  int cta_arg[2];
  int last;
};

// What is left of the current node's row after the rejections so far.
template <int MODE> struct Residual {
  const float* p;
  const float* q;
  const int* tried;
  double c;
  int n_tried;
  __device__ __forceinline__ double of(int x, float pv, float qv) const {
    const double w = (double)pv;
    if constexpr (MODE == kModeDraft) {
      const double rest = __dsub_rn(w, __dmul_rn(c, (double)qv));
      return rest < 0.0 ? 0.0 : rest;                // a NaN stays one
    } else {
      for (int e = 0; e < n_tried; ++e)
        if (tried[e] == x) return 0.0;
      return w;
    }
  }
  __device__ __forceinline__ bool with_q() const { return MODE == kModeDraft && c != 0.0; }
  __device__ __forceinline__ double at(int x) const { return of(x, p[x], with_q() ? q[x] : 0.f); }
};

// Sum over this warp's range.
template <int MODE> __device__ __forceinline__ double range_sum(const Residual<MODE>& w, int lo, int hi) {
  const int lane = threadIdx.x & 31;
  const bool with_q = w.with_q();
  double s[2] = {0.0, 0.0};
  for (int x0 = lo + lane; x0 < hi; x0 += 32 * kUnroll) {
    float pv[kUnroll], qv[kUnroll];
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      const int x = x0 + 32 * e;
      pv[e] = x < hi ? w.p[x] : 0.f;
      qv[e] = with_q && x < hi ? w.q[x] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) s[e & 1] += w.of(x0 + 32 * e, pv[e], qv[e]);
  }
  return warp_sum(s[0] + s[1]);
}

template <int MODE, int kVerifyThreads>
__global__ void __launch_bounds__(kVerifyThreads, 1024 / kVerifyThreads) verify_draft_kernel(VerifyParams p) {
  constexpr int kVerifyWarps = kVerifyThreads / 32;
  __shared__ VerifyShared sh;
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int b = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
      sh.p[tid] = p.target[row0 + (int64_t)pa * p.vocab + x];
      if (MODE == kModeDraft) sh.q[tid] = p.draft[row0 + (int64_t)pa * p.vocab + x];
    }
  }
  int status = __syncthreads_or(bad) ? NGC_DEV_BAD_TREE : NGC_DEV_OK;

  // slices of the CTAs, ranges of the warps
  const int per_cta = (p.vocab + ctas - 1) / ctas, cta_lo = min(p.vocab, rank * per_cta), cta_hi = min(p.vocab, cta_lo + per_cta);
  const int per_warp = (per_cta + kVerifyWarps - 1) / kVerifyWarps;
  const int lo = min(cta_hi, cta_lo + warp * per_warp), hi = min(cta_hi, lo + per_warp);
  int exchange = 0;
  double share = 0.0;                                // lane i of every warp: the sum of CTA i's slice

  // sum of a residual over the vocabulary: the same value in every thread of the cluster; the shares of warps and CTAs stay
  auto vocab_sum = [&](const Residual<MODE>& w) {
    const double s = range_sum(w, lo, hi);
    __syncthreads();
    if (lane == 0) sh.warp_sum[warp] = s;
    __syncthreads();
    if (warp == 0) {
      const double t = warp_sum(lane < kVerifyWarps ? sh.warp_sum[lane] : 0.0);
      if (lane == 0) sh.cta_sum[exchange & 1] = t;
    }
    cluster.sync();
    share = lane < ctas ? cluster.map_shared_rank(sh.cta_sum, lane)[exchange & 1] : 0.0;
    ++exchange;
    return warp_sum(share);
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
    for (int x0 = lo + lane; x0 < hi; x0 += 32 * kUnroll) {
      float v[kUnroll];
#pragma unroll
      for (int e = 0; e < kUnroll; ++e) v[e] = x0 + 32 * e < hi ? row[x0 + 32 * e] : -INFINITY;
#pragma unroll
      for (int e = 0; e < kUnroll; ++e) {
        nan = nan || v[e] != v[e];
        if (x0 + 32 * e < hi) better(v[e], x0 + 32 * e, best, arg);
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
    int cur = 0;
    double mass = 1.0;
    bool summed = false;                             // mass is the sum of w as it stands, its shares are in shared memory
    Residual<MODE> w = {p.target + row0, MODE == kModeDraft ? p.draft + row0 : nullptr, sh.tried, 0.0, 0};
    int best = MODE == kModeGreedy ? row_argmax(w.p) : 0;
    if (tid == 0) sh.path[0] = 0;
    n_path = 1;
    for (int i = 1; i < n && status == NGC_DEV_OK && best >= 0; ++i) {
      if (sh.parent[i] != cur) continue;
      const int x = sh.token[i];
      bool ok;
      if (MODE == kModeGreedy) {
        ok = x == best;
      } else {
        const double wx = w.of(x, sh.p[i], MODE == kModeDraft ? sh.q[i] : 0.f), u = (double)sh.u[i];
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
            __syncthreads();                         // (reads of the list by w.of above are done)
            if (tid == 0) sh.tried[w.n_tried] = x;
            __syncthreads();
            ++w.n_tried;
          }
        }
      }
      if (ok) {
        cur = i;
        if (tid == 0) sh.path[n_path] = i;
        ++n_path;
        w.p = p.target + row0 + (int64_t)i * p.vocab;
        if (MODE == kModeDraft) w.q = p.draft + row0 + (int64_t)i * p.vocab;
        w.c = 0.0;
        w.n_tried = 0;
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
          const double shares = lane < kVerifyWarps ? sh.warp_sum[lane] : 0.0;
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
          double s = 0.0;
          int tail = -1;
          for (int x = x0; x < x1; ++x) {
            const double wx = w.at(x);
            s += wx;
            if (wx > 0.0) tail = x;
          }
          double c = s;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += y;
          }
          __syncthreads();                           // (warp_sum has been read)
          if (tid == 0) { sh.last = -1; sh.warp_arg[0] = 0x7fffffff; }
          if (lane == 31) sh.warp_sum[warp] = c;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < kVerifyWarps; ++i) before += i < warp ? sh.warp_sum[i] : 0.0;
          double upto = before + (c - s);
          int hit = -1;
          if (upto + s > t)
            for (int x = x0; x < x1 && hit < 0; ++x) {
              upto += w.at(x);
              if (upto > t) hit = x;
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
  // CTAs per sequence: a slice of at least 2048 tokens each, at most 8, and no more than one round of CTAs in all: a
  // sequence that rejects many children takes many passes, which others should not queue behind.  Few sequences get
  // twice the threads: then a pass is bound by each SM's conversions and latencies (4 rejections in 131072 tokens: 18.5 us
  // with 512 threads, 24.8 us with 256), else by how many CTAs are there at once (64 sequences: 46.7 and 42.3 us).
  const bool wide = (int64_t)B * kMaxCluster <= 2 * 148;
  int cluster = vocab / 2048;
  if (cluster > 4 * 148 / B) cluster = 4 * 148 / B;
  if (cluster > kMaxCluster) cluster = kMaxCluster;
  if (cluster < 1) cluster = 1;
  if ((int64_t)B * cluster > 0x7fffffffLL) return NGC_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(B * cluster)), block(wide ? 512 : 256);
  auto kernel = greedy ? (wide ? verify_draft_kernel<kModeGreedy, 512> : verify_draft_kernel<kModeGreedy, 256>)
              : draft_probs ? (wide ? verify_draft_kernel<kModeDraft, 512> : verify_draft_kernel<kModeDraft, 256>)
                            : (wide ? verify_draft_kernel<kModePoint, 512> : verify_draft_kernel<kModePoint, 256>);
  NGC_CUDA_TRY(launch_pdl_cluster(kernel, grid, block, (unsigned)cluster, (cudaStream_t)stream, p));
  return NGC_OK;
}
