// ngc_verify_draft: multi-round speculative sampling over a drafted tree.
//
// One CTA per sequence.  Nodes are numbered with parents before children, so one ascending sweep over
// the nodes visits the children of the current node in index order.  With draft rows, k rejections at
// a node leave w = max(p - c q, 0): the max of nested subtractions of non-negative multiples of q is the
// subtraction of their sum, so one number c stands for the whole residual and nothing is stored.  All
// decisions and sums are in fp64 (fp32 inputs are exact in it); multiplications and subtractions are
// kept apart (no fused multiply-add), so that the arithmetic is the one written down.
// The final draw is an inverse CDF: every warp owns a contiguous range of the vocabulary, the sums of the
// ranges give the range that the target falls into, and its warp walks it.
#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

enum { kModeDraft = 0, kModePoint = 1, kModeGreedy = 2 };
constexpr int kVerifyThreads = 1024, kVerifyWarps = kVerifyThreads / 32;

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
  float u[NGC_TREE_MAX_NODES];
  double warp_sum[kVerifyWarps];
  float warp_max[kVerifyWarps];
  int warp_arg[kVerifyWarps];
  int next;
};

// What is left of token x at the current node.
template <int MODE> struct Residual {
  const float* p;
  const float* q;
  const int* tried;
  double c;
  int n_tried;
  __device__ __forceinline__ double at(int x) const {
    double w = (double)p[x];
    if (MODE == kModeDraft) {
      w = __dsub_rn(w, __dmul_rn(c, (double)q[x]));
      return w < 0.0 ? 0.0 : w;                      // a NaN stays one
    }
    for (int e = 0; e < n_tried; ++e)
      if (tried[e] == x) return 0.0;
    return w;
  }
};

// Sum over the vocabulary; the warps' shares stay in sh.warp_sum.  Every thread gets the same value.
template <int MODE> __device__ double residual_sum(const Residual<MODE>& w, int lo, int hi, VerifyShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double s = 0.0;
  for (int x = lo + lane; x < hi; x += 32) s += w.at(x);
  s = warp_sum(s);
  __syncthreads();
  if (lane == 0) sh.warp_sum[warp] = s;
  __syncthreads();
  s = 0.0;
  for (int i = 0; i < kVerifyWarps; ++i) s += sh.warp_sum[i];
  return s;
}

// argmax of a row (the smallest index of equal values), or -1 if the row holds a NaN.
__device__ int row_argmax(const float* p, int lo, int hi, VerifyShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float best = -INFINITY;
  int arg = 0x7fffffff;
  bool nan = false;
  for (int x = lo + lane; x < hi; x += 32) {
    const float v = p[x];
    nan = nan || v != v;
    if (v > best || arg == 0x7fffffff) { best = v; arg = x; }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v = __shfl_xor_sync(0xffffffffu, best, o);
    const int a = __shfl_xor_sync(0xffffffffu, arg, o);
    if (v > best || (v == best && a < arg)) { best = v; arg = a; }
  }
  if (__syncthreads_or(nan)) return -1;
  if (lane == 0) { sh.warp_max[warp] = best; sh.warp_arg[warp] = arg; }
  __syncthreads();
  best = sh.warp_max[0];
  arg = sh.warp_arg[0];
  for (int i = 1; i < kVerifyWarps; ++i) {
    const float v = sh.warp_max[i];
    const int a = sh.warp_arg[i];
    if (v > best || (v == best && a < arg)) { best = v; arg = a; }
  }
  return arg;
}

template <int MODE> __global__ void __launch_bounds__(kVerifyThreads) verify_draft_kernel(VerifyParams p) {
  __shared__ VerifyShared sh;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  int n = p.n_nodes ? p.n_nodes[b] : p.N;
  bool bad = n < 0 || n > p.N;
  if (bad) n = 0;
  for (int i = tid; i < n; i += kVerifyThreads) {
    const int pa = p.parent[(int64_t)b * p.N + i], x = p.tokens[(int64_t)b * p.N + i];
    bad = bad || (i == 0 ? pa != -1 : (pa < 0 || pa >= i || x < 0 || x >= p.vocab));
    sh.parent[i] = pa;
    sh.token[i] = x;
    if (MODE != kModeGreedy) sh.u[i] = p.uniforms[(int64_t)b * p.N + i];
  }
  int status = __syncthreads_or(bad) ? NGC_DEV_BAD_TREE : NGC_DEV_OK;

  const int per_warp = (p.vocab + kVerifyWarps - 1) / kVerifyWarps;
  const int lo = min(p.vocab, warp * per_warp), hi = min(p.vocab, lo + per_warp);
  int n_path = 0, next = -1;
  if (status == NGC_DEV_OK && n > 0) {
    const int64_t row0 = (int64_t)b * p.N * p.vocab;
    int cur = 0;
    double mass = 1.0;
    Residual<MODE> w = {p.target + row0, MODE == kModeDraft ? p.draft + row0 : nullptr, sh.tried, 0.0, 0};
    int best = MODE == kModeGreedy ? row_argmax(w.p, lo, hi, sh) : 0;
    if (tid == 0) sh.path[0] = 0;
    n_path = 1;
    for (int i = 1; i < n && status == NGC_DEV_OK && best >= 0; ++i) {
      if (sh.parent[i] != cur) continue;
      const int x = sh.token[i];
      bool ok;
      if (MODE == kModeGreedy) {
        ok = x == best;
      } else {
        const double wx = w.at(x), u = (double)sh.u[i];
        ok = MODE == kModeDraft ? __dmul_rn(__dmul_rn(u, (double)w.q[x]), mass) < wx : __dmul_rn(u, mass) < wx;
        if (!ok && MODE == kModeDraft) {
          const double c = w.c;
          w.c = __dadd_rn(c, mass);
          const double rest = residual_sum(w, lo, hi, sh);
          if (!isfinite(rest)) status = NGC_DEV_BAD_PROBS;
          else if (rest > 0.0) mass = rest;
          else w.c = c;
        } else if (!ok) {
          const double rest = __dsub_rn(mass, wx);
          if (rest > 0.0) {
            mass = rest;
            __syncthreads();                         // (reads of the list by w.at above are done)
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
        if (MODE == kModeGreedy) best = row_argmax(w.p, lo, hi, sh);
      }
    }
    if (MODE == kModeGreedy) {
      next = best;
      if (best < 0) status = NGC_DEV_BAD_PROBS;
    } else if (status == NGC_DEV_OK) {
      const double total = residual_sum(w, lo, hi, sh);
      if (!isfinite(total) || !(total > 0.0)) {
        status = NGC_DEV_BAD_PROBS;
      } else {
        double t = __dmul_rn((double)sh.u[0], total), before = 0.0;
        int own = -1, last = 0;                      // the range the target falls into; the last one with mass
        for (int i = 0; i < kVerifyWarps; ++i) {
          const double s = sh.warp_sum[i];
          if (s > 0.0) last = i;
          if (own < 0 && before + s > t) own = i;
          if (own < 0) before += s;
        }
        if (own < 0) { own = last; t = INFINITY; }   // rounding left the target at the very end: the last token with mass
        if (warp == own) {
          int hit = -1, tail = lo;
          double run = before;
          for (int x0 = lo; x0 < hi; x0 += 32) {
            const double wx = x0 + lane < hi ? w.at(x0 + lane) : 0.0;
            double c = wx;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
              const double y = __shfl_up_sync(0xffffffffu, c, o);
              if (lane >= o) c += y;
            }
            const uint32_t over = __ballot_sync(0xffffffffu, run + c > t), live = __ballot_sync(0xffffffffu, wx > 0.0);
            if (over) { hit = x0 + __ffs(over) - 1; break; }
            if (live) tail = x0 + 31 - __clz(live);
            run += __shfl_sync(0xffffffffu, c, 31);
          }
          if (lane == 0) sh.next = hit >= 0 ? hit : tail;
        }
        __syncthreads();
        next = sh.next;
      }
    }
  }
  if (status != NGC_DEV_OK) {
    if (tid == 0) set_dev_status(p.dev_status, status);
    n_path = 0;
    next = -1;
  }
  __syncthreads();
  for (int i = tid; i < p.N; i += kVerifyThreads) p.path[(int64_t)b * p.N + i] = i < n_path ? sh.path[i] : -1;
  if (tid == 0) { p.n_path[b] = n_path; p.next_token[b] = next; }
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
  if (N > NGC_TREE_MAX_NODES) return NGC_ERR_UNSUPPORTED;
  const VerifyParams p = {tokens, parent, n_nodes, target_probs, draft_probs, uniforms, path, n_path, next_token, dev_status, N, vocab};
  const dim3 grid((unsigned)B), block(kVerifyThreads);
  cudaStream_t s = (cudaStream_t)stream;
  if (greedy) NGC_CUDA_TRY(launch_pdl(verify_draft_kernel<kModeGreedy>, grid, block, 0, s, p));
  else if (draft_probs) NGC_CUDA_TRY(launch_pdl(verify_draft_kernel<kModeDraft>, grid, block, 0, s, p));
  else NGC_CUDA_TRY(launch_pdl(verify_draft_kernel<kModePoint>, grid, block, 0, s, p));
  return NGC_OK;
}
