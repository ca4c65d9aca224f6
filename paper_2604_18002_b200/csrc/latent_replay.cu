// ngc_latent_replay_attn and its gradient: entries, argument checks, and the kernels that prepare the masks.
#include "latent_pool.cuh"
#include "latent_replay.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

// When each token was evicted.  Kept lists of all rounds become one number per token: the sequence length at the first
// round that fired after the token was there and did not keep it.  (Tokens are marked with the last round that names
// them; a token named by none goes at the first round that it was there for.)  A CTA takes kSpan tokens of a (sequence, list) and
// looks through all rounds' lists for them: their entries are read many times over, from L2, but all at once.  Bound by latency:
// two sequences of 8192 tokens and seven rounds take 9 us, 13 with one CTA per list.
constexpr int kSpan = 1024;
__global__ void __launch_bounds__(kSpan) latent_gone_kernel(LatentReplayParams p) {
  __shared__ int mark[kSpan];
  const int gi = blockIdx.y % p.G, b = blockIdx.y / p.G, tid = threadIdx.x, t0 = blockIdx.x * kSpan, t = t0 + tid;
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  int64_t row0;
  const int T = latent_seq(p, b, row0);
  if (t0 >= T) return;
  const int64_t list = (int64_t)b * p.G + gi;
  mark[tid] = -1;
  __syncthreads();
  const bool report = blockIdx.x == 0;
  for (int r = 0; r < p.n_rounds; ++r) {
    const int64_t at = ((int64_t)r * p.B + b) * p.G + gi;
    const int n = p.alive_count[at], fired = p.total_before[r * p.B + b];
    if (fired >= T) break;                             // no query of the sequence comes after this round
    if (n < 0 || n > p.kt_max) {                       // (a list that failed has count -1 from its round on)
      if (report && tid == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_KEPT);
      continue;
    }
    for (int i = tid; i < n; i += kSpan) {
      const int x = p.alive_pos[at * p.kt_max + i];
      if (x < 0 || x >= fired) {
        if (report) set_dev_status(p.dev_status, NGC_DEV_BAD_KEPT);
      } else if (x >= t0 && x < t0 + kSpan) {
        atomicMax(&mark[x - t0], r);
      }
    }
  }
  __syncthreads();
  int r = mark[tid] + 1;                               // the first round that does not name it ...
  while (r < p.n_rounds && p.total_before[r * p.B + b] <= t) ++r;        // ... among those that it was there for
  const int gone = t >= T ? 0 : (r < p.n_rounds ? p.total_before[r * p.B + b] : kNeverGone);
  if (t < p.gone_cap) p.gone[list * p.gone_cap + t] = gone;
  int lo = t < T ? gone : kNeverGone, hi = gone;
  for (int o = 16; o > 0; o >>= 1) { lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o)); hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o)); }
  __syncthreads();
  int2* warps = reinterpret_cast<int2*>(mark);
  if ((tid & 31) == 0) warps[tid >> 5] = make_int2(lo, hi);
  __syncthreads();
  if (tid < kSpan / kLatTile && t0 + tid * kLatTile < T) {
    const int2* w = warps + 4 * tid;
    p.tile_gone[list * (p.gone_cap / kLatTile) + t0 / kLatTile + tid] =
        make_int4(min(w[0].x, w[1].x), max(w[0].y, w[1].y), min(w[2].x, w[3].x), max(w[2].y, w[3].y));
  }
}

// delta = sum over channels of out * grad_out: 16 lanes per (token, head), 8 channels each.  Bound by HBM: both are read once,
// 120 MB in 24 us for 14.7 thousand tokens of 16 heads (5 TB/s).
__device__ __forceinline__ float dot8(uint4 a, const float* o) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s += __uint_as_float(w[i] << 16) * o[2 * i] + __uint_as_float(w[i] & 0xffff0000u) * o[2 * i + 1];
  return s;
}
__global__ void __launch_bounds__(256) latent_delta_kernel(LatentReplayParams p) {
  const int c = 8 * (threadIdx.x & 15), b = blockIdx.y % p.B, l = blockIdx.y / p.B;
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  int64_t row0;
  const int64_t T = latent_seq(p, b, row0), x0 = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 4);
#pragma unroll
  for (int k = 0; k < 4; ++k) {                        // (token, head) pairs in the order of memory
    const int64_t x = x0 + 16 * k, t = x / p.H;
    const int h = (int)(x - t * p.H);
    float s = 0.f;
    if (t < T) {
      const int64_t at = (((int64_t)l * p.rows + row0) * p.H + x) * kLatV + c;
      const uint4 g = *reinterpret_cast<const uint4*>(p.go + at);
      float o[8];
      if (p.out_bf16) {
        const uint4 v = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)p.out + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { o[2 * i] = __uint_as_float(w[i] << 16); o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
      } else {
        const float4 v0 = *reinterpret_cast<const float4*>((const float*)p.out + at), v1 = *reinterpret_cast<const float4*>((const float*)p.out + at + 4);
        o[0] = v0.x; o[1] = v0.y; o[2] = v0.z; o[3] = v0.w; o[4] = v1.x; o[5] = v1.y; o[6] = v1.z; o[7] = v1.w;
      }
      s = dot8(g, o);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (c == 0 && t < T) p.delta[((int64_t)l * p.H + h) * p.rows + row0 + t] = s;
  }
}

cudaError_t launch_gone(const LatentReplayParams& p, cudaStream_t stream) {
  return launch_pdl(latent_gone_kernel, dim3((p.max_len + kSpan - 1) / kSpan, p.G * p.B), dim3(kSpan), 0, stream, p);
}

bool valid_seqs(const ngc_latent_seqs* s) {
  return s && s->seq_off && s->lens && s->rows >= 0 && s->L > 0 && s->B > 0 && s->H > 0 && s->d_nope > 0 && s->d_v > 0 && s->d_rope > 0 &&
         s->max_len >= 0 && (s->dtype == NGC_F32 || s->dtype == NGC_BF16);
}

struct Space { size_t gone, tiles, delta, dkr, all; };
int gone_cap(const ngc_latent_seqs* s) { return (int)(((int64_t)s->max_len + kLatTile - 1) / kLatTile * kLatTile); }
Space space_of(const ngc_latent_seqs* s, int lists, int n_rounds, int backward) {
  Space w = {0, 0, 0, 0, 0};
  const size_t BG = (size_t)s->B * lists_G(lists, s->L, 1);
  size_t at = 0;
  if (n_rounds > 0) {
    w.gone = at; at += align256(BG * gone_cap(s) * 4);
    w.tiles = at; at += align256(BG * (gone_cap(s) / kLatTile) * 16);
  }
  if (backward) {
    w.delta = at; at += align256((size_t)s->L * s->H * s->rows * 4);
    w.dkr = at; at += align256((size_t)s->L * s->H * s->rows * s->d_rope * 4);
  }
  w.all = at;
  return w;
}

int prepare(const ngc_latent_seqs* s, const void* q, const void* kv, const void* k_rope, const int32_t* alive_pos, const int32_t* alive_count,
            const int32_t* total_before, int n_rounds, int kt_max, int lists, float scale, int out_dtype, void* ws, size_t ws_bytes,
            int32_t* dev_status, int backward, LatentReplayParams* p) {
  // (tensors without rows have no address)
  if (!valid_seqs(s) || (s->rows > 0 && (!q || !kv || !k_rope)) || n_rounds < 0 || lists < 0 || lists > 2 || (out_dtype != NGC_F32 && out_dtype != NGC_BF16) ||
      (n_rounds > 0 && (!alive_pos || !alive_count || !total_before || kt_max < 1)) || !(scale > 0.f && scale <= 2e38f) || !aligned16(q) ||
      !aligned16(kv) || !aligned16(k_rope))
    return NGC_ERR_INVALID_ARG;
  if (s->dtype != NGC_BF16 || s->d_nope != kLatNope || s->d_v != kLatV || s->d_rope % 16 != 0 || s->d_rope > 64 ||
      s->rows * s->L > 0x7fffffffLL || s->max_len > 0x7fffff00 || (int64_t)s->L * s->B > 65535)
    return NGC_ERR_UNSUPPORTED;
  const Space w = space_of(s, lists, n_rounds, backward);
  if (w.all > 0 && (!ws || ws_bytes < w.all || ((uintptr_t)ws & 255))) return NGC_ERR_WORKSPACE;
  *p = LatentReplayParams{};
  uint8_t* base = (uint8_t*)ws;
  p->seq_off = s->seq_off; p->lens = s->lens; p->rows = s->rows;
  p->q = (const __nv_bfloat16*)q; p->kv = (const __nv_bfloat16*)kv; p->kr = (const __nv_bfloat16*)k_rope;
  p->alive_pos = alive_pos; p->alive_count = alive_count; p->total_before = total_before;
  if (n_rounds > 0) { p->gone = (int32_t*)(base + w.gone); p->tile_gone = (int4*)(base + w.tiles); }
  if (backward) { p->delta = (float*)(base + w.delta); p->dkr_part = (float*)(base + w.dkr); }
  p->L = s->L; p->B = s->B; p->H = s->H; p->G = lists_G(lists, s->L, 1); p->dr = s->d_rope; p->lists = lists; p->n_rounds = n_rounds;
  p->kt_max = kt_max; p->max_len = s->max_len; p->gone_cap = gone_cap(s); p->out_bf16 = out_dtype == NGC_BF16;
  p->scale = scale; p->scale_log2 = scale * 1.4426950408889634f; p->dev_status = dev_status;
  return NGC_OK;
}

}  // namespace
}  // namespace ngc

extern "C" size_t ngc_latent_replay_workspace_bytes(const ngc_latent_seqs* s, int lists, int n_rounds, int backward) {
  return s && lists >= 0 && lists <= 2 ? ngc::space_of(s, lists, n_rounds, backward).all : 0;
}

extern "C" int ngc_latent_replay_attn(const ngc_latent_seqs* s, const void* q, const void* kv, const void* k_rope, const int32_t* alive_pos,
                                      const int32_t* alive_count, const int32_t* total_before, int n_rounds, int kt_max, int lists, float scale,
                                      void* out, int out_dtype, float* lse, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_latent_replay_attn");
  LatentReplayParams p;
  const int rc = prepare(s, q, kv, k_rope, alive_pos, alive_count, total_before, n_rounds, kt_max, lists, scale, out_dtype, ws, ws_bytes, dev_status, 0, &p);
  if (rc != NGC_OK) return rc;
  if (s->rows == 0) return NGC_OK;
  if (!out || !aligned16(out)) return NGC_ERR_INVALID_ARG;
  if (s->max_len == 0) return NGC_OK;
  p.out = out; p.lse = lse;
  if (n_rounds > 0) NGC_CUDA_TRY(launch_gone(p, stream));
  return launch_latent_fwd(p, stream);
}

extern "C" int ngc_latent_replay_attn_backward(const ngc_latent_seqs* s, const void* q, const void* kv, const void* k_rope, const int32_t* alive_pos,
                                               const int32_t* alive_count, const int32_t* total_before, int n_rounds, int kt_max, int lists,
                                               float scale, const void* out, int out_dtype, const float* lse, const void* grad_out, void* grad_q,
                                               void* grad_kv, void* grad_k_rope, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_latent_replay_attn_backward");
  LatentReplayParams p;
  const int rc = prepare(s, q, kv, k_rope, alive_pos, alive_count, total_before, n_rounds, kt_max, lists, scale, out_dtype, ws, ws_bytes, dev_status, 1, &p);
  if (rc != NGC_OK) return rc;
  if (s->rows == 0) return NGC_OK;
  if (!out || !lse || !grad_out || !grad_q || !grad_kv || !grad_k_rope || !aligned16(out) || !aligned16(grad_out) || !aligned16(grad_q) ||
      !aligned16(grad_kv) || !aligned16(grad_k_rope))
    return NGC_ERR_INVALID_ARG;
  if (s->max_len == 0) return NGC_OK;
  p.out = const_cast<void*>(out); p.lse = const_cast<float*>(lse); p.go = (const __nv_bfloat16*)grad_out;
  p.gq = (__nv_bfloat16*)grad_q; p.gkv = (__nv_bfloat16*)grad_kv; p.gkr = (__nv_bfloat16*)grad_k_rope;
  if (n_rounds > 0) NGC_CUDA_TRY(launch_gone(p, stream));
  NGC_CUDA_TRY(launch_pdl(latent_delta_kernel, dim3((unsigned)(((int64_t)p.max_len * p.H + 63) / 64), p.L * p.B), dim3(256), 0, stream, p));
  return launch_latent_bwd(p, stream);
}
