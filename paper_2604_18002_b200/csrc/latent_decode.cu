// ngc_latent_decode: absorbed latent attention of one token per sequence over a pool of pages.
#include <cuda_bf16.h>

#include "latent_pool.cuh"
#include "ptx.cuh"

namespace ngc {
namespace {

struct LatentDecodeParams {
  const __nv_bfloat16* rows;
  const int32_t* table;
  const int32_t* lens;
  const __nv_bfloat16* ql;
  const __nv_bfloat16* qr;
  void* out;
  int32_t* dev_status;
  int B, H, G, dc, dr, page, cap, n_pages, lists, layer_begin, out_bf16;
  float scale_log2;
};

// One CTA per (head, sequence, layer), its warps take tokens in turn; online softmax per warp, joined at the end.
__global__ void __launch_bounds__(256) latent_decode_kernel(LatentDecodeParams p) {
  __shared__ float so[8][512];
  __shared__ float sm[8], sl[8];
  const int h = blockIdx.x, b = blockIdx.y, l = p.layer_begin + blockIdx.z;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gi = list_of(p.lists, l, 0, 1);
  const int64_t list = (int64_t)b * p.G + gi;
  const int len = p.lens[list];
  if (len < 0 || len > p.cap * p.page) {
    if (threadIdx.x == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_COUNTS);
    return;
  }
  const int D = p.dc + p.dr, per = p.dc / 32;
  const int64_t qi = ((int64_t)l * p.B + b) * p.H + h;
  float q[18], acc[16];
  for (int i = 0; i < 16; ++i) { acc[i] = 0.f; q[i] = i < per ? __bfloat162float(p.ql[qi * p.dc + 32 * i + lane]) : 0.f; }
  for (int i = 0; i < 2; ++i) q[16 + i] = 32 * i + lane < p.dr ? __bfloat162float(p.qr[qi * p.dr + 32 * i + lane]) : 0.f;
  float m = -INFINITY, sum = 0.f;
  for (int t = warp; t < len; t += 8) {
    int pg = p.table[list * p.cap + t / p.page];
    if ((uint32_t)pg >= (uint32_t)p.n_pages) { if (lane == 0) set_dev_status(p.dev_status, NGC_DEV_BAD_PAGE); pg = 0; }
    const __nv_bfloat16* x = p.rows + (((int64_t)l * p.n_pages + pg) * p.page + t % p.page) * D;
    float v[16], z = 0.f;
    for (int i = 0; i < 16; ++i) if (i < per) { v[i] = __bfloat162float(x[32 * i + lane]); z += v[i] * q[i]; }
    for (int i = 0; i < 2; ++i) if (32 * i + lane < p.dr) z += __bfloat162float(x[p.dc + 32 * i + lane]) * q[16 + i];
    z = warp_sum(z) * p.scale_log2;
    const float mn = fmaxf(m, z), a = exp2f(m - mn), w = exp2f(z - mn);
    sum = sum * a + w;
    for (int i = 0; i < 16; ++i) if (i < per) acc[i] = acc[i] * a + w * v[i];
    m = mn;
  }
  for (int i = 0; i < 16; ++i) if (i < per) so[warp][32 * i + lane] = acc[i];
  if (lane == 0) { sm[warp] = m; sl[warp] = sum; }
  __syncthreads();
  float mm = -INFINITY, ll = 0.f;
  for (int w = 0; w < 8; ++w) if (sl[w] > 0.f || sl[w] != sl[w]) mm = fmaxf(mm, sm[w]);
  for (int w = 0; w < 8; ++w) if (sm[w] != -INFINITY) ll += sl[w] * exp2f(sm[w] - mm);
  for (int c = threadIdx.x; c < p.dc; c += 256) {
    float o = 0.f;
    for (int w = 0; w < 8; ++w) if (sm[w] != -INFINITY) o += so[w][c] * exp2f(sm[w] - mm);
    o = len == 0 ? 0.f : o / ll;
    if (p.out_bf16) ((__nv_bfloat16*)p.out)[qi * p.dc + c] = __float2bfloat16(o);
    else ((float*)p.out)[qi * p.dc + c] = o;
  }
}

}  // namespace
}  // namespace ngc

extern "C" size_t ngc_latent_decode_workspace_bytes(const ngc_latent_pool* c, int H) { return c && H > 0 ? 256 : 0; }

extern "C" int ngc_latent_decode(const ngc_latent_pool* c, const void* q_latent, const void* q_rope, int H, int layer_begin, int layer_end,
                                 float scale, void* out, int out_dtype, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream) {
  using namespace ngc;
  NGC_API_RANGE("ngc_latent_decode");
  if (!valid_latent_pool(c) || !q_latent || !q_rope || !out || layer_begin < 0 || layer_begin >= layer_end || layer_end > c->L || H < 1 ||
      !(scale > 0.f && scale <= 2e38f) || (out_dtype != NGC_F32 && out_dtype != NGC_BF16) || !aligned16(c->rows) || !aligned16(q_latent) ||
      !aligned16(q_rope) || !aligned16(out))
    return NGC_ERR_INVALID_ARG;
  if (c->dtype != NGC_BF16 || !built_latent_dims(c->d_latent, c->d_rope) || H > 128) return NGC_ERR_UNSUPPORTED;
  if (ws_bytes < ngc_latent_decode_workspace_bytes(c, H) || !ws || ((uintptr_t)ws & 255)) return NGC_ERR_WORKSPACE;
  LatentDecodeParams p;
  p.rows = (const __nv_bfloat16*)c->rows; p.table = c->page_table; p.lens = c->lens;
  p.ql = (const __nv_bfloat16*)q_latent; p.qr = (const __nv_bfloat16*)q_rope; p.out = out; p.dev_status = dev_status;
  p.B = c->B; p.H = H; p.G = lists_G(c->lists, c->L, 1); p.dc = c->d_latent; p.dr = c->d_rope; p.page = c->page; p.cap = c->pages_cap;
  p.n_pages = c->n_pages; p.lists = c->lists; p.layer_begin = layer_begin; p.out_bf16 = out_dtype == NGC_BF16;
  p.scale_log2 = scale * 1.4426950408889634f;
  latent_decode_kernel<<<dim3(H, c->B, layer_end - layer_begin), 256, 0, stream>>>(p);
  return launch_status();
}
