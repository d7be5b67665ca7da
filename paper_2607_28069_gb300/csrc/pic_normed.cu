// pic_append_normed: per-head norm, rotation and append of new tokens.
//
//   y = R(p) (x rsqrt(mean x^2 + eps) w)     for every query and key head x
//
// in 32 bits, rounded to bf16 once (a Reader that norms in bf16 first would round twice); the
// angle p theta_i is reduced exactly, as whole numbers.  q, k and v are read where the
// projection left them: any strides of requests, tokens and heads.
//
// One CTA per token, a thread per chunk of 8 pairs of a query or key head (and per 16 bytes
// of a value head), KC = d / 16 neighbouring lanes a head: the mean of squares takes log2 KC
// shuffles.  The rotation's cos and sin are formed once a token for all heads.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace normed {

constexpr int kMaxThreads = 512;

struct Params {
  int batch, max_tokens, Hq, Hkv, G, r_pad, rows, max_pages, layer;
  long long num_pages;
  const __nv_bfloat16 *q, *k, *v, *wq, *wk;
  long long qs[3], ks[3], vs[3];  // strides of requests, tokens, heads in elements
  const int32_t *num_tokens, *pos, *row, *ctx_len, *block_table;
  __nv_bfloat16 *k_cache, *v_cache;  // at the layer
  __nv_bfloat16 *q_out;              // [batch][max_tokens][Hq][d], or with r_pad the prefill's packed rows
  float eps;
  int32_t *status;
};

template <int D>
__global__ void __launch_bounds__(kMaxThreads) append_kernel(Params p, RopeParams rp) {
  constexpr int KC = D / 16, VC = D / 8;
  pdl_entry();
  __shared__ float2 cs[D / 2];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int b = blockIdx.x / p.max_tokens, t = blockIdx.x % p.max_tokens;
  // The token's projections go out before anything is known of its request.  (The threads are
  // a multiple of KC: a thread's chunk of a head is always the same.)
  const int units = (p.Hq + p.Hkv) * KC, pieces = p.Hkv * VC;
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);
  uint4 xa = make_uint4(0, 0, 0, 0), xb = xa, vn = xa;
  auto load = [&](int u) {
    const int h = u / KC;
    const __nv_bfloat16 *src = h < p.Hq ? p.q + b * p.qs[0] + t * p.qs[1] + h * p.qs[2]
                                        : p.k + b * p.ks[0] + t * p.ks[1] + (h - p.Hq) * p.ks[2];
    xa = ld_stream(src + pc.off_a);
    xb = ld_stream(src + pc.off_b);
  };
  auto value = [&](int u) { return ld_stream(p.v + b * p.vs[0] + t * p.vs[1] + (u / VC) * p.vs[2] + u % VC * 8); };
  if (tid < units) load(tid);
  if (tid < pieces) vn = value(tid);
  const uint64_t turn = tid < D / 2 ? rope_turn(rope_theta(rp, p.layer, tid)) : 0;
  const int row = p.row ? p.row[b] : b;
  int n = p.num_tokens ? p.num_tokens[b] : p.max_tokens;
  bool twice = false;  // the row named before
  if (p.row)
    for (int j = tid; j < b; j += threads) twice |= p.row[j] == row;
  const bool known = !__syncthreads_or(twice) && row >= 0 && row < p.rows && n >= 0 && n <= p.max_tokens;
  if (!known) {
    if (tid == 0 && t == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    n = 0;
  }
  auto q_row = [&](int h) {
    return p.r_pad ? ((size_t)(b * p.Hkv + h / p.G) * p.r_pad + t * p.G + h % p.G) * D
                   : (((size_t)b * p.max_tokens + t) * p.Hq + h) * D;
  };
  if (t >= n) {
    if (p.r_pad)  // the prefill multiplies every packed row
      for (int u = tid; u < p.Hq * VC; u += threads)
        st_global16(p.q_out + q_row(u / VC) + u % VC * 8, make_uint4(0, 0, 0, 0));
    return;
  }
  const long long at = p.pos ? (long long)p.pos[(size_t)b * p.max_tokens + t] : (long long)p.ctx_len[row] + t;
  const bool ok = at >= 0 && at < (long long)p.max_pages * 16;
  int page = ok ? p.block_table[(size_t)row * p.max_pages + at / 16] : -1;
  if (tid == 0) {
    if (at < 0) dev_fail(p.status, PIC_DEV_BAD_POSITION, b);
    else if (!ok) dev_fail(p.status, PIC_DEV_BLOCK_TABLE_SHORT, b);
    else if (page < 0 || page >= p.num_pages) dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
  }
  if (page >= p.num_pages) page = -1;
  if (tid < D / 2) cs[tid] = rope_cos_sin_turn(ok ? (int)at : 0, turn);
  __syncthreads();
  const int slot = (int)(at & 15);
#pragma unroll 1
  for (int u0 = 0; u0 < units; u0 += threads) {
    const int u = u0 + tid, h = u / KC;
    if (u0 && u < units) load(u);
    float a[8], c[8];
    unpack8(xa, a);
    unpack8(xb, c);
    const __nv_bfloat16 *w = h < p.Hq ? p.wq : p.wk;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(a[i], a[i], fmaf(c[i], c[i], s));
#pragma unroll
    for (int o = 1; o < KC; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (u >= units) continue;
    if (w) {
      const float f = rsqrtf(fmaf(s, 1.f / D, p.eps));
      float wa[8], wc[8];
      unpack8(__ldg(reinterpret_cast<const uint4 *>(w + pc.off_a)), wa);
      unpack8(__ldg(reinterpret_cast<const uint4 *>(w + pc.off_b)), wc);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] *= f * wa[i], c[i] *= f * wc[i];
    }
    __nv_bfloat16 *dst = nullptr;
    if (h < p.Hq)
      dst = p.q_out + q_row(h);
    else if (page >= 0)
      dst = p.k_cache + (((size_t)page * p.Hkv + h - p.Hq) * 16 + slot) * D;
    if (!dst) continue;
    const float2 *r = cs + 8 * (tid % KC);
    if (rp.style == PIC_ROPE_HALF) {
      rotate8(a, c, r);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 r0 = r[i], r1 = r[4 + i];
        const float u0_ = a[2 * i], w0 = a[2 * i + 1], u1 = c[2 * i], w1 = c[2 * i + 1];
        a[2 * i] = fmaf(u0_, r0.x, -w0 * r0.y), a[2 * i + 1] = fmaf(u0_, r0.y, w0 * r0.x);
        c[2 * i] = fmaf(u1, r1.x, -w1 * r1.y), c[2 * i + 1] = fmaf(u1, r1.y, w1 * r1.x);
      }
    }
    st_global16(dst + pc.off_a, pack8(a));
    st_global16(dst + pc.off_b, pack8(c));
  }
  if (page >= 0)
#pragma unroll 1
    for (int u = tid; u < pieces; u += threads) {
      if (u != tid) vn = value(u);
      st_global16(p.v_cache + (((size_t)page * p.Hkv + u / VC) * 16 + slot) * D + u % VC * 8, vn);
    }
}

}  // namespace normed
}  // namespace pic

extern "C" pic_status_t pic_append_normed(const pic_geom_t *geom, int32_t layer, int32_t batch,
                                          int32_t max_tokens, const void *q, const int64_t *q_stride,
                                          const void *k_new, const int64_t *k_stride,
                                          const void *v_new, const int64_t *v_stride,
                                          const void *q_weight, const void *k_weight, float eps,
                                          const int32_t *num_tokens, const int32_t *pos,
                                          const int32_t *row, const int32_t *ctx_len, int32_t rows,
                                          const int32_t *block_table, int32_t max_pages,
                                          int64_t num_pages, void *k_cache, void *v_cache,
                                          void *q_out, void *workspace, size_t workspace_bytes,
                                          pic_stream_t stream) {
  using namespace pic;
  using namespace pic::normed;
  static const char *who = "pic_append_normed";
  RopeParams rp;
  pic_status_t st = make_rope(geom, &rp);
  if (st != PIC_OK) return st;
  if (layer < 0 || layer >= geom->num_layers)
    return fail(PIC_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", who, layer, geom->num_layers);
  if (batch <= 0 || max_tokens <= 0 || rows <= 0 || max_pages <= 0 || num_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (!q || !k_new || !v_new || !q_stride || !k_stride || !v_stride || !block_table || !k_cache || !v_cache)
    return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if (!pos && !ctx_len)
    return fail(PIC_ERR_INVALID_ARG, "%s: neither positions nor lengths", who);
  if (!row && batch > rows)
    return fail(PIC_ERR_INVALID_ARG, "%s: batch %d, block table of %d rows", who, batch, rows);
  if (!q_out == !workspace)
    return fail(PIC_ERR_INVALID_ARG, "%s: one of q_out and workspace takes the queries", who);
  if (!(eps >= 0.f) || std::isinf(eps))
    return fail(PIC_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
  uintptr_t low = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) |
                  reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(q_weight) |
                  reinterpret_cast<uintptr_t>(k_weight) | reinterpret_cast<uintptr_t>(k_cache) |
                  reinterpret_cast<uintptr_t>(v_cache) | reinterpret_cast<uintptr_t>(q_out);
  for (int i = 0; i < 3; ++i) {
    low |= (uintptr_t)((q_stride[i] | k_stride[i] | v_stride[i]) * 2);
    if (q_stride[i] < 0 || k_stride[i] < 0 || v_stride[i] < 0)
      return fail(PIC_ERR_INVALID_ARG, "%s: negative stride", who);
  }
  if (low & 15)
    return fail(PIC_ERR_INVALID_ARG, "%s: bf16 tensors and their strides must be multiples of 16 bytes", who);
  if ((long long)batch * max_tokens >= INT32_MAX || max_pages > INT32_MAX / 16 - 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: 2^31 tokens or positions", who);
  Params p;
  p.batch = batch;
  p.max_tokens = max_tokens;
  p.Hq = geom->num_q_heads;
  p.Hkv = geom->num_kv_heads;
  p.G = p.Hq / p.Hkv;
  p.r_pad = 0;
  if (workspace) {
    const size_t need = pic_prefill_workspace_size(geom, batch, max_tokens, 1, 1);
    if (workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255))
      return fail(PIC_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", who, need);
    p.r_pad = (int)(((long long)max_tokens * p.G + 127) / 128 * 128);
  }
  p.rows = rows;
  p.max_pages = max_pages;
  p.layer = layer;
  p.num_pages = num_pages;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.k = static_cast<const __nv_bfloat16 *>(k_new);
  p.v = static_cast<const __nv_bfloat16 *>(v_new);
  p.wq = static_cast<const __nv_bfloat16 *>(q_weight);
  p.wk = static_cast<const __nv_bfloat16 *>(k_weight);
  for (int i = 0; i < 3; ++i) p.qs[i] = q_stride[i], p.ks[i] = k_stride[i], p.vs[i] = v_stride[i];
  p.num_tokens = num_tokens;
  p.pos = pos;
  p.row = row;
  p.ctx_len = ctx_len;
  p.block_table = block_table;
  const int D = geom->head_dim;
  const size_t layer_elems = (size_t)num_pages * p.Hkv * 16 * D;
  p.k_cache = static_cast<__nv_bfloat16 *>(k_cache) + layer * layer_elems;
  p.v_cache = static_cast<__nv_bfloat16 *>(v_cache) + layer * layer_elems;
  p.q_out = static_cast<__nv_bfloat16 *>(workspace ? workspace : q_out);
  p.eps = eps;
  p.status = device_status_ptr();
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  const int units = (p.Hq + p.Hkv) * (D / 16);
  const int threads = std::min(kMaxThreads, std::max(D / 2, (units + 31) / 32 * 32));
  const dim3 grid((unsigned)(batch * max_tokens));
  const cudaError_t e = D == 128 ? launch_dependent(append_kernel<128>, grid, dim3(threads), 0, stream, p, rp)
                                 : launch_dependent(append_kernel<64>, grid, dim3(threads), 0, stream, p, rp);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
