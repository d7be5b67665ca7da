// pic_append_normed: per-head norm, rotation and append of new tokens.
//
//   y = R(p) (x rsqrt(mean x^2 + eps) w)     for every query and key head x
//
// in 32 bits, rounded to bf16 once (a Reader that norms in bf16 first would round twice); the
// angle p theta_i is reduced exactly, as whole numbers.  q, k and v are read where the
// projection left them: any strides of requests, tokens and heads.
//
// A CTA takes a run of tokens of a request, a thread of it a chunk of 8 pairs of a query or
// key head (and 16 bytes of a value head), KC = d / 16 neighbouring lanes a head: the mean of
// squares takes log2 KC shuffles.  Positions, pages and the rotation's cos and sin are formed
// for the run at once, while the first tokens' projections are under way to shared memory;
// each thread copies what it will read itself, so the ring needs no barrier.
#include <algorithm>
#include <cstdlib>

#include "pic_internal.cuh"

namespace pic {
namespace normed {

constexpr int kMaxThreads = 512;
constexpr int kMaxRun = 16;  // tokens of a CTA
constexpr int kStages = 4;   // tokens in flight

struct Params {
  int batch, max_tokens, Hq, Hkv, G, r_pad, rows, max_pages, layer;
  long long num_pages;
  const __nv_bfloat16 *q, *k, *v, *wq, *wk;
  long long qs[3], ks[3], vs[3];  // strides of requests, tokens, heads in elements
  const int32_t *num_tokens, *pos, *row, *ctx_len, *block_table;
  __nv_bfloat16 *k_cache, *v_cache;  // at the layer
  __nv_bfloat16 *q_out;              // [batch][max_tokens][Hq][d], or with r_pad the prefill's packed rows
  uint64_t turn[64];  // of the frequencies (where the geometry has one table)
  float eps;
  int run;
  int32_t *status;
};

PIC_DEV void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
PIC_DEV void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
PIC_DEV void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

#ifndef MAXREG
#define MAXREG
#endif
template <int D>
__global__ void MAXREG __launch_bounds__(kMaxThreads) append_kernel(Params p, RopeParams rp) {
  constexpr int KC = D / 16, VC = D / 8;
  pdl_entry();
  extern __shared__ __align__(16) uint8_t ring[];  // [kStages][48 bytes of each thread], 16 at a time
  __shared__ float2 cs[kMaxRun][D / 2];
  __shared__ int at_s[kMaxRun], page_s[kMaxRun];
  __shared__ uint64_t turn_s[D / 2];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int runs = (p.max_tokens + p.run - 1) / p.run;
  const int b = blockIdx.x / runs, t0 = blockIdx.x % runs * p.run;
  const int slots = min(p.run, p.max_tokens - t0);
  // (The threads are a multiple of KC: a thread's chunk of a head is always the same.)
  const int units = (p.Hq + p.Hkv) * KC, pieces = p.Hkv * VC;
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);
  auto head = [&](int u, int t) {
    const int h = u / KC;
    return h < p.Hq ? p.q + b * p.qs[0] + t * p.qs[1] + h * p.qs[2]
                    : p.k + b * p.ks[0] + t * p.ks[1] + (h - p.Hq) * p.ks[2];
  };
  auto value = [&](int u, int t) { return p.v + b * p.vs[0] + t * p.vs[1] + (u / VC) * p.vs[2] + u % VC * 8; };
  const uint32_t mine = smem_u32(ring) + tid * 16, third = threads * 16;
  auto fetch = [&](int j) {  // token t0 + j
    if (j < slots) {
      const uint32_t dst = mine + j % kStages * 3 * third;
      if (tid < units) {
        const __nv_bfloat16 *src = head(tid, t0 + j);
        copy16(dst, src + pc.off_a);
        copy16(dst + third, src + pc.off_b);
      }
      if (tid < pieces) copy16(dst + 2 * third, value(tid, t0 + j));
    }
    copies_commit();
  };
  // The projections go out before anything is known of the request.
#pragma unroll
  for (int j = 0; j < kStages - 1; ++j) fetch(j);
  uint4 wa = make_uint4(0, 0, 0, 0), wb = wa;  // this thread's weights
  auto weights = [&](int u) {
    const __nv_bfloat16 *w = u / KC < p.Hq ? p.wq : p.wk;
    if (w) wa = __ldg(reinterpret_cast<const uint4 *>(w + pc.off_a)), wb = __ldg(reinterpret_cast<const uint4 *>(w + pc.off_b));
    return w != nullptr;
  };
  bool norm = weights(tid);
  const int row = p.row ? p.row[b] : b;
  int n = p.num_tokens ? p.num_tokens[b] : p.max_tokens;
  const long long pos = p.pos && tid < slots ? (long long)p.pos[(size_t)b * p.max_tokens + t0 + tid] : 0;
  for (int i = tid; i < D / 2; i += threads)
    turn_s[i] = rp.layer_theta ? rope_turn(rope_theta(rp, p.layer, i)) : p.turn[i];
  bool twice = false;  // the row named before
  if (p.row)
    for (int j = tid; j < b; j += threads) twice |= p.row[j] == row;
  const bool known = row >= 0 && row < p.rows && n >= 0 && n <= p.max_tokens;
  if (tid < slots && known) {
    const long long at = p.pos ? pos : (long long)p.ctx_len[row] + t0 + tid;
    const bool ok = at >= 0 && at < (long long)p.max_pages * 16;
    int page = ok && t0 + tid < n ? p.block_table[(size_t)row * p.max_pages + at / 16] : -1;
    at_s[tid] = ok ? (int)at : 0;
    if (t0 + tid < n) {
      if (at < 0) dev_fail(p.status, PIC_DEV_BAD_POSITION, b);
      else if (!ok) dev_fail(p.status, PIC_DEV_BLOCK_TABLE_SHORT, b);
      else if (page < 0 || page >= p.num_pages) dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
    }
    page_s[tid] = page >= p.num_pages ? -1 : page;
  }
  if (__syncthreads_or(twice) || !known) {
    if (tid == 0 && t0 == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    n = 0;
  }
  auto q_row = [&](int h, int t) {
    return p.r_pad ? ((size_t)(b * p.Hkv + h / p.G) * p.r_pad + t * p.G + h % p.G) * D
                   : (((size_t)b * p.max_tokens + t) * p.Hq + h) * D;
  };
  const int live = min(max(n - t0, 0), slots);
  if (p.r_pad)  // the prefill multiplies every packed row
    for (int t = t0 + live; t < t0 + slots; ++t)
      for (int u = tid; u < p.Hq * VC; u += threads)
        st_global16(p.q_out + q_row(u / VC, t) + u % VC * 8, make_uint4(0, 0, 0, 0));
  for (int e = tid; e < live * (D / 2); e += threads)
    cs[e / (D / 2)][e % (D / 2)] = rope_cos_sin_turn(at_s[e / (D / 2)], turn_s[e % (D / 2)]);
  __syncthreads();
  // one chunk: norm, rotation, store
  auto work = [&](int u, int j, const uint4 &xa, const uint4 &xb) {
    float a[8], c[8];
    unpack8(xa, a);
    unpack8(xb, c);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(a[i], a[i], fmaf(c[i], c[i], s));
#pragma unroll
    for (int o = 1; o < KC; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (u >= units) return;
    if (norm) {
      const float f = rsqrtf(fmaf(s, 1.f / D, p.eps));
      float w[8];
      unpack8(wa, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] *= f * w[i];
      unpack8(wb, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] *= f * w[i];
    }
    const int h = u / KC, page = page_s[j];
    __nv_bfloat16 *dst = nullptr;
    if (h < p.Hq)
      dst = p.q_out + q_row(h, t0 + j);
    else if (page >= 0)
      dst = p.k_cache + (((size_t)page * p.Hkv + h - p.Hq) * 16 + (at_s[j] & 15)) * D;
    if (!dst) return;
    const float2 *r = cs[j] + 8 * (tid % KC);
    if (rp.style == PIC_ROPE_HALF) {
      rotate8(a, c, r);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 r0 = r[i], r1 = r[4 + i];
        const float x0 = a[2 * i], y0 = a[2 * i + 1], x1 = c[2 * i], y1 = c[2 * i + 1];
        a[2 * i] = fmaf(x0, r0.x, -y0 * r0.y), a[2 * i + 1] = fmaf(x0, r0.y, y0 * r0.x);
        c[2 * i] = fmaf(x1, r1.x, -y1 * r1.y), c[2 * i + 1] = fmaf(x1, r1.y, y1 * r1.x);
      }
    }
    st_global16(dst + pc.off_a, pack8(a));
    st_global16(dst + pc.off_b, pack8(c));
  };
  auto store_value = [&](int u, int j, const uint4 &x) {
    if (page_s[j] >= 0)
      st_global16(p.v_cache + (((size_t)page_s[j] * p.Hkv + u / VC) * 16 + (at_s[j] & 15)) * D + u % VC * 8, x);
  };
#pragma unroll 1
  for (int j = 0; j < live; ++j) {
    copies_wait<kStages - 2>();
    const uint32_t src = mine + j % kStages * 3 * third;
    const uint4 xa = lds128(src), xb = lds128(src + third), xv = lds128(src + 2 * third);
    fetch(j + kStages - 1);
    work(tid, j, xa, xb);
    if (tid < pieces) store_value(tid, j, xv);
  }
  copies_wait<0>();
  // heads beyond the CTA's threads
#pragma unroll 1
  for (int u0 = threads; u0 < units; u0 += threads) {
    const int u = u0 + tid;
    if (u < units) norm = weights(u);
#pragma unroll 1
    for (int j = 0; j < live; ++j) {
      const __nv_bfloat16 *src = head(min(u, units - 1), t0 + j);
      work(u, j, ld_stream(src + pc.off_a), ld_stream(src + pc.off_b));
    }
  }
#pragma unroll 1
  for (int u = threads + tid; u < pieces; u += threads)
    for (int j = 0; j < live; ++j) store_value(u, j, ld_stream(value(u, t0 + j)));
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
  // as rope_turn: 2^64 times the turns per position
  for (int i = 0; i < D / 2 && !rp.layer_theta; ++i) {
    double turns = rp.theta[i] * (1.0 / 6.283185307179586476925286766559);
    turns -= std::floor(turns);
    p.turn[i] = (uint64_t)(turns * 18446744073709551616.0);
  }
  p.status = device_status_ptr();
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  const int units = (p.Hq + p.Hkv) * (D / 16);
  const int threads = std::min(kMaxThreads, (units + 31) / 32 * 32);
  const char *env = getenv("PIC_RUN");
  // as many CTAs as an SM holds, if that leaves each a token
  const long long tokens = (long long)batch * max_tokens, resident = 152ll * std::max(1, 65536 / (64 * threads));
  p.run = env ? atoi(env) : (int)std::min<long long>(kMaxRun, (tokens + resident - 1) / resident);
  const dim3 grid((unsigned)(batch * ((max_tokens + p.run - 1) / p.run)));
  const size_t smem = (size_t)kStages * 48 * threads;
  cudaError_t e = cudaFuncSetAttribute(D == 128 ? append_kernel<128> : append_kernel<64>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * 48 * kMaxThreads);
  if (e == cudaSuccess)
    e = D == 128 ? launch_dependent(append_kernel<128>, grid, dim3(threads), smem, stream, p, rp)
                 : launch_dependent(append_kernel<64>, grid, dim3(threads), smem, stream, p, rp);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
