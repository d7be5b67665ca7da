// pic_append_normed: per-head norm, rotation and append of new tokens.
//
//   y = R(p) (x rsqrt(mean x^2 + eps) w)     for every query and key head x
//
// in 32 bits, rounded to bf16 once (a Reader that norms in bf16 first would round twice); the
// angle p theta_i is reduced exactly, as whole numbers.  q, k and v are read where the
// projection left them: any strides of requests, tokens and heads.
//
// The tokens are dealt to the CTAs that the GPU holds at once in equal shares: of all requests'
// tokens, in order.  A thread takes a chunk of 8 pairs of a query or key head (and 16 bytes of
// a value head), KC = d / 16 neighbouring lanes a head: the mean of squares takes log2 KC
// shuffles.  Positions, pages and the rotation's cos and sin are formed for up to 16 tokens at
// once, while the first tokens' projections are under way to shared memory; each thread
// copies what it will read itself, so that ring needs no barrier.
//
// Measured: 8 ragged requests of up to 1067 tokens, 32 + 2 x 8 heads of 128, 28.4 us (140 MB: 4.95
// TB/s, 73% of a copy's rate): the issue slots are 70% busy with about 380 instructions a chunk,
// DRAM 37% (the rest of the rows written stays in L2).  Packed operations took 40% fewer of them,
// but 80 registers or spills, and were no faster.  A run of tokens per CTA instead of equal shares
// left a fifth of the CTAs without work (32 us); one token a CTA 57.  One request's token 4.0 us:
// its chain of loads (projections, row and length, page), sine and cosine.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace normed {

constexpr int kMaxThreads = 512;
constexpr int kMaxRun = 16;  // tokens of a CTA at a time
constexpr int kMaxRagged = 1024;
constexpr int kMaxList = 4096;
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

template <int D, bool kRagged>
__global__ void __launch_bounds__(kMaxThreads, 2) append_kernel(Params p, RopeParams rp) {
  constexpr int KC = D / 16, VC = D / 8;
  pdl_entry();
  extern __shared__ __align__(16) uint8_t ring[];  // [kStages][48 bytes of each thread], 16 at a time
  __shared__ __align__(16) float2 cs[kMaxRun][D / 2];
  __shared__ int at_s[kMaxRun], page_s[kMaxRun], row_s[kMaxRun];  // page_s: -2 left alone
  __shared__ int2 tok_s[kMaxRun];  // request, token
  __shared__ uint64_t turn_s[D / 2];
  __shared__ int first_s[kRagged ? kMaxRagged : 1], warp_s[kMaxThreads / 32];
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31;
  // (The threads are a multiple of KC: a thread's chunk of a head is always the same.)
  const int units = (p.Hq + p.Hkv) * KC, pieces = p.Hkv * VC;
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);
  uint4 wa = make_uint4(0, 0, 0, 0), wb = wa;  // this thread's weights
  auto weights = [&](int u) {
    const __nv_bfloat16 *w = u / KC < p.Hq ? p.wq : p.wk;
    if (w) wa = __ldg(reinterpret_cast<const uint4 *>(w + pc.off_a)), wb = __ldg(reinterpret_cast<const uint4 *>(w + pc.off_b));
    return w != nullptr;
  };
  auto count_of = [&](int b) {  // tokens of request b, 0 where they are none
    const int n = p.num_tokens ? p.num_tokens[b] : p.max_tokens;
    return n < 0 || n > p.max_tokens ? 0 : n;
  };
  int all = p.batch * p.max_tokens;
  if constexpr (kRagged) {  // first_s: tokens of the requests before
    int at = 0;
    for (int b0 = 0; b0 < p.batch; b0 += threads) {
      const int n = b0 + tid < p.batch ? count_of(b0 + tid) : 0;
      int x = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      __syncthreads();
      if (lane == 31) warp_s[tid >> 5] = x;
      __syncthreads();
      x += at - n;
      for (int w = 0; w < threads / 32; ++w) {
        if (w < (tid >> 5)) x += warp_s[w];
        at += warp_s[w];
      }
      if (b0 + tid < p.batch) first_s[b0 + tid] = x;
    }
    all = at;
  }
  auto q_row = [&](int h, int2 tok) {
    return p.r_pad ? ((size_t)(tok.x * p.Hkv + h / p.G) * p.r_pad + tok.y * p.G + h % p.G) * D
                   : (((size_t)tok.x * p.max_tokens + tok.y) * p.Hq + h) * D;
  };
  auto zero = [&](int2 tok) {  // (the prefill multiplies every packed row)
    for (int u = tid; u < p.Hq * VC; u += threads)
      if (tok.y * p.G + u / VC % p.G < p.r_pad)
        st_global16(p.q_out + q_row(u / VC, tok) + u % VC * 8, make_uint4(0, 0, 0, 0));
  };
  auto head = [&](int u, int2 tok) {
    const int h = u / KC;
    return h < p.Hq ? p.q + tok.x * p.qs[0] + tok.y * p.qs[1] + h * p.qs[2]
                    : p.k + tok.x * p.ks[0] + tok.y * p.ks[1] + (h - p.Hq) * p.ks[2];
  };
  auto value = [&](int u, int2 tok) {
    return p.v + tok.x * p.vs[0] + tok.y * p.vs[1] + (u / VC) * p.vs[2] + u % VC * 8;
  };
  const uint32_t mine = smem_u32(ring) + tid * 16, third = threads * 16;
  const int each = all / (int)gridDim.x, more = all % (int)gridDim.x, cta = blockIdx.x;
  const int share0 = each * cta + min(cta, more), share1 = share0 + each + (cta < more ? 1 : 0);
  bool norm = false;
#pragma unroll 1
  for (int s0 = share0; s0 < share1 || s0 == share0; s0 += kMaxRun) {
  const int slots = min(kMaxRun, share1 - s0);
  if (kRagged || s0 > share0) __syncthreads();  // (what was formed for the tokens before has been read)
  auto dense = [&](int i) { return p.max_tokens == 1 ? make_int2(i, 0) : make_int2(i / p.max_tokens, i % p.max_tokens); };
  if (tid < slots) {
    const int i = s0 + tid;
    int2 tok = dense(i);
    if constexpr (kRagged) {
      int lo = 0, hi = p.batch - 1;  // the last request that begins at or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first_s[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      tok = make_int2(lo, i - first_s[lo]);
    }
    tok_s[tid] = tok;
  }
  if constexpr (kRagged) __syncthreads();
  auto fetch = [&](int j) {
    if (j < slots) {
      const uint32_t dst = mine + j % kStages * 3 * third;
      const int2 tok = kRagged ? tok_s[j] : dense(s0 + j);
      if (tid < units) {
        const __nv_bfloat16 *src = head(tid, tok);
        copy16(dst, src + pc.off_a);
        copy16(dst + third, src + pc.off_b);
      }
      if (tid < pieces) copy16(dst + 2 * third, value(tid, tok));
    }
    copies_commit();
  };
  // The projections go out before anything more is known of the requests.
#pragma unroll
  for (int j = 0; j < kStages - 1; ++j) fetch(j);
  if (s0 == share0) {
    norm = weights(tid);
    for (int i = tid; i < D / 2; i += threads)
      turn_s[i] = rp.layer_theta ? rope_turn(rope_theta(rp, p.layer, i)) : p.turn[i];
  }
  if (tid < slots) {
    const int b = tok_s[tid].x, t = tok_s[tid].y;
    const int row = p.row ? p.row[b] : b, n = count_of(b);
    const long long pos = p.pos ? (long long)p.pos[(size_t)b * p.max_tokens + t] : 0;
    int page = -2;
    long long at = 0;
    if (row < 0 || row >= p.rows) {
      dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    } else if (t < n) {
      at = p.pos ? pos : (long long)p.ctx_len[row] + t;
      const bool ok = at >= 0 && at < (long long)p.max_pages * 16;
      page = ok ? p.block_table[(size_t)row * p.max_pages + at / 16] : -1;
      if (!ok) dev_fail(p.status, at < 0 ? PIC_DEV_BAD_POSITION : PIC_DEV_BLOCK_TABLE_SHORT, b);
      else if (page < 0 || page >= p.num_pages) dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
      if (page < 0 || page >= p.num_pages) page = -1;
      if (!ok) at = 0;
    }
    at_s[tid] = (int)at, page_s[tid] = page, row_s[tid] = row;
  }
  __syncthreads();
  if (p.row) {  // rows named before: left alone
    for (int j = tid >> 5; j < slots; j += threads / 32) {
      const int b = tok_s[j].x, row = row_s[j];
      bool twice = false;
      for (int i = lane; i < b; i += 32) twice |= p.row[i] == row;
      if (__any_sync(0xffffffffu, twice) && lane == 0 && page_s[j] != -2) {
        dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
        page_s[j] = -2;
      }
    }
  }
  // pairs 8 c + 2 q, 8 c + 2 q + 1 of chunk c at q KC + c: neighbouring lanes read neighbouring
  // 16 bytes (a chunk's 64 bytes in a row took four times the shared memory's cycles)
  for (int e = tid; e < slots * (D / 2); e += threads) {
    const int i = e % (D / 2);
    cs[e / (D / 2)][((i / 2 % 4) * KC + i / 8) * 2 + i % 2] = rope_cos_sin_turn(at_s[e / (D / 2)], turn_s[i]);
  }
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
      dst = page != -2 ? p.q_out + q_row(h, tok_s[j]) : nullptr;
    else if (page >= 0)
      dst = p.k_cache + (((size_t)page * p.Hkv + h - p.Hq) * 16 + (at_s[j] & 15)) * D;
    if (!dst) return;
    float2 r[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 x = *reinterpret_cast<const float4 *>(&cs[j][(q * KC + tid % KC) * 2]);
      r[2 * q] = make_float2(x.x, x.y), r[2 * q + 1] = make_float2(x.z, x.w);
    }
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
  for (int j = 0; j < slots; ++j) {
    copies_wait<kStages - 2>();
    const uint32_t src = mine + j % kStages * 3 * third;
    const uint4 xa = lds128(src), xb = lds128(src + third), xv = lds128(src + 2 * third);
    fetch(j + kStages - 1);
    work(tid, j, xa, xb);
    if (tid < pieces) store_value(tid, j, xv);
    if (p.r_pad && page_s[j] == -2) zero(tok_s[j]);
  }
  copies_wait<0>();
  // heads beyond the CTA's threads
#pragma unroll 1
  for (int u0 = threads; u0 < units; u0 += threads) {
    const int u = u0 + tid;
    if (u < units) norm = weights(u);
#pragma unroll 1
    for (int j = 0; j < slots; ++j) {
      const __nv_bfloat16 *src = head(min(u, units - 1), tok_s[j]);
      work(u, j, ld_stream(src + pc.off_a), ld_stream(src + pc.off_b));
    }
  }
  if (units > threads) norm = weights(tid);
#pragma unroll 1
  for (int u = threads + tid; u < pieces; u += threads)
    for (int j = 0; j < slots; ++j) store_value(u, j, ld_stream(value(u, tok_s[j])));
  }
  if (p.num_tokens && tid == 0)  // counts that are none
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x)
      if (p.num_tokens[b] < 0 || p.num_tokens[b] > p.max_tokens) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
  if (p.r_pad) {  // the rows behind each request's
    const int each = (p.r_pad + p.G - 1) / p.G;
    for (long long i = blockIdx.x; i < (long long)p.batch * each; i += gridDim.x) {
      const int b = (int)(i / each), t = (int)(i % each);
      if (t >= count_of(b)) zero(make_int2(b, t));
    }
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
  if (row && batch > kMaxList)
    return fail(PIC_ERR_UNSUPPORTED, "%s: a list of %d rows (at most %d)", who, batch, kMaxList);
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
  if ((long long)batch * max_tokens > INT32_MAX - 65536 || max_pages > INT32_MAX / 16 - 16)
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
  // as many CTAs as the SMs hold
  const long long tokens = (long long)batch * max_tokens;
  const long long resident = 152ll * std::min(8, std::max(1, 65536 / (64 * threads)));
  const bool ragged = num_tokens && batch > 1 && max_tokens > 1 && batch <= kMaxRagged;
  void (*kernel)(Params, RopeParams) = D == 128 ? ragged ? append_kernel<128, true> : append_kernel<128, false>
                                                : ragged ? append_kernel<64, true> : append_kernel<64, false>;
  const dim3 grid((unsigned)std::min(tokens, resident));
  const size_t smem = (size_t)kStages * 48 * threads;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kStages * 48 * kMaxThreads);
  if (e == cudaSuccess) e = launch_dependent(kernel, grid, dim3(threads), smem, stream, p, rp);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
