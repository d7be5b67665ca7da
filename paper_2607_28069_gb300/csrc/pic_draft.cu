// pic_attend_draft: one layer of one step over the drafted tokens of every
// request (a chain or a tree of up to 64 tokens behind the cached context).
//
// The attention reads each key and value of a request once for all its drafted
// tokens and query heads: a request's queries of one kv head are packed into
// rows r = token * G + head of 128-row tiles (one TMEM lane per row), so with up
// to 128 rows a key costs 4 d flops a row for the 4 d bytes that it and its
// value take: HBM-bound below about 280 rows.  What a chain's causal mask or a
// tree's ancestor mask hides lies within the last 64 slots; every earlier key
// is visible to every row.
//
// Launches:
//  1. draft_append_kernel: per token its depth and ancestor bits, the rotated
//     key and the value into their slots, the rotated queries packed.
//  2. draft_attn_kernel: one persistent CTA per SM.  All (request, kv head, row
//     tile) units' key tiles form one sequence, unit after unit, of which every
//     CTA takes an equal share (the lengths are only known on the device, and
//     batches are ragged), so no SM waits for a longer request's.  A CTA's share
//     is a run of segments, each a range of one unit's key tiles; a unit that
//     lies within one CTA is finished there, the others leave partial states.
//  3. draft_merge_kernel: log-sum-exp merge of those.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace draft {

constexpr int BM = 128, BN = 128;  // rows of a tile, keys of a tile
constexpr int kMaxDraft = 64;
constexpr int kCtas = 152;         // one per SM
constexpr int NSK = 3, NSV = 2;    // ring stages of K and V
constexpr int NQB = 2;             // query tiles: the present segment's and the next one's
constexpr int kThreads = 256;      // K producer, MMA, V producer, -, four softmax warps
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;    // S at 0 and 128, O at 256 and 256 + D

template <int D>
struct Layout {
  static constexpr int kTile = BN * D * 2;
  static constexpr int kQ = 0;
  static constexpr int kK = kQ + NQB * kTile;
  static constexpr int kV = kK + NSK * kTile;
  static constexpr int kBar = kV + NSV * kTile;
  static constexpr int kAlloc = kBar + 256 + 1024;
};

enum {
  B_QFULL = 0,
  B_QEMPTY = B_QFULL + NQB,
  B_KFULL = B_QEMPTY + NQB,
  B_KEMPTY = B_KFULL + NSK,
  B_VFULL = B_KEMPTY + NSK,
  B_VEMPTY = B_VFULL + NSV,
  B_VFIX = B_VEMPTY + NSV,   // per V stage: the rows behind the last draft are cleared
  B_SFULL = B_VFIX + NSV,    // S(g) in buffer g % 2
  B_P = B_SFULL + 2,         // P(g) in buffer g % 2
  B_PV = B_P + 2,            // PV(g) done, g % 2
  B_OEMPTY = B_PV + 2,       // O buffer read
  B_END = B_OEMPTY + 2,
  B_COUNT = B_END + 1
};
static_assert(B_COUNT * 8 + 16 <= 256, "barrier area");

struct Params {
  int batch, max_draft, Hq, Hkv, G, r_pad, rt_max, max_pages, oob_row, layer;
  long long num_pages, layer_row0;
  const int32_t *ctx_len, *draft_len, *parent, *block_table;
  const __nv_bfloat16 *q, *k_new, *v_new;
  __nv_bfloat16 *k_cache, *v_cache;  // at the layer
  __nv_bfloat16 *qp;                 // workspace: packed rotated queries
  uint64_t *mask;                    // workspace: [batch][max_draft] ancestor bits
  int2 *unit;                        // workspace: [batch][Hkv][rt_max] first and last CTA
  float *part_o;                     // workspace: [2 kCtas][BM][D]
  float2 *part_ml;                   // workspace: [2 kCtas][BM]
  __nv_bfloat16 *out;
  float *lse;
  int32_t *status;
  float scale_log2;
};

// What a request brings: its key tiles and row tiles (0 for one left alone).
struct Request {
  int ctx, n, tiles, rt;
};
PIC_DEV Request request_of(const Params &p, int b) {
  Request r;
  r.ctx = p.ctx_len[b];
  r.n = p.draft_len[b];
  const bool ok = r.ctx >= 0 && r.n > 0 && r.n <= p.max_draft &&
                  (long long)r.ctx + r.n <= (long long)p.max_pages * 16;
  if (!ok) r.ctx = r.n = 0;
  r.tiles = ok ? (r.ctx + r.n + BN - 1) / BN : 0;
  r.rt = (r.n * p.G + BM - 1) / BM;
  return r;
}

// ------------------------------------------------------------------ append
template <int D>
__global__ void __launch_bounds__(128) draft_append_kernel(Params p, RopeParams rp) {
  constexpr int KC = D / 16;
  pdl_entry();
  __shared__ float2 cs[D / 2];
  __shared__ int32_t par[kMaxDraft];
  __shared__ int depth;
  const int b = blockIdx.y, i = blockIdx.x, tid = threadIdx.x;
  const int ctx = p.ctx_len[b], n = p.draft_len[b];
  const bool bad = ctx < 0 || n < 0 || n > p.max_draft;
  if (bad || (long long)ctx + n > (long long)p.max_pages * 16) {
    if (i == 0 && tid == 0)
      dev_fail(p.status, bad ? PIC_DEV_BAD_REQUEST : PIC_DEV_BLOCK_TABLE_SHORT, b);
    return;
  }
  if (i >= n) return;
  if (tid < n) {
    int q = tid - 1;
    if (p.parent) {
      q = p.parent[(size_t)b * p.max_draft + tid];
      if (q < -1 || q >= tid) {
        if (tid == i) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
        q = -1;
      }
    }
    par[tid] = q;
  }
  __syncthreads();
  if (tid == 0) {
    uint64_t m = 1ull << i;
    int d = 0;
    for (int q = par[i]; q >= 0; q = par[q]) m |= 1ull << q, ++d;
    p.mask[(size_t)b * p.max_draft + i] = m;
    depth = d;
  }
  __syncthreads();
  const int pos = ctx + depth, slot = ctx + i;
  if (tid < D / 2) cs[tid] = rope_cos_sin_turn(pos, rope_turn(rope_theta(rp, p.layer, tid)));
  int page = p.block_table[(size_t)b * p.max_pages + slot / 16];
  if (page < 0 || page >= p.num_pages) {
    if (tid == 0) dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
    page = -1;
  }
  __syncthreads();
  const size_t tok = (size_t)b * p.max_draft + i;
  for (int u = tid; u < (p.Hq + p.Hkv) * KC; u += 128) {
    const int h = u / KC, c = u % KC;
    if (h < p.Hq) {
      const int hk = h / p.G, g = h % p.G;
      rotate_chunk(p.q + (tok * p.Hq + h) * D,
                   p.qp + ((size_t)(b * p.Hkv + hk) * p.r_pad + i * p.G + g) * D, c, D / 2, rp.style,
                   cs + 8 * c, true);
    } else if (page >= 0) {
      const int hk = h - p.Hq;
      rotate_chunk(p.k_new + (tok * p.Hkv + hk) * D,
                   p.k_cache + (((size_t)page * p.Hkv + hk) * 16 + slot % 16) * D, c, D / 2, rp.style,
                   cs + 8 * c, true);
    }
  }
  if (page >= 0)
    for (int u = tid; u < p.Hkv * (D / 8); u += 128) {
      const int hk = u / (D / 8), c = u % (D / 8);
      st_global16(p.v_cache + (((size_t)page * p.Hkv + hk) * 16 + slot % 16) * D + c * 8,
                  ld_stream(p.v_new + (tok * p.Hkv + hk) * D + c * 8));
    }
}

// ---------------------------------------------------------------- schedule
// The segments of one CTA, walked by each role's warp for itself.
struct Segments {
  const Params &p;
  long long total, pos, end;  // key tiles of the batch, next tile, end of this CTA's share
  long long base;             // first tile of request b
  int b, cta, ctas;
  Request r;
  // the present segment
  int hk, rt, kt0, n;
  bool first, last;  // holds the unit's first, last key tile
  long long unit0;   // the unit's first tile

  PIC_DEV long long work(const Request &x) const { return (long long)p.Hkv * x.rt * x.tiles; }

  PIC_DEV Segments(const Params &pp, int cta_, int grid) : p(pp), cta(cta_) {
    const int lane = threadIdx.x & 31;
    total = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      long long w = b0 + lane < p.batch ? work(request_of(p, b0 + lane)) : 0;
#pragma unroll
      for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
      total += w;
    }
    // every CTA that takes part has a tile
    ctas = (int)min((long long)grid, total);
    base = pos = end = 0;
    b = 0;
    if (cta >= ctas) return;
    pos = total * cta / ctas;
    end = total * (cta + 1) / ctas;
    // the request that holds tile `pos`
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      long long w = b0 + lane < p.batch ? work(request_of(p, b0 + lane)) : 0, x = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + x > pos);
      if (past) {
        const int l = __ffs(past) - 1;
        b = b0 + l;
        base += __shfl_sync(0xffffffffu, x - w, l);
        break;
      }
      base += __shfl_sync(0xffffffffu, x, 31);
    }
    r = request_of(p, b);
  }
  PIC_DEV bool next() {
    if (pos >= end) return false;
    while (pos - base >= work(r)) {
      base += work(r);
      r = request_of(p, ++b);
    }
    const int u = (int)((pos - base) / r.tiles);
    unit0 = base + (long long)u * r.tiles;
    kt0 = (int)(pos - unit0);
    n = (int)min((long long)(r.tiles - kt0), end - pos);
    hk = u / r.rt;
    rt = u % r.rt;
    first = kt0 == 0;
    last = kt0 + n == r.tiles;
    pos += n;
    return true;
  }
  // the CTA whose share holds tile t
  PIC_DEV int owner(long long t) const { return (int)(((t + 1) * ctas - 1) / total); }
  // the partial slot of the present segment: a CTA has at most one segment
  // that ends a unit begun elsewhere or lies inside one (0), and one that begins
  // a unit and leaves its end to others (1)
  PIC_DEV int slot() const { return 2 * cta + (first ? 1 : 0); }
};

// --------------------------------------------------------------- attention
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    draft_attn_kernel(const __grid_constant__ CUtensorMap tm_q,
                      const __grid_constant__ CUtensorMap tm_k,
                      const __grid_constant__ CUtensorMap tm_v, Params p) {
  using L = Layout<D>;
  constexpr int PANELS = D / 64;
  constexpr uint32_t IDESC_QK = idesc_bf16(BM, BN, false, false);
  constexpr uint32_t IDESC_PV = idesc_bf16(BM, D, false, true);
  // K/V tiles page by page, as the prefill's: [8-row half][panel][8 rows][128 B]
  constexpr uint32_t kPageBytes = 16 * D * 2;
  constexpr uint32_t kGroupStride = PANELS == 2 ? 2048 : 1024;
  constexpr uint32_t kPanelOff = PANELS == 2 ? 1024 : BN * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                              ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem);
  auto bar = [&](int i) { return sbase + L::kBar + 8u * (uint32_t)i; };
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::kBar + 8 * B_COUNT);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kBar + 8 * B_COUNT + 8);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < B_COUNT; ++i)
      mbar_init(bar(i), (i == B_P || i == B_P + 1 || i == B_OEMPTY || i == B_OEMPTY + 1) ? 4 : 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (lane == 0 && warp < 3) prefetch_tmap(warp == 0 ? &tm_k : warp == 1 ? &tm_q : &tm_v);
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int detail = -2;

  Segments sg(p, (int)blockIdx.x, (int)gridDim.x);
  if (warp == 0 || warp == 2) {
    // ===================================================== TMA producers
    // Warp 0 the query tile of each segment and K, warp 2 V.  Lane l < 8
    // moves page l of a tile as one box.
    const bool is_k = warp == 0;
    const int nst = is_k ? NSK : NSV;
    const int b_full = is_k ? B_KFULL : B_VFULL, b_empty = is_k ? B_KEMPTY : B_VEMPTY;
    const uint32_t ring = sbase + (is_k ? L::kK : L::kV);
    const CUtensorMap *tmap = is_k ? &tm_k : &tm_v;
    int g = 0, s = 0;   // tiles and segments issued
    bool ok = true;
    while (ok && sg.next()) {
      if (is_k) {
        if (s >= NQB)
          ok = __all_sync(0xffffffffu, mbar_wait(bar(B_QEMPTY + s % NQB), (s / NQB - 1) & 1,
                                                 abort_flag, p.status, detail));
        if (!ok) break;
        if (lane == 0) {
          mbar_expect_tx(bar(B_QFULL + s % NQB), L::kTile);
          const int row = (sg.b * p.Hkv + sg.hk) * p.r_pad + sg.rt * BM;
#pragma unroll
          for (int pn = 0; pn < PANELS; ++pn)
            tma_load_2d(sbase + L::kQ + (s % NQB) * L::kTile + pn * BM * 128, &tm_q, pn * 64, row,
                        bar(B_QFULL + s % NQB));
        }
        __syncwarp();
      }
      ++s;
      const int32_t *bt = p.block_table + (size_t)sg.b * p.max_pages;
      const int keys = sg.r.ctx + sg.r.n;
      for (int j = 0; j < sg.n; ++j, ++g) {
        const int st = g % nst, kt = sg.kt0 + j;
        int y = p.oob_row;  // zeros
        const int pidx = kt * 8 + lane;
        if (lane < 8 && (long long)pidx * 16 < keys && pidx < p.max_pages) {
          const int page = bt[pidx];
          if (page >= 0 && page < p.num_pages)
            y = (int)(p.layer_row0 + ((long long)page * p.Hkv + sg.hk) * 16);
          else if (is_k)
            dev_fail(p.status, PIC_DEV_BAD_PAGE, sg.b);
        }
        if (g >= nst) {
          ok = __all_sync(0xffffffffu, mbar_wait(bar(b_empty + st), (g / nst - 1) & 1, abort_flag,
                                                 p.status, detail));
          if (!ok) break;
        }
        if (lane == 0) mbar_expect_tx(bar(b_full + st), L::kTile);
        __syncwarp();
        if (lane < 8) {
          const uint32_t dst = ring + st * L::kTile + lane * kPageBytes;
          if constexpr (PANELS == 2)
            tma_load_4d(dst, tmap, 0, 0, 0, y >> 3, bar(b_full + st));
          else
            tma_load_2d(dst, tmap, 0, y, bar(b_full + st));
        }
        if (!is_k && kt != sg.r.tiles - 1) {
          if (lane == 0) mbar_arrive(bar(B_VFIX + st));
        } else if (!is_k) {
          // Rows behind the last draft may hold anything, and a weight of zero
          // does not silence an infinity: they are cleared before PV reads them
          ok = __all_sync(0xffffffffu, mbar_wait(bar(b_full + st), (g / nst) & 1, abort_flag,
                                                 p.status, detail));
          if (!ok) {
            ++g;
            break;
          }
          const int r0 = keys - kt * BN, r1 = (r0 + 15) & ~15;  // the rest of its page
          constexpr int CH = D / 8;
          for (int e = lane; e < (r1 - r0) * CH; e += 32) {
            const int row = r0 + e / CH, ch = e % CH, rr = row & 15;
            const uint32_t off =
                PANELS == 2 ? (uint32_t)((rr >> 3) * 2048 + (ch >> 3) * 1024 + (rr & 7) * 128 +
                                         (((ch & 7) ^ (rr & 7)) << 4))
                            : (uint32_t)(rr * 128 + ((ch ^ (rr & 7)) << 4));
            sts128(ring + st * L::kTile + (row >> 4) * kPageBytes + off, make_uint4(0, 0, 0, 0));
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_VFIX + st));
        }
      }
    }
    // what was issued lands before the CTA exits
    if (lane == 0) {
      for (int j = max(0, g - nst); j < g; ++j)
        mbar_wait_no_flag(bar(b_full + j % nst), (j / nst) & 1, p.status, detail, kWaitLimitNs);
      if (is_k)
        for (int j = max(0, s - NQB); j < s; ++j)
          mbar_wait_no_flag(bar(B_QFULL + j % NQB), (j / NQB) & 1, p.status, detail, kWaitLimitNs);
    }
  } else if (warp == 1) {
    // ===================================================== MMA issuer
    // The tiles of all segments in one sequence g: QK(g + 1) is issued before
    // PV(g), so the scores of the next tile are there when a softmax ends.
    const uint32_t el = elect_one();
    const uint32_t ub = __shfl_sync(0xffffffffu, tbase, 0);
    const MatDesc dQ = sdesc_sw128(sbase + L::kQ, 16, 1024);
    const MatDesc dK = sdesc_sw128(sbase + L::kK, 16, kGroupStride);
    const MatDesc dV = sdesc_sw128(sbase + L::kV, kPanelOff, kGroupStride);
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      if (ok)
        ok = __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, p.status, detail));
      return ok;
    };
    // the tile whose QK was issued last waits for its PV
    int g = 0, s = 0;
    bool have = false, pv_first = false, pv_lasttile = false;
    int pv_s = 0;
    auto pv = [&](int gg) {
      const int st = gg % NSV, ob = pv_s & 1;
      wait(B_VFULL + st, (gg / NSV) & 1);
      if (pv_lasttile) wait(B_VFIX + st, (gg / NSV) & 1);
      if (pv_first && pv_s >= 2) wait(B_OEMPTY + ob, (pv_s / 2 - 1) & 1);
      wait(B_P + (gg & 1), (gg >> 1) & 1);
      if (!ok) return;
      tc_fence_after();
      const uint32_t tO = ub + kColO + ob * D, tP = ub + (gg & 1) * 128;
      const MatDesc dv = dV.at(st * L::kTile);
#pragma unroll
      for (int kk = 0; kk < BN / 16; ++kk)
        mma_ts(tO, tP + kk * 8, dv.at(kk * kPageBytes), IDESC_PV, !(pv_first && kk == 0), el);
      mma_commit(bar(B_VEMPTY + st), el);
      mma_commit(bar(B_PV + (gg & 1)), el);
    };
    while (ok && sg.next()) {
      wait(B_QFULL + s % NQB, (s / NQB) & 1);
      for (int j = 0; ok && j < sg.n; ++j, ++g) {
        const int st = g % NSK;
        if (!wait(B_KFULL + st, (g / NSK) & 1)) break;
        tc_fence_after();
        const uint32_t tS = ub + (g & 1) * 128;
        const MatDesc dq = dQ.at((s % NQB) * L::kTile), dk = dK.at(st * L::kTile);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_ss(tS, dq.at((kk >> 2) * (BM * 128) + (kk & 3) * 32),
                 dk.at((kk >> 2) * kPanelOff + (kk & 3) * 32), IDESC_QK, kk > 0, el);
        mma_commit(bar(B_KEMPTY + st), el);
        if (j == sg.n - 1) mma_commit(bar(B_QEMPTY + s % NQB), el);
        mma_commit(bar(B_SFULL + (g & 1)), el);
        if (have) pv(g - 1);
        have = true;
        pv_first = j == 0;
        pv_lasttile = sg.kt0 + j == sg.r.tiles - 1;
        pv_s = s;
      }
      ++s;
    }
    if (ok && have) pv(g - 1);
    mma_commit(bar(B_END), el);
    if (lane == 0) mbar_wait_no_flag(bar(B_END), 0, p.status, detail, 4 * kWaitLimitNs);
    __syncwarp();
  } else if (warp >= 4) {
    // ===================================================== softmax
    // One thread per row; tile g's scores from TMEM, the exponentials back as
    // bf16 over them.  O is rescaled only when a row's maximum grew by more than
    // 2^8; sums and O stay within fp32 (exponents up to 2^8, P in bf16).
    const int wq = warp & 3, row = wq * 32 + lane;
    const uint32_t tl = tbase + ((uint32_t)(wq * 32) << 16);
    int g = 0, s = 0;
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      if (ok)
        ok = __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, p.status, detail));
      return ok;
    };
    while (ok && sg.next()) {
      const int ob = s & 1;
      const uint32_t tO = tl + kColO + ob * D;
      const int rr = sg.rt * BM + row;
      const bool valid = rr < sg.r.n * p.G;
      const int tok = valid ? rr / p.G : 0, head = sg.hk * p.G + (valid ? rr % p.G : 0);
      const uint64_t mask = valid ? p.mask[(size_t)sg.b * p.max_draft + tok] : 0;
      if (sg.first && threadIdx.x == 128)
        p.unit[((size_t)sg.b * p.Hkv + sg.hk) * p.rt_max + sg.rt] =
            make_int2((int)blockIdx.x, sg.owner(sg.unit0 + sg.r.tiles - 1));
      float m_used = -INFINITY, l = 0.f;
      for (int j = 0; j < sg.n; ++j, ++g) {
        if (!wait(B_SFULL + (g & 1), (g >> 1) & 1)) break;
        // PV(g - 2) is done (its commit precedes that of S(g)); waited for all the
        // same, so that this barrier is never more than one phase ahead of its waiter
        if (g >= 2 && !wait(B_PV + (g & 1), ((g >> 1) - 1) & 1)) break;
        tc_fence_after();
        const uint32_t tS = tl + (g & 1) * 128;
        float x[BN];
#pragma unroll
        for (int c = 0; c < BN / 32; ++c) tmem_ld32(tS + c * 32, reinterpret_cast<uint32_t *>(x + c * 32));
        tmem_wait_ld();
        const int off = (sg.kt0 + j) * BN - sg.r.ctx;  // key c of the tile is draft off + c
        if (off > -BN) {
          // its visible keys as 128 bits: all below the context's end, then the
          // ancestors' bits
          uint32_t w[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int o = off + 32 * q;  // draft of bit 0 of the word
            w[q] = o >= 64 ? 0u : o >= 0 ? (uint32_t)(mask >> o)
                 : o <= -32 ? 0xffffffffu
                            : (0xffffffffu >> (32 + o)) | ((uint32_t)mask << -o);
          }
#pragma unroll
          for (int c = 0; c < BN; ++c)
            if (!((w[c >> 5] >> (c & 31)) & 1u)) x[c] = -INFINITY;
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < BN; c += 8)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx[i] = max3f(mx[i], x[c + 2 * i], x[c + 2 * i + 1]);
        const float m_new = fmaxf(m_used, max3f(mx[0], mx[1], fmaxf(mx[2], mx[3])) * p.scale_log2);
        const bool resc = m_new > m_used + 8.f;
        float alpha = 1.f;
        if (resc) {
          alpha = ex2(m_used - m_new);
          m_used = m_new;
        }
        if (j > 0 && __any_sync(0xffffffffu, resc)) {
          if (!wait(B_PV + ((g - 1) & 1), ((g - 1) >> 1) & 1)) break;  // PV(g - 1) has finished
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            float o[16];
            tmem_ld16(tO + c * 16, reinterpret_cast<uint32_t *>(o));
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < 16; ++q) o[q] *= alpha;
            tmem_st16(tO + c * 16, reinterpret_cast<uint32_t *>(o));
          }
        }
        const float mref = m_used == -INFINITY ? 0.f : m_used;
        const uint64_t sc2 = f2pack(p.scale_log2, p.scale_log2), nm2 = f2pack(-mref, -mref);
        uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int c0 = 0; c0 < BN; c0 += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const uint64_t e = exp2_mufu2(fma2(f2pack(x[c0 + 2 * q], x[c0 + 2 * q + 1]), sc2, nm2));
            acc[q & 3] = add2(acc[q & 3], e);
            float e0, e1;
            f2unpack(e, e0, e1);
            pk[q] = pack2(e0, e1);
          }
          tmem_st16(tS + c0 / 2, pk);
        }
        float l0, l1;
        f2unpack(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), l0, l1);
        l = fmaf(l, alpha, l0 + l1);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_P + (g & 1)));
      }
      if (!ok) break;
      // ---- the segment's last PV, then its rows
      if (!wait(B_PV + ((g - 1) & 1), ((g - 1) >> 1) & 1)) break;
      tc_fence_after();
      const bool whole = sg.first && sg.last;
      const size_t o_row = (((size_t)sg.b * p.max_draft + tok) * p.Hq + head);
      const size_t p_row = (size_t)sg.slot() * BM + row;
      const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float o[32];
        tmem_ld32(tO + c * 32, reinterpret_cast<uint32_t *>(o));
        tmem_wait_ld();
        if (whole) {
#pragma unroll
          for (int q = 0; q < 32; ++q) o[q] *= inv;
          if (valid)
#pragma unroll
            for (int q = 0; q < 4; ++q) st_global16(p.out + o_row * D + c * 32 + q * 8, pack8(o + q * 8));
        } else if (valid) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            *reinterpret_cast<float4 *>(p.part_o + p_row * D + c * 32 + q * 4) =
                make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_OEMPTY + ob));
      if (whole) {
        if (valid && p.lse)
          p.lse[o_row] = l > 0.f ? (m_used + __log2f(l)) * 0.69314718055994531f : -INFINITY;
      } else if (valid) {
        p.part_ml[p_row] = make_float2(l > 0.f ? m_used : -INFINITY, l);
      }
      ++s;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tbase, kTmemCols);
  }
}

// ------------------------------------------------------------------- merge
// o = sum_c w_c O_c / sum_c w_c l_c, w_c = 2^(m_c - M), over the CTAs that hold
// key tiles of a row's unit: one CTA per (token, query head), its four warps
// over the partials, combined in shared memory in a fixed order.
template <int D>
__global__ void __launch_bounds__(128) draft_merge_kernel(Params p) {
  constexpr int CPL = D / 32;
  __shared__ float acc_s[4][D], m_s[4], l_s[4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
  const Request r = request_of(p, b);
  if (i >= r.n) return;
  const int hk = h / p.G, rr = i * p.G + h % p.G, rt = rr / BM, row = rr % BM;
  const int2 u = p.unit[((size_t)b * p.Hkv + hk) * p.rt_max + rt];
  if (u.x == u.y) return;  // finished by its CTA
  float m = -INFINITY, l = 0.f, acc[CPL];
#pragma unroll
  for (int q = 0; q < CPL; ++q) acc[q] = 0.f;
  for (int c = u.x + warp; c <= u.y; c += 4) {
    const size_t pr = (size_t)(2 * c + (c == u.x ? 1 : 0)) * BM + row;
    const float2 ml = p.part_ml[pr];
    float v[CPL];
#pragma unroll
    for (int q = 0; q < CPL; ++q) v[q] = p.part_o[pr * D + q * 32 + lane];
    if (ml.y <= 0.f) continue;
    const float mn = fmaxf(m, ml.x), wa = m == -INFINITY ? 0.f : ex2(m - mn), wb = ex2(ml.x - mn);
    l = l * wa + ml.y * wb;
#pragma unroll
    for (int q = 0; q < CPL; ++q) acc[q] = acc[q] * wa + v[q] * wb;
    m = mn;
  }
#pragma unroll
  for (int q = 0; q < CPL; ++q) acc_s[warp][q * 32 + lane] = acc[q];
  if (lane == 0) m_s[warp] = m, l_s[warp] = l;
  __syncthreads();
  const float M = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
  float L = 0.f, w[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    w[c] = m_s[c] == -INFINITY ? 0.f : ex2(m_s[c] - M);
    L = fmaf(w[c], l_s[c], L);
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  const size_t o_row = ((size_t)b * p.max_draft + i) * p.Hq + h;
  for (int e = threadIdx.x; e < D; e += 128) {
    float a = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) a = fmaf(w[c], acc_s[c][e], a);
    p.out[o_row * D + e] = __float2bfloat16_rn(a * inv);
  }
  if (threadIdx.x == 0 && p.lse)
    p.lse[o_row] = L > 0.f ? (M + __log2f(L)) * 0.69314718055994531f : -INFINITY;
}

// -------------------------------------------------------------------- host
struct Plan {
  int r_pad, rt_max;
  size_t q_bytes, mask_bytes, unit_bytes, o_bytes, ml_bytes, total;
};
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline Plan plan(const pic_geom_t *g, int batch, int max_draft) {
  Plan pl;
  const int G = g->num_q_heads / g->num_kv_heads;
  pl.rt_max = (int)(((long long)max_draft * G + BM - 1) / BM);
  pl.r_pad = pl.rt_max * BM;
  pl.q_bytes = align256((size_t)batch * g->num_kv_heads * pl.r_pad * g->head_dim * 2);
  pl.mask_bytes = align256((size_t)batch * max_draft * 8);
  pl.unit_bytes = align256((size_t)batch * g->num_kv_heads * pl.rt_max * sizeof(int2));
  pl.o_bytes = align256((size_t)2 * kCtas * BM * g->head_dim * 4);
  pl.ml_bytes = align256((size_t)2 * kCtas * BM * sizeof(float2));
  pl.total = pl.q_bytes + pl.mask_bytes + pl.unit_bytes + pl.o_bytes + pl.ml_bytes;
  return pl;
}

template <int D>
static cudaError_t launch(const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv,
                          const Params &p, const RopeParams &rp, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(draft_attn_kernel<D>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       Layout<D>::kAlloc);
  if (e != cudaSuccess) return e;
  e = launch_dependent(draft_append_kernel<D>, dim3(p.max_draft, p.batch), dim3(128), 0, stream, p, rp);
  if (e != cudaSuccess) return e;
  e = launch_dependent(draft_attn_kernel<D>, dim3(kCtas), dim3(kThreads), Layout<D>::kAlloc, stream,
                       tq, tk, tv, p);
  if (e != cudaSuccess) return e;
  return launch_dependent(draft_merge_kernel<D>, dim3(p.Hq, p.max_draft, p.batch), dim3(128), 0,
                          stream, p);
}

}  // namespace draft
}  // namespace pic

extern "C" size_t pic_draft_workspace_size(const pic_geom_t *geom, int32_t batch,
                                           int32_t max_draft) {
  if (!geom || batch <= 0 || max_draft <= 0 || max_draft > pic::draft::kMaxDraft ||
      geom->num_kv_heads <= 0 || geom->num_q_heads <= 0 ||
      geom->num_q_heads % geom->num_kv_heads || (geom->head_dim != 64 && geom->head_dim != 128))
    return 0;
  return pic::draft::plan(geom, batch, max_draft).total;
}

extern "C" pic_status_t pic_attend_draft(const pic_geom_t *geom, int32_t layer, int32_t batch,
                                         int32_t max_draft, const void *q, const void *k_new,
                                         const void *v_new, const int32_t *ctx_len,
                                         const int32_t *draft_len, const int32_t *parent,
                                         const int32_t *block_table, int32_t max_pages,
                                         int64_t num_pages, void *k_cache, void *v_cache,
                                         void *out, float *lse, void *workspace,
                                         size_t workspace_bytes, pic_stream_t stream) {
  using namespace pic;
  using namespace pic::draft;
  static const char *who = "pic_attend_draft";
  RopeParams rp;
  pic_status_t st = make_rope(geom, &rp);
  if (st != PIC_OK) return st;
  if (layer < 0 || layer >= geom->num_layers)
    return fail(PIC_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", who, layer, geom->num_layers);
  if (batch <= 0 || max_draft <= 0 || max_pages <= 0 || num_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (max_draft > kMaxDraft)
    return fail(PIC_ERR_UNSUPPORTED, "%s: max_draft %d (at most %d)", who, max_draft, kMaxDraft);
  if (!q || !k_new || !v_new || !ctx_len || !draft_len || !block_table || !k_cache || !v_cache || !out)
    return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) |
       reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(k_cache) |
       reinterpret_cast<uintptr_t>(v_cache) | reinterpret_cast<uintptr_t>(out)) & 15)
    return fail(PIC_ERR_INVALID_ARG, "%s: bf16 tensors must be 16-byte aligned", who);
  const int D = geom->head_dim, Hkv = geom->num_kv_heads;
  const long long rows_total = (long long)geom->num_layers * num_pages * Hkv * 16;
  const Plan pl = plan(geom, batch, max_draft);
  if (rows_total + 16 >= INT32_MAX || (long long)batch * Hkv * pl.r_pad >= INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: cache or queries have more than 2^31 rows", who);
  if (batch > 65535) return fail(PIC_ERR_UNSUPPORTED, "%s: grid too large", who);
  if (!workspace || workspace_bytes < pl.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return fail(PIC_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", who, pl.total);

  Params p;
  p.batch = batch;
  p.max_draft = max_draft;
  p.Hq = geom->num_q_heads;
  p.Hkv = Hkv;
  p.G = p.Hq / Hkv;
  p.r_pad = pl.r_pad;
  p.rt_max = pl.rt_max;
  p.max_pages = max_pages;
  p.oob_row = (int)((rows_total + 15) / 16 * 16);
  p.layer = layer;
  p.num_pages = num_pages;
  p.layer_row0 = (long long)layer * num_pages * Hkv * 16;
  p.ctx_len = ctx_len;
  p.draft_len = draft_len;
  p.parent = parent;
  p.block_table = block_table;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
  p.v_new = static_cast<const __nv_bfloat16 *>(v_new);
  const size_t layer_elems = (size_t)num_pages * Hkv * 16 * D;
  p.k_cache = static_cast<__nv_bfloat16 *>(k_cache) + layer * layer_elems;
  p.v_cache = static_cast<__nv_bfloat16 *>(v_cache) + layer * layer_elems;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.qp = reinterpret_cast<__nv_bfloat16 *>(ws);
  ws += pl.q_bytes;
  p.mask = reinterpret_cast<uint64_t *>(ws);
  ws += pl.mask_bytes;
  p.unit = reinterpret_cast<int2 *>(ws);
  ws += pl.unit_bytes;
  p.part_o = reinterpret_cast<float *>(ws);
  ws += pl.o_bytes;
  p.part_ml = reinterpret_cast<float2 *>(ws);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.status = device_status_ptr();
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)D));

  CUtensorMap tq, tk, tv;
  st = encode_tmap_2d(&tq, p.qp, D, (uint64_t)batch * Hkv * pl.r_pad, (uint64_t)D * 2, 64, BM);
  if (D == 128) {
    const uint64_t heads = (uint64_t)geom->num_layers * num_pages * Hkv;
    if (st == PIC_OK) st = encode_tmap_pages128(&tk, k_cache, heads);
    if (st == PIC_OK) st = encode_tmap_pages128(&tv, v_cache, heads);
  } else {
    if (st == PIC_OK) st = encode_tmap_2d(&tk, k_cache, D, rows_total, (uint64_t)D * 2, 64, 16);
    if (st == PIC_OK) st = encode_tmap_2d(&tv, v_cache, D, rows_total, (uint64_t)D * 2, 64, 16);
  }
  if (st != PIC_OK) return st;
  cudaError_t e = D == 128 ? launch<128>(tq, tk, tv, p, rp, stream) : launch<64>(tq, tk, tv, p, rp, stream);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
