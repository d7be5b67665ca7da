// pic_attend_draft: one layer of one step over the drafted tokens of every
// request (a chain or a tree of up to 64 tokens behind the cached context).
//
// The attention reads each key and value of a request once for all its drafted
// tokens and query heads: a request's queries of one kv head are packed into
// rows r = token * G + head of 128-row tiles (one TMEM lane per row), so with up
// to 128 rows a key costs 4 d flops a row for the 4 d bytes that it and its
// value take: below about 280 rows a key tile's bytes take longer than its MMAs.  What a chain's causal mask or a
// tree's ancestor mask hides lies within the last 64 slots; every earlier key
// is visible to every row.
//
// Launches:
//  1. draft_append_kernel: per token its depth and ancestor bits, the rotated
//     key and the value into their slots, the rotated queries packed.
//  2. draft_attn_kernel: one persistent CTA per SM.  All (request, kv head, pair of
//     row tiles) units' key tiles form one sequence, unit after unit, of which
//     every CTA takes an equal share (the lengths are only known on the device,
//     and batches are ragged), so no SM waits for a longer request's.  A CTA's
//     share is a run of segments, each a range of one unit's key tiles; a unit
//     that lies within one CTA is finished there, the others leave partial states.
//  3. draft_merge_kernel: log-sum-exp merge of those.
//
// Measured, whole calls: 4 requests of 139k keys, 32 rows of each of 8 kv heads, 330
// us (2.29 GB: 6.92 TB/s; a plain copy runs at 6.79); 16 of 33k, 112 rows of 4 kv
// heads, 169 us (6.4 TB/s); 4 of 16k, 256 rows of 8 kv heads, 67.6 us (4.0 TB/s; the
// attention 58.6 of them); d = 64, 16 of 139k, 64 rows of 2 kv heads, 204 us (5.6 TB/s),
// 8 of 100k 85 us (4.8); one of 4288 keys 14.5 us, three dependent launches.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace draft {

constexpr int BM = 128, BN = 128;  // rows of a tile, keys of a tile
constexpr int kMaxDraft = 64;
constexpr int kCtas = 152;         // one per SM
constexpr int NSK = 3, NSV = 2;    // ring stages of K and V
constexpr int NQB = 2;             // query tiles
constexpr int kThreads = 384;      // K producer, MMA, V producer, ring, two softmax warpgroups
// The bound for the compiler: 127 registers a thread instead of 154.  With those, and with
// no shared memory to spare for an alignment, CTAs of the append and of the merge (one warp
// a row: none of either) fit beside one on an SM and begin early.  us with and without:
// 5 ragged requests, d = 64, 21.1 and 23.2; 24, d = 64, 20.0 and 21.9; d = 128, 4 of 16k
// with 256 rows 67.9 and 68.5, 4 of 139k 333.7 and 334.4, 24 tokens of 4 x 1000 15.3 and 14.9.
constexpr int kBoundThreads = 448;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;    // S_t at 128 t, O_t at 256 + D t
// Named barriers (0: __syncthreads): P_t from warpgroup t to the MMA warp, the
// ring warp's word to the MMA warp, the two warpgroups' exchange.
constexpr int kNbP = 1, kNbRing = 3, kNbPair = 4;

template <int D>
struct Layout {
  static constexpr int kTile = BN * D * 2;
  static constexpr int kQ = 0;
  static constexpr int kK = kQ + NQB * kTile;
  static constexpr int kV = kK + NSK * kTile;
  static constexpr int kML = kV + NSV * kTile;  // float [2][BM]: the warpgroups' m, then l
  static constexpr int kBar = kML + 2 * BM * 4;
  static constexpr int kAlloc = kBar + 256;
};

enum {
  B_QFULL = 0,
  B_QEMPTY = B_QFULL + NQB,
  B_KFULL = B_QEMPTY + NQB,
  B_KEMPTY = B_KFULL + NSK,
  B_VFULL = B_KEMPTY + NSK,
  B_VEMPTY = B_VFULL + NSV,
  B_VFIX = B_VEMPTY + NSV,   // per V stage: what must not meet a weight of zero is cleared
  B_SFULL = B_VFIX + NSV,    // S_t
  B_OEND = B_SFULL + 2,      // a segment's last PV of warpgroup t
  B_ODONE = B_OEND + 2,      // a segment's O read by both warpgroups
  B_END = B_ODONE + 1,
  B_COUNT = B_END + 1
};
static_assert(B_COUNT * 8 + 16 <= 256, "barrier area");

struct Params {
  int batch, max_draft, Hq, Hkv, G, r_pad, max_pages, oob_row, layer;
  long long num_pages, layer_row0;
  const int32_t *ctx_len, *draft_len, *parent, *block_table;
  const __nv_bfloat16 *q, *k_new, *v_new;
  __nv_bfloat16 *k_cache, *v_cache;  // at the layer
  __nv_bfloat16 *qp;                 // workspace: packed rotated queries
  uint64_t *mask;                    // workspace: [batch][max_draft] ancestor bits
  int32_t *wild;                     // workspace: [batch][max_draft] the value has an infinity or NaN
  struct Share *share;               // workspace: [kCtas] each CTA's start
  int32_t *rows;                     // workspace: [kCtas][32] K/V rows of its first 32 pages
  int4 *req;                         // workspace: [batch] first step, ctx_len, draft_len as dealt
  float *part_o;                     // workspace: [kCtas][2][row tile of the pair][BM][D]
  float2 *part_ml;                   // the same without [D]
  __nv_bfloat16 *out;
  float *lse;
  int32_t *status;
  float scale_log2;
};

// The ring warp's waits, in one place in the code: 11 KB less of it, which a call with
// cold instruction caches feels (one request of 4288 keys 14.5 and 14.2 us); the
// producers' waits as calls too cost 0.3% of long contexts.
__device__ __noinline__ bool ring_wait(uint32_t bar, uint32_t parity, volatile int *abort, int32_t *status,
                                       int detail) {
  return mbar_wait(bar, parity, abort, status, detail);
}

PIC_DEV void st_global32(void *p, const float *f) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]),
               "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
               : "memory");
}

// What a request brings: its key tiles and row tiles (0 for one left alone).
struct Request {
  int ctx, n, tiles, rt;
};
PIC_DEV Request request_of(const Params &p, int ctx, int n) {
  Request r;
  r.ctx = ctx;
  r.n = n;
  const bool ok = r.ctx >= 0 && r.n > 0 && r.n <= p.max_draft &&
                  (long long)r.ctx + r.n <= (long long)p.max_pages * 16;
  if (!ok) r.ctx = r.n = 0;
  r.tiles = ok ? (r.ctx + r.n + BN - 1) / BN : 0;
  r.rt = (r.n * p.G + BM - 1) / BM;
  return r;
}
PIC_DEV Request request_of(const Params &p, int b) {
  return request_of(p, p.ctx_len[b], p.draft_len[b]);
}

// The work is counted in steps, a row tile times a key tile: a unit of two row tiles
// has 2 `tiles` of them, two for each key tile, one of one row tile `tiles`; the
// pairs of a kv head come first.  (Two row tiles take nearly twice the time of one
// unless HBM sets the pace.)  A key tile belongs to the CTA whose share holds its
// last step.
//
// A CTA's share of the batch's `total` steps, which are dealt to `ctas` CTAs: steps
// [pos, end), the first of them in request b, whose first step is `base`, and
// there in the unit of (hk, pair) that begins at unit0.
struct alignas(16) Share {
  int total, ctas, pos, end, b, base, ctx, n;  // ctx, n: request b's
  int unit0, hk, pair, per;                    // per: total / ctas
};

PIC_DEV int work_of(const Params &p, const Request &r) { return p.Hkv * r.rt * r.tiles; }

// The unit of step pos of request r, whose first step is base.
PIC_DEV void unit_of(const Request &r, int base, int pos, int *unit0, int *hk, int *pair) {
  const int per = r.rt * r.tiles;  // of a kv head
  *hk = (pos - base) / per;
  *pair = (pos - base - *hk * per) / (2 * r.tiles);
  *unit0 = base + *hk * per + *pair * 2 * r.tiles;
}

// The first step of CTA c's share, floor(total c / ctas), without a 64-bit product
// or a division: total = q ctas + r, and r c < 2^15 leaves (r c + 1/2) / ctas at least
// 1 / 304 away from a whole number, far more than its rounding.
struct Deal {
  int ctas, q, r;
  float inv;
  PIC_DEV Deal(int total, int n, int quotient) : ctas(n), q(quotient), r(total - q * n), inv(1.f / (float)max(n, 1)) {}
  PIC_DEV int first(int c) const { return q * c + (int)(((float)(r * c) + 0.5f) * inv); }
  // The CTA whose share holds step t: a rounded estimate, then exact.
  PIC_DEV int owner(int t, int total) const {
    int c = min(ctas - 1, (int)((float)(t + 1) * (float)ctas / (float)total));
    while (first(c) > t) --c;
    while (first(c + 1) <= t) ++c;
    return c;
  }
};

// The K/V row (of the whole cache) of page pidx of request b's kv head hk; zeros
// are read for a page past the last key or outside the cache.
PIC_DEV int page_row(const Params &p, int page, int pidx, int keys, int hk) {
  if ((long long)pidx * 16 >= keys || page < 0 || page >= p.num_pages) return p.oob_row;
  return (int)(p.layer_row0 + ((long long)page * p.Hkv + hk) * 16);
}

// The shares of CTAs first .. first + 3 (every CTA that takes part has a tile), by
// one warp, lane l < 4 for CTA first + l; the warp of CTA 0 also notes every
// request's first step and lengths, from which the later kernels work: all roles of
// a CTA have to walk the same segments, whatever is written to ctx_len meanwhile.
constexpr int kDealt = 4;
PIC_DEV void deal_shares(const Params &p, int first) {
  const int lane = threadIdx.x & 31, c = first + lane;
  auto request = [&](int b) { return b < p.batch ? request_of(p, b) : Request{0, 0, 0, 0}; };
  const Request first32 = request(lane);  // mostly all of them: read once
  int total = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    int w = work_of(p, b0 ? request(b0 + lane) : first32);
#pragma unroll
    for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
    total += w;
  }
  // two steps at least, one for each softmax warpgroup: half as many are no faster
  // and leave twice the partials to merge
  const int ctas = min(kCtas, max(1, total / 2));
  Share sh{total, ctas, 0, 0, -1, 0, 0, 0, 0, 0, 0, total / ctas};
  const Deal deal(total, ctas, total / ctas);
  if (lane < kDealt && c < ctas && total > 0) sh.pos = deal.first(c), sh.end = deal.first(c + 1);
  int base = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const Request r = b0 ? request(b0 + lane) : first32;
    const int w = work_of(p, r);
    int x = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (first == 0 && b0 + lane < p.batch) p.req[b0 + lane] = make_int4(base + x - w, r.ctx, r.n, 0);
    // lane l's request holds steps [base + x - w, base + x): the one of step pos
#pragma unroll
    for (int k = 0; k < kDealt; ++k) {
      const int pos = __shfl_sync(0xffffffffu, sh.pos, k), end = __shfl_sync(0xffffffffu, sh.end, k);
      const unsigned in = __ballot_sync(0xffffffffu, end > 0 && pos >= base + x - w && pos < base + x);
      if (in) {
        const int l = __ffs(in) - 1;
        const int lo = base + __shfl_sync(0xffffffffu, x - w, l);
        const int ctx = __shfl_sync(0xffffffffu, r.ctx, l), n = __shfl_sync(0xffffffffu, r.n, l);
        if (lane == k) sh.b = b0 + l, sh.base = lo, sh.ctx = ctx, sh.n = n;
      }
    }
    base += __shfl_sync(0xffffffffu, x, 31);
  }
  const Request r = request_of(p, sh.ctx, sh.n);
  int kt0 = 0;
  if (r.tiles > 0) {
    unit_of(r, sh.base, sh.pos, &sh.unit0, &sh.hk, &sh.pair);
    kt0 = (sh.pos - sh.unit0) >> (2 * sh.pair + 1 < r.rt ? 1 : 0);
  }
  if (lane < kDealt && c < kCtas) p.share[c] = sh;
  // the rows of each CTA's first 32 pages: its producers then start from one round
  // trip
  int page[kDealt], pidx[kDealt], keys[kDealt], hk[kDealt];
#pragma unroll
  for (int k = 0; k < kDealt; ++k) {
    const int b = __shfl_sync(0xffffffffu, sh.b, k);
    pidx[k] = __shfl_sync(0xffffffffu, kt0, k) * 8 + lane;
    keys[k] = __shfl_sync(0xffffffffu, sh.ctx + sh.n, k);
    hk[k] = __shfl_sync(0xffffffffu, sh.hk, k);
    page[k] = -1;
    if (b >= 0 && (long long)pidx[k] * 16 < keys[k])
      page[k] = p.block_table[(size_t)b * p.max_pages + pidx[k]];
  }
#pragma unroll
  for (int k = 0; k < kDealt; ++k) {
    const int b = __shfl_sync(0xffffffffu, sh.b, k);
    if (b >= 0 && (long long)pidx[k] * 16 < keys[k] && (page[k] < 0 || page[k] >= p.num_pages))
      dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
    if (first + k < kCtas)
      p.rows[(first + k) * 32 + lane] = page_row(p, page[k], pidx[k], keys[k], hk[k]);
  }
}

// Of 8 bf16 values: whether there is an infinity or a NaN among them; zeros in their place.
PIC_DEV uint32_t wild_halves(uint32_t w) { return __vcmpeq2(w & 0x7f807f80u, 0x7f807f80u); }
PIC_DEV bool has_wild(const uint4 &v) {
  return (wild_halves(v.x) | wild_halves(v.y) | wild_halves(v.z) | wild_halves(v.w)) != 0;
}
PIC_DEV uint4 without_wild(const uint4 &v) {
  return make_uint4(v.x & ~wild_halves(v.x), v.y & ~wild_halves(v.y), v.z & ~wild_halves(v.z),
                    v.w & ~wild_halves(v.w));
}
// Request b's tokens with such a value, from what lane l read for tokens l and l + 32.
struct Wild {
  int a, b;
  PIC_DEV Wild(const Params &p, int req, int n) {
    const int lane = threadIdx.x & 31;
    const int32_t *w = p.wild + (size_t)req * p.max_draft;
    a = lane < n ? w[lane] : 0;
    b = lane + 32 < n ? w[lane + 32] : 0;
  }
  PIC_DEV uint64_t tokens() const {
    return __ballot_sync(0xffffffffu, a != 0) | (uint64_t)__ballot_sync(0xffffffffu, b != 0) << 32;
  }
};

// ------------------------------------------------------------------ append
// One CTA per token, behind `dealers` CTAs that deal out the work.  A thread takes
// a chunk (8 pairs) of a query or key head, and a value piece: the host gives the
// CTAs as many threads as there are chunks, up to kAppendMax.  Bound by its chain of
// loads (lengths and parents, the page, cos/sin): 3.6 to 5.5 us for 4 to 256 tokens.  One
// place in the code rotates, because a call starts with cold instruction caches (three chunks a
// thread, their rotations unrolled, took 5.3 us instead of 4.9, 16 x 16 tokens).
constexpr int kAppendMax = 512;

// Token i and its ancestors as bits, by one warp whose lanes hold the parents of
// tokens lane and lane + 32: each round doubles the ancestors that a token knows.
// (A walk up took 1.7 us for a line of 64.)  A parent that is none is read as -1.
PIC_DEV uint64_t ancestors(const Params &p, const int (&parent)[2], int b, int i) {
  const int lane = threadIdx.x & 31;
  uint64_t m[2];
  int up[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int q = lane + 32 * k;
    const bool bad = parent[k] < -1 || parent[k] >= q;
    if (bad && q == i) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    m[k] = 1ull << q;
    up[k] = bad ? -1 : parent[k];
  }
  while (__any_sync(0xffffffffu, up[0] >= 0 || up[1] >= 0)) {
    uint64_t nm[2];
    int nu[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int from = up[k] & 31;
      const uint64_t m0 = __shfl_sync(0xffffffffu, m[0], from), m1 = __shfl_sync(0xffffffffu, m[1], from);
      const int u0 = __shfl_sync(0xffffffffu, up[0], from), u1 = __shfl_sync(0xffffffffu, up[1], from);
      nm[k] = up[k] < 0 ? m[k] : m[k] | (up[k] < 32 ? m0 : m1);
      nu[k] = up[k] < 0 ? -1 : up[k] < 32 ? u0 : u1;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) m[k] = nm[k], up[k] = nu[k];
  }
  const uint64_t m0 = __shfl_sync(0xffffffffu, m[0], i & 31), m1 = __shfl_sync(0xffffffffu, m[1], i & 31);
  return i < 32 ? m0 : m1;
}

template <int D>
__global__ void __launch_bounds__(kAppendMax) draft_append_kernel(Params p, RopeParams rp, int dealers) {
  constexpr int KC = D / 16;
  pdl_entry();
  __shared__ float2 cs[D / 2];
  __shared__ int depth;
  // (the dealers first: theirs is the longer chain)
  const int tid = threadIdx.x, threads = blockDim.x;
  if ((int)blockIdx.x < dealers) {
    deal_shares(p, ((int)blockIdx.x * (threads >> 5) + (tid >> 5)) * kDealt);
    return;
  }
  const int item = (int)blockIdx.x - dealers;
  const int b = item / p.max_draft, i = item % p.max_draft;
  const size_t tok = (size_t)b * p.max_draft + i;
  // The token's projections go out before anything is known of its request
  const int units = (p.Hq + p.Hkv) * KC;
  // (the CTA's threads are a multiple of KC: a thread's chunk of a row is always the
  // same)
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);
  uint4 qa = make_uint4(0, 0, 0, 0), qb = qa, vn = qa;
  auto load = [&](int u) {
    const int h = u / KC;
    const __nv_bfloat16 *src =
        h < p.Hq ? p.q + (tok * p.Hq + h) * D : p.k_new + (tok * p.Hkv + h - p.Hq) * D;
    qa = ld_stream(src + pc.off_a);
    qb = ld_stream(src + pc.off_b);
  };
  if (tid < units) load(tid);
  const int pieces = p.Hkv * (D / 8);
  const __nv_bfloat16 *v_src = p.v_new + tok * p.Hkv * D;
  if (tid < pieces) vn = ld_stream(v_src + tid * 8);
  int up[2] = {-1, -1};  // warp 0: the parents of tokens tid and tid + 32
  if (p.parent && tid < 32)
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (tid + 32 * k < p.max_draft) up[k] = p.parent[(size_t)b * p.max_draft + tid + 32 * k];
  const uint64_t turn = tid < D / 2 ? rope_turn(rope_theta(rp, p.layer, tid)) : 0;
  const int ctx = p.ctx_len[b], n = p.draft_len[b];
  const bool bad = ctx < 0 || n < 0 || n > p.max_draft;
  if (bad || (long long)ctx + n > (long long)p.max_pages * 16) {
    if (i == 0 && tid == 0)
      dev_fail(p.status, bad ? PIC_DEV_BAD_REQUEST : PIC_DEV_BLOCK_TABLE_SHORT, b);
    return;
  }
  if (i >= n) return;
  const int slot = ctx + i;
  int page = p.block_table[(size_t)b * p.max_pages + slot / 16];
  if (tid < 32) {
    uint64_t line = ~0ull >> (63 - i);  // token i and its ancestors
    if (p.parent) line = ancestors(p, up, b, i);
    if (tid == 0) {
      p.mask[tok] = line;
      p.wild[tok] = 0;  // (a thread that finds one writes 1 behind a barrier)
      depth = __popcll(line) - 1;
      if (page < 0 || page >= p.num_pages) dev_fail(p.status, PIC_DEV_BAD_PAGE, b);
    }
  }
  if (page >= p.num_pages) page = -1;
  __syncthreads();
  if (tid < D / 2) cs[tid] = rope_cos_sin_turn(ctx + depth, turn);
  __syncthreads();
#pragma unroll 1
  for (int u = tid; u < units; u += threads) {
    if (u != tid) load(u);
    const int h = u / KC, hk = h < p.Hq ? h / p.G : h - p.Hq;
    __nv_bfloat16 *dst = nullptr;
    if (h < p.Hq)
      dst = p.qp + ((size_t)(b * p.Hkv + hk) * p.r_pad + i * p.G + h - hk * p.G) * D;
    else if (page >= 0)
      dst = p.k_cache + (((size_t)page * p.Hkv + hk) * 16 + slot % 16) * D;
    if (dst) rotate_store(qa, qb, dst, pc, rp.style, cs + 8 * (tid % KC));
  }
  bool wild = false;
  if (page >= 0)
#pragma unroll 1
    for (int u = tid; u < pieces; u += threads) {
      const int hk = u / (D / 8), c = u % (D / 8);
      if (u != tid) vn = ld_stream(v_src + u * 8);
      wild |= has_wild(vn);
      st_global16(p.v_cache + (((size_t)page * p.Hkv + hk) * 16 + slot % 16) * D + c * 8, vn);
    }
  if (wild) p.wild[tok] = 1;
}

// ---------------------------------------------------------------- schedule
// The segments of one CTA, walked by each role's warp for itself.
struct Segments {
  const Params &p;
  int pos, end;         // next step (the host keeps them below 2^31), end of this CTA's share
  int base;             // first step of request b
  int b, cta;
  Request r;
  // the present segment
  int hk, pair, kt0, n;
  bool two;          // the pair has two row tiles
  bool first, last;  // holds the unit's first, last key tile
  int unit0;         // the unit's first step

  PIC_DEV Segments(const Params &pp, int cta_) : p(pp), cta(cta_) {
    const int4 *q = reinterpret_cast<const int4 *>(p.share + cta);
    const int4 x = q[0], y = q[1], z = q[2];
    pos = x.z, end = x.w;
    b = y.x, base = y.y;
    r = request_of(p, y.z, y.w);
    unit0 = z.x, hk = z.y, pair = z.z;  // the first segment's unit
    two = 2 * pair + 1 < r.rt;
  }
  PIC_DEV bool next() {
    if (pos >= end) return false;
    if (pos >= unit0 + (r.tiles << (two ? 1 : 0))) {  // a unit behind the first segment's
      while (pos - base >= work_of(p, r)) {
        if (++b >= p.batch) {
          pos = end;
          return false;
        }
        const int4 x = p.req[b];
        base = x.x;
        r = request_of(p, x.y, x.z);
      }
      unit_of(r, base, pos, &unit0, &hk, &pair);
      two = 2 * pair + 1 < r.rt;
    }
    const int shift = two ? 1 : 0;
    kt0 = (pos - unit0) >> shift;
    n = min(r.tiles, (end - unit0) >> shift) - kt0;
    if (n <= 0) return false;  // half a key tile of the next CTA's
    first = kt0 == 0;
    last = kt0 + n == r.tiles;
    pos = last ? unit0 + (r.tiles << shift) : end;
    return true;
  }
  // the partial slot of row tile t of the present segment: a CTA has at most
  // one segment that ends a unit begun elsewhere or lies inside one (0), and one
  // that begins a unit and leaves its end to others (1)
  PIC_DEV int slot(int t) const { return (2 * cta + (first ? 1 : 0)) * 2 + t; }
  // key tiles of warpgroup t (see draft_attn_kernel)
  PIC_DEV int count(int t) const { return two ? n : (n + 1 - t) / 2; }
  PIC_DEV int drafts() const { return (kt0 + n) * BN > r.ctx ? r.n : 0; }  // 0: the segment holds none
};

// --------------------------------------------------------------- attention
// Two softmax warpgroups, one query row per thread, each with its scores S_t and
// its accumulator O_t in TMEM.  Where a unit has two row tiles, warpgroup t takes
// row tile t, and both read every key tile; with one row tile, warpgroup t takes
// the key tiles of parity t, and the two states are joined at the segment's end
// (each warpgroup half of the columns).  Either way one warpgroup's softmax runs
// beside the other's MMAs.  MMA order, for t = 0, 1, 0, ...: PV_t of warpgroup t's
// tile before, QK_t of its next one, across segments.  MMAs complete in order, so
// S_t full means that PV_t has finished and O_t may be rescaled; O_t is only
// rescaled when a row's maximum grew by more than 2^8.
//
// Scores, maxima, sums and O are held in fp32, partial states too.  P is rounded to
// bf16, the type in which the tensor core multiplies it with V: against 64 bits a
// row's output is off by 0.0026 to 0.0029, where 32-bit weights give 0.0023 to 0.0024
// (most of that the output's own rounding; 0.0034 to 0.0038 and 0.0033 to 0.0036 with
// queries scaled by 2).
//
// Bound by HBM with one row tile of d = 128: 325 us for 4 x 139k keys (7.0 TB/s), 163 us cold
// for 16 x 33k (6.6 TB/s, DRAM 84% busy, tensor pipe 37%).  With two row tiles (4 x 16k keys, 256
// rows: 58.6 us, DRAM 58% busy, tensor pipe 60%) and with d = 64, whose key tile is half the
// bytes (16 x 139k: 200 us, DRAM 72%; 8 x 100k: 81 us, 65%; tensor pipe 30%, issue slots 40%),
// neither is at its limit: the chain of a key tile's MMAs and softmax.  With 512 rows a key tile of
// two row tiles takes about 2750 cycles where its MMAs need 2080; for short contexts
// set-up, first tiles and the epilogue count (7.2 us with two key tiles in all).
// Against the short loops below: all scores of a row in registers were 6% slower; half
// of them kept from the maximum for the exponentials, or no maximum after the first
// tile, 1% faster at best and up to 9% slower in short calls.
//
// Waits: the MMA warp meets the ring warp (which waits for K, V, Q and the
// accumulators on its behalf) and the softmax warps on named barriers only.  These
// have no limit, so after a wait that ran out every role still walks all segments
// and meets each barrier; the MMA warp then issues nothing but its commits.
template <int D>
__global__ void __launch_bounds__(kBoundThreads, 1)
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
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  if (sbase & 1023) {  // the tiles' swizzle counts on the array's alignment
    if (threadIdx.x == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, -1);
    return;
  }
  auto bar = [&](int i) { return sbase + L::kBar + 8u * (uint32_t)i; };
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::kBar + 8 * B_COUNT);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kBar + 8 * B_COUNT + 8);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < B_COUNT; ++i) mbar_init(bar(i), i == B_ODONE ? 8 : 1);
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

  Segments sg(p, (int)blockIdx.x);
  if (warp >= 4) {
    // ===================================================== softmax
    const int t = (warp - 4) >> 2, wq = warp & 3, row = wq * 32 + lane;
    const uint32_t tl = tbase + ((uint32_t)(wq * 32) << 16);
    const uint32_t tS = tl + t * 128, tO = tl + kColO + t * D;
    float *ml_s = reinterpret_cast<float *>(smem + L::kML);
    int nS = 0, nEnd = 0;  // tiles and segments of this warpgroup
    bool ok = true;
    // The MMA warp commits every S_t and every segment's end, also after an abort
    auto wait = [&](int i, uint32_t parity) {
      const bool was = ok;
      ok = mbar_wait_while(ok, bar(i), parity, p.status, detail, 4 * kWaitLimitNs);
      if (was && !ok) *abort_flag = 1;
    };
    while (sg.next()) {
      const int n = sg.count(t);
      const Wild wild(p, sg.b, sg.drafts());
      // this thread's row: token rr / G, query head hk G + rr % G
      auto row_of = [&]() { return (2 * sg.pair + (sg.two ? t : 0)) * BM + row; };
      float m_used = -INFINITY, l = 0.f;
      for (int i = 0; i < n; ++i, ++nS) {
        const int kt = sg.kt0 + (sg.two ? i : 2 * i + t);
        wait(B_SFULL + t, nS & 1);
        tc_fence_after();
        // The scores are read twice, 32 columns at a time, once for the maximum and
        // once for the exponentials: the loops stay short, and short code counts
        // for more than the second read, because each call begins with cold
        // instruction caches (with a row's 128 scores in registers and everything
        // unrolled, a request of 4k keys spent half of its 12600 cycles on that).
        float x0[32], x1[32];
        auto load = [&](float *x, int c) { tmem_ld32(tS + c * 32, reinterpret_cast<uint32_t *>(x)); };
        auto chunks = [&](auto &&work) {  // work(x, c), the next chunk on its way meanwhile
          load(x0, 0);
          tmem_wait_ld();
#pragma unroll 1
          for (int c = 0; c < BN / 32; c += 2) {
            load(x1, c + 1);
            work(x0, c);
            tmem_wait_ld();
            if (c + 2 < BN / 32) load(x0, c + 2);
            work(x1, c + 1);
            tmem_wait_ld();
          }
        };
        const int off = kt * BN - sg.r.ctx;  // key c of the tile is draft off + c
        if (off > -BN) {
          // hide what the row does not see: of a chunk's keys as 32 bits, those below
          // the context's end are visible, then the ancestors' bits
          const int rr = row_of();
          const uint64_t mask =
              rr < sg.r.n * p.G ? p.mask[(size_t)sg.b * p.max_draft + rr / p.G] : 0;
#pragma unroll 1
          for (int c = 0; c < BN / 32; ++c) {
            const int o = off + 32 * c;  // draft of the chunk's first key
            if (o <= -32) continue;
            const uint32_t w = o >= 64 ? 0u : o >= 0 ? (uint32_t)(mask >> o)
                               : (0xffffffffu >> (32 + o)) | ((uint32_t)mask << -o);
            load(x0, c);
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (!((w >> q) & 1u)) x0[q] = -INFINITY;
            tmem_st32(tS + c * 32, reinterpret_cast<uint32_t *>(x0));
          }
          tmem_wait_st();
        }
        float mx[2] = {-INFINITY, -INFINITY};
        chunks([&](const float *x, int) {
#pragma unroll
          for (int q = 0; q < 32; q += 4) {
            mx[0] = max3f(mx[0], x[q], x[q + 1]);
            mx[1] = max3f(mx[1], x[q + 2], x[q + 3]);
          }
        });
        const float m_new = fmaxf(m_used, fmaxf(mx[0], mx[1]) * p.scale_log2);
        const bool resc = m_new > m_used + 8.f;
        float alpha = 1.f;
        if (resc) {
          alpha = ex2(m_used - m_new);
          m_used = m_new;
        }
        if (i > 0 && __any_sync(0xffffffffu, resc)) {
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
        uint64_t acc[2] = {0, 0};
        // P of chunk c over columns 16 c .. 16 c + 15, whose scores have been read
        chunks([&](const float *x, int c) {
          uint32_t pk[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const uint64_t e = exp2_mufu2(fma2(f2pack(x[2 * q], x[2 * q + 1]), sc2, nm2));
            acc[q & 1] = add2(acc[q & 1], e);
            float e0, e1;
            f2unpack(e, e0, e1);
            pk[q] = pack2(e0, e1);
          }
          tmem_st16(tS + c * 16, pk);
        });
        float l0, l1;
        f2unpack(add2(acc[0], acc[1]), l0, l1);
        l = fmaf(l, alpha, l0 + l1);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        named_bar_arrive(kNbP + t, 128 + 32);
      }
      // ---- the segment's rows: after its last PV, o = w_0 O_0 + w_1 O_1 (with one
      // row tile), or O_t alone
      if (n > 0) {
        wait(B_OEND + t, nEnd & 1);
        ++nEnd;
        tc_fence_after();
      }
      float M = m_used, w0 = 1.f, w1 = 0.f;
      if (!sg.two) {  // m, then l through one array of shared memory
        auto exchange = [&](float v) {
          ml_s[t * BM + row] = v;
          named_bar_sync(kNbPair, 256);
          const float other = ml_s[(t ^ 1) * BM + row];
          named_bar_sync(kNbPair, 256);
          return other;
        };
        tc_fence_before();
        const float mo = exchange(m_used), lo = exchange(l);
        tc_fence_after();
        M = fmaxf(m_used, mo);
        const float wt = m_used == -INFINITY ? 0.f : ex2(m_used - M);
        const float wo = mo == -INFINITY ? 0.f : ex2(mo - M);
        l = t ? fmaf(lo, wo, l * wt) : fmaf(l, wt, lo * wo);  // l_0 w_0 + l_1 w_1 in both
        w0 = t ? wo : wt;
        w1 = t ? wt : wo;
      }
      const int rr = row_of();
      const bool valid = rr < sg.r.n * p.G;
      const bool store = valid && ok && !*abort_flag, whole = sg.first && sg.last;
      const size_t o_row = ((size_t)sg.b * p.max_draft + rr / p.G) * p.Hq + sg.hk * p.G + rr % p.G;
      const size_t p_row = (size_t)sg.slot(sg.two ? t : 0) * BM + row;
      const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
      const int c_begin = sg.two ? 0 : t * (D / 64), c_end = sg.two ? D / 32 : (t + 1) * (D / 64);
      const uint32_t tA = sg.two ? tO : tl + kColO;
#pragma unroll 1
      for (int c = c_begin; c < c_end; ++c) {
        float o[32];
        tmem_ld32(tA + c * 32, reinterpret_cast<uint32_t *>(o));
        tmem_wait_ld();
        if (!sg.two) {
#pragma unroll
          for (int q = 0; q < 32; ++q) o[q] *= w0;
          if (sg.n > 1) {  // (with one tile O_1 was never written)
            float o1[32];
            tmem_ld32(tA + D + c * 32, reinterpret_cast<uint32_t *>(o1));
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < 32; ++q) o[q] = fmaf(o1[q], w1, o[q]);
          }
        }
        if (whole) {
#pragma unroll
          for (int q = 0; q < 32; ++q) o[q] *= inv;
          if (store)
#pragma unroll
            for (int q = 0; q < 4; ++q) st_global16(p.out + o_row * D + c * 32 + q * 8, pack8(o + q * 8));
        } else if (store) {
          // 32 bytes at a time: a lane's row is its own, so each store of 16 would
          // be half a sector
#pragma unroll
          for (int q = 0; q < 32; q += 8) st_global32(p.part_o + p_row * D + c * 32 + q, o + q);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_ODONE));
      // infinities and NaN in the values of the segment's drafts lo .. hi - 1, which were
      // taken out of PV, for the rows that see them
      const int lo = max(0, sg.kt0 * BN - sg.r.ctx), hi = min(kMaxDraft, (sg.kt0 + sg.n) * BN - sg.r.ctx);
      uint64_t seen = hi > lo ? wild.tokens() : 0;
      if (seen && store) {
        seen &= p.mask[(size_t)sg.b * p.max_draft + rr / p.G] & (~0ull >> (64 - hi + lo) << lo);
#pragma unroll 1
        for (; seen; seen &= seen - 1) {
          const size_t token = (size_t)sg.b * p.max_draft + __ffsll((long long)seen) - 1;
          const __nv_bfloat16 *v = p.v_new + (token * p.Hkv + sg.hk) * D;
#pragma unroll 1
          for (int e = c_begin * 32; e < c_end * 32; ++e) {
            const float x = __bfloat162float(v[e]);
            if (fabsf(x) <= 3.4e38f) continue;
            if (whole)
              p.out[o_row * D + e] = __float2bfloat16(__bfloat162float(p.out[o_row * D + e]) + x);
            else
              p.part_o[p_row * D + e] += x;
          }
        }
      }
      __syncwarp();
      if (store && (sg.two || t == 0)) {
        if (!whole)
          p.part_ml[p_row] = make_float2(l == 0.f ? -INFINITY : M, l);
        else if (p.lse)
          p.lse[o_row] = l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994531f;
      }
    }
  } else if (warp == 0 || warp == 2) {
    // ===================================================== TMA producers
    // Warp 0 the query tiles of each segment and K, warp 2 V.  Lane l < 8
    // moves page l of a tile as one box.
    const bool is_k = warp == 0;
    const int nst = is_k ? NSK : NSV;
    const int b_full = is_k ? B_KFULL : B_VFULL, b_empty = is_k ? B_KEMPTY : B_VEMPTY;
    const uint32_t ring = sbase + (is_k ? L::kK : L::kV);
    const CUtensorMap *tmap = is_k ? &tm_k : &tm_v;
    int g = 0, nq = 0;  // key and query tiles issued
    const int rows_first = p.rows[blockIdx.x * 32 + lane];
    bool at_start = true;  // in the share's first segment
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      if (ok)
        ok = __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, p.status, detail));
      return ok;
    };
    while (ok && sg.next()) {
      const int keys = sg.r.ctx + sg.r.n;
      const Wild wild(p, sg.b, is_k ? 0 : sg.drafts());
      if (is_k)
        for (int t = 0; t <= (sg.two ? 1 : 0); ++t, ++nq) {
          const int qb = nq % NQB;
          if (nq >= NQB && !wait(B_QEMPTY + qb, (nq / NQB - 1) & 1)) break;
          if (lane == 0) {
            mbar_expect_tx(bar(B_QFULL + qb), L::kTile);
            const int row = (sg.b * p.Hkv + sg.hk) * p.r_pad + (2 * sg.pair + t) * BM;
#pragma unroll
            for (int pn = 0; pn < PANELS; ++pn)
              tma_load_2d(sbase + L::kQ + qb * L::kTile + pn * BM * 128, &tm_q, pn * 64, row,
                          bar(B_QFULL + qb));
          }
          __syncwarp();
        }
      // The block-table entries of four tiles at a time, a lane per page, read four
      // tiles ahead of their use.
      const int32_t *bt = p.block_table + (size_t)sg.b * p.max_pages;
      auto entry = [&](int j) {  // of page `lane` of the four tiles from tile j on
        const int pidx = (sg.kt0 + j) * 8 + lane;
        return j < sg.n && (long long)pidx * 16 < keys ? bt[pidx] : -1;
      };
      int next = -1, y4 = rows_first;
      if (!at_start) next = entry(0);
      for (int j = 0; ok && j < sg.n; ++j) {
        const int st = g % nst, kt = sg.kt0 + j;
        if ((j & 3) == 0 && (j > 0 || !at_start)) {
          const int pidx = kt * 8 + lane;
          if (is_k && (long long)pidx * 16 < keys && j + lane / 8 < sg.n &&
              (next < 0 || next >= p.num_pages))
            dev_fail(p.status, PIC_DEV_BAD_PAGE, sg.b);
          y4 = page_row(p, next, pidx, keys, sg.hk);
        }
        const int y = __shfl_sync(0xffffffffu, y4, (j & 3) * 8 + (lane & 7));
        if (g >= nst && !wait(b_empty + st, (g / nst - 1) & 1)) break;
        if (lane == 0) mbar_expect_tx(bar(b_full + st), L::kTile);
        __syncwarp();
        if (lane < 8) {
          const uint32_t dst = ring + st * L::kTile + lane * kPageBytes;
          if constexpr (PANELS == 2)
            tma_load_4d(dst, tmap, 0, 0, 0, y >> 3, bar(b_full + st));
          else
            tma_load_2d(dst, tmap, 0, y, bar(b_full + st));
        }
        if ((j & 3) == 0) next = entry(j + 4);
        ++g;
        if (is_k) continue;
        // A weight of zero does not silence an infinity.  Before PV reads them, rows
        // behind the last draft, which may hold anything, are cleared, and the drafts'
        // own infinities and NaN (rows that do not see them have weight zero there).
        const bool end = kt == sg.r.tiles - 1;
        if ((kt + 1) * BN > sg.r.ctx && (end || wild.tokens())) {
          if (!wait(b_full + st, ((g - 1) / nst) & 1)) break;
          const int r0 = keys - kt * BN, r1 = (r0 + 15) & ~15;  // the rest of its page
          constexpr int CH = D / 8;
          auto piece = [&](int row, int ch) {
            const int rr = row & 15;
            const uint32_t off =
                PANELS == 2 ? (uint32_t)((rr >> 3) * 2048 + (ch >> 3) * 1024 + (rr & 7) * 128 +
                                         (((ch & 7) ^ (rr & 7)) << 4))
                            : (uint32_t)(rr * 128 + ((ch ^ (rr & 7)) << 4));
            return ring + st * L::kTile + (row >> 4) * kPageBytes + off;
          };
          const int z0 = wild.tokens() ? max(0, sg.r.ctx - kt * BN) : r0, z1 = end ? r1 : BN;
          for (int e = lane; e < (z1 - z0) * CH; e += 32) {
            const uint32_t at = piece(z0 + e / CH, e % CH);
            sts128(at, z0 + e / CH >= r0 ? make_uint4(0, 0, 0, 0) : without_wild(lds128(at)));
          }
          fence_proxy_async();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(bar(B_VFIX + st));
      }
      at_start = false;
    }
    // what was issued lands before the CTA exits
    if (lane == 0) {
      for (int j = max(0, g - nst); j < g; ++j)
        mbar_wait_no_flag(bar(b_full + j % nst), (j / nst) & 1, p.status, detail, kWaitLimitNs);
      if (is_k)
        for (int j = max(0, nq - NQB); j < nq; ++j)
          mbar_wait_no_flag(bar(B_QFULL + j % NQB), (j / NQB) & 1, p.status, detail, kWaitLimitNs);
    }
  } else if (warp == 1) {
    // ===================================================== MMA issuer
    const uint32_t el = elect_one();
    const uint32_t ub = __shfl_sync(0xffffffffu, tbase, 0);
    const MatDesc dQ = sdesc_sw128(sbase + L::kQ, 16, 1024);
    const MatDesc dK = sdesc_sw128(sbase + L::kK, 16, kGroupStride);
    const MatDesc dV = sdesc_sw128(sbase + L::kV, kPanelOff, kGroupStride);
    // the tile of warpgroup t whose QK was issued last and whose PV comes next
    int pv_g[2] = {-1, -1};
    bool pv_first[2] = {}, pv_end[2] = {}, pv_free[2] = {};  // its segment's first, last of this warpgroup; V free behind it
    auto pv = [&](int t, bool go) {
      named_bar_sync(kNbP + t, 128 + 32);  // P_t
      tc_fence_after();
      const int st = pv_g[t] % NSV;
      const uint32_t tO = ub + kColO + t * D, tP = ub + t * 128;
      const MatDesc dv = dV.at(st * L::kTile);
      if (go)
#pragma unroll
        for (int kk = 0; kk < BN / 16; ++kk)
          mma_ts(tO, tP + kk * 8, dv.at(kk * kPageBytes), IDESC_PV, !(pv_first[t] && kk == 0), el);
      if (pv_free[t]) mma_commit(bar(B_VEMPTY + st), el);
      if (pv_end[t]) mma_commit(bar(B_OEND + t), el);
    };
    int g0 = 0, q0 = 0;  // key and query tiles of the segments before
    while (sg.next()) {
      const int macros = sg.count(0);
      for (int m = 0; m < macros; ++m)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bool cur = m < sg.count(t);
          if (!cur && pv_g[t] < 0) continue;
          const bool go = !named_bar_or(kNbRing, 64, false);
          tc_fence_after();
          if (pv_g[t] >= 0) pv(t, go);
          pv_g[t] = -1;
          if (!cur) continue;
          const int j = sg.two ? m : 2 * m + t, g = g0 + j, st = g % NSK;
          const int qb = (q0 + (sg.two ? t : 0)) % NQB;
          const uint32_t tS = ub + t * 128;
          const MatDesc dq = dQ.at(qb * L::kTile), dk = dK.at(st * L::kTile);
          if (go)
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              mma_ss(tS, dq.at((kk >> 2) * (BM * 128) + (kk & 3) * 32),
                     dk.at((kk >> 2) * kPanelOff + (kk & 3) * 32), IDESC_QK, kk > 0, el);
          mma_commit(bar(B_SFULL + t), el);
          if (!sg.two || t == 1) mma_commit(bar(B_KEMPTY + st), el);
          if (j == sg.n - 1) mma_commit(bar(B_QEMPTY + qb), el);
          pv_g[t] = g;
          pv_first[t] = m == 0;
          pv_end[t] = m == sg.count(t) - 1;
          pv_free[t] = !sg.two || t == 1;
        }
      g0 += sg.n;
      q0 += sg.two ? 2 : 1;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (pv_g[t] >= 0) {
        const bool go = !named_bar_or(kNbRing, 64, false);
        tc_fence_after();
        pv(t, go);
      }
    mma_commit(bar(B_END), el);
    if (lane == 0) mbar_wait_no_flag(bar(B_END), 0, p.status, detail, 4 * kWaitLimitNs);
    __syncwarp();
  } else if (warp == 3) {
    // ===================================================== ring warp
    // The MMA warp's waits, in its order.
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      if (ok) ok = ring_wait(bar(i), parity, abort_flag, p.status, detail);
    };
    auto meet = [&]() {
      ok = __all_sync(0xffffffffu, ok);
      named_bar_or(kNbRing, 64, !ok);
    };
    int pv_g[2] = {-1, -1}, pv_s[2] = {};  // pv_s: its segment where it is the first of it, else 0
    bool pv_fix[2] = {};
    auto wait_pv = [&](int t) {
      const int st = pv_g[t] % NSV;
      wait(B_VFULL + st, (pv_g[t] / NSV) & 1);
      if (pv_fix[t]) wait(B_VFIX + st, (pv_g[t] / NSV) & 1);
      if (pv_s[t] > 0) wait(B_ODONE, (pv_s[t] - 1) & 1);
    };
    int g0 = 0, q0 = 0, s = 0;
    while (sg.next()) {
      const int macros = sg.count(0);
      for (int m = 0; m < macros; ++m)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bool cur = m < sg.count(t);
          if (!cur && pv_g[t] < 0) continue;
          if (pv_g[t] >= 0) wait_pv(t);
          pv_g[t] = -1;
          if (cur) {
            const int j = sg.two ? m : 2 * m + t, g = g0 + j;
            if (m == 0) {
              const int q = q0 + (sg.two ? t : 0);
              wait(B_QFULL + q % NQB, (q / NQB) & 1);
            }
            wait(B_KFULL + g % NSK, (g / NSK) & 1);
            pv_g[t] = g;
            pv_s[t] = m == 0 ? s : 0;
            pv_fix[t] = (sg.kt0 + j + 1) * BN > sg.r.ctx;  // holds drafts
          }
          meet();
        }
      g0 += sg.n;
      q0 += sg.two ? 2 : 1;
      ++s;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (pv_g[t] >= 0) {
        wait_pv(t);
        meet();
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
// key tiles of a row's unit.  kWarps warps per (token, query head), each with its
// share of the partials: the (m, l) pairs of all of them first (a lane per
// partial), then the O rows, U loads in flight; the warps' sums are combined in
// shared memory in a fixed order.  One warp per row where there are many rows, four
// where a unit may be split over many CTAs (see `launch`; 76 partials of two units by
// one load after the other had cost 11 of 27.5 us).  Bound by its chain of loads (the
// request and the deal, then the partials): 2.7 us for 16 rows, 4.5 for 1024 rows of
// about five partials, 5.5 for 3200 rows of d = 64, 7.6 for 8192 rows.
// acc + w v.  A weight that has underflowed to 0 does not hide an infinity or a NaN.
constexpr float kFloatMax = 3.402823466e38f;
PIC_DEV float weigh(float w, float v, float acc) {
  return w != 0.f || fabsf(v) <= kFloatMax ? fmaf(w, v, acc) : acc + v;
}

template <int D, int kWarps, int U>
__global__ void __launch_bounds__(128) draft_merge_kernel(Params p) {
  constexpr int CPL = D / 32, kRows = 4 / kWarps;
  constexpr int KW = ((kCtas + kWarps - 1) / kWarps + 31) / 32;  // partials of a lane
  __shared__ float acc_s[4][D], m_s[4], l_s[4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.x * kRows + warp / kWarps, i = blockIdx.y, b = blockIdx.z;
  const int4 rq = p.req[b];  // one round trip with the deal's figures
  const int total = p.share[0].total;
  const Deal deal(total, p.share[0].ctas, p.share[0].per);
  const Request r = request_of(p, rq.y, rq.z);
  if (i >= r.n || h >= p.Hq) return;  // (kWarps = 4: the whole CTA)
  const int hk = h / p.G, rr = i * p.G + h % p.G, rt = rr / BM, row = rr % BM, pair = rt / 2;
  const int step = 2 * pair + 1 < r.rt ? 2 : 1, t0 = rq.x + (hk * r.rt + pair * 2) * r.tiles;
  const int2 u = make_int2(deal.owner(t0 + step - 1, total), deal.owner(t0 + step * r.tiles - 1, total));
  if (u.x == u.y) return;  // finished by its CTA
  const int parts = u.y - u.x + 1, t = 2 * pair + 1 < r.rt ? rt & 1 : 0;
  // partial c is the one of CTA u.x + c; this warp's are c = w0, w0 + kWarps, ...
  const int w0 = warp % kWarps, mine = (parts - w0 + kWarps - 1) / kWarps;
  auto part_row = [&](int c) {
    c = c * kWarps + w0;
    return (size_t)((2 * (u.x + c) + (c == 0 ? 1 : 0)) * 2 + t) * BM + row;
  };
  float v[U][CPL], M = -INFINITY, l = 0.f, acc[CPL];
  auto load = [&](int c0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float *src = p.part_o + part_row(min(c0 + k, mine - 1)) * D + lane * CPL;
      if constexpr (CPL == 4) {
        const float4 f = *reinterpret_cast<const float4 *>(src);
        v[k][0] = f.x, v[k][1] = f.y, v[k][2] = f.z, v[k][3] = f.w;
      } else {
        const float2 f = *reinterpret_cast<const float2 *>(src);
        v[k][0] = f.x, v[k][1] = f.y;
      }
    }
  };
  if (mine > 0) load(0);  // beside the (m, l) pairs
  float w[KW];  // lane's partials: c = lane, lane + 32, ...
  float2 ml[KW];
#pragma unroll
  for (int k = 0; k < KW; ++k) {
    ml[k] = lane + 32 * k < mine ? p.part_ml[part_row(lane + 32 * k)] : make_float2(-INFINITY, 0.f);
    M = fmaxf(M, ml[k].x);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
  for (int k = 0; k < KW; ++k) {
    w[k] = ml[k].x == -INFINITY ? 0.f : ex2(ml[k].x - M);
    l = fmaf(w[k], ml[k].y, l);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
  for (int e = 0; e < CPL; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int c0 = 0; c0 < mine; c0 += U) {
    if (c0) load(c0);
    float wc = w[0];
#pragma unroll
    for (int k = 1; k < KW; ++k) wc = c0 >= 32 * k ? w[k] : wc;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float wk = __shfl_sync(0xffffffffu, wc, (c0 + k) & 31);  // 0 past the end
      if (wk != 0.f)
#pragma unroll
        for (int e = 0; e < CPL; ++e) acc[e] = fmaf(wk, v[k][e], acc[e]);
    }
  }
  // Infinities and NaN of parts whose weight underflowed to 0 (rare: in the loop above
  // they cost 5 ragged requests, d = 64, 1.3 us of 20.1, apart 0.2).  Adding those of the
  // other parts once more changes nothing.
  bool under = false;
#pragma unroll
  for (int k = 0; k < KW; ++k) under |= lane + 32 * k < mine && w[k] == 0.f;
  if (__any_sync(0xffffffffu, under))
#pragma unroll 1
    for (int c = 0; c < mine; ++c)
#pragma unroll 1
      for (int e = 0; e < CPL; ++e) {
        const float x = p.part_o[part_row(c) * D + lane * CPL + e];
        if (fabsf(x) <= kFloatMax) continue;
#pragma unroll
        for (int q = 0; q < CPL; ++q)
          if (q == e) acc[q] += x;
      }
  const size_t o_row = ((size_t)b * p.max_draft + i) * p.Hq + h;
  if constexpr (kWarps == 4) {
#pragma unroll
    for (int e = 0; e < CPL; ++e) acc_s[warp][lane * CPL + e] = acc[e];
    if (lane == 0) m_s[warp] = M, l_s[warp] = l;
    __syncthreads();
    if (warp) return;
    const float mw[4] = {m_s[0], m_s[1], m_s[2], m_s[3]};
    M = fmaxf(fmaxf(mw[0], mw[1]), fmaxf(mw[2], mw[3]));
    l = 0.f;
#pragma unroll
    for (int e = 0; e < CPL; ++e) acc[e] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float wc = mw[c] == -INFINITY ? 0.f : ex2(mw[c] - M);
      l = fmaf(wc, l_s[c], l);
#pragma unroll
      for (int e = 0; e < CPL; ++e) acc[e] = weigh(wc, acc_s[c][lane * CPL + e], acc[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
  __nv_bfloat162 *dst = reinterpret_cast<__nv_bfloat162 *>(p.out + o_row * D + lane * CPL);
#pragma unroll
  for (int e = 0; e < CPL; e += 2) dst[e / 2] = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
  if (lane == 0 && p.lse)
    p.lse[o_row] = l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994531f;
}

// -------------------------------------------------------------------- host
struct Plan {
  int r_pad;
  size_t q_bytes, mask_bytes, wild_bytes, share_bytes, rows_bytes, req_bytes, o_bytes, ml_bytes, total;
};
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline Plan plan(const pic_geom_t *g, int batch, int max_draft) {
  Plan pl;
  const int G = g->num_q_heads / g->num_kv_heads;
  const int rt_max = (int)(((long long)max_draft * G + BM - 1) / BM);
  pl.r_pad = rt_max * BM;
  pl.q_bytes = align256((size_t)batch * g->num_kv_heads * pl.r_pad * g->head_dim * 2);
  pl.mask_bytes = align256((size_t)batch * max_draft * 8);
  pl.wild_bytes = align256((size_t)batch * max_draft * 4);
  pl.share_bytes = align256(kCtas * sizeof(Share));
  pl.rows_bytes = align256(kCtas * 32 * 4);
  pl.req_bytes = align256((size_t)batch * sizeof(int4));
  pl.o_bytes = align256((size_t)4 * kCtas * BM * g->head_dim * 4);
  pl.ml_bytes = align256((size_t)4 * kCtas * BM * sizeof(float2));
  pl.total = pl.q_bytes + pl.mask_bytes + pl.wild_bytes + pl.share_bytes + pl.rows_bytes + pl.req_bytes + pl.o_bytes + pl.ml_bytes;
  return pl;
}

template <int D>
static cudaError_t launch(const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv,
                          const Params &p, const RopeParams &rp, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(draft_attn_kernel<D>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       Layout<D>::kAlloc);
  if (e != cudaSuccess) return e;
  const int threads = std::min(kAppendMax, std::max(128, ((p.Hq + p.Hkv) * (D / 16) + 31) / 32 * 32));
  const int dealers = (kCtas + threads / 32 * kDealt - 1) / (threads / 32 * kDealt);
  e = launch_dependent(draft_append_kernel<D>, dim3(dealers + p.max_draft * p.batch), dim3(threads), 0,
                       stream, p, rp, dealers);
  if (e != cudaSuccess) return e;
  e = launch_dependent(draft_attn_kernel<D>, dim3(kCtas), dim3(kThreads), Layout<D>::kAlloc, stream,
                       tq, tk, tv, p);
  if (e != cudaSuccess) return e;
  // A unit is split over about 152 / units CTAs or more; with four warps a row the rows
  // should fit about one wave of CTAs.  us of the call, four warps and one: 16 units of
  // 32 rows, 20k keys 38.0 and 39.9; 8 of 256 36.2 and 38.0; 4 of 128, d = 64, 25.1
  // and 28.3; but 16 of 256 58.0 and 54.4, 64 of 32 53.7 and 51.9, 64 of 112 176 and 168,
  // 24 of 32, d = 64, 21.8 and 21.1.
  const long long units = (long long)p.batch * p.Hkv * ((p.r_pad / BM + 1) / 2);
  const long long rows = (long long)p.batch * p.max_draft * p.Hq;
  // Four loads in flight instead of eight where units are few CTAs' (64 units of 112 rows
  // 171.0 and 169.8 us, 48 of 40, d = 64, 15.1 and 14.5; but 40 of 32 19.4 and 20.1).
  const bool one = units >= 24 || rows > 20 * kCtas;
  void (*merge)(Params) = !one ? draft_merge_kernel<D, 4, 8>
                               : units >= 48 ? draft_merge_kernel<D, 1, 4> : draft_merge_kernel<D, 1, 8>;
  return launch_dependent(merge, dim3(one ? (p.Hq + 3) / 4 : p.Hq, p.max_draft, p.batch), dim3(128), 0, stream, p);
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
  if (rows_total + 16 >= INT32_MAX || (long long)batch * Hkv * pl.r_pad >= INT32_MAX ||
      (double)batch * Hkv * (pl.r_pad / BM) * (max_pages / 8 + 1) >= INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: cache or queries have more than 2^31 rows", who);
  if (batch > 65535) return fail(PIC_ERR_UNSUPPORTED, "%s: grid too large", who);
  if (max_pages > INT32_MAX / 16 - 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: max_pages %d: positions beyond 32 bits", who, max_pages);
  if (!workspace || workspace_bytes < pl.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return fail(PIC_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", who, pl.total);

  Params p;
  p.batch = batch;
  p.max_draft = max_draft;
  p.Hq = geom->num_q_heads;
  p.Hkv = Hkv;
  p.G = p.Hq / Hkv;
  p.r_pad = pl.r_pad;
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
  p.wild = reinterpret_cast<int32_t *>(ws);
  ws += pl.wild_bytes;
  p.share = reinterpret_cast<Share *>(ws);
  ws += pl.share_bytes;
  p.rows = reinterpret_cast<int32_t *>(ws);
  ws += pl.rows_bytes;
  p.req = reinterpret_cast<int4 *>(ws);
  ws += pl.req_bytes;
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
