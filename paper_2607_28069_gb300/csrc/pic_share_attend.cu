// pic_attend_shared: attention of one new token per entry over a batch whose entries share
// pages, every shared key and value read once for all entries of a node of the plan.
//
// The queries of a node's entries that belong to one kv head are the rows of 128-row tiles
// (one TMEM lane per row): row e G + g is head g of the group of the tile's entry e, 128 / G
// entries a tile, read by TMA straight from q.  Up to two row tiles share a key tile.  A node
// of m entries costs 4 d flops a row and key for 4 d bytes a key: m G rows of 128 make the
// difference between reading a prefix m times and once.
//
// Launches:
//  1. attend_kernel: one persistent CTA per SM, its share of the units' key tiles as the plan
//     dealt it.  An entry whose keys all lie in one node within one CTA is finished there; the
//     others leave partial states.
//  2. merge_kernel: log-sum-exp merge along each entry's chain of nodes.
//
// Measured, whole calls on inputs that change from call to call: 16 branches of one context of
// 139k, 8 kv heads (605 MB), 101 us (6.0 TB/s; the attention 93 of them, DRAM 80% busy); 64 branches
// of one of 33k, 7 heads of 4 kv heads, 48 us, the attention 37 with the tensor pipe 39% busy: first
// tiles after 4.5 us (plan, pages, keys: dependent round trips), then 1.5 us a key tile of two
// row tiles, where its MMAs need 1.1 and its exponentials as much, 2 for the epilogue's 128 KB a CTA,
// and the branches' own tiles at 0.85 us each and 2.5 a branch; 48 entries of 8 nested contexts,
// d = 64, 19.6 us; 4 of 160 keys 9, two dependent launches.
//
// Where rows share nothing, pic_attend_decode (append and attention in one call) is as fast or
// faster: us a layer, 32 + 2 x 8 heads of 128, that call, and this one with its append: 1 row of 4k
// keys 8.7 and 15.3, 8 of 16k 86.8 and 90.2, 64 of 16k 593 and 600.  4 rows of a common 33k take 88.5
// and 36.5, 64 of them 801 and 54.5.
#include <algorithm>

#include "pic_plan.cuh"

namespace pic {
namespace share {

constexpr int NSK = 3, NSV = 2;  // ring stages of K and V
constexpr int NQB = 2;           // query tiles
constexpr int kThreads = 384;    // K producer, MMA, V producer, ring, two softmax warpgroups
// The bound is 448 threads: 14 warps, four of them on one of the SM's quarters of 16384 registers,
// so at most 128 a thread (d = 128 spills 8 bytes).  The 12 warps launched then leave each quarter
// 4096 registers, two warps of the merge (64 a thread): two of its CTAs fit beside one of these.
constexpr int kBoundThreads = 448;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColO = 256;  // S_t at 128 t, O_t at 256 + D t
// Named barriers (0: __syncthreads): P_t from warpgroup t to the MMA warp, the ring warp's
// word to the MMA warp, the two warpgroups' exchange.
constexpr int kNbP = 1, kNbRing = 3, kNbPair = 4;

template <int D>
struct Layout {
  static constexpr int kTile = BN * D * 2;
  static constexpr int kQ = 0;
  static constexpr int kK = kQ + NQB * kTile;
  static constexpr int kV = kK + NSK * kTile;
  static constexpr int kML = kV + NSV * kTile;  // float2 [2][BM / 2]: the warpgroups' m and l
  static constexpr int kBar = kML + BM * 8;
  static constexpr int kAlloc = kBar + 256;
};
// (CTAs of the merge, without shared memory, fit beside one on an SM and begin early.)
static_assert(Layout<128>::kAlloc <= 227 * 1024, "shared memory");

enum {
  B_QFULL = 0,
  B_QEMPTY = B_QFULL + NQB,
  B_KFULL = B_QEMPTY + NQB,
  B_KEMPTY = B_KFULL + NSK,
  B_VFULL = B_KEMPTY + NSK,
  B_VEMPTY = B_VFULL + NSV,
  B_VFIX = B_VEMPTY + NSV,  // per V stage: rows behind the last key are cleared
  B_SFULL = B_VFIX + NSV,   // S_t
  B_OEND = B_SFULL + 2,     // a segment's last PV of warpgroup t
  B_ODONE = B_OEND + 2,     // a segment's O read by both warpgroups
  B_END = B_ODONE + 1,
  B_COUNT = B_END + 1
};
static_assert(B_COUNT * 8 + 16 <= 256, "barrier area");

struct Params {
  int n, Hq, Hkv, G, ept, rows, max_pages, oob_row;
  long long num_pages, layer_row0;
  const int32_t *block_table;
  void *plan;
  float *part_o;    // workspace: pieces [kCtas][2][2][BM][D], then whole units' rows [kDepth][n][Hq][D]
  float2 *part_ml;  // the same without [D]
  __nv_bfloat16 *out;
  float *lse;
  int32_t *status;
  float scale_log2;
};
constexpr long long kPieceRows = (long long)kCtas * 4 * BM;

PIC_DEV bool plan_fits(const Params &p, const Header &h) {
  return h.magic == kMagic && h.n == p.n && h.hkv == p.Hkv && h.ept == p.ept && h.rows == p.rows &&
         h.max_pages == p.max_pages;
}

// The segments of one CTA, walked by each role's warp for itself: ranges of key tiles of its
// units.
struct Segments {
  const Params &p;
  const View v;
  int n_items;
  long long pos, end, unit0, cost;
  int item, cta;
  bool started;
  Item it, ahead;  // the item; the one behind it, on its way
  int rt, hk, pair;
  // the present segment
  int kt0, n;        // of the item's tiles
  bool two;          // two row tiles
  bool first, last;  // holds the unit's first, last key tile

  PIC_DEV Segments(const Params &pp, int cta_) : p(pp), v(pp.plan, pp.n), cta(cta_), started(false) {
    const Header h = *v.head;
    const Share s = v.shares[cta];
    pos = s.pos, end = plan_fits(p, h) ? s.end : s.pos;
    unit0 = s.unit0, item = s.item, n_items = h.items;
    hk = s.hk, pair = s.pair;
    it = s.it;
    rt = (it.m + p.ept - 1) / p.ept;
    kt0 = n = 0;
    two = first = last = false;
    cost = 0;
    if (pos < end) look_ahead();
  }
  PIC_DEV void take(const Segments &o) {
    pos = o.pos, unit0 = o.unit0, cost = o.cost, item = o.item, started = o.started, it = o.it, ahead = o.ahead;
    rt = o.rt, hk = o.hk, pair = o.pair, kt0 = o.kt0, n = o.n, two = o.two, first = o.first, last = o.last;
  }
  PIC_DEV void look_ahead() { ahead = v.items[min(item + 1, n_items - 1)]; }
  PIC_DEV bool next() {
    for (;;) {
      if (pos >= end) return false;
      if (!started) {
        started = true;
      } else {
        unit0 += cost;
        if (unit0 >= end) {
          pos = end;
          return false;
        }
        if (2 * ++pair >= rt) {
          pair = 0;
          if (++hk >= p.Hkv) {
            hk = 0;
            if (++item >= n_items) {
              pos = end;
              return false;
            }
            it = ahead;
            rt = (it.m + p.ept - 1) / p.ept;
            look_ahead();
          }
        }
      }
      two = 2 * pair + 1 < rt;
      const int w = two ? kTwo : kOne;
      cost = kUnit + (long long)it.tiles * w;
      // key tile k's first step is unit0 + kUnit + k w: those in [pos, end)
      const int lo = (int)max(pos - unit0 - kUnit + w - 1, 0ll), hi = (int)min(max(end - unit0 - kUnit + w - 1, 0ll), cost);
      kt0 = two ? lo / kTwo : lo / kOne;
      n = min(it.tiles, two ? hi / kTwo : hi / kOne) - kt0;
      if (n <= 0) continue;
      first = kt0 == 0;
      last = kt0 + n == it.tiles;
      return true;
    }
  }
  // key tiles of warpgroup t: with two row tiles all, else those of parity t
  PIC_DEV int count(int t) const { return two ? n : (n + 1 - t) / 2; }
  PIC_DEV int tile() const { return it.tile_begin + kt0; }
  // of the segment: whether its last key tile is cut by the end of the keys
  PIC_DEV bool cut() const { return last && (it.tile_begin + it.tiles) * BN > it.keys; }
  // rows of row tile t of the pair
  PIC_DEV int tile_rows(int t) const { return min(p.ept, it.m - (2 * pair + t) * p.ept) * p.G; }
};

// The K/V row (of the whole cache) of a page's kv head hk; zeros are read for none.
PIC_DEV int page_row(const Params &p, int page, int hk) {
  if (page < 0 || page >= p.num_pages) return p.oob_row;
  return (int)(p.layer_row0 + ((long long)page * p.Hkv + hk) * 16);
}

PIC_DEV void arrive_twice(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], 2;" ::"r"(bar) : "memory");
}
PIC_DEV void st_global32(void *p, const float *f) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]),
               "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
               : "memory");
}

// Of four neighbouring lanes' 32 values each, a row a lane: piece l (8 values) of the four rows to
// lane l, row k at o + 8 k.  The lanes then store a row's 128 bytes together: a lane's own row 32
// bytes at a time, each in a line of its own, took the load-store unit 3 us for two row tiles.
PIC_DEV void turn_quads(float *o) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int b = 1; b <= 2; b <<= 1) {
    const bool up = lane & b;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (!(k & b))
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          float &x = o[8 * k + q], &y = o[8 * (k | b) + q];
          const float z = __shfl_xor_sync(0xffffffffu, up ? x : y, b);
          (up ? x : y) = z;
        }
  }
}

// --------------------------------------------------------------- attention
// Two softmax warpgroups, one query row per thread, each with its scores S_t and its
// accumulator O_t in TMEM.  Where a unit has two row tiles, warpgroup t takes row tile t, and
// both read every key tile; with one row tile, warpgroup t takes the key tiles of parity t,
// and the two states are joined at the segment's end (each warpgroup half of the columns).
// MMA order, for t = 0, 1, 0, ...: PV_t of warpgroup t's tile before, QK_t of its next one,
// across segments.  MMAs complete in order, so S_t full means that PV_t has finished and O_t
// may be rescaled; O_t is only rescaled when a row's maximum grew by more than 2^8.
//
// Scores, maxima, sums, O and the partial states are held in fp32.  P is rounded to bf16, the
// type in which the tensor core multiplies it with V.  Rows of a tile that belong to no entry
// (an entry of its own has G of 128) hold whatever shared memory held: an MMA's rows do not
// meet, and a warp without a row of an entry leaves its scores alone.
//
// Waits: as in the attention of drafts, the MMA warp meets the ring warp and the softmax warps
// on named barriers only.  These have no limit, so after a wait that ran out every role still
// walks all segments and meets each barrier; the MMA warp then issues nothing but its commits.
__device__ __noinline__ bool ring_wait(uint32_t bar, uint32_t parity, volatile int *abort, int32_t *status,
                                       int detail) {
  return mbar_wait(bar, parity, abort, status, detail);
}

template <int D>
__global__ void __launch_bounds__(kBoundThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q1,
                  const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  Params p) {
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
    asm volatile("griddepcontrol.wait;" ::: "memory");
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
  if (lane == 0 && warp < 4) prefetch_tmap(warp == 0 ? &tm_k : warp == 1 ? &tm_q : warp == 2 ? &tm_v : &tm_q1);
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

  int first4 = -1;  // (the producers': the first pages come with the share)
  if (warp == 0 || warp == 2) first4 = View(p.plan, p.n).first_pages[blockIdx.x * kFirstPages + lane];
  Segments sg(p, (int)blockIdx.x);
  if (threadIdx.x == 0 && blockIdx.x == 0 && !plan_fits(p, *sg.v.head)) dev_fail(p.status, PIC_DEV_BAD_REQUEST, -1);
  if (warp >= 4) {
    // ===================================================== softmax
    const int t = (warp - 4) >> 2, wq = warp & 3, row = wq * 32 + lane;
    const uint32_t tl = tbase + ((uint32_t)(wq * 32) << 16);
    const uint32_t tS = tl + t * 128, tO = tl + kColO + t * D;
    float2 *ml_s = reinterpret_cast<float2 *>(smem + L::kML);
    int nS = 0, nEnd = 0;  // tiles and segments of this warpgroup
    bool ok = true;
    // The MMA warp commits every S_t and every segment's end, also after an abort
    auto wait = [&](int i, uint32_t parity) {
      const bool was = ok;
      ok = mbar_wait_while(ok, bar(i), parity, p.status, detail, 4 * kWaitLimitNs);
      if (was && !ok) *abort_flag = 1;
    };
    bool more = sg.next();
    while (more) {
      const int n = sg.count(t);
      const int rows = sg.tile_rows(sg.two ? t : 0);
      const bool live = wq * 32 < rows;  // of the warp
      float m_used = -INFINITY, l = 0.f;
      for (int i = 0; i < n; ++i, ++nS) {
        wait(B_SFULL + t, nS & 1);
        if (!live) {
          named_bar_arrive(kNbP + t, 128 + 32);
          continue;
        }
        tc_fence_after();
        const int kt = sg.tile() + (sg.two ? i : 2 * i + t);
        // The scores are read twice, 32 columns at a time, once for the maximum and once for
        // the exponentials: short loops, because each call begins with cold instruction caches.
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
        const int keys = sg.it.keys - kt * BN;  // of this tile
        if (keys < BN) {  // hide what lies behind them
#pragma unroll 1
          for (int c = keys / 32; c < BN / 32; ++c) {
            load(x0, c);
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (c * 32 + q >= keys) x0[q] = -INFINITY;
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
      // ---- the segment's rows: after its last PV, o = w_0 O_0 + w_1 O_1 (with one row tile
      // and several key tiles), or O_t alone.  Where they go, and the next segment, while the
      // PV is under way.
      const bool two = sg.two, both = !two && sg.n > 1, whole = sg.first && sg.last;
      const int tile = 2 * sg.pair + (two ? t : 0);
      const int entry = sg.it.begin + tile * p.ept + row / p.G;
      const size_t o_row = (size_t)entry * p.Hq + sg.hk * p.G + row % p.G;
      const bool done = whole && sg.it.leaf && sg.it.level == 0;  // all of the entry's keys
      // partial states: a CTA has at most one segment that ends a unit begun elsewhere or lies
      // inside one (0), and one that begins a unit and leaves its end to others (1)
      const size_t p_row = whole ? kPieceRows + (size_t)sg.it.level * p.n * p.Hq + o_row
                                 : ((size_t)(2 * sg.cta + (sg.first ? 1 : 0)) * 2 + (two ? t : 0)) * BM + row;
      more = sg.next();
      if (n > 0) {
        wait(B_OEND + t, nEnd & 1);
        ++nEnd;
        tc_fence_after();
      }
      float M = m_used, w0 = 1.f, w1 = 0.f;
      if (both) {  // (read before the next segment's PV, and so before the next write)
        constexpr int kHalf = BM / 2;
        float2 o = make_float2(0.f, 0.f);
        tc_fence_before();
#pragma unroll 1
        for (int half = 0; half * kHalf < rows; ++half) {
          const bool mine = row / kHalf == half;
          if (half) named_bar_sync(kNbPair, 256);  // (the first half has been read)
          if (mine) ml_s[t * kHalf + row % kHalf] = make_float2(m_used, l);
          named_bar_sync(kNbPair, 256);
          if (mine) o = ml_s[(t ^ 1) * kHalf + row % kHalf];
        }
        tc_fence_after();
        M = fmaxf(m_used, o.x);
        const float wt = m_used == -INFINITY ? 0.f : ex2(m_used - M);
        const float wo = o.x == -INFINITY ? 0.f : ex2(o.x - M);
        l = t ? fmaf(o.y, wo, l * wt) : fmaf(l, wt, o.y * wo);  // l_0 w_0 + l_1 w_1 in both
        w0 = t ? wo : wt;
        w1 = t ? wt : wo;
      }
      if (live && (two || both || t == 0)) {
        const bool store = row < rows && ok && !*abort_flag;
        const unsigned stores = __ballot_sync(0xffffffffu, store);
        const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
        const int c_begin = both ? t * (D / 64) : 0, c_end = both ? (t + 1) * (D / 64) : D / 32;
        const uint32_t tA = two ? tO : tl + kColO;
#pragma unroll 1
        for (int c = c_begin; c < c_end; ++c) {
          float o[32];
          tmem_ld32(tA + c * 32, reinterpret_cast<uint32_t *>(o));
          tmem_wait_ld();
          if (both) {
            float o1[32];
            tmem_ld32(tA + D + c * 32, reinterpret_cast<uint32_t *>(o1));
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < 32; ++q) o[q] = fmaf(o1[q], w1, o[q] * w0);
          }
          if (done) {
#pragma unroll
            for (int q = 0; q < 32; ++q) o[q] *= inv;
            if (store)
#pragma unroll
              for (int q = 0; q < 4; ++q) st_global16(p.out + o_row * D + c * 32 + q * 8, pack8(o + q * 8));
          } else if (rows <= 32) {  // (few: the turning would cost more)
            if (store)
#pragma unroll
              for (int q = 0; q < 32; q += 8) st_global32(p.part_o + p_row * D + c * 32 + q, o + q);
          } else {
            turn_quads(o);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t r = __shfl_sync(0xffffffffu, (uint32_t)p_row, (lane & 28) + k);
              if (stores >> ((lane & 28) + k) & 1)
                st_global32(p.part_o + (size_t)r * D + c * 32 + (lane & 3) * 8, o + 8 * k);
            }
          }
        }
        if (store && (two || t == 0)) {
          if (!done)
            p.part_ml[p_row] = make_float2(l == 0.f ? -INFINITY : M, l);
          else if (p.lse)
            p.lse[o_row] = l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994531f;
        }
      }
      tc_fence_before();
      __syncwarp();
      // Of a segment of a single tile warpgroup 1 has nothing: it does not wait for the segment
      // and would be ahead with its arrivals, so warpgroup 0 arrives for both.
      if (lane == 0 && (two || both))
        mbar_arrive(bar(B_ODONE));
      else if (lane == 0 && t == 0)
        arrive_twice(bar(B_ODONE));
    }
  } else if (warp == 0 || warp == 2) {
    // ===================================================== TMA producers
    // Warp 0 the query tiles of each segment and K, warp 2 V.  Lane l < 8 moves page l of a
    // tile as one box.
    const bool is_k = warp == 0;
    const int nst = is_k ? NSK : NSV;
    const int b_full = is_k ? B_KFULL : B_VFULL, b_empty = is_k ? B_KEMPTY : B_VEMPTY;
    const uint32_t ring = sbase + (is_k ? L::kK : L::kV);
    const CUtensorMap *tmap = is_k ? &tm_k : &tm_v;
    int g = 0, nq = 0;  // key and query tiles issued
    // block-table entries of four tiles at a time, a lane per page, read four tiles ahead of
    // their use; those of a segment's first four while the segment before is worked on
    auto entry = [&](const Segments &a, int j) {  // of page `lane` of the four tiles from tile j on
      const long long pidx = (long long)(a.tile() + j) * 8 + lane;
      return j + lane / 8 < a.n && pidx * 16 < a.it.keys ? p.block_table[(size_t)a.it.row * p.max_pages + pidx] : -2;
    };
    Segments ahead = sg;
    bool more = ahead.next();
    if (more && (ahead.item != sg.item || ahead.hk != sg.hk || ahead.pair != sg.pair))
      first4 = entry(ahead, 0);  // (no tile of the share's first unit begins in it)
    else if (more && ((long long)ahead.tile() * 8 + lane) * 16 >= ahead.it.keys)
      first4 = -2;
    bool ok = true;
    auto wait = [&](int i, uint32_t parity) {
      if (ok)
        ok = __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, p.status, detail));
      return ok;
    };
    while (ok && more) {
      sg.take(ahead);
      const int keys = sg.it.keys;
      int now = first4;
      if (is_k)
        for (int t = 0; t <= (sg.two ? 1 : 0); ++t, ++nq) {
          const int qb = nq % NQB;
          if (nq >= NQB && !wait(B_QEMPTY + qb, (nq / NQB - 1) & 1)) break;
          if (lane == 0) {
            const bool one = sg.it.m == 1;
            mbar_expect_tx(bar(B_QFULL + qb), (one ? 1 : p.ept) * p.G * D * 2);
#pragma unroll
            for (int pn = 0; pn < PANELS; ++pn)
              tma_load_3d(sbase + L::kQ + qb * L::kTile + pn * BM * 128, one ? &tm_q1 : &tm_q, pn * 64,
                          sg.hk * p.G, sg.it.begin + (2 * sg.pair + t) * p.ept, bar(B_QFULL + qb));
          }
          __syncwarp();
        }
      int y4 = p.oob_row, next = -2;
      for (int j = 0; ok && j < sg.n; ++j) {
        const int st = g % nst, kt = sg.tile() + j;
        if ((j & 3) == 0) {
          if (j) now = next;
          if (is_k && now != -2 && j + lane / 8 < sg.n && (now < 0 || now >= p.num_pages))
            dev_fail(p.status, PIC_DEV_BAD_PAGE, sg.it.begin);
          y4 = page_row(p, now, sg.hk);
          next = entry(sg, j + 4);
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
        ++g;
        // the next segment and its first pages, when this one's first tiles are on their way
        if (j == min(2, sg.n - 1)) {
          more = ahead.next();
          if (more) first4 = entry(ahead, 0);
        }
        if (is_k) continue;
        // A weight of zero does not silence an infinity: of the last key tile, rows behind the
        // keys, which may hold anything, are cleared before PV reads them (to the end of their
        // page; further pages read as zeros).
        if (j == sg.n - 1 && sg.cut()) {
          if (!wait(b_full + st, ((g - 1) / nst) & 1)) break;
          const int r0 = keys - kt * BN, r1 = (r0 + 15) & ~15;
          constexpr int CH = D / 8;
          for (int e = lane; e < (r1 - r0) * CH; e += 32) {
            const int r = r0 + e / CH, ch = e % CH, rr = r & 15;
            const uint32_t off =
                PANELS == 2 ? (uint32_t)((rr >> 3) * 2048 + (ch >> 3) * 1024 + (rr & 7) * 128 +
                                         (((ch & 7) ^ (rr & 7)) << 4))
                            : (uint32_t)(rr * 128 + ((ch ^ (rr & 7)) << 4));
            sts128(ring + st * L::kTile + (r >> 4) * kPageBytes + off, make_uint4(0, 0, 0, 0));
          }
          fence_proxy_async();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(bar(B_VFIX + st));
      }
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
            pv_fix[t] = j == sg.n - 1 && sg.cut();
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
// o = sum_c w_c O_c / sum_c w_c l_c, w_c = 2^(m_c - M), over the parts of an entry's nodes: one
// state for a unit that lay within a CTA, else one for each of its CTAs.  kWarps warps per
// (entry, query head), each with its share of the parts, 32 at a time: their (m, l) pairs, a lane
// each, and their O rows, U loads in flight; the warps' sums are combined in shared memory in a
// fixed order.  Short loops: a call begins with cold instruction caches.
constexpr float kFloatMax = 3.402823466e38f;
// acc + w v.  A weight that has underflowed to 0 does not hide an infinity or a NaN.
PIC_DEV float weigh(float w, float v, float acc) {
  return w != 0.f || fabsf(v) <= kFloatMax ? fmaf(w, v, acc) : acc + v;
}

template <int D, int kWarps, int U>
__global__ void __launch_bounds__(128) merge_kernel(Params p) {
  constexpr int CPL = D / 32, kRows = 4 / kWarps;
  pdl_entry();
  __shared__ float acc_s[kWarps == 4 ? 4 : 1][kWarps == 4 ? D : 1], m_s[4], l_s[4];  // (with one warp a row unused)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int work = blockIdx.x * kRows + warp / kWarps;
  const int entry = work / p.Hq, h = work - entry * p.Hq;
  if (entry >= p.n) return;  // (kWarps = 4: the whole CTA)
  const View v(p.plan, p.n);
  const Header hd = *v.head;
  const int keys = v.keys[entry];
  // lane j < kDepth: the parts of the chain's node of level j
  Link k{0, 0, 0, 0, 0, {0, 0}};
  if (lane < kDepth) k = v.chain[(size_t)entry * kDepth + lane];
  if (!plan_fits(p, hd) || keys < 0) return;  // an entry that is left alone
  int count = 0, c0 = 0, piece = 0;
  if (k.tiles > 0) {
    const Deal deal(hd.total, hd.ctas, hd.q);
    const int e = entry - k.begin, tile = e / p.ept, pair = tile / 2;
    const Units u(k.m, k.tiles, p.ept);
    const long long unit0 = k.base + h / p.G * u.per_head() + pair * u.pair_cost();
    const int w = u.weight(pair);
    c0 = deal.owner(tile_step(unit0, 0, w));
    count = deal.owner(tile_step(unit0, k.tiles - 1, w)) - c0 + 1;
    piece = (u.two(pair) ? tile & 1 : 0) * BM + (e - tile * p.ept) * p.G + h % p.G;
  }
  int end = count;  // parts up to this level's
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, end, o);
    if (lane >= o) end += y;
  }
  const int parts = __shfl_sync(0xffffffffu, end, kDepth - 1);
  if (parts == 1 && __any_sync(0xffffffffu, k.alone)) return;  // done by its CTA
  // this warp's parts are w0, w0 + kWarps, ...
  const int w0 = warp % kWarps, mine = (parts - w0 + kWarps - 1) / kWarps;
  float l = 0.f, M = -INFINITY, acc[CPL];
#pragma unroll
  for (int e = 0; e < CPL; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int b = 0; b < mine; b += 32) {
    const int c = (b + lane) * kWarps + w0;
    uint32_t row = 0;  // of the lane's part
#pragma unroll 1
    for (int j = 0; j < kDepth; ++j) {
      const int e1 = __shfl_sync(0xffffffffu, end, j), n = __shfl_sync(0xffffffffu, count, j);
      const int at = __shfl_sync(0xffffffffu, c0, j), off = __shfl_sync(0xffffffffu, piece, j), i = c - (e1 - n);
      if (i >= 0 && i < n)
        row = n == 1 ? (uint32_t)kPieceRows + ((uint32_t)j * p.n + entry) * p.Hq + h
                     : (uint32_t)((at + i) * 2 + (i == 0 ? 1 : 0)) * 2 * BM + off;
    }
    const bool there = b + lane < mine;
    const float2 ml = there ? p.part_ml[row] : make_float2(-INFINITY, 0.f);
    const int last = min(32, mine - b) - 1;
    float x[U][CPL];
    auto load = [&](int k) {
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const float *src = p.part_o + (size_t)__shfl_sync(0xffffffffu, row, min(k + q, last)) * D + lane * CPL;
        if constexpr (CPL == 4) {
          const float4 f = *reinterpret_cast<const float4 *>(src);
          x[q][0] = f.x, x[q][1] = f.y, x[q][2] = f.z, x[q][3] = f.w;
        } else {
          const float2 f = *reinterpret_cast<const float2 *>(src);
          x[q][0] = f.x, x[q][1] = f.y;
        }
      }
    };
    load(0);  // beside the (m, l) pairs
    float m = ml.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = fmaxf(m, M);
    const float old = M == -INFINITY ? 0.f : ex2(M - m), w = ml.x == -INFINITY ? 0.f : ex2(ml.x - m);
    if (b) {
      l *= old;
#pragma unroll
      for (int e = 0; e < CPL; ++e) acc[e] = weigh(old, acc[e], 0.f);
    }
    M = m;
    l = fmaf(w, ml.y, l);
#pragma unroll 1
    for (int k = 0; k <= last; k += U) {
      if (k) load(k);
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const float wk = k + q <= last ? __shfl_sync(0xffffffffu, w, (k + q) & 31) : 0.f;
        if (wk != 0.f)
#pragma unroll
          for (int e = 0; e < CPL; ++e) acc[e] = fmaf(wk, x[q][e], acc[e]);
      }
    }
    // Infinities and NaN of parts whose weight underflowed to 0 (rare)
    unsigned under = __ballot_sync(0xffffffffu, there && w == 0.f);
#pragma unroll 1
    for (; under; under &= under - 1) {
      const size_t r = __shfl_sync(0xffffffffu, row, __ffs(under) - 1);
#pragma unroll
      for (int e = 0; e < CPL; ++e) acc[e] = weigh(0.f, p.part_o[r * D + lane * CPL + e], acc[e]);
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  const size_t o_row = (size_t)entry * p.Hq + h;
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
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t partial_rows(const pic_geom_t *g, int n) {
  return (size_t)kPieceRows + (size_t)kDepth * n * g->num_q_heads;
}

template <int D>
static cudaError_t launch(const CUtensorMap &tq, const CUtensorMap &tq1, const CUtensorMap &tk,
                          const CUtensorMap &tv, const Params &p, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(attend_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       Layout<D>::kAlloc);
  if (e != cudaSuccess) return e;
  e = launch_dependent(attend_kernel<D>, dim3(kCtas), dim3(kThreads), Layout<D>::kAlloc, stream, tq,
                       tq1, tk, tv, p);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)p.n * p.Hq;
  // Four warps a row where one or two units are split over all CTAs, which leaves each row many
  // parts (us of the call, one warp and four: 2 entries of 4 heads of one kv head, 60k keys, 24.4
  // and 15.9, 3 of 4 heads of 2, 100k keys, 32.0 and 30.7; but 16 of 7 heads of 4, 20k keys, 25.4
  // and 26.4, 64 of 7 heads of 4, 33k keys, 47.8 and 49.9).
  const int units = p.Hkv * (((p.n + p.ept - 1) / p.ept + 1) / 2);
  const bool one = units > 2 || (long long)units * (p.max_pages / 8) < 2 * kCtas;
  return launch_dependent(one ? merge_kernel<D, 1, 8> : merge_kernel<D, 4, 8>,
                          dim3((unsigned)(one ? (rows + 3) / 4 : rows)), dim3(128), 0, stream, p);
}

}  // namespace share
}  // namespace pic

extern "C" size_t pic_shared_workspace_size(const pic_geom_t *geom, int32_t n) {
  using namespace pic::share;
  if (!geom || n <= 0 || n > kMaxEntries || geom->num_kv_heads <= 0 || geom->num_q_heads <= 0 ||
      geom->num_q_heads % geom->num_kv_heads || (geom->head_dim != 64 && geom->head_dim != 128))
    return 0;
  const size_t rows = partial_rows(geom, n);
  return align256(rows * geom->head_dim * 4) + align256(rows * sizeof(float2));
}

extern "C" pic_status_t pic_attend_shared(const pic_geom_t *geom, int32_t layer, int32_t n,
                                          const void *q, int32_t rows, const int32_t *block_table,
                                          int32_t max_pages, int64_t num_pages, const void *k_cache,
                                          const void *v_cache, const int32_t *plan,
                                          size_t plan_bytes, void *out, float *lse, void *workspace,
                                          size_t workspace_bytes, pic_stream_t stream) {
  using namespace pic;
  using namespace pic::share;
  static const char *who = "pic_attend_shared";
  RopeParams rp;
  pic_status_t st = make_rope(geom, &rp);
  if (st != PIC_OK) return st;
  if (layer < 0 || layer >= geom->num_layers)
    return fail(PIC_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", who, layer, geom->num_layers);
  if (n <= 0 || rows <= 0 || max_pages <= 0 || num_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (n > kMaxEntries) return fail(PIC_ERR_UNSUPPORTED, "%s: n %d (at most %d)", who, n, kMaxEntries);
  if (!q || !block_table || !k_cache || !v_cache || !plan || !out)
    return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_cache) |
       reinterpret_cast<uintptr_t>(v_cache) | reinterpret_cast<uintptr_t>(out)) & 15)
    return fail(PIC_ERR_INVALID_ARG, "%s: bf16 tensors must be 16-byte aligned", who);
  const int D = geom->head_dim, Hkv = geom->num_kv_heads, G = geom->num_q_heads / Hkv;
  if (G > BM) return fail(PIC_ERR_UNSUPPORTED, "%s: %d query heads a kv head (at most %d)", who, G, BM);
  const long long rows_total = (long long)geom->num_layers * num_pages * Hkv * 16;
  if (num_pages > INT32_MAX || rows_total + 16 >= INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: cache has more than 2^31 rows", who);
  if (kPieceRows + (long long)kDepth * n * geom->num_q_heads >= INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: grid too large", who);
  if (max_pages > INT32_MAX / 16 - 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: max_pages %d: positions beyond 32 bits", who, max_pages);
  if (plan_bytes < pic_share_plan_size(n) || (reinterpret_cast<uintptr_t>(plan) & 15))
    return fail(PIC_ERR_WORKSPACE, "%s: plan needs %zu bytes, 16-aligned", who, pic_share_plan_size(n));
  const size_t need = pic_shared_workspace_size(geom, n);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return fail(PIC_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", who, need);

  Params p;
  p.n = n;
  p.Hq = geom->num_q_heads;
  p.Hkv = Hkv;
  p.G = G;
  p.ept = entries_per_tile(G);
  p.rows = rows;
  p.max_pages = max_pages;
  p.oob_row = (int)((rows_total + 15) / 16 * 16);
  p.num_pages = num_pages;
  p.layer_row0 = (long long)layer * num_pages * Hkv * 16;
  p.block_table = block_table;
  p.plan = const_cast<int32_t *>(plan);
  p.part_o = static_cast<float *>(workspace);
  p.part_ml = reinterpret_cast<float2 *>(static_cast<uint8_t *>(workspace) +
                                         align256(partial_rows(geom, n) * D * 4));
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.status = device_status_ptr();
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)D));

  // a box of G heads of ept entries (or of one): row e G + g of a row tile's panel
  CUtensorMap tq, tq1, tk, tv;
  const uint64_t head = (uint64_t)D * 2, ent = head * p.Hq;
  st = encode_tmap_3d(&tq, q, D, p.Hq, n, head, ent, 64, G, p.ept);
  if (st == PIC_OK) st = encode_tmap_3d(&tq1, q, D, p.Hq, n, head, ent, 64, G, 1);
  if (D == 128) {
    const uint64_t heads = (uint64_t)geom->num_layers * num_pages * Hkv;
    if (st == PIC_OK) st = encode_tmap_pages128(&tk, k_cache, heads);
    if (st == PIC_OK) st = encode_tmap_pages128(&tv, v_cache, heads);
  } else {
    if (st == PIC_OK) st = encode_tmap_2d(&tk, k_cache, D, rows_total, (uint64_t)D * 2, 64, 16);
    if (st == PIC_OK) st = encode_tmap_2d(&tv, v_cache, D, rows_total, (uint64_t)D * 2, 64, 16);
  }
  if (st != PIC_OK) return st;
  const cudaError_t e = D == 128 ? launch<128>(tq, tq1, tk, tv, p, stream)
                                 : launch<64>(tq, tq1, tk, tv, p, stream);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
