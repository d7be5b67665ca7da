// pic_page_reserve, pic_page_fork, pic_page_compact, pic_page_free and
// pic_page_copy: the pages of a cache while its contexts branch, grow and
// shrink.
//
// The state is the block table (which pages a row uses, in logical order) and
// one count per page (how many rows use it; 0 = free).  There is no list of free
// pages: an allocation scans the counts and takes the lowest free numbers in the
// order of the call, so the result depends on the state alone and a page may be
// given back by any number of CTAs in any order.
//
// All data movement is HBM-bound: each byte is read once and written once, in
// 16-byte pieces with several loads of a thread in flight.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace pages {

constexpr int kPage = 16;
constexpr int kMaxRows = 4096;  // rows a call may list

// Bounded spin on a flag that another CTA of this launch sets (ld.acquire).
PIC_DEV int ld_acquire(const int32_t *p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
PIC_DEV bool wait_flag(const int32_t *flag, int32_t *status, int detail) {
  if (ld_acquire(flag)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t i = 1;; ++i) {
    if (ld_acquire(flag)) return true;
    if ((i & 63u) == 0 && globaltimer_ns() - t0 > kWaitLimitNs) {
      dev_fail(status, PIC_DEV_TIMEOUT, detail);
      return false;
    }
  }
}

// ------------------------------------------------------------- allocation
struct PlanParams {
  int n, rows, max_pages, extra;
  long long num_pages;
  const int32_t *row, *src_row;  // src_row: fork
  int32_t *ctx_len, *block_table, *page_refs, *result;
  int32_t *status;
};

constexpr int kPlanThreads = 1024;
constexpr int kScanBytes = 2 * 32 * 4;  // static shared memory
// A large pool's first pages are mostly all in use: kSkip loads of a thread pass over
// 32768 of them by one barrier.  16 rows x 4 pages (us, without and with, the calls'
// other work included): the first 130000 of 140000 pages in use 24 and 13, 950000 of
// 10^6 142 and 33; with 20000 pages or fewer the loop's code would cost 0.1 to 0.2.
constexpr int kSkip = 8, kSkipped = 4 * kSkip * kPlanThreads;

// Exclusive prefix sum over the block; *total gets the sum.  One barrier: every
// warp adds up the warps' sums itself.  The caller alternates between two buffers
// of 32, so that a buffer is written again only behind a later barrier.
PIC_DEV int block_scan(int v, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int s = warp_sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  *total = __shfl_sync(0xffffffffu, s, 31);
  const int before = __shfl_sync(0xffffffffu, s, max(warp - 1, 0));
  return (warp ? before : 0) + x - v;
}
static_assert(kPlanThreads == 32 * 32, "a lane per warp sum");

// Whether a row may not be appended to in page `page` of its table (-1: none yet), because
// other rows read it.  Rows share pages from their starts on (a fork shares the full pages
// of its source's context, and nothing else shares any), so if the page of a row's next
// position is its own, those behind are.
PIC_DEV bool used_by_others(int page, const int32_t *page_refs, long long num_pages) {
  return page >= 0 && page < num_pages && page_refs[page] > 1;
}

// One CTA: what each listed row needs, then the free pages in ascending order,
// the k-th of them to the row whose range of the needs' prefix sum holds k.  One CTA,
// because the k-th free page depends on all below it and the counts are few (a pool
// of 280 GB has some 10^5 pages).  Bound by dependent loads and barriers: 4.6 to 5 us
// for 8 rows (0.4 of it the use count of each row's next page), 5.2 to 5.7 for 64 branches.
// kLarge: pools of kSkipped pages or more.
template <bool kFork, bool kLarge>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PlanParams p) {
  pdl_entry();
  extern __shared__ int32_t sh[];
  int32_t *first = sh, *col0 = sh + p.n + 1, *len_of = col0 + p.n;  // len_of: fork
  __shared__ int warp_sums[2][32];
  static_assert(sizeof(warp_sums) == kScanBytes, "the host counts with it");
  const int tid = threadIdx.x;
  int carry = 0, turn = 0;
  // the counts of four pages; the first ones go out before the needs are known
  const bool vec = (reinterpret_cast<uintptr_t>(p.page_refs) & 15) == 0;
  auto counts = [&](long long pg) {
    int4 v = make_int4(1, 1, 1, 1);
    if (vec && pg + 3 < p.num_pages) {
      v = *reinterpret_cast<const int4 *>(p.page_refs + pg);
    } else {
      if (pg < p.num_pages) v.x = p.page_refs[pg];
      if (pg + 1 < p.num_pages) v.y = p.page_refs[pg + 1];
      if (pg + 2 < p.num_pages) v.z = p.page_refs[pg + 2];
      if (pg + 3 < p.num_pages) v.w = p.page_refs[pg + 3];
    }
    return v;
  };
  int4 ahead = counts(4 * tid);
  for (int j0 = 0; j0 < p.n; j0 += kPlanThreads) {
    const int j = j0 + tid;
    int need = 0, at = 0, res = -1, len = -1;
    if (j < p.n) {
      const int r = p.row[j];  // the row that gets the pages
      const int a = kFork ? p.src_row[j] : r;
      int code = PIC_DEV_OK;
      if (r < 0 || r >= p.rows || a < 0 || a >= p.rows || (kFork && a == r)) {
        code = PIC_DEV_BAD_REQUEST;
      } else {
        const int32_t *ta = p.block_table + (size_t)a * p.max_pages;
        const int32_t *tr = p.block_table + (size_t)r * p.max_pages;
        len = p.ctx_len[a];
        const long long want = ((long long)len + p.extra + kPage - 1) / kPage;
        if (len < 0 || (kFork && tr[0] >= 0)) {
          code = PIC_DEV_BAD_REQUEST;
        } else if (want > p.max_pages) {
          code = PIC_DEV_BLOCK_TABLE_SHORT;
        } else if constexpr (kFork) {
          at = len / kPage;
          need = (int)want - at;
          res = len;
          if (len % kPage && (ta[at] < 0 || ta[at] >= p.num_pages)) code = PIC_DEV_BAD_PAGE;
        } else {
          int lo = (len + kPage - 1) / kPage, hi = (int)want;  // the first entry without a page
          if (lo < hi) {  // mostly all or none are there
            const bool none = tr[lo] < 0, all = tr[hi - 1] >= 0;
            if (none) hi = lo;
            else if (all) lo = hi;
          }
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (tr[mid] >= 0) lo = mid + 1;
            else hi = mid;
          }
          at = lo;
          need = max(0, (int)want - lo);
          res = (int)want;
          if (p.extra > 0 && used_by_others(tr[len / kPage], p.page_refs, p.num_pages))
            code = PIC_DEV_SHARED_PAGE;
        }
      }
      if (code != PIC_DEV_OK) {
        dev_fail(p.status, code, j);
        need = 0, res = -1;
      }
    }
    int total;
    const int before = block_scan(need, warp_sums[turn ^= 1], &total);
    if (j < p.n) {
      first[j] = carry + before;
      col0[j] = at;
      if constexpr (kFork) len_of[j] = res;
      else p.result[j] = res;
    }
    carry += total;
  }
  if (tid == 0) first[p.n] = carry;
  __syncthreads();
  const int want_all = carry;

  int found = 0;
  long long base = 0;
  if constexpr (kLarge) {
    for (; vec && want_all > 0 && base + kSkipped <= p.num_pages; base += kSkipped) {
      int4 v[kSkip];
#pragma unroll
      for (int q = 0; q < kSkip; ++q)
        v[q] = *reinterpret_cast<const int4 *>(p.page_refs + base + 4 * (q * kPlanThreads + tid));
      bool any = false;
#pragma unroll
      for (int q = 0; q < kSkip; ++q) any |= v[q].x == 0 || v[q].y == 0 || v[q].z == 0 || v[q].w == 0;
      if (__syncthreads_or(any)) break;
    }
    if (base > 0) ahead = counts(base + 4 * tid);
  }
  for (; base < p.num_pages && found < want_all; base += 4 * kPlanThreads) {
    const long long pg = base + 4 * tid;
    const int4 v = ahead;
    ahead = counts(pg + 4 * kPlanThreads);
    // a bit per page of the thread's
    unsigned free_pages = (v.x == 0) | (v.y == 0) << 1 | (v.z == 0) << 2 | (v.w == 0) << 3;
    int total;
    int k = found + block_scan(__popc(free_pages), warp_sums[turn ^= 1], &total);
    for (; free_pages && k < want_all; free_pages &= free_pages - 1, ++k) {
      const int i = __ffs(free_pages) - 1;
      int lo = 0, hi = p.n;  // the last row with first <= k
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= k) lo = mid;
        else hi = mid;
      }
      p.block_table[(size_t)p.row[lo] * p.max_pages + col0[lo] + (k - first[lo])] = (int32_t)(pg + i);
      p.page_refs[pg + i] = 1;
    }
    found += total;
  }
  found = min(found, want_all);
  __syncthreads();
  // rows beyond the free pages are refused, what one of them got goes back
  for (int j = tid; j < p.n; j += kPlanThreads) {
    const bool served = first[j + 1] <= found || first[j + 1] == first[j];
    if (!served) {
      dev_fail(p.status, PIC_DEV_NO_FREE_PAGE, j);
      int32_t *t = p.block_table + (size_t)p.row[j] * p.max_pages + col0[j];
      for (int k = first[j]; k < found; ++k) {
        p.page_refs[t[k - first[j]]] = 0;
        t[k - first[j]] = -1;
      }
    }
    if constexpr (kFork) {
      const int res = served ? len_of[j] : -1;
      p.result[j] = res;
      if (res >= 0) p.ctx_len[p.row[j]] = res;
    } else if (!served) {
      p.result[j] = -1;
    }
  }
}

// ------------------------------------------------------------------- fork
struct ForkParams {
  int n, max_pages, hkv, piece_row, layers, table_blocks;  // piece_row: 16-byte pieces of a row
  long long num_pages, layer_pieces;
  const int32_t *src_row, *dst_row, *result;
  int32_t *block_table, *page_refs;
  uint4 *k, *v;  // at layer_begin
  int32_t *status;
};

// After the plan: blocks [0, table_blocks) enter the shared pages into the
// branches' rows and count their new users, one thread per entry; the others
// copy the valid rows of each context's last page, one warp per (branch, layer,
// kv head), K and V, up to 16 16-byte loads of a lane in flight.  Two dependent loads
// (length, page) and the rows: 8.5 us for 64 branches of 28 layers x 4 heads (53 MB
// with each branch's own read of the rows: 6.2 TB/s, part of it from L2).  Several
// heads a warp were slower, 16.5 us of the call instead of 15.0.
__global__ void __launch_bounds__(256) fork_kernel(ForkParams p) {
  pdl_entry();
  if ((int)blockIdx.x < p.table_blocks) {
    const int per = (p.max_pages + 255) / 256;
    const int j = (int)blockIdx.x / per, e = ((int)blockIdx.x % per) * 256 + (int)threadIdx.x;
    const int len = p.result[j];
    if (len < 0 || e >= len / kPage) return;
    const int page = p.block_table[(size_t)p.src_row[j] * p.max_pages + e];
    if (page < 0 || page >= p.num_pages) {
      dev_fail(p.status, PIC_DEV_BAD_PAGE, j);
      return;
    }
    atomicAdd(p.page_refs + page, 1);
    p.block_table[(size_t)p.dst_row[j] * p.max_pages + e] = page;
    return;
  }
  const int lane = threadIdx.x & 31;
  const long long w = ((long long)blockIdx.x - p.table_blocks) * 8 + (threadIdx.x >> 5);
  const int j = (int)(w / ((long long)p.layers * p.hkv));
  if (j >= p.n) return;
  const int len = p.result[j], src = p.src_row[j], dst = p.dst_row[j];  // one round trip
  const int full = len / kPage, rows = len % kPage;
  if (len < 0 || rows == 0) return;
  const int rem = (int)(w % ((long long)p.layers * p.hkv)), l = rem / p.hkv, h = rem % p.hkv;
  const int from = p.block_table[(size_t)src * p.max_pages + full];
  const int to = p.block_table[(size_t)dst * p.max_pages + full];
  const int pieces = rows * p.piece_row;  // at most 16 * 16
  const long long layer = (long long)l * p.layer_pieces;
  const long long a = layer + ((long long)from * p.hkv + h) * kPage * p.piece_row;
  const long long z = layer + ((long long)to * p.hkv + h) * kPage * p.piece_row;
  uint4 x[8], y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < pieces) {
      x[i] = p.k[a + lane + 32 * i];
      y[i] = p.v[a + lane + 32 * i];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < pieces) {
      p.k[z + lane + 32 * i] = x[i];
      p.v[z + lane + 32 * i] = y[i];
    }
}

// ------------------------------------------------------------------- free
struct FreeParams {
  int n, rows, max_pages;
  long long num_pages;
  const int32_t *row;
  const int32_t *result;  // compact: the rows' new lengths (-1: refused); null: free
  int reserve;
  int32_t *ctx_len, *block_table, *page_refs, *status;
};

// One CTA per listed row: the entries from the cut on are taken out one by
// one (an exchange, so that a page goes back once whatever the call lists) and
// their pages lose a user.  A row's entries are contiguous: the first kReleaseThreads
// without any page end the walk.  Bound by dependent loads and atomics: 3.1 us for 64
// rows of a few pages, 4.6 for one row that gives back 375.
constexpr int kReleaseThreads = 512;
__global__ void __launch_bounds__(kReleaseThreads) release_kernel(FreeParams p) {
  pdl_entry();
  const int j = blockIdx.x, r = p.row[j];
  int cut = 0;
  if (p.result) {
    const int len = p.result[j];
    if (len < 0) return;
    cut = (int)min((long long)p.max_pages, ((long long)len + p.reserve + kPage - 1) / kPage);
    if (threadIdx.x == 0) p.ctx_len[r] = len;
  } else {
    if (r < 0 || r >= p.rows) {
      if (threadIdx.x == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, j);
      return;
    }
    if (threadIdx.x == 0) p.ctx_len[r] = 0;
  }
  int32_t *t = p.block_table + (size_t)r * p.max_pages;
  for (int e0 = cut; e0 < p.max_pages; e0 += kReleaseThreads) {
    const int e = e0 + (int)threadIdx.x;
    const int page = e < p.max_pages ? atomicExch(t + e, -1) : -1;
    if (page >= p.num_pages) {
      dev_fail(p.status, PIC_DEV_BAD_PAGE, j);
    } else if (page >= 0 && atomicSub(p.page_refs + page, 1) <= 0) {
      atomicAdd(p.page_refs + page, 1);  // nobody used it
      dev_fail(p.status, PIC_DEV_BAD_PAGE, j);
    }
    if (!__syncthreads_or(page >= 0)) break;
  }
}

// ---------------------------------------------------------------- compact
constexpr int kSeg = 16;      // kept positions that a CTA holds at once
constexpr int kShort = 64;    // longest list that one CTA per (row, layer, heads) works off
constexpr int kUnits = 4;     // 32-byte units of a thread
constexpr int kMoveCtas = 4;  // of an SM
constexpr int kMoveThreads = 256;
static_assert(kSeg == 16, "half a warp looks a segment's positions up");
constexpr int kCheckThreads = 1024;  // kept positions of a checking CTA

struct CompactParams {
  int n, rows, max_pages, max_keep, segs, hkv, hgroup, hgroups, lgroup, lhs, layers, layer_begin, rotate, dim, reserve;
  long long num_pages, layer_elems;
  const int32_t *row, *start, *keep, *keep_len;
  const int32_t *ctx_len, *block_table, *page_refs;
  int32_t *result;
  __nv_bfloat16 *k, *v;  // at layer_begin
  // lists beyond kShort (workspace): from and to row of every kept position (elements
  // from the layer's begin to head 0's; as page and row, with the products at each use,
  // 9001 of 15001 positions took 72.0 us instead of 70.7), per (row, segment) the first
  // and last segment to wait for, a ticket, and per (row, layer and head group, segment)
  // "reads done"
  longlong2 *slot;       // [n][max_keep]
  int2 *wait;            // [n][segs]
  int32_t *bad;          // [n][checks]: a checking CTA found a fault
  int checks;
  int32_t *ticket, *flags;
  int32_t *status;
};

// The start of row j's window, or -1 with *code set.
PIC_DEV int compact_start(const CompactParams &p, int j, int *code) {
  const int r = p.row[j], m = p.keep_len[j];
  if (r < 0 || r >= p.rows || m < 0 || m > p.max_keep) {
    *code = PIC_DEV_BAD_REQUEST;
    return -1;
  }
  const int s = p.start ? p.start[j] : p.ctx_len[r];
  if (s < 0 || (long long)s + m > (long long)p.max_pages * kPage) {
    *code = s < 0 ? PIC_DEV_BAD_REQUEST : PIC_DEV_BLOCK_TABLE_SHORT;
    return -1;
  }
  return s;
}

// Room behind the kept positions, from s on, is asked for: the page of the next position.
PIC_DEV int compact_end(const CompactParams &p, int j, int s) {
  const int r = p.row[j], e = (s + p.keep_len[j]) / kPage;
  if (p.reserve == 0 || e >= p.max_pages) return PIC_DEV_OK;
  return used_by_others(p.block_table[(size_t)r * p.max_pages + e], p.page_refs, p.num_pages)
             ? PIC_DEV_SHARED_PAGE : PIC_DEV_OK;
}

// Entry i of a keep list: its checks and its slots, as page * 16 + row of the page.
PIC_DEV int compact_entry(const CompactParams &p, int j, int s, int i, int *k_out,
                          longlong2 *slot) {
  const int32_t *t = p.block_table + (size_t)p.row[j] * p.max_pages;
  const int32_t *kp = p.keep + (size_t)j * p.max_keep;
  const int k = kp[i], before = i > 0 ? kp[i - 1] : -1;
  // Ascending from >= 0 on: never below i.  The entry before is judged here too: it may
  // be another CTA's, and what follows here takes it as an index.
  if (k < i || before < i - 1 || before >= k) return PIC_DEV_BAD_POSITION;
  if ((long long)s + k >= (long long)p.max_pages * kPage) return PIC_DEV_BLOCK_TABLE_SHORT;
  const int a = t[(s + k) / kPage], z = t[(s + i) / kPage];
  if (a < 0 || a >= p.num_pages || z < 0 || z >= p.num_pages) return PIC_DEV_BAD_PAGE;
  if (k != i && p.page_refs[z] != 1) return PIC_DEV_SHARED_PAGE;
  *k_out = k;
  *slot = make_longlong2((long long)a * kPage + (s + k) % kPage, (long long)z * kPage + (s + i) % kPage);
  return PIC_DEV_OK;
}

// Lists beyond kShort, one CTA per 1024 entries of a listed row: every
// check before anything moves, the slots, the segments to wait for, the flags
// cleared.  An entry is a chain of three loads: 5.2 us for a list of 9001 (15 by one
// CTA).
__global__ void __launch_bounds__(kCheckThreads) compact_check_kernel(CompactParams p) {
  pdl_entry();
  const int j = blockIdx.y, tid = threadIdx.x, i0 = blockIdx.x * kCheckThreads;
  const long long per = (long long)p.lhs * p.segs;
  for (long long i = i0 + tid; i < per; i += (long long)p.checks * kCheckThreads)
    p.flags[j * per + i] = 0;
  if (j == 0 && i0 == 0 && tid == 0) *p.ticket = 0;
  int code = PIC_DEV_OK;
  const int s = compact_start(p, j, &code);
  const int m = s >= 0 ? p.keep_len[j] : 0;
  if (i0 + tid < m) {
    int k;
    longlong2 slot;
    code = compact_entry(p, j, s, i0 + tid, &k, &slot);
    auto elem = [&](long long sl) { return (sl / kPage * p.hkv * kPage + sl % kPage) * p.dim; };
    if (code == PIC_DEV_OK)
      p.slot[(size_t)j * p.max_keep + i0 + tid] = make_longlong2(elem(slot.x), elem(slot.y));
  }
  // (a thread that mostly has no entry)
  if (blockIdx.x == gridDim.x - 1 && tid == kCheckThreads - 1 && s >= 0 && code == PIC_DEV_OK)
    code = compact_end(p, j, s);
  if (code != PIC_DEV_OK && (s >= 0 || (tid == 0 && i0 == 0))) dev_fail(p.status, code, j);
  const bool bad = __syncthreads_or(code != PIC_DEV_OK);
  if (tid == 0) p.bad[j * p.checks + blockIdx.x] = bad;
  if (bad) return;
  // Segment s2 reads positions keep[16 s2] .. its last entry, segment seg writes
  // 16 seg .. 16 seg + 15: the ones to wait for are the first s2 that reads as far as
  // 16 seg to the last that begins at or below 16 seg + 15.  Each s2 notes itself as
  // the first for the segments from behind s2 - 1's last source to its own, and as
  // the last for those from its first source to ahead of s2 + 1's.
  const int32_t *kp = p.keep + (size_t)j * p.max_keep;
  const int segs = (m + kSeg - 1) / kSeg, s2 = i0 / kSeg + tid;
  if (tid < kCheckThreads / kSeg && s2 < segs) {
    int2 *w = p.wait + (size_t)j * p.segs;
    const int begin = kp[s2 * kSeg] / kSeg;
    const int end = min(s2 + 1 < segs ? kp[(s2 + 1) * kSeg] / kSeg : segs, segs);
    const int lo = s2 ? kp[s2 * kSeg - 1] / kSeg : -1;
    const int hi = min(kp[min((s2 + 1) * kSeg, m) - 1] / kSeg, segs - 1);
    for (int seg = s2 ? begin : 0; seg < end; ++seg) w[seg].y = seg < begin ? -1 : s2;
    for (int seg = lo + 1; seg <= hi; ++seg) w[seg].x = s2;
  }
}

// A CTA moves 16 kept positions x a group of kv heads (and layers) of one row: it
// reads them all on chip, says so, waits for the CTAs whose sources lie in what it
// overwrites (few, and long past where much was left out), and stores.  keep is
// ascending, so those are CTAs of earlier segments of the same (row, group) only; a
// segment comes from a ticket, so they have started before it, and they read before
// they wait: every wait ends.  Keys move by i - keep[i] positions and are re-rotated by
// that, with cos/sin formed once per CTA.
// Long lists (compact_move_kernel) are checked by compact_check_kernel, and moved by
// CTAs that stay and look up the next segment's positions while they wait.  Short ones
// (compact_short_kernel: windows of drafts, up to kShort entries, mostly few of them
// kept) are worked off by a CTA per (row, layer, head group), which needs no flags -- a
// segment's targets lie below the next one's sources -- and checks the list itself,
// so the call is a launch shorter.
// Measured: 9001 of 15001 positions, 8 heads, 4 layers, 58 us (295 MB read and
// written: 5.1 TB/s; 53 without the rotation): a row of a head is 256 bytes, reads and
// writes of that size alternate, and issue slots are over half busy with addresses and
// rotations.  The short form: 8 rows that keep 5 of 16, 32 layers, 5 us, latency.

// The units of a segment of group lh (heads, with kLayers of several layers): unit u =
// (position, K or V, row of the group, chunk), thread tid's are tid, tid + kMoveThreads, ...
template <int D, bool kLayers>
struct Units {
  static constexpr int KC = D / 16;  // 8-pair chunks of a row
  int layer, h0, heads, per, count, magic, head_magic;  // per: units of a position's K or V
  long long base;
  PIC_DEV Units(const CompactParams &p, int lh, int positions) {
    layer = lh / p.hgroups * (kLayers ? p.lgroup : 1);
    h0 = (lh % p.hgroups) * p.hgroup;
    heads = min(p.hgroup, p.hkv - h0);
    per = KC * heads * (kLayers ? min(p.lgroup, p.layers - layer) : 1);
    count = positions * 2 * per;
    // (division by per <= 32 as a product: exact for u < 1024; by heads: for 8 of them)
    magic = ((1 << 20) + per - 1) / per;
    head_magic = (256 + heads - 1) / heads;
    base = (long long)layer * p.layer_elems;
  }
  PIC_DEV int pair_of(int u) const { return (u * magic) >> 20; }  // 2 * position + (0 K, 1 V)
  PIC_DEV int head_of(int u, int w) const { return h0 + (u - w * per) / KC; }  // without kLayers
  // unit u's row in its (position, K or V) w, from the position's row of layer 0, head 0
  PIC_DEV long long row_of(const CompactParams &p, int u, int w) const {
    const int g = (u - w * per) / KC, l = kLayers ? (g * head_magic) >> 8 : 0;
    return base + l * p.layer_elems + (h0 + g - l * heads) * (kPage * D);
  }
};

// Short lists: a CTA takes all segments of a (row, layer, head group) in turn.
template <int D>
__global__ void __launch_bounds__(kMoveThreads, kMoveCtas) compact_short_kernel(CompactParams p, RopeParams rp) {
  constexpr int KC = D / 16;
  pdl_entry();
  __shared__ float2 cs[kSeg][D / 2];
  __shared__ int32_t k_of[kShort / kSeg][kSeg];
  __shared__ longlong2 slot_of[kShort / kSeg][kSeg];
  const int tid = threadIdx.x, lhs = p.lhs;
  const int lh = blockIdx.x % lhs, j = blockIdx.x / lhs;
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);
  int code = PIC_DEV_OK;
  const int s = compact_start(p, j, &code), m = s >= 0 ? p.keep_len[j] : 0;
  if (tid < m) {
    int k = 0;
    longlong2 slot = make_longlong2(0, 0);
    code = compact_entry(p, j, s, tid, &k, &slot);
    k_of[tid / kSeg][tid % kSeg] = k;
    slot_of[tid / kSeg][tid % kSeg] = slot;
  }
  if (tid == kMoveThreads - 1 && s >= 0) code = compact_end(p, j, s);
  const bool bad = __syncthreads_or(code != PIC_DEV_OK);
  if (lh == 0) {  // one CTA of a row reports
    if (code != PIC_DEV_OK && (tid == 0 || s >= 0)) dev_fail(p.status, code, j);
    if (tid == 0) p.result[j] = bad ? -1 : s + m;
  }
  if (bad) return;
  const int f = tid % (D / 2);  // the frequency this thread forms cos/sin of
  const uint64_t turn = p.rotate ? rope_turn(rope_theta(rp, p.layer_begin + lh / p.hgroups, f)) : 0;
  for (int seg = 0; seg * kSeg < m; ++seg) {
    const int i0 = seg * kSeg, cnt = min(kSeg, m - i0);
    const Units<D, false> un(p, lh, cnt);
    auto where = [&](int u, int w, bool to) {
      const long long sl = to ? slot_of[seg][w >> 1].y : slot_of[seg][w >> 1].x;
      return (w & 1 ? p.v : p.k) + un.base + (((sl >> 4) * p.hkv + un.head_of(u, w)) * kPage + (sl & 15)) * D;
    };
    uint4 a[kUnits], b[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int u = tid + q * kMoveThreads, w = un.pair_of(u);
      if (u < un.count && k_of[seg][w >> 1] != i0 + (w >> 1)) {
        const __nv_bfloat16 *src = where(u, w, false);
        a[q] = *reinterpret_cast<const uint4 *>(src + pc.off_a);
        b[q] = *reinterpret_cast<const uint4 *>(src + pc.off_b);
      }
    }
    if (p.rotate)
      for (int i = tid / (D / 2); i < cnt; i += kMoveThreads / (D / 2))
        cs[i][f] = rope_cos_sin_turn(i0 + i - k_of[seg][i], turn);
    __syncthreads();  // all are read: the targets lie below the next segment's sources
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int u = tid + q * kMoveThreads, w = un.pair_of(u), i = w >> 1;
      if (u < un.count && k_of[seg][i] != i0 + i) {
        __nv_bfloat16 *dst = where(u, w, true);
        if (p.rotate && !(w & 1)) {
          rotate_store(a[q], b[q], dst, pc, rp.style, &cs[i][8 * (tid % KC)]);
        } else {
          st_global16(dst + pc.off_a, a[q]);
          st_global16(dst + pc.off_b, b[q]);
        }
      }
    }
    if (i0 + kSeg < m) __syncthreads();  // cs may be written again
  }
}

// Long lists.  A thread's units wait in its own part of shared memory, so that it keeps
// the registers for addresses and rotations (in registers 70.3 us for the call above,
// now 68.9; two buffers, the next segment's rows on their way during the stores, leave
// three CTAs an SM: 72.2, and 57 instead of 51 with 2 heads of 64).
constexpr int kLongCtas = 4;  // of an SM
constexpr int kHeldBytes = kUnits * 2 * kMoveThreads * 16;
PIC_DEV void cp_async16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
PIC_DEV void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// kLayers: several layers of narrow rows a CTA (lgroup; 2 rows of 32 layers x 2 heads of
// 64, 1500 of 3000 positions, 51.6 and 31.1 us).
template <int D, bool kLayers>
__global__ void __launch_bounds__(kMoveThreads, kLongCtas) compact_move_kernel(CompactParams p, RopeParams rp) {
  constexpr int KC = D / 16;
  pdl_entry();
  extern __shared__ __align__(16) uint4 held[];  // [kUnits][a, b][thread]: a thread's own units
  __shared__ float2 cs[kSeg][D / 2];
  __shared__ int32_t k_of[2][kSeg];
  __shared__ longlong2 slot_of[2][kSeg];
  __shared__ int next_at, cnt_of[2];
  __shared__ int2 wait_of[2];
  const int tid = threadIdx.x, lhs = p.lhs;
  const int all = lhs * p.n * p.segs;  // (the host keeps it below 2^30)
  const PairChunk pc = pair_chunk(tid % KC, D / 2, rp.style);

  // the positions of item `at` into buffer `buf` (the count 0: nothing to move), by
  // the last 16 threads: their loads run beside the others' polls
  auto look_up = [&](int at, int buf) {
    const int j = at / lhs % p.n, seg = at / lhs / p.n;
    const int t = tid - (kMoveThreads - kSeg);
    if (t >= 0) {
      const size_t i = (size_t)j * p.max_keep + min(seg * kSeg + t, p.max_keep - 1);
      bool bad = false;
      for (int c = t; c < p.checks; c += kSeg) bad |= p.bad[j * p.checks + c] != 0;
      bad = __any_sync(0xffffu << (32 - kSeg), bad);
      const int k = p.keep[i], m = p.keep_len[j];
      const int2 wait = p.wait[(size_t)j * p.segs + seg];
      slot_of[buf][t] = p.slot[i];
      k_of[buf][t] = k;
      if (t == 0) {
        cnt_of[buf] = bad ? 0 : max(0, min(kSeg, m - seg * kSeg));
        wait_of[buf] = make_int2(wait.x, min(wait.y, seg - 1));
        if (at % lhs == 0 && seg == 0) {  // one CTA of a row reports
          int code;
          p.result[j] = bad ? -1 : compact_start(p, j, &code) + m;
        }
      }
    }
  };
  auto held_at = [&](int q) { return 2 * q * kMoveThreads + tid; };
  auto row_of = [&](const Units<D, kLayers> &un, int u, int w, long long sl) {
    return (w & 1 ? p.v : p.k) + un.row_of(p, u, w) + sl;
  };
  auto read = [&](int at, int buf) {
    const int i0 = at / lhs / p.n * kSeg;
    const Units<D, kLayers> un(p, at % lhs, cnt_of[buf]);
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int u = tid + q * kMoveThreads, w = un.pair_of(u);
      if (u < un.count && k_of[buf][w >> 1] != i0 + (w >> 1)) {
        const __nv_bfloat16 *src = row_of(un, u, w, slot_of[buf][w >> 1].x);
        const uint32_t dst = smem_u32(held + held_at(q));
        cp_async16(dst, src + pc.off_a);
        cp_async16(dst + kMoveThreads * 16, src + pc.off_b);
      }
    }
  };

  if (tid == 0) next_at = atomicAdd(p.ticket, 1);
  __syncthreads();
  int at = next_at, buf = 0, turn_layer = -1;
  const int f = tid % (D / 2);  // the frequency this thread forms cos/sin of
  uint64_t turn = 0;            // (fp64 work: once, not once per segment)
  if (at < all) look_up(at, 0);
  __syncthreads();
  if (at < all) read(at, 0);
  while (at < all) {
    const int lh = at % lhs, j = at / lhs % p.n, seg = at / lhs / p.n, i0 = seg * kSeg;
    const int cnt = cnt_of[buf];
    const Units<D, kLayers> un(p, lh, cnt);
    if (tid == 0) next_at = atomicAdd(p.ticket, 1);
    unsigned runs = 0;
    if (p.rotate) {
      // positions of a run that stayed together move alike: cos/sin for its first only
      const int i = tid & 31;
      runs = __ballot_sync(0xffffffffu, i < cnt && (i == 0 || k_of[buf][i] != k_of[buf][i - 1] + 1));
      if (un.layer != turn_layer && (turn_layer < 0 || rp.layer_theta))
        turn = rope_turn(rope_theta(rp, p.layer_begin + un.layer, f));
      turn_layer = un.layer;
      unsigned left = runs;
      auto drop = [&](int n) {
        for (int k = 0; k < n; ++k) left &= left - 1;
      };
      for (drop(tid / (D / 2)); left; drop(kMoveThreads / (D / 2))) {
        const int r = __ffs(left) - 1;
        cs[r][f] = rope_cos_sin_turn(i0 + r - k_of[buf][r], turn);
      }
    }
    cp_async_wait();
    int32_t *fl = p.flags + ((long long)j * lhs + lh) * p.segs;
    // every thread's loads are done at the barrier; thread 0's fence orders them,
    // and not only its own, before the flag
    __syncthreads();
    const int after = next_at;
    bool ok = true;
    if (cnt > 0 && tid == 0) {
      __threadfence();
      atomicExch(fl + seg, 1);
    }
    if (after < all) look_up(after, buf ^ 1);
    if (cnt > 0)
      for (int s2 = wait_of[buf].x + tid; ok && s2 <= wait_of[buf].y; s2 += kMoveThreads)
        ok = wait_flag(fl + s2, p.status, j);
    if (__syncthreads_or(!ok)) return;
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int u = tid + q * kMoveThreads, w = un.pair_of(u), i = w >> 1;
      if (u < un.count && k_of[buf][i] != i0 + i) {
        const uint4 a = held[held_at(q)], b = held[held_at(q) + kMoveThreads];
        __nv_bfloat16 *dst = row_of(un, u, w, slot_of[buf][i].y);
        if (p.rotate && !(w & 1)) {
          rotate_store(a, b, dst, pc, rp.style, &cs[31 - __clz(runs & ((2u << i) - 1))][8 * (tid % KC)]);
        } else {
          st_global16(dst + pc.off_a, a);
          st_global16(dst + pc.off_b, b);
        }
      }
    }
    if (after < all) read(after, buf ^ 1);
    __syncthreads();  // cs and the buffer may be written again
    at = after;
    buf ^= 1;
  }
}

// ------------------------------------------------------------------- copy
struct CopyParams {
  int n, layers, pieces_page;  // 2 KB pieces of a page of one layer
  long long src_pages, dst_pages, total;  // total: pieces in all
  const int32_t *src_page, *dst_page;
  const uint4 *ks, *vs;
  uint4 *kd, *vd;  // all at layer_begin
  int32_t *status;
};

constexpr int kCopyPieces = 4;  // pieces of a warp (8 KB)

// A page of a layer is contiguous: a warp moves four consecutive 2 KB pieces,
// all 16 16-byte loads of a lane before its stores.  HBM-bound: 308 us for 512 pages
// of 32 layers x 8 heads (2.15 GB: 7.0 TB/s, DRAM 87% busy).
__global__ void __launch_bounds__(256) copy_kernel(CopyParams p) {
  pdl_entry();
  const int lane = threadIdx.x & 31;
  const long long w0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kCopyPieces;
  uint4 x[kCopyPieces][4];
  uint4 *to[kCopyPieces];
#pragma unroll
  for (int i = 0; i < kCopyPieces; ++i) {
    to[i] = nullptr;
    const long long w = w0 + i;
    if (w >= p.total) continue;
    const int piece = (int)(w % p.pieces_page);
    const long long item = w / p.pieces_page;  // ((pair * layers) + layer) * 2 + kv
    const int kv = (int)(item & 1), layer = (int)((item >> 1) % p.layers);
    const int pair = (int)((item >> 1) / p.layers);
    const int s = p.src_page[pair], d = p.dst_page[pair];
    if (s < 0 || s >= p.src_pages || d < 0 || d >= p.dst_pages) {
      if (piece == 0 && (item % (2 * p.layers)) == 0 && lane == 0 && !(s == -1 && d == -1))
        dev_fail(p.status, PIC_DEV_BAD_PAGE, pair);
      continue;
    }
    const long long from = (((long long)layer * p.src_pages + s) * p.pieces_page + piece) * 128;
    const uint4 *src = (kv ? p.vs : p.ks) + from + lane;
    to[i] = (kv ? p.vd : p.kd) +
            (((long long)layer * p.dst_pages + d) * p.pieces_page + piece) * 128 + lane;
#pragma unroll
    for (int q = 0; q < 4; ++q) x[i][q] = src[q * 32];
  }
#pragma unroll
  for (int i = 0; i < kCopyPieces; ++i)
    if (to[i])
#pragma unroll
      for (int q = 0; q < 4; ++q) st_global16(to[i] + q * 32, x[i][q]);
}

// ------------------------------------------------------------------- host
static pic_status_t check_table(const char *who, int32_t n, const int32_t *row, int32_t rows,
                                const int32_t *ctx_len, const int32_t *block_table,
                                int32_t max_pages, int64_t num_pages, const int32_t *page_refs) {
  if (n < 0 || n > kMaxRows)
    return fail(n < 0 ? PIC_ERR_INVALID_ARG : PIC_ERR_UNSUPPORTED, "%s: %d rows (at most %d)", who,
                n, kMaxRows);
  if (rows <= 0 || max_pages <= 0 || num_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (num_pages > INT32_MAX || max_pages > INT32_MAX / kPage ||
      (long long)n * max_pages > INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: page numbers or positions beyond 32 bits", who);
  if (n && (!row || !ctx_len || !block_table || !page_refs))
    return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  return PIC_OK;
}

static pic_status_t check_cache(const char *who, const pic_geom_t *geom, RopeParams *rp,
                                const void *k, const void *v, int32_t layer_begin,
                                int32_t layer_end) {
  pic_status_t st = make_rope(geom, rp);
  if (st != PIC_OK) return st;
  if (layer_begin < 0 || layer_end > geom->num_layers || layer_begin > layer_end)
    return fail(PIC_ERR_INVALID_ARG, "%s: layers [%d, %d) outside [0, %d)", who, layer_begin,
                layer_end, geom->num_layers);
  if (!k || !v) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15)
    return fail(PIC_ERR_INVALID_ARG, "%s: bf16 tensors must be 16-byte aligned", who);
  return PIC_OK;
}

static pic_status_t launched(const char *who, cudaError_t e) {
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}

template <bool kFork, bool kLarge>
static cudaError_t launch_plan(const PlanParams &pp, pic_stream_t stream) {
  const size_t smem = (size_t)(pp.n + 1 + pp.n * (kFork ? 2 : 1)) * 4;
  if (smem + kScanBytes > 48 * 1024) {  // (the default limit counts the static part too)
    const cudaError_t e = cudaFuncSetAttribute(plan_kernel<kFork, kLarge>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)smem);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(plan_kernel<kFork, kLarge>, dim3(1), dim3(kPlanThreads), smem, stream, pp);
}
template <bool kFork>
static cudaError_t launch_plan(const PlanParams &pp, pic_stream_t stream) {
  return pp.num_pages >= kSkipped ? launch_plan<kFork, true>(pp, stream)
                                  : launch_plan<kFork, false>(pp, stream);
}

// Head groups of a compaction: as many heads as 16 positions of a CTA hold.
static int heads_per_group(const pic_geom_t *g) {
  return kMoveThreads * kUnits / (kSeg * 2 * (g->head_dim / 16));
}
struct CompactSpace {  // byte offsets in the workspace
  size_t wait, bad, ticket, flags, total;
};
static int compact_checks(int max_keep) { return (max_keep + kCheckThreads - 1) / kCheckThreads; }
static CompactSpace compact_space(const pic_geom_t *g, int n, int max_keep, int layers) {
  const int hg = heads_per_group(g);
  const size_t groups = (size_t)(g->num_kv_heads + hg - 1) / hg;
  const size_t segs = ((size_t)max_keep + kSeg - 1) / kSeg;
  CompactSpace c;
  c.wait = (size_t)n * max_keep * sizeof(longlong2);
  c.bad = c.wait + (size_t)n * segs * sizeof(int2);
  c.ticket = c.bad + (size_t)n * compact_checks(max_keep) * 4;
  c.flags = c.ticket + 4;
  c.total = max_keep <= kShort ? 0 : c.flags + (size_t)n * layers * groups * segs * 4;
  return c;
}

template <int D>
static cudaError_t launch_move(const CompactParams &cp, const RopeParams &rp, long long items,
                               pic_stream_t stream) {
  if (!cp.flags)
    return launch_dependent(compact_short_kernel<D>, dim3((unsigned)items), dim3(kMoveThreads), 0, stream,
                            cp, rp);
  void (*kernel)(CompactParams, RopeParams) =
      cp.lgroup > 1 ? compact_move_kernel<D, true> : compact_move_kernel<D, false>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldBytes);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)std::min(items, kLongCtas * 152LL)), dim3(kMoveThreads),
                          kHeldBytes, stream, cp, rp);
}

}  // namespace pages
}  // namespace pic

extern "C" pic_status_t pic_page_reserve(int32_t n, const int32_t *row, int32_t extra, int32_t rows,
                                         const int32_t *ctx_len, int32_t *block_table,
                                         int32_t max_pages, int64_t num_pages, int32_t *page_refs,
                                         int32_t *result, pic_stream_t stream) {
  using namespace pic;
  using namespace pic::pages;
  static const char *who = "pic_page_reserve";
  pic_status_t st = check_table(who, n, row, rows, ctx_len, block_table, max_pages, num_pages, page_refs);
  if (st != PIC_OK) return st;
  if (extra < 0) return fail(PIC_ERR_INVALID_ARG, "%s: extra %d is negative", who, extra);
  if (n == 0) return PIC_OK;
  if (!result) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  PlanParams pp{n, rows, max_pages, extra, num_pages, row, nullptr, const_cast<int32_t *>(ctx_len),
                block_table, page_refs, result, device_status_ptr()};
  if (!pp.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  return launched(who, launch_plan<false>(pp, stream));
}

extern "C" pic_status_t pic_page_fork(const pic_geom_t *geom, int32_t n, const int32_t *src_row,
                                      const int32_t *dst_row, int32_t reserve, int32_t rows,
                                      int32_t *ctx_len, int32_t *block_table, int32_t max_pages,
                                      int64_t num_pages, int32_t *page_refs, void *k_cache,
                                      void *v_cache, int32_t layer_begin, int32_t layer_end,
                                      int32_t *result, pic_stream_t stream) {
  using namespace pic;
  using namespace pic::pages;
  static const char *who = "pic_page_fork";
  RopeParams rp;
  pic_status_t st = check_cache(who, geom, &rp, k_cache, v_cache, layer_begin, layer_end);
  if (st == PIC_OK)
    st = check_table(who, n, dst_row, rows, ctx_len, block_table, max_pages, num_pages, page_refs);
  if (st != PIC_OK) return st;
  if (reserve < 0) return fail(PIC_ERR_INVALID_ARG, "%s: reserve %d is negative", who, reserve);
  if (n == 0) return PIC_OK;
  if (!src_row || !result) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  const int layers = layer_end - layer_begin, hkv = geom->num_kv_heads;
  const long long table_blocks = (long long)n * ((max_pages + 255) / 256);
  const long long copy_blocks = ((long long)n * layers * hkv + 7) / 8;
  if (table_blocks + copy_blocks > INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%s: problem too large for one launch", who);
  int32_t *status = device_status_ptr();
  if (!status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  PlanParams pp{n, rows, max_pages, reserve, num_pages, dst_row, src_row, ctx_len, block_table,
                page_refs, result, status};
  cudaError_t e = launch_plan<true>(pp, stream);
  if (e != cudaSuccess) return cuda_fail(e, who);
  ForkParams fp;
  fp.n = n;
  fp.max_pages = max_pages;
  fp.hkv = hkv;
  fp.piece_row = geom->head_dim * 2 / 16;
  fp.layers = layers;
  fp.table_blocks = (int)table_blocks;
  fp.num_pages = num_pages;
  fp.layer_pieces = (long long)num_pages * fp.hkv * kPage * fp.piece_row;
  fp.src_row = src_row;
  fp.dst_row = dst_row;
  fp.result = result;
  fp.block_table = block_table;
  fp.page_refs = page_refs;
  fp.k = static_cast<uint4 *>(k_cache) + layer_begin * fp.layer_pieces;
  fp.v = static_cast<uint4 *>(v_cache) + layer_begin * fp.layer_pieces;
  fp.status = status;
  return launched(who, launch_dependent(fork_kernel, dim3((unsigned)(table_blocks + copy_blocks)),
                                        dim3(256), 0, stream, fp));
}

extern "C" size_t pic_page_compact_workspace_size(const pic_geom_t *geom, int32_t n,
                                                  int32_t max_keep) {
  if (!geom || n <= 0 || max_keep <= 0 || geom->num_layers <= 0 || geom->num_kv_heads <= 0 ||
      (geom->head_dim != 64 && geom->head_dim != 128))
    return 0;
  return pic::pages::compact_space(geom, n, max_keep, geom->num_layers).total;
}

extern "C" pic_status_t pic_page_compact(const pic_geom_t *geom, int32_t n, const int32_t *row,
                                         const int32_t *start, const int32_t *keep,
                                         int32_t max_keep, const int32_t *keep_len,
                                         int32_t reserve, int32_t rotate, int32_t rows,
                                         int32_t *ctx_len, int32_t *block_table, int32_t max_pages,
                                         int64_t num_pages, int32_t *page_refs, void *k_cache,
                                         void *v_cache, int32_t layer_begin, int32_t layer_end,
                                         int32_t *result, void *workspace, size_t workspace_bytes,
                                         pic_stream_t stream) {
  using namespace pic;
  using namespace pic::pages;
  static const char *who = "pic_page_compact";
  RopeParams rp;
  pic_status_t st = check_cache(who, geom, &rp, k_cache, v_cache, layer_begin, layer_end);
  if (st == PIC_OK)
    st = check_table(who, n, row, rows, ctx_len, block_table, max_pages, num_pages, page_refs);
  if (st != PIC_OK) return st;
  if (reserve < 0 || max_keep <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: reserve %d, max_keep %d", who, reserve, max_keep);
  if (n == 0) return PIC_OK;
  if (!keep || !keep_len || !result) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  CompactParams cp;
  cp.n = n;
  cp.rows = rows;
  cp.max_pages = max_pages;
  cp.max_keep = max_keep;
  cp.segs = (max_keep + kSeg - 1) / kSeg;
  cp.hkv = geom->num_kv_heads;
  cp.hgroup = std::min(heads_per_group(geom), cp.hkv);
  cp.hgroups = (cp.hkv + cp.hgroup - 1) / cp.hgroup;
  cp.layers = layer_end - layer_begin;
  // Long lists of narrow rows: as many layers a CTA as it holds, if they turn alike and
  // two segments an SM are left
  cp.lgroup = 1;
  if (max_keep > kShort && !rp.layer_theta)
    cp.lgroup = (int)std::max(1LL, std::min<long long>(heads_per_group(geom) / cp.hkv,
                                                       (long long)n * cp.layers * cp.segs / (2 * 152)));
  cp.lhs = (cp.layers + cp.lgroup - 1) / cp.lgroup * cp.hgroups;
  cp.layer_begin = layer_begin;
  cp.rotate = rotate != 0;
  cp.num_pages = num_pages;
  cp.dim = geom->head_dim;
  cp.reserve = reserve;
  cp.layer_elems = (long long)num_pages * cp.hkv * kPage * geom->head_dim;
  cp.row = row;
  cp.start = start;
  cp.keep = keep;
  cp.keep_len = keep_len;
  cp.ctx_len = ctx_len;
  cp.block_table = block_table;
  cp.page_refs = page_refs;
  cp.result = result;
  cp.k = static_cast<__nv_bfloat16 *>(k_cache) + layer_begin * cp.layer_elems;
  cp.v = static_cast<__nv_bfloat16 *>(v_cache) + layer_begin * cp.layer_elems;
  cp.flags = cp.ticket = cp.bad = nullptr;
  cp.wait = nullptr;
  cp.checks = compact_checks(max_keep);
  cp.slot = nullptr;
  const CompactSpace cw = compact_space(geom, n, max_keep, cp.layers);
  if (cw.total) {
    if (!workspace || workspace_bytes < cw.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
      return fail(PIC_ERR_WORKSPACE, "%s: workspace needs %zu bytes, 256-aligned", who, cw.total);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    cp.slot = reinterpret_cast<longlong2 *>(ws);
    cp.wait = reinterpret_cast<int2 *>(ws + cw.wait);
    cp.bad = reinterpret_cast<int32_t *>(ws + cw.bad);
    cp.ticket = reinterpret_cast<int32_t *>(ws + cw.ticket);
    cp.flags = reinterpret_cast<int32_t *>(ws + cw.flags);
  }
  const long long items = (long long)n * cp.lhs * (cp.flags ? cp.segs : 1);
  if (items > INT32_MAX / 2)
    return fail(PIC_ERR_UNSUPPORTED, "%s: problem too large for one launch", who);
  if (items == 0) return fail(PIC_ERR_INVALID_ARG, "%s: no layers", who);
  cp.status = device_status_ptr();
  if (!cp.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  cudaError_t e = cudaSuccess;
  if (cp.flags)
    e = launch_dependent(compact_check_kernel, dim3(cp.checks, n), dim3(kCheckThreads), 0, stream, cp);
  if (e == cudaSuccess)
    e = geom->head_dim == 128 ? launch_move<128>(cp, rp, items, stream)
                              : launch_move<64>(cp, rp, items, stream);
  if (e != cudaSuccess) return cuda_fail(e, who);
  FreeParams fp{n, rows, max_pages, num_pages, row, result, reserve, ctx_len, block_table, page_refs,
                cp.status};
  return launched(who, launch_dependent(release_kernel, dim3(n), dim3(kReleaseThreads), 0, stream, fp));
}

extern "C" pic_status_t pic_page_free(int32_t n, const int32_t *row, int32_t rows, int32_t *ctx_len,
                                      int32_t *block_table, int32_t max_pages, int64_t num_pages,
                                      int32_t *page_refs, pic_stream_t stream) {
  using namespace pic;
  using namespace pic::pages;
  static const char *who = "pic_page_free";
  pic_status_t st = check_table(who, n, row, rows, ctx_len, block_table, max_pages, num_pages, page_refs);
  if (st != PIC_OK || n == 0) return st;
  FreeParams fp{n, rows, max_pages, num_pages, row, nullptr, 0, ctx_len, block_table, page_refs,
                device_status_ptr()};
  if (!fp.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  return launched(who, launch_dependent(release_kernel, dim3(n), dim3(kReleaseThreads), 0, stream, fp));
}

extern "C" pic_status_t pic_page_copy(const pic_geom_t *geom, int32_t n, const int32_t *src_page,
                                      const int32_t *dst_page, const void *k_src, const void *v_src,
                                      int64_t src_pages, void *k_dst, void *v_dst,
                                      int64_t dst_pages, int32_t layer_begin, int32_t layer_end,
                                      pic_stream_t stream) {
  using namespace pic;
  using namespace pic::pages;
  static const char *who = "pic_page_copy";
  RopeParams rp;
  pic_status_t st = check_cache(who, geom, &rp, k_src, v_src, layer_begin, layer_end);
  if (st == PIC_OK) st = check_cache(who, geom, &rp, k_dst, v_dst, layer_begin, layer_end);
  if (st != PIC_OK) return st;
  if (n < 0 || src_pages <= 0 || dst_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: n %d, pages must be positive", who, n);
  if (n == 0 || layer_begin == layer_end) return PIC_OK;
  if (!src_page || !dst_page) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  CopyParams cp;
  cp.n = n;
  cp.layers = layer_end - layer_begin;
  cp.pieces_page = geom->num_kv_heads * kPage * geom->head_dim * 2 / 2048;
  cp.src_pages = src_pages;
  cp.dst_pages = dst_pages;
  cp.total = (long long)n * cp.layers * 2 * cp.pieces_page;
  cp.src_page = src_page;
  cp.dst_page = dst_page;
  const long long so = (long long)layer_begin * src_pages * cp.pieces_page * 128;
  const long long to = (long long)layer_begin * dst_pages * cp.pieces_page * 128;
  cp.ks = static_cast<const uint4 *>(k_src) + so;
  cp.vs = static_cast<const uint4 *>(v_src) + so;
  cp.kd = static_cast<uint4 *>(k_dst) + to;
  cp.vd = static_cast<uint4 *>(v_dst) + to;
  cp.status = device_status_ptr();
  if (!cp.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  const long long blocks = (cp.total + 8 * kCopyPieces - 1) / (8 * kCopyPieces);
  if (blocks > INT32_MAX) return fail(PIC_ERR_UNSUPPORTED, "%s: problem too large for one launch", who);
  return launched(who, launch_dependent(copy_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, cp));
}
