// pic_share_plan: which listed rows of a block table read the same pages, as a forest, and
// the deal of the attention's work over it to the SMs.
//
// Two neighbours of the list share the tiles (128 positions, 8 pages) from their starts on in
// which their block tables name the same pages.  Entries i..j share what the least of the
// neighbours' counts between them is, so the nodes of the forest are the runs of entries
// around each count that are bounded by smaller ones: nearest smaller values on both sides,
// found in a tree of minima.
//
// Launches:
//  1. common_kernel: a CTA per entry, its length and its count with the next one (all block
//     table entries are read at once).
//  2. plan_kernel: one CTA: the forest, every entry's chain of nodes, the units' costs added
//     up, and each of the attention's CTAs its first unit and pages.
//
// Measured, on inputs that change from call to call: 4 branches of 4.3k positions 10.4 us, 32
// 11.7, 64 entries of 8 contexts 13.5, 256 of four of 139k 19.8 (17.9 MB of table entries, each read for both its neighbours, 8.9 from DRAM).  Not
// bytes but dependent steps by one CTA: counts and tree 2 us, nearest values 1 to 2.5, nodes and
// their sums 1.5, the CTAs' first units and pages 2 to 3.5, each on cold instructions (nodes formed
// again where they can be read back cost 0.5 us more).  It is made once a step, for all layers.
#include <algorithm>

#include "pic_plan.cuh"

namespace pic {
namespace share {

struct PlanParams {
  int n, rows, max_pages, pos_offset, hkv, ept, tree;  // tree: leaves of the tree of minima
  long long num_pages;
  const int32_t *row, *ctx_len, *block_table;
  void *plan;
  int32_t *status;
};

// Entry i's row and its keys (-1: left alone).
struct Entry {
  int row, keys;
  int code;
};
PIC_DEV Entry entry_of(const PlanParams &p, int i) {
  Entry e{p.row ? p.row[i] : i, -1, PIC_DEV_OK};
  if (e.row < 0 || e.row >= p.rows) {
    e.row = -1, e.code = PIC_DEV_BAD_REQUEST;
    return e;
  }
  const int len = p.ctx_len[e.row];
  const long long keys = (long long)len + p.pos_offset + 1;
  if (len < 0 || keys < 0)
    e.code = PIC_DEV_BAD_REQUEST;
  else if (keys > (long long)p.max_pages * 16)
    e.code = PIC_DEV_BLOCK_TABLE_SHORT;
  else
    e.keys = (int)keys;
  return e;
}

__global__ void __launch_bounds__(1024) common_kernel(PlanParams p) {
  pdl_entry();
  __shared__ int first_diff;
  const int i = blockIdx.x, tid = threadIdx.x;
  View v(p.plan, p.n);
  const Entry a = entry_of(p, i);
  Entry b{-1, -1, 0};
  if (i + 1 < p.n) b = entry_of(p, i + 1);
  const int pages = a.keys < 0 || b.keys < 0 ? 0 : min(a.keys, b.keys) / BN * 8;
  if (tid == 0) first_diff = pages;
  __syncthreads();
  if (pages > 0) {
    const int32_t *ta = p.block_table + (size_t)a.row * p.max_pages;
    const int32_t *tb = p.block_table + (size_t)b.row * p.max_pages;
    int diff = pages;
    constexpr int U = 10;  // entries in flight
    for (int j0 = tid; j0 < pages; j0 += U * blockDim.x) {
      int x[U], y[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int j = min(j0 + k * (int)blockDim.x, pages - 1);
        x[k] = ta[j], y[k] = tb[j];
      }
#pragma unroll
      for (int k = U - 1; k >= 0; --k) {
        const int j = j0 + k * (int)blockDim.x;
        if (j < pages && (x[k] != y[k] || x[k] < 0 || x[k] >= p.num_pages)) diff = min(diff, j);
      }
    }
    if (diff < pages) atomicMin(&first_diff, diff);
  }
  __syncthreads();
  if (tid == 0) {
    v.keys[i] = a.keys;
    v.common[i] = first_diff / 8;
    if (a.code) dev_fail(p.status, a.code, i);
  }
}

// Nearest value of at most x left (or right) of leaf c of a tree of minima with `leaves` leaves
// (node 1 the root, leaf c at leaves + c); -1: none.
__device__ __noinline__ int nearest(const int *tree, int leaves, int c, int x, bool right) {
  int at = leaves + c;
  for (;;) {  // up until a sibling on the wanted side holds one
    if (at == 1) return -1;
    if (((at & 1) != 0) != right && tree[at ^ 1] <= x) {
      at ^= 1;
      break;
    }
    at >>= 1;
  }
  while (at < leaves) {
    at = 2 * at + (right ? 0 : 1);
    if (tree[at] > x) at ^= 1;
  }
  return at - leaves;
}

struct Scratch {  // plan_kernel's shared memory, by columns: boundary i (entries i, i + 1) is column i + 1
  int *tree, *keys, *row;
  uint16_t *left, *right, *rep, *jump;  // of every column with a count
  long long *base;                      // first step of node k in the order of the work
  uint16_t *item;                       // items ahead of it
  uint8_t *level;
  size_t bytes;
  __host__ __device__ Scratch(void *smem, int n, int leaves) {
    uint8_t *p = static_cast<uint8_t *>(smem), *p0 = p;
    auto take = [&](size_t b) {
      uint8_t *at = p;
      p += (b + 15) & ~(size_t)15;
      return at;
    };
    base = reinterpret_cast<long long *>(take(8 * (size_t)2 * n));
    tree = reinterpret_cast<int *>(take(8 * (size_t)leaves));
    keys = reinterpret_cast<int *>(take(4 * (size_t)n));
    row = reinterpret_cast<int *>(take(4 * (size_t)n));
    left = reinterpret_cast<uint16_t *>(take(2 * (size_t)(n + 1)));
    right = reinterpret_cast<uint16_t *>(take(2 * (size_t)(n + 1)));
    rep = reinterpret_cast<uint16_t *>(take(2 * (size_t)(n + 1)));
    jump = reinterpret_cast<uint16_t *>(take(2 * (size_t)(n + 1)));
    item = reinterpret_cast<uint16_t *>(take(2 * (size_t)2 * n));
    level = take((size_t)n + 1);
    bytes = (size_t)(p - p0);
  }
};
constexpr int kNoLevel = 255;

// a / b for 0 <= a, 0 < b and a quotient below 2^20: a rounded estimate, then exact.
PIC_DEV int quotient(long long a, long long b) {
  int q = (int)((float)a / (float)b);
  while (q > 0 && q * b > a) --q;
  while ((q + 1) * b <= a) ++q;
  return q;
}

__global__ void __launch_bounds__(1024) plan_kernel(PlanParams p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ long long warp_cost[32];
  __shared__ int warp_items[32];
  const int n = p.n, tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, leaves = p.tree;
  Scratch s(smem, n, leaves);
  View v(p.plan, n);
  int *val = s.tree + leaves;  // column c: entries c - 1 and c; 0 at both ends
  for (int c = tid; c < leaves; c += threads) val[c] = c >= 1 && c < n ? v.common[c - 1] : 0;
  for (int i = tid; i < n; i += threads) s.keys[i] = v.keys[i], s.row[i] = p.row ? p.row[i] : i;
  for (int w = leaves >> 1; w >= 1; w >>= 1) {
    __syncthreads();
    for (int k = tid; k < w; k += threads) s.tree[w + k] = min(s.tree[2 * (w + k)], s.tree[2 * (w + k) + 1]);
  }
  __syncthreads();
  // each column's run, and the first column of its count there: the node's
  for (int c = tid; c <= n; c += threads) {
    const int x = val[c];
    int l = 0, r = n, rep = 0;
    if (x > 0) {
      l = nearest(s.tree, leaves, c, x - 1, false);
      r = nearest(s.tree, leaves, c, x - 1, true);
      rep = nearest(s.tree, leaves, l, x, true);
    }
    s.left[c] = l, s.right[c] = r, s.rep[c] = rep;
    s.level[c] = kNoLevel;
  }
  __syncthreads();
  // the node above one's own: the run bounded by the larger neighbour (0: none)
  auto parent_of = [&](int c) {
    const int l = s.left[c], r = s.right[c];
    const int up = val[l] >= val[r] ? l : r;
    return val[up] > 0 ? (int)s.rep[up] : 0;
  };
  bool all = true;
  for (int level = 0; level <= kLevels; ++level) {
    bool left_out = false;
    for (int c = tid; c <= n; c += threads)
      if (val[c] > 0 && s.rep[c] == c && s.level[c] == kNoLevel) {
        const int up = parent_of(c);
        s.jump[c] = up;
        if (level < kLevels && (up == 0 ? level == 0 : level > 0 && s.level[up] == level - 1))
          s.level[c] = level, s.jump[c] = c;
        else
          left_out = true;
      }
    all = !__syncthreads_or(left_out);
    if (all) break;
  }
  // nodes too deep are left out: their nearest ancestor that is not
  if (!all)
    for (int w = 1; w < 2 * n; w *= 2) {
      for (int c = tid; c <= n; c += threads)
        if (val[c] > 0 && s.rep[c] == c && s.jump[c] > 0) s.jump[c] = s.jump[s.jump[c]];
      __syncthreads();
    }

  // Node k in the order of the work, shared nodes (k = column - 1) first; its number is k + n,
  // or k - n for an entry's own tiles.
  auto node_of = [&](int k, Node *o) {
    *o = Node{0, 0, 0, 0, -1, 0, -1, -1};
    int up;
    if (k < n) {
      const int c = k + 1;
      if (c >= n || val[c] == 0 || s.rep[c] != c || s.level[c] == kNoLevel) return;
      up = parent_of(c);
      o->begin = s.left[c], o->end = s.right[c];
      o->tile_end = val[c];
      o->row = s.row[o->begin];
      o->keys = val[c] * BN;
      o->level = s.level[c];
    } else {
      const int i = k - n, keys = s.keys[i];
      o->begin = i, o->end = i + 1;
      o->keys = keys;
      if (keys < 0) return;
      const int c = val[i] >= val[i + 1] ? i : i + 1;  // the deeper node beside it
      up = val[c] > 0 ? (int)s.jump[s.rep[c]] : 0;
      o->tile_end = (keys + BN - 1) / BN;
      o->row = s.row[i];
      o->level = up ? s.level[up] + 1 : 0;
    }
    o->tile_begin = up ? val[up] : 0;
    o->parent = up ? n + up - 1 : -1;
  };
  long long at = 0;  // steps and items of the rounds before
  int items = 0;
#pragma unroll 1
  for (int k0 = 0; k0 < 2 * n; k0 += threads) {
    const int k = k0 + tid;
    Node o{0, 0, 0, 0, -1, 0, -1, -1};
    if (k < 2 * n) {
      node_of(k, &o);
      int4 *dst = reinterpret_cast<int4 *>(v.nodes + (k < n ? k + n : k - n));
      dst[0] = make_int4(o.begin, o.end, o.tile_begin, o.tile_end);
      dst[1] = make_int4(o.row, o.keys, o.parent, o.level);
    }
    const int tiles = o.tile_end - o.tile_begin, m = o.end - o.begin;
    const long long cost = tiles > 0 ? p.hkv * Units(m, tiles, p.ept).per_head() : 0;
    // steps and items ahead, over the CTA
    const unsigned there = __ballot_sync(0xffffffffu, tiles > 0);
    long long x = cost;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, w);
      if (lane >= w) x += y;
    }
    __syncthreads();
    if (lane == 31) warp_cost[warp] = x, warp_items[warp] = __popc(there);
    __syncthreads();
    long long of_warps = lane < threads / 32 ? warp_cost[lane] : 0;
    int items_of = lane < threads / 32 ? warp_items[lane] : 0;
    const long long mine = __shfl_sync(0xffffffffu, of_warps, warp);
    const int items_mine = __shfl_sync(0xffffffffu, items_of, warp);
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, of_warps, w);
      const int z = __shfl_up_sync(0xffffffffu, items_of, w);
      if (lane >= w) of_warps += y, items_of += z;
    }
    const long long ahead = at + __shfl_sync(0xffffffffu, of_warps, warp) - mine + x - cost;
    const int item = items + __shfl_sync(0xffffffffu, items_of, warp) - items_mine + __popc(there & ((1u << lane) - 1));
    at += __shfl_sync(0xffffffffu, of_warps, 31), items += __shfl_sync(0xffffffffu, items_of, 31);
    if (k < 2 * n) s.base[k] = ahead, s.item[k] = item;
    if (tiles > 0) {
      int4 *dst = reinterpret_cast<int4 *>(v.items + item);
      dst[0] = make_int4(o.begin, m, o.tile_begin, tiles);
      dst[1] = make_int4(o.row, o.keys, o.level, k >= n);
    }
  }
  const long long total = at;
  __syncthreads();
  // each CTA's first unit: lane l < kShares of a warp finds the one of CTA kShares warp + l
  const int ctas = (int)min((long long)kCtas, max(1ll, total / kLeast));
  const Deal deal(total, ctas);
  if (tid == 0) *v.head = Header{kMagic, n, p.hkv, p.ept, p.rows, p.max_pages, items, ctas, total, deal.q};
  constexpr int kShares = 5;
  static_assert(kShares * 32 >= kCtas, "a warp's share of the CTAs");
  for (int c0 = warp * kShares; c0 < kCtas; c0 += threads / 32 * kShares) {
    const int c = c0 + lane;
    int first_page = 0, row = -1, last_page = 0;  // of its first tiles
    if (lane < kShares && c < kCtas) {
      Share sh{0, 0, 0, 0, 0, 0, 0, 0, Item{0, 0, 0, 0, -1, 0, 0, 0}};
      if (c < ctas && total > 0) {
        sh.pos = deal.first(c), sh.end = deal.first(c + 1);
        int lo = 0, hi = 2 * n - 1;  // the last node that begins at or before pos
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (s.base[mid] <= sh.pos) lo = mid;
          else hi = mid - 1;
        }
        const Node o = v.nodes[lo < n ? lo + n : lo - n];
        const Units u(o.end - o.begin, o.tile_end - o.tile_begin, p.ept);
        sh.item = s.item[lo];
        sh.it = Item{o.begin, o.end - o.begin, o.tile_begin, o.tile_end - o.tile_begin, o.row, o.keys, o.level, lo >= n};
        const long long off = sh.pos - s.base[lo], head = u.per_head();
        sh.hk = quotient(off, head);
        const long long in = off - sh.hk * head;
        sh.pair = quotient(in, u.pair_cost());
        sh.unit0 = s.base[lo] + sh.hk * head + sh.pair * u.pair_cost();
        const int w = u.weight(sh.pair);
        const int kt = max(0, (int)(sh.pos - sh.unit0) - kUnit + w - 1) / w;
        first_page = (o.tile_begin + kt) * 8, row = o.row, last_page = (o.keys + 15) / 16;
      }
      v.shares[c] = sh;
    }
#pragma unroll
    for (int j = 0; j < kShares; ++j) {
      const int r = __shfl_sync(0xffffffffu, row, j), pg = __shfl_sync(0xffffffffu, first_page, j) + lane;
      const int end = __shfl_sync(0xffffffffu, last_page, j);
      int page = -1;
      if (r >= 0 && pg < end) page = p.block_table[(size_t)r * p.max_pages + pg];
      if (c0 + j < kCtas) v.first_pages[(c0 + j) * kFirstPages + lane] = page;
    }
  }
  // each entry's chain, by level (the last warps first, which have no shares)
  for (int i = threads - 1 - tid; i < n; i += threads) {
    Link *chain = v.chain + (size_t)i * kDepth;
    Node o = v.nodes[i];
    int k = n + i;
#pragma unroll 1
    for (int level = kDepth - 1; level >= 0; --level) {
      Link l{0, 0, 0, 0, 0, {0, 0}};
      if (level == o.level && o.tile_end > o.tile_begin)
        l = Link{s.base[k], o.tile_end - o.tile_begin, o.begin, o.end - o.begin, k >= n && o.level == 0, {0, 0}};
      *reinterpret_cast<int4 *>(chain + level) = *reinterpret_cast<int4 *>(&l);
      *(reinterpret_cast<int4 *>(chain + level) + 1) = *(reinterpret_cast<int4 *>(&l) + 1);
      if (level == o.level && o.parent >= 0) k = o.parent - n, o = v.nodes[o.parent];
    }
  }
}

}  // namespace share
}  // namespace pic

extern "C" size_t pic_share_plan_size(int32_t n) {
  if (n <= 0 || n > pic::share::kMaxEntries) return 0;
  return pic::share::View(nullptr, n).bytes;
}

extern "C" pic_status_t pic_share_plan(const pic_geom_t *geom, int32_t n, const int32_t *row,
                                       int32_t rows, const int32_t *ctx_len, int32_t pos_offset,
                                       const int32_t *block_table, int32_t max_pages,
                                       int64_t num_pages, int32_t *plan, size_t plan_bytes,
                                       pic_stream_t stream) {
  using namespace pic;
  using namespace pic::share;
  static const char *who = "pic_share_plan";
  RopeParams rp;
  pic_status_t st = make_rope(geom, &rp);
  if (st != PIC_OK) return st;
  if (n <= 0 || rows <= 0 || max_pages <= 0 || num_pages <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (n > kMaxEntries) return fail(PIC_ERR_UNSUPPORTED, "%s: n %d (at most %d)", who, n, kMaxEntries);
  const int G = geom->num_q_heads / geom->num_kv_heads;
  if (G > BM) return fail(PIC_ERR_UNSUPPORTED, "%s: %d query heads a kv head (at most %d)", who, G, BM);
  if (max_pages > INT32_MAX / 16 - 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: max_pages %d: positions beyond 32 bits", who, max_pages);
  if (!ctx_len || !block_table) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if (!row && n > rows)
    return fail(PIC_ERR_INVALID_ARG, "%s: %d entries, block table of %d rows", who, n, rows);
  const size_t need = pic_share_plan_size(n);
  if (!plan || plan_bytes < need || (reinterpret_cast<uintptr_t>(plan) & 15))
    return fail(PIC_ERR_WORKSPACE, "%s: plan needs %zu bytes, 16-aligned", who, need);
  PlanParams p;
  p.n = n;
  p.rows = rows;
  p.max_pages = max_pages;
  p.pos_offset = pos_offset;
  p.hkv = geom->num_kv_heads;
  p.ept = entries_per_tile(G);
  p.tree = 2;
  while (p.tree < n + 1) p.tree *= 2;
  p.num_pages = num_pages;
  p.row = row;
  p.ctx_len = ctx_len;
  p.block_table = block_table;
  p.plan = plan;
  p.status = device_status_ptr();
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  const size_t smem = Scratch(nullptr, n, p.tree).bytes;
  cudaError_t e = cudaSuccess;
  if (smem > 40 * 1024)
    e = cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)Scratch(nullptr, kMaxEntries, 2 * kMaxEntries).bytes);
  const int wide = std::min(1024, std::max(128, (max_pages / 8 + 31) / 32 * 32));
  if (e == cudaSuccess) e = launch_dependent(common_kernel, dim3(n), dim3(wide), 0, stream, p);
  if (e == cudaSuccess) e = launch_dependent(plan_kernel, dim3(1), dim3(1024), smem, stream, p);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
