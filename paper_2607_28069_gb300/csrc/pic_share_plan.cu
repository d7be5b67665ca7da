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
    for (int j0 = tid; j0 < pages; j0 += 8 * blockDim.x) {
      int x[8], y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int j = min(j0 + k * (int)blockDim.x, pages - 1);
        x[k] = ta[j], y[k] = tb[j];
      }
#pragma unroll
      for (int k = 7; k >= 0; --k) {
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

// Nearest value below x (kEqual: at most x) left or right of leaf c of a tree of minima with
// `leaves` leaves (node 1 the root, leaf c at leaves + c); -1: none.
template <bool kEqual>
PIC_DEV int nearest(const int *tree, int leaves, int c, int x, bool right) {
  auto has = [&](int node) { return kEqual ? tree[node] <= x : tree[node] < x; };
  int at = leaves + c;
  for (;;) {  // up until a sibling on the wanted side holds one
    if (at == 1) return -1;
    const bool is_right = at & 1;
    if (is_right != right && has(at ^ 1)) {
      at ^= 1;
      break;
    }
    at >>= 1;
  }
  while (at < leaves) {
    at = 2 * at + (right ? 0 : 1);
    if (!has(at)) at ^= 1;
  }
  return at - leaves;
}

struct Scratch {  // plan_kernel's shared memory, by columns: boundary i (entries i, i + 1) is column i + 1
  int *tree;
  uint16_t *left, *right, *rep, *jump;  // of every column with a count
  uint8_t *level;
  long long *base;      // first step of node k in the order of the work
  uint16_t *item;       // items ahead of it
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

PIC_DEV long long scan_add(long long v, long long *warp_sums, long long *total) {
  const int tid = threadIdx.x, lane = tid & 31, warps = blockDim.x / 32;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[tid >> 5] = x;
  __syncthreads();
  long long before = 0, all = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < (tid >> 5)) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return before + x - v;  // exclusive
}

__global__ void __launch_bounds__(1024) plan_kernel(PlanParams p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ long long warp_sums[32];
  const int n = p.n, tid = threadIdx.x, threads = blockDim.x, leaves = p.tree;
  Scratch s(smem, n, leaves);
  View v(p.plan, n);
  int *val = s.tree + leaves;  // column c: entries c - 1 and c; 0 at both ends
  for (int c = tid; c < leaves; c += threads) val[c] = c >= 1 && c < n ? v.common[c - 1] : 0;
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
      l = nearest<false>(s.tree, leaves, c, x, false);
      r = nearest<false>(s.tree, leaves, c, x, true);
      rep = nearest<true>(s.tree, leaves, l, x, true);
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

  auto leaf_up = [&](int i) {  // the column of the node above entry i's own tiles, or 0
    const int c = val[i] >= val[i + 1] ? i : i + 1;
    return val[c] > 0 ? (int)s.jump[s.rep[c]] : 0;
  };
  // Node k in the order of the work, shared nodes first: its entries and tiles; returns its number.
  auto node_of = [&](int k, Node *o) {
    *o = Node{0, 0, 0, 0, -1, 0, -1, -1};
    if (k < n) {  // node n + k: column k + 1
      const int c = k + 1;
      if (c >= n || val[c] == 0 || s.rep[c] != c || s.level[c] == kNoLevel) return n + k;
      const int up = parent_of(c);
      o->begin = s.left[c], o->end = s.right[c];
      o->tile_begin = up ? val[up] : 0, o->tile_end = val[c];
      o->row = p.row ? p.row[o->begin] : o->begin;
      o->keys = val[c] * BN;
      o->parent = up ? n + up - 1 : -1;
      o->level = s.level[c];
      return n + k;
    }
    const int i = k - n, keys = v.keys[i];
    o->begin = i, o->end = i + 1;
    if (keys < 0) {
      o->keys = -1;
      return i;
    }
    const int up = leaf_up(i);
    o->tile_begin = up ? val[up] : 0;
    o->tile_end = (keys + BN - 1) / BN;
    o->row = p.row ? p.row[i] : i;
    o->keys = keys;
    o->parent = up ? n + up - 1 : -1;
    o->level = up ? s.level[up] + 1 : 0;
    return i;
  };
  const int per = (2 * n + threads - 1) / threads;
  long long cost = 0, items = 0, total, count;
  for (int k = tid * per; k < min(2 * n, (tid + 1) * per); ++k) {
    Node o;
    const int j = node_of(k, &o);
    v.nodes[j] = o;
    const int tiles = o.tile_end - o.tile_begin;
    if (tiles > 0) cost += p.hkv * Units(o.end - o.begin, tiles, p.ept).per_head(), ++items;
  }
  long long at = scan_add(cost, warp_sums, &total);
  int item = (int)scan_add(items, warp_sums, &count);
  for (int k = tid * per; k < min(2 * n, (tid + 1) * per); ++k) {
    Node o;
    node_of(k, &o);
    const int tiles = o.tile_end - o.tile_begin, m = o.end - o.begin;
    s.base[k] = at, s.item[k] = item;
    if (tiles <= 0) continue;
    v.items[item] = Item{o.begin, m, o.tile_begin, tiles, o.row, o.keys, o.level, k >= n};
    at += p.hkv * Units(m, tiles, p.ept).per_head();
    ++item;
  }
  __syncthreads();
  // each entry's chain, by level
  for (int i = tid; i < n; i += threads) {
    Link *chain = v.chain + (size_t)i * kDepth;
    Node o;
    int k = n + i;
    node_of(k, &o);
    for (int level = kDepth - 1; level >= 0; --level) {
      const bool there = level == o.level && o.tile_end > o.tile_begin;
      chain[level] = there ? Link{s.base[k], o.tile_end - o.tile_begin, o.begin, o.end - o.begin,
                                  k >= n && o.level == 0, {0, 0}}
                           : Link{0, 0, 0, 0, 0, {0, 0}};
      if (level == o.level && o.parent >= 0) k = o.parent - n, node_of(k, &o);
    }
  }
  const int ctas = (int)min((long long)kCtas, max(1ll, total / (kUnit + kOne)));
  const Deal deal(total, ctas);
  if (tid == 0) *v.head = Header{kMagic, n, p.hkv, p.ept, p.rows, p.max_pages, (int)count, ctas, total, 0};
  // each CTA's first unit and pages, a warp each
  const int lane = tid & 31;
  for (int c = tid >> 5; c < kCtas; c += threads / 32) {
    Share sh{0, 0, 0, 0, 0, 0, 0, 0};
    int page = -1;
    if (c < ctas && total > 0) {
      sh.pos = deal.first(c), sh.end = deal.first(c + 1);
      int lo = 0, hi = 2 * n - 1;  // the last node that begins at or before pos
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.base[mid] <= sh.pos) lo = mid;
        else hi = mid - 1;
      }
      const Item it = v.items[s.item[lo]];
      const Units u(it.m, it.tiles, p.ept);
      sh.item = s.item[lo];
      const long long off = sh.pos - s.base[lo], head = u.per_head();
      sh.hk = (int)(off / head);
      const long long in = off - sh.hk * head;
      sh.pair = (int)(in / u.pair_cost());
      sh.unit0 = s.base[lo] + sh.hk * head + sh.pair * u.pair_cost();
      const int w = u.weight(sh.pair);
      const int kt = max(0, (int)((sh.pos - sh.unit0 - kUnit + w - 1) / w));
      const long long pidx = (long long)(it.tile_begin + kt) * 8 + lane;
      if (pidx * 16 < it.keys) page = p.block_table[(size_t)it.row * p.max_pages + pidx];
    }
    if (lane == 0) v.shares[c] = sh;
    v.first_pages[c * kFirstPages + lane] = page;
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
  cudaError_t e = cudaFuncSetAttribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)Scratch(nullptr, kMaxEntries, 2 * kMaxEntries).bytes);
  const int wide = std::min(1024, std::max(128, (max_pages / 8 + 31) / 32 * 32));
  if (e == cudaSuccess) e = launch_dependent(common_kernel, dim3(n), dim3(wide), 0, stream, p);
  if (e == cudaSuccess) e = launch_dependent(plan_kernel, dim3(1), dim3(1024), smem, stream, p);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
