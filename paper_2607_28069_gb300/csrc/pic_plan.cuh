// The plan of a batch whose rows share pages, as pic_share_plan writes it and
// pic_attend_shared reads it (never installed).
//
// Nodes: ranges of 128-position tiles that a run of listed entries reads in the same pages.
// Node j < n holds entry j's own tiles, node n + i those that a run around entries i and
// i + 1 shares, below its parent's.  Every (node, kv head, pair of row tiles) is a unit of
// work; the units' costs form one sequence, of which every CTA gets an equal share.
#pragma once

#include "pic_internal.cuh"

namespace pic {
namespace share {

constexpr int kMaxEntries = 4096;
constexpr int kLevels = 4;         // shared nodes above an entry
constexpr int kDepth = kLevels + 1;
constexpr int kCtas = 152;         // one per SM
constexpr int BM = 128, BN = 128;  // rows of a row tile, positions of a key tile
constexpr int kFirstPages = 32;
constexpr int32_t kMagic = 0x50534831;
// Costs of a key tile in a unit of one and of two row tiles, and of a unit besides (0.3 us each: a
// key tile of two row tiles takes 1.5 us, one of one 0.85, a short unit's last softmax, exchange
// and stores about 2.5).  Between 7 and 13 the third makes no difference beyond the noise; 3 made
// 64 entries of 33k keys 62 us instead of 52, as the CTAs of short units were late.
constexpr int kOne = 3, kTwo = 5, kUnit = 8;
// A CTA's least share: it holds the first step of a key tile of any unit around it.
constexpr int kLeast = 2 * kOne;
static_assert(kLeast >= kTwo && kLeast >= kOne, "every CTA within a unit has a tile of it");

struct alignas(16) Node {  // public: include/pic.h
  int32_t begin, end, tile_begin, tile_end, row, keys, parent, level;
};
struct alignas(16) Header {
  int32_t magic, n, hkv, ept, rows, max_pages, items, ctas;
  long long total, q;  // steps; q: total / ctas
};
struct alignas(16) Item {  // a node with tiles
  int32_t begin, m, tile_begin, tiles, row, keys, level, leaf;
};
struct alignas(16) Share {  // of a CTA: its first unit
  long long pos, end, unit0;
  int32_t item, hk, pair, pad;
  long long pad2;
  Item it;  // the item
};
struct alignas(16) Link {  // a node of an entry's chain, by level
  long long base;
  int32_t tiles, begin, m, alone, pad[2];  // alone: all keys of an entry
};

struct View {
  Node *nodes;           // [2 n]
  Header *head;
  Share *shares;         // [kCtas]
  int32_t *first_pages;  // [kCtas][kFirstPages]
  Item *items;           // [2 n]
  Link *chain;           // [n][kDepth]
  int32_t *keys;         // [n] -1: left alone
  int32_t *common;       // [n] of entries i and i + 1
  size_t bytes;
  __host__ __device__ View(void *plan, int n) {
    uint8_t *p = static_cast<uint8_t *>(plan), *p0 = p;
    auto take = [&](size_t b) {
      uint8_t *at = p;
      p += (b + 15) & ~(size_t)15;
      return at;
    };
    nodes = reinterpret_cast<Node *>(take(sizeof(Node) * 2 * n));
    head = reinterpret_cast<Header *>(take(sizeof(Header)));
    shares = reinterpret_cast<Share *>(take(sizeof(Share) * kCtas));
    first_pages = reinterpret_cast<int32_t *>(take(4 * kCtas * kFirstPages));
    items = reinterpret_cast<Item *>(take(sizeof(Item) * 2 * n));
    chain = reinterpret_cast<Link *>(take(sizeof(Link) * (size_t)n * kDepth));
    keys = reinterpret_cast<int32_t *>(take(4 * (size_t)n));
    common = reinterpret_cast<int32_t *>(take(4 * (size_t)n));
    bytes = (size_t)(p - p0);
  }
};

// Entries of a row tile: their query heads of one kv head are its rows.
__host__ __device__ inline int entries_per_tile(int G) { return BM / G; }

// The units of a node of m entries and `tiles` key tiles: of a kv head first the pairs of row
// tiles, then a single one.
struct Units {
  int rt, tiles;
  __host__ __device__ Units(int m, int tiles_, int ept) : rt((m + ept - 1) / ept), tiles(tiles_) {}
  __host__ __device__ bool two(int pair) const { return 2 * pair + 1 < rt; }
  __host__ __device__ int weight(int pair) const { return two(pair) ? kTwo : kOne; }
  __host__ __device__ long long cost(int pair) const { return kUnit + (long long)tiles * weight(pair); }
  __host__ __device__ long long pair_cost() const { return kUnit + (long long)tiles * kTwo; }
  __host__ __device__ long long per_head() const {  // steps of a kv head
    return (rt >> 1) * pair_cost() + (rt & 1) * (kUnit + (long long)tiles * kOne);
  }
};

// Steps are dealt to `ctas` CTAs in equal shares: CTA c's first is floor(total c / ctas) =
// q c + floor(r c / ctas).
struct Deal {
  long long q;
  int ctas, r;
  float part, inv;  // 1 / ctas, ctas / total
  PIC_DEV Deal(long long total, int n, long long quotient)
      : q(quotient), ctas(n), r((int)(total - quotient * n)), part(1.f / (float)n), inv((float)n / (float)max(total, 1ll)) {}
  PIC_DEV Deal(long long total, int n) : Deal(total, n, total >> 31 ? total / n : (long long)((int)total / n)) {}
  // (r c < 2^15: (r c + 1/2) / ctas is at least 1 / 304 away from a whole number, far more than
  // its rounding)
  PIC_DEV long long first(int c) const { return q * c + (int)(((float)(r * c) + 0.5f) * part); }
  // The CTA whose share holds step t: an estimate, then exact.
  PIC_DEV int owner(long long t) const {
    int c = max(0, min(ctas - 1, (int)((float)t * inv)));
    while (c > 0 && first(c) > t) --c;
    while (c + 1 < ctas && first(c + 1) <= t) ++c;
    return c;
  }
};
// A key tile belongs to the CTA whose share holds its first step.
PIC_DEV long long tile_step(long long unit0, int tile, int weight) { return unit0 + kUnit + (long long)tile * weight; }

}  // namespace share
}  // namespace pic
