// pic_sample: the next token of every row of logits, from given random numbers: temperature,
// top-k, top-p and min-p.
//
// The weights 2^((x - M) log2(e) / T) are formed by a fixed rule of fp32 operations and taken as
// whole numbers of 2^-36 (as the drafts' verification takes probabilities), so that every sum
// is exact in 64 bits in any order, and the token the same however the row is split.  What
// top-k and top-p keep is a prefix of the order "logit descending, index ascending": a last
// entry (its logit, its index), found without sorting: a histogram over the exponent's range
// gives the bin that holds it, the few entries of that bin are gathered and ranked.  (A bin of
// many entries is divided again over the bits of its logits; equal logits by index.)
//
// One cluster per row, its CTAs a part of the row each, which they keep in shared memory as
// far as it fits; sums go through distributed shared memory.  A warp takes chunks of 1024
// entries, 16 bytes a lane from aligned addresses whatever the row's start.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace sample {

constexpr int kMaxVocab = 1 << 24;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kChunk = 1024;
constexpr int kMaxCluster = 16;
constexpr int kBins = 2048;
constexpr float kBinsPerOctave = 54.f;  // 37 octaves of weights in 1998 bins
constexpr int kList = 256;              // entries of a bin that are ranked
constexpr int kSlots = 8;

struct Params {
  int vocab, hold_chunks, bins;  // bins: shared memory holds the histogram and the list
  long long stride;
  const void *logits;
  const float *temperature, *top_p, *min_p, *uniform;
  const int32_t *top_k;
  int32_t *token, *kept;
  float *logprob;
};

struct alignas(16) Fixed {
  uint64_t slot[kSlots][kMaxCluster][2];  // values from every CTA of the cluster
  uint64_t warp[kWarps][2];
  uint64_t tile[32 * 33];                 // the measures of the chunk that is searched
  int32_t found, pad[3];
};
struct alignas(16) Bins {
  uint64_t sum[kBins], all_sum[kBins];      // this CTA's, the cluster's
  uint32_t count[kBins], all_count[kBins];
  uint64_t list_w[kList];
  uint32_t list_key[kList], list_idx[kList];
  uint32_t list_n, first, pick[2];          // pick: the entry found
  uint64_t pick_sum, before_sum;
  uint32_t bin, before_count;
};

PIC_DEV void st_cluster64(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
PIC_DEV void st_cluster32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
PIC_DEV uint64_t ld_cluster64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
PIC_DEV uint32_t ld_cluster32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
PIC_DEV int cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return (int)r;
}
PIC_DEV uint64_t warp_sum(uint64_t s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
PIC_DEV uint64_t scan64(uint64_t v) {  // inclusive prefix sum over the warp
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}
// floor(total floor(2^24 u) / 2^24) for u taken into [0, top]
PIC_DEV uint64_t share_of(uint64_t total, float u, float top) {
  const uint64_t n = (uint64_t)fminf(fmaxf(u, 0.f) * 16777216.f, top);
  return (__umul64hi(total, n) << 40) | ((total * n) >> 24);
}
// Logits as whole numbers in the same order (a NaN counts as -infinity; -0 as 0).
PIC_DEV uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The rule of the weights: e = 2^z for z = fl((x - M) s) >= -37, else 0, by rounding z to a
// whole number and a polynomial of degree 5 in the rest, each operation rounded to fp32; the
// weight is trunc(2^36 e).
struct Rule {
  float max, scale;
  PIC_DEV float z(float x) const { return __fmul_rn(x == max ? 0.f : __fsub_rn(x, max), scale); }
  PIC_DEV float e(float x) const {
    const float z_ = z(x);
    const float r = __fadd_rn(z_, 12582912.f);  // 1.5 2^23: the whole number in the low bits
    const float f = __fsub_rn(z_, __fsub_rn(r, 12582912.f));
    float p = __fadd_rn(__fmul_rn(f, 0.001326472731307149f), 0.009671512991189957f);
    p = __fadd_rn(__fmul_rn(p, f), 0.05550733581185341f);
    p = __fadd_rn(__fmul_rn(p, f), 0.24022242426872253f);
    p = __fadd_rn(__fmul_rn(p, f), 0.6931470036506653f);
    p = __fadd_rn(__fmul_rn(p, f), 1.f);
    const float v = __uint_as_float(__float_as_uint(p) + (__float_as_uint(r) << 23));
    return z_ >= -37.f && x > -INFINITY ? v : 0.f;
  }
  PIC_DEV uint64_t weight(float x) const { return (uint64_t)(e(x) * 68719476736.f); }
};
// Sums of weights in two 32-bit parts: hi = trunc(2^13 e), lo the next 23 bits, taken from the
// low bits of a float by adding 2^23 with rounding towards zero (the 2^23's are taken out once).
struct Sum {
  uint32_t hi = 0, lo = 0, n = 0;
  PIC_DEV void add(float e) {
    const float h = __fmaf_rz(e, 8192.f, 8388608.f);
    const float r = fmaf(e, 8192.f, 8388608.f - h);  // exact, in [0, 1)
    hi += __float_as_uint(h);
    lo += __float_as_uint(__fmaf_rz(r, 8388608.f, 8388608.f));
    n += e >= 1.4551915228366852e-11f;  // 2^-36: a weight
  }
  PIC_DEV uint64_t total(uint32_t entries) const {
    constexpr uint32_t kTwo23 = 0x4b000000u;  // the bits of 2^23
    return ((uint64_t)(hi - entries * kTwo23) << 23) + (lo - entries * kTwo23);
  }
};

// A CTA's part of a row: chunks [c0, c1) of 1024 entries from the aligned address at or below
// the row's start (`lead` entries before it); the first `hold` of them are in shared memory.
template <typename T>
struct Part {
  static constexpr int E = 16 / (int)sizeof(T);        // entries of 16 bytes
  static constexpr int G = kChunk / 32 / E;            // such pieces of a lane
  const uint4 *base;
  uint4 *held;
  int lead, vocab, c0, c1, hold;
  // Entries of piece g of chunk c: x[0 .. E), NaN and what is outside the row as -infinity.
  // kLoad: from memory, and into shared memory where that has room.
  PIC_DEV int index(int c, int g) const { return c * kChunk + (g * 32 + (threadIdx.x & 31)) * E - lead; }
  template <bool kLoad>
  PIC_DEV uint4 raw(int c, int g) const {
    const int lane = threadIdx.x & 31;
    const int at = (c - c0) * (kChunk / E) + g * 32 + lane;
    if (!kLoad && c - c0 < hold) return held[at];
    const int i = index(c, g);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i + E > 0 && i < vocab) v = __ldg(base + (size_t)c * (kChunk / E) + g * 32 + lane);
    return v;
  }
  PIC_DEV void keep(int c, int g, const uint4 &v) const {
    if (c - c0 < hold) held[(c - c0) * (kChunk / E) + g * 32 + (threadIdx.x & 31)] = v;
  }
  PIC_DEV void entries(int c, int g, const uint4 &v, float *x) const {
    if constexpr (E == 4) {
      x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y);
      x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    } else {
      unpack8(v, x);
    }
    const int i = index(c, g);
    const bool inside = i >= 0 && i + E <= vocab;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      x[k] = fmaxf(x[k], -INFINITY);
      if (!inside && (i + k < 0 || i + k >= vocab)) x[k] = -INFINITY;
    }
  }
  // work(c, g, x) for this warp's chunks
  template <typename F>
  PIC_DEV void pieces(int c, F &&work) const {
#pragma unroll 2
    for (int g = 0; g < G; ++g) {
      float x[E];
      entries(c, g, raw<false>(c, g), x);
      work(g, x);
    }
  }
};

template <typename T>
struct Row {
  Part<T> part;
  Fixed &fx;
  uint64_t *chunk;  // a sum for each of this CTA's chunks
  int rank, C, turn;
  PIC_DEV Row(Fixed &f) : fx(f) {}

  // Two values of each CTA of the cluster (given by thread 0) to all of them: slot to read.
  PIC_DEV int exchange(uint64_t a, uint64_t b) {
    const int t = turn;
    turn = (turn + 1) % kSlots;
    // thread j writes to CTA j
    if ((int)threadIdx.x < C) {
      const uint32_t dst = map_to_rank(smem_u32(&fx.slot[t][rank][0]), threadIdx.x);
      st_cluster64(dst, a);
      st_cluster64(dst + 8, b);
    }
    cluster_sync_all();
    return t;
  }
  // Sums of a and b (lane 0 of each warp) over the CTA: in all threads of warp 0.
  PIC_DEV void cta_sum(uint64_t &a, uint64_t &b) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) fx.warp[warp][0] = a, fx.warp[warp][1] = b;
    __syncthreads();
    if (warp == 0) {
      a = warp_sum(lane < kWarps ? fx.warp[lane][0] : 0);
      b = warp_sum(lane < kWarps ? fx.warp[lane][1] : 0);
    }
  }
  // measure(x, i): a whole number for an entry.  Every chunk's sum stays in `chunk`; gives the
  // row's total, this CTA's part [before, before + own) of it, and the number of entries with
  // a measure.
  template <typename F>
  PIC_DEV void sums(F &&chunk_sum, uint64_t &total, uint64_t &before, uint64_t &own, uint64_t &count) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t mine = 0, num = 0;
#pragma unroll 1
    for (int c = part.c0 + warp; c < part.c1; c += kWarps) {
      uint32_t n = 0;
      const uint64_t s = warp_sum(chunk_sum(c, n));
      if (lane == 0) chunk[c - part.c0] = s;
      mine += s;
      num += __reduce_add_sync(0xffffffffu, n);
    }
    cta_sum(mine, num);
    const int t = exchange(mine, num);
    total = before = own = count = 0;
    for (int c = 0; c < C; ++c) {
      const uint64_t v = fx.slot[t][c][0];
      if (c < rank) before += v;
      if (c == rank) own = v;
      total += v;
      count += fx.slot[t][c][1];
    }
  }
  // The first entry whose running sum of measures exceeds `at` (below the total), by the CTA that
  // holds it: done(index, its measure) in one warp, all lanes.
  template <typename F, typename D>
  PIC_DEV void find(uint64_t at, uint64_t before, uint64_t own, F &&measure, D &&done) {
    if (threadIdx.x >= 32 || at < before || at >= before + own) return;
    const int lane = threadIdx.x & 31, n = part.c1 - part.c0;
    uint64_t left = at - before;
    int c = 0;
    for (int i = 0;; i += 32) {
      const uint64_t v = i + lane < n ? chunk[i + lane] : 0, x = scan64(v);
      const unsigned past = __ballot_sync(0xffffffffu, x > left);
      if (past || i + 32 >= n) {
        const int l = past ? __ffs(past) - 1 : 0;
        left -= __shfl_sync(0xffffffffu, x - v, l);
        c = part.c0 + i + l;
        break;
      }
      left -= __shfl_sync(0xffffffffu, x, 31);
    }
    part.pieces(c, [&](int g, const float *x) {
      const int i = part.index(c, g);
#pragma unroll
      for (int k = 0; k < Part<T>::E; ++k) {
        const int at_ = (g * 32 + lane) * Part<T>::E + k;
        fx.tile[(at_ >> 5) * 33 + (at_ & 31)] = measure(x[k], i + k);
      }
    });
    __syncwarp();
    uint64_t v = 0;  // lane l: entries 32 l .. 32 l + 31
#pragma unroll 8
    for (int k = 0; k < 32; ++k) v += fx.tile[lane * 33 + k];
    uint64_t x = scan64(v);
    const int row = __ffs(__ballot_sync(0xffffffffu, x > left)) - 1;
    left -= __shfl_sync(0xffffffffu, x - v, row & 31);
    v = fx.tile[(row & 31) * 33 + lane];
    x = scan64(v);
    const int l = __ffs(__ballot_sync(0xffffffffu, x > left)) - 1;
    done(c * kChunk + (row & 31) * 32 + (l & 31) - part.lead, __shfl_sync(0xffffffffu, v, l & 31));
  }
};

// What is kept so far: entries before or at (key, index) in the order.
struct Last {
  uint32_t key = 0;
  int index = 0x7fffffff;
  PIC_DEV bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(Params p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  Fixed &fx = *reinterpret_cast<Fixed *>(smem);
  // every CTA of the cluster runs before another one writes to its shared memory
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  Row<T> row(fx);
  row.rank = (int)cluster_rank(), row.C = cluster_size(), row.turn = 0;
  const int b = blockIdx.x / row.C;
  Part<T> &part = row.part;
  {
    const uintptr_t a = reinterpret_cast<uintptr_t>(static_cast<const T *>(p.logits) + b * p.stride);
    part.base = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
    part.lead = (int)(a & 15) / (int)sizeof(T);
    part.vocab = p.vocab;
    const int chunks = (part.lead + p.vocab + kChunk - 1) / kChunk;
    part.c0 = (int)((long long)chunks * row.rank / row.C);
    part.c1 = (int)((long long)chunks * (row.rank + 1) / row.C);
    part.hold = p.hold_chunks;
  }
  uint8_t *at = smem + sizeof(Fixed);
  Bins *bins = p.bins ? reinterpret_cast<Bins *>(at) : nullptr;
  if (p.bins) at += sizeof(Bins);
  part.held = reinterpret_cast<uint4 *>(at);
  row.chunk = reinterpret_cast<uint64_t *>(at + (size_t)p.hold_chunks * kChunk * sizeof(T));
  // this row's settings
  const float temp = p.temperature ? p.temperature[b] : 1.f, u = p.uniform[b];
  const int top_k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;

  // ---- the largest logit, and as much of the row as fits into shared memory
  float m = -INFINITY;
#pragma unroll 1
  for (int c = part.c0 + warp; c < part.c1; c += kWarps) {
    uint4 v[Part<T>::G];
#pragma unroll
    for (int g = 0; g < Part<T>::G; ++g) v[g] = part.template raw<true>(c, g);
#pragma unroll
    for (int g = 0; g < Part<T>::G; ++g) {
      part.keep(c, g, v[g]);
      float x[Part<T>::E];
      part.entries(c, g, v[g], x);
#pragma unroll
      for (int k = 0; k < Part<T>::E; ++k) m = fmaxf(m, x[k]);
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float *warp_max = reinterpret_cast<float *>(fx.tile);
  if (lane == 0) warp_max[warp] = m;
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  __syncthreads();
  if (warp == 0) {
    m = lane < kWarps ? warp_max[lane] : -INFINITY;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  {
    const int t = row.exchange(__float_as_uint(m), 0);
    m = -INFINITY;
    for (int c = 0; c < row.C; ++c) m = fmaxf(m, __uint_as_float((uint32_t)fx.slot[t][c][0]));
  }
  const bool writer = row.rank == 0 && tid == 0;
  if (m == -INFINITY) {  // no entry has a weight
    if (writer) {
      p.token[b] = -1;
      if (p.kept) p.kept[b] = 0;
      if (p.logprob) p.logprob[b] = __int_as_float(0x7fffffff);
    }
    return;
  }
  uint64_t total, before, own, count;
  if (!(temp > 0.f)) {  // the first entry of the largest logit
    auto first = [&](float x, int) -> uint64_t { return x == m; };
    row.sums([&](int c, uint32_t &) {
      uint64_t s = 0;
      part.pieces(c, [&](int, const float *x) {
#pragma unroll
        for (int k = 0; k < Part<T>::E; ++k) s += x[k] == m;
      });
      return s;
    }, total, before, own, count);
    row.find(0, before, own, first, [&](int i, uint64_t) {
      if (lane) return;
      p.token[b] = i;
      if (p.kept) p.kept[b] = 1;
      if (p.logprob) p.logprob[b] = 0.f;
    });
    return;
  }
  const Rule rule{m, fminf(__fdiv_rn(1.4426950408889634f, temp), 1e30f)};
  row.sums([&](int c, uint32_t &n) {
    Sum s;
    part.pieces(c, [&](int, const float *x) {
#pragma unroll
      for (int k = 0; k < Part<T>::E; ++k) s.add(rule.e(x[k]));
    });
    n = s.n;
    return s.total(32);
  }, total, before, own, count);

  // ---- the last entry that top-k and then top-p keep
  Last last;
  bool cut = false;
  auto select = [&](bool by_count, uint64_t target, float z_min) {
    // the first entry, in the order, with which the count or the sum reaches `target`; entries
    // with z < z_min come behind it
    Bins &bn = *bins;
    uint32_t lo = 0, hi = 0xffffffffu;  // its key is one of [lo, hi]
    int shift = -1, zbin = -1;          // shift < 0: bins over z
    uint64_t sum0 = 0;                  // of the entries ahead of the bin
    uint32_t count0 = 0;
    auto bin_of = [&](float x, uint32_t key) -> int {
      const int zb = min(kBins - 1, (int)(-rule.z(x) * kBinsPerOctave));
      if (shift < 0) return zb;
      return zb != zbin || key < lo || key > hi ? -1 : (int)((hi - key) >> shift);
    };
    auto each = [&](auto &&work) {  // work(x, key, index, weight) for what is kept so far
#pragma unroll 1
      for (int c = part.c0 + warp; c < part.c1; c += kWarps)
        part.pieces(c, [&](int g, const float *x) {
#pragma unroll
          for (int k = 0; k < Part<T>::E; ++k) {
            if (!(rule.z(x[k]) >= z_min)) continue;
            const int i = part.index(c, g) + k;
            const uint32_t key = key_of(x[k]);
            if (!last.keeps(key, i)) continue;
            const uint64_t w = rule.weight(x[k]);
            if (w) work(x[k], key, i, w);
          }
        });
    };
    for (;;) {
      for (int i = tid; i < kBins; i += kThreads) bn.sum[i] = 0, bn.count[i] = 0;
      if (tid == 0) bn.list_n = 0, bn.bin = 0, bn.before_sum = sum0, bn.before_count = count0;
      __syncthreads();
      each([&](float x, uint32_t key, int, uint64_t w) {
        const int k = bin_of(x, key);
        if (k < 0) return;
        atomicAdd(&bn.count[k], 1u);
        atomicAdd(reinterpret_cast<unsigned long long *>(&bn.sum[k]), (unsigned long long)w);
      });
      cluster_sync_all();
      const int per = kBins / row.C;  // bins that this CTA adds up for all
      for (int i = row.rank * per + tid; i < (row.rank + 1) * per; i += kThreads) {
        uint64_t s = 0;
        uint32_t n = 0;
        for (int c = 0; c < row.C; ++c) {
          s += ld_cluster64(map_to_rank(smem_u32(&bn.sum[i]), c));
          n += ld_cluster32(map_to_rank(smem_u32(&bn.count[i]), c));
        }
        for (int c = 0; c < row.C; ++c) {
          st_cluster64(map_to_rank(smem_u32(&bn.all_sum[i]), c), s);
          st_cluster32(map_to_rank(smem_u32(&bn.all_count[i]), c), n);
        }
      }
      cluster_sync_all();
      // the bin in which the target is reached (every CTA for itself)
      {
        constexpr int kPer = kBins / kThreads;
        uint64_t s = 0;
        uint64_t n = 0;
        for (int k = 0; k < kPer; ++k) s += bn.all_sum[tid * kPer + k], n += bn.all_count[tid * kPer + k];
        const uint64_t s_in = scan64(s), n_in = scan64(n);
        if (lane == 31) fx.warp[warp][0] = s_in, fx.warp[warp][1] = n_in;
        __syncthreads();
        uint64_t s_at = sum0 + s_in - s, n_at = count0 + n_in - n;
        for (int w = 0; w < warp; ++w) s_at += fx.warp[w][0], n_at += fx.warp[w][1];
        for (int k = 0; k < kPer; ++k) {
          const uint64_t ds = bn.all_sum[tid * kPer + k], dn = bn.all_count[tid * kPer + k];
          const uint64_t now = by_count ? n_at : s_at, then = by_count ? n_at + dn : s_at + ds;
          if (now < target && then >= target) {
            bn.bin = tid * kPer + k, bn.before_sum = s_at, bn.before_count = (uint32_t)n_at;
          }
          s_at += ds, n_at += dn;
        }
        __syncthreads();
      }
      const int bin = bn.bin;
      sum0 = bn.before_sum, count0 = bn.before_count;
      const uint32_t members = bn.all_count[bin];
      if (members <= kList) {
        // gathered by every CTA: this one's entries behind those of the CTAs before it
        if (tid == 0) {
          uint32_t first = 0;
          for (int c = 0; c < row.rank; ++c) first += ld_cluster32(map_to_rank(smem_u32(&bn.count[bin]), c));
          bn.first = first;
        }
        __syncthreads();
        each([&](float x, uint32_t key, int i, uint64_t w) {
          if (bin_of(x, key) != bin) return;
          const uint32_t at_ = bn.first + atomicAdd(&bn.list_n, 1u);
          for (int c = 0; c < row.C; ++c) {
            st_cluster64(map_to_rank(smem_u32(&bn.list_w[at_]), c), w);
            st_cluster32(map_to_rank(smem_u32(&bn.list_key[at_]), c), key);
            st_cluster32(map_to_rank(smem_u32(&bn.list_idx[at_]), c), (uint32_t)i);
          }
        });
        cluster_sync_all();
        for (int i = warp; i < (int)members; i += kWarps) {
          const uint32_t key = bn.list_key[i], idx = bn.list_idx[i];
          uint64_t s = 0;
          uint32_t n = 0;
          for (int j = lane; j < (int)members; j += 32) {
            const uint32_t kj = bn.list_key[j];
            if (kj > key || (kj == key && bn.list_idx[j] <= idx)) s += bn.list_w[j], ++n;
          }
          s = sum0 + warp_sum(s);
          n = count0 + __reduce_add_sync(0xffffffffu, n);
          const uint64_t w = bn.list_w[i];
          const bool here = by_count ? n == target : s >= target && s - w < target;
          if (here && lane == 0) bn.pick[0] = key, bn.pick[1] = idx, bn.pick_sum = s;
        }
        __syncthreads();
        last.key = bn.pick[0], last.index = (int)bn.pick[1];
        return bn.pick_sum;
      }
      if (shift == 0) {  // entries of one key
        const uint32_t key = hi - (uint32_t)bin;
        const uint64_t w = bn.all_sum[bin] / members;
        const uint64_t r = by_count ? target - count0 : (target - sum0 + w - 1) / w;
        auto same = [&](float x, int i) -> uint64_t {
          const uint32_t k = key_of(x);
          return k == key && last.keeps(k, i);
        };
        uint64_t tot, bef, mine, num;
        row.sums([&](int c, uint32_t &) {
          uint64_t s = 0;
          part.pieces(c, [&](int g, const float *x) {
#pragma unroll
            for (int k = 0; k < Part<T>::E; ++k) s += same(x[k], part.index(c, g) + k);
          });
          return s;
        }, tot, bef, mine, num);
        row.find(r - 1, bef, mine, same, [&](int i, uint64_t) {
          if (lane < row.C) st_cluster32(map_to_rank(smem_u32(&fx.found), lane), (uint32_t)i);
        });
        cluster_sync_all();
        last.key = key, last.index = fx.found;
        return sum0 + r * w;
      }
      if (shift < 0) {  // the bin's keys
        zbin = bin;
        uint32_t k_lo = 0xffffffffu, k_hi = 0;
        each([&](float x, uint32_t key, int, uint64_t) {
          if (bin_of(x, key) != bin) return;
          k_lo = min(k_lo, key), k_hi = max(k_hi, key);
        });
        k_lo = __reduce_min_sync(0xffffffffu, k_lo), k_hi = __reduce_max_sync(0xffffffffu, k_hi);
        __syncthreads();
        if (lane == 0) fx.warp[warp][0] = k_lo, fx.warp[warp][1] = k_hi;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) k_lo = min(k_lo, (uint32_t)fx.warp[w][0]), k_hi = max(k_hi, (uint32_t)fx.warp[w][1]);
        const int t = row.exchange(k_lo, k_hi);
        lo = 0xffffffffu, hi = 0;
        for (int c = 0; c < row.C; ++c)
          lo = min(lo, (uint32_t)fx.slot[t][c][0]), hi = max(hi, (uint32_t)fx.slot[t][c][1]);
      } else {
        const uint32_t top = hi - ((uint32_t)bin << shift);
        lo = max(lo, top - ((1u << shift) - 1));
        hi = top;
      }
      shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
      // (the histogram is read by the other CTAs until here)
      cluster_sync_all();
    }
  };
  if (bins) {
    uint64_t sum_k = total;
    if (top_k > 0 && (uint64_t)top_k < count) sum_k = select(true, (uint64_t)top_k, -38.f), cut = true;
    if (top_p < 1.f) {
      const uint64_t target = max(share_of(sum_k, top_p, 16777216.f), (uint64_t)1);
      // entries whose weights are too small to add up to what top-p leaves out: all of them
      // together have less than (sum_k - target)
      const float rest = (float)(sum_k - target) * (0.999f / (float)p.vocab);
      const float z_min = rest >= 1.f ? __log2f(rest) - 36.01f : -38.f;
      if (cut) cluster_sync_all();  // (the first selection's lists are read until here)
      select(false, target, z_min);
      cut = true;
    }
  }
  const uint64_t least = (uint64_t)(fminf(fmaxf(min_p, 0.f), 1.f) * 68719476736.f);
  auto measure = [&](float x, int i) -> uint64_t {
    if (cut && !last.keeps(key_of(x), i)) return 0;
    const uint64_t w = rule.weight(x);
    return w >= least ? w : 0;
  };
  if (cut || least > 1) {
    const uint32_t key_min = cut ? last.key : 0;
    row.sums([&](int c, uint32_t &n) {
      uint64_t s = 0;
      part.pieces(c, [&](int g, const float *x) {
        const int i = part.index(c, g);
#pragma unroll
        for (int k = 0; k < Part<T>::E; ++k)
          if (key_of(x[k]) >= key_min) {
            const uint64_t w = measure(x[k], i + k);
            s += w, n += w > 0;
          }
      });
      return s;
    }, total, before, own, count);
  }
  const uint64_t draw = share_of(total, u, 16777215.f);
  row.find(draw, before, own, measure, [&](int i, uint64_t w) {
    if (lane) return;
    p.token[b] = i;
    if (p.logprob) p.logprob[b] = (float)log((double)w / (double)total);
  });
  if (writer && p.kept) p.kept[b] = (int32_t)count;
}

template <typename T>
static cudaError_t launch(Params p, int batch, cudaStream_t stream) {
  constexpr size_t kSmem = 113 * 1024;  // two CTAs an SM
  auto attempt = [&](int C) {
    const int chunks = (p.vocab + 16 / (int)sizeof(T) - 1 + kChunk - 1) / kChunk;
    const int mine = (chunks + C - 1) / C;
    const size_t fixed = sizeof(Fixed) + (p.bins ? sizeof(Bins) : 0) + (size_t)mine * 8 + 16;
    const size_t room = fixed < kSmem ? kSmem - fixed : 0;
    p.hold_chunks = (int)std::min<size_t>(mine, room / (kChunk * sizeof(T)));
    const size_t smem = fixed + (size_t)p.hold_chunks * kChunk * sizeof(T);
    cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)std::max(smem, kSmem));
    if (e == cudaSuccess && C > 8)
      e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    return launch_dependent_cluster(sample_kernel<T>, dim3((unsigned)(batch * C)), dim3(kThreads), smem,
                                    stream, C, p);
  };
  if (batch <= 12) {
    if (attempt(16) == cudaSuccess) return cudaSuccess;
    cudaGetLastError();  // (where the device places no such clusters)
  }
  return attempt(batch <= 38 ? 8 : 4);
}

}  // namespace sample
}  // namespace pic

extern "C" pic_status_t pic_sample(int32_t batch, int32_t vocab, const void *logits, int32_t bf16,
                                   int64_t stride, const float *temperature, const int32_t *top_k,
                                   const float *top_p, const float *min_p, const float *uniform,
                                   int32_t *token, float *logprob, int32_t *kept,
                                   pic_stream_t stream) {
  using namespace pic;
  using namespace pic::sample;
  static const char *who = "pic_sample";
  if (batch <= 0 || vocab <= 0) return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (vocab > kMaxVocab || batch > INT32_MAX / 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: batch %d, vocab %d (at most %d)", who, batch, vocab, kMaxVocab);
  if (!logits || !uniform || !token) return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if (stride < 0) return fail(PIC_ERR_INVALID_ARG, "%s: negative stride", who);
  if (reinterpret_cast<uintptr_t>(logits) % (bf16 ? 2 : 4))
    return fail(PIC_ERR_INVALID_ARG, "%s: misaligned logits", who);
  Params p{vocab, 0, top_k || top_p, stride, logits, temperature, top_p, min_p, uniform, top_k, token, kept,
           logprob};
  const cudaError_t e = bf16 ? launch<__nv_bfloat16>(p, batch, stream) : launch<float>(p, batch, stream);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
