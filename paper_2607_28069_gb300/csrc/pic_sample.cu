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
// far as it fits.  What they tell each other goes as asynchronous stores that an mbarrier of
// the receiver counts: about 0.7 us, where a barrier of the cluster and a load took 1.3 to 2.
// A warp takes chunks of 256 entries, 16 bytes a lane from aligned addresses whatever the row's
// start.
//
// Measured, us, on inputs that change from call to call: 1 x 50001, top-p 0.9, 12.1, of which the
// load and the largest 1.3, the histogram and its sums 3, the bin 2, its entries gathered and ranked
// 2, the kept ones' sums 1.5, the token 0.3; 64 x 131072 at a temperature alone 19.5 (33.6 MB): load
// and largest 3.7, the weights' sums 5.5 to 9 (19 packed operations a pair of entries; two CTAs an SM
// on two thirds of the SMs), the token 2; the same with top-p 59.6; 48 x 100003 of mixed settings
// 42.4: where top-p's border lies among most of a flat row, its histogram takes 9, two 32-bit
// shared-memory atomics an entry.  64 registers, for two CTAs an SM, spill 50 bytes (fp32) and 14
// (bf16).
#include <algorithm>
#include <type_traits>

#include "pic_internal.cuh"

namespace pic {
namespace sample {

constexpr int kMaxVocab = 1 << 24;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kChunk = 256;  // entries of a warp at a time, 8 a lane
constexpr int kMaxCluster = 16;
constexpr int kBins = 2048;
constexpr float kBinsPerOctave = 56.f;  // the 36 octaves of weights in 2017 bins
constexpr int kList = 256;              // entries of a bin that are ranked
constexpr int kSlots = 8;
constexpr int kSmall = 4096;             // entries of a CTA's part that go into a histogram at once

struct Params {
  int vocab, hold_chunks, bins;  // bins: shared memory holds the histogram and the list
  long long stride;
  const void *logits;
  const float *temperature, *top_p, *min_p, *uniform;
  const int32_t *top_k;
  int32_t *token, *kept;
  float *logprob;
  int32_t *status;
};

struct alignas(16) Fixed {
  uint64_t slot[kSlots][kMaxCluster][2];  // values from every CTA of the cluster
  uint64_t warp[kWarps][2];
  uint64_t bar[kSlots];                   // mbarriers of the slots
  uint64_t list_bar[2], seg_bar, bin_bar[2];
  int32_t found, pad[3];
};
struct alignas(16) Sum2 {
  uint64_t sum, count;
};
struct alignas(16) Entry {
  uint64_t weight, place;  // place: key << 32 | ~index, larger for what comes ahead in the order
};
constexpr int kSegs = 32, kSegBins = kBins / kSegs;
struct alignas(16) Bins {
  uint32_t count[kBins], low[kBins], high[kBins];  // entries; their weights' sum in 64 bits
  // (two each: a CTA may be at its second selection while another is at its first)
  Entry list[2][kList];
  Sum2 rank[kList];         // of the second half of the list ahead of an entry
  uint64_t pick, pick_sum;
  uint32_t list_n, pad[3];
  Sum2 seg[kSegs];  // the row's
  uint32_t where[4];
  uint64_t where_sum, pad2;
  Sum2 in[1];  // from every CTA [cluster size]: of each segment [kSegs], then twice of a segment's bins [kSegBins]
};
__host__ __device__ constexpr size_t bins_bytes(int C) {
  return sizeof(Bins) - sizeof(Sum2) + sizeof(Sum2) * C * (kSegs + 2 * kSegBins);
}

// 16 bytes to another CTA of the cluster (addresses from map_to_rank), counted by its mbarrier.
PIC_DEV void send(uint32_t addr, uint64_t a, uint64_t b, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.u64 [%0], {%1, %2}, [%3];" ::"r"(addr),
               "l"(a), "l"(b), "r"(bar)
               : "memory");
}
PIC_DEV void st_cluster32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
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
// floor(total floor(2^24 u) / 2^24) for 2^24 u taken into [0, top]
PIC_DEV uint64_t share_of(uint64_t total, float u, float top) {
  const uint64_t n = (uint64_t)fminf(fmaxf(u, 0.f) * 16777216.f, top);
  return (__umul64hi(total, n) << 40) | ((total * n) >> 24);
}
// Logits as whole numbers in the same order (-0 as 0).
PIC_DEV uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
PIC_DEV float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
// Of two packed floats: a b + c rounded towards zero.
PIC_DEV uint64_t fma2_rz(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
PIC_DEV uint32_t lo32(uint64_t v) { return (uint32_t)v; }
PIC_DEV uint32_t hi32(uint64_t v) { return (uint32_t)(v >> 32); }
PIC_DEV uint64_t both(float v) { return f2pack(v, v); }

// The rule of the weights: for z = fl((x - M) s), e = 2^z by rounding z to a whole number and a
// polynomial of degree 5 in the rest, each operation rounded to fp32; the weight is
// trunc(2^36 e).  That is 0 exactly where z < -36 (z is kept at -38 or above, a NaN too), and
// at least 1 from -36 on.  Pairs of entries go through packed operations.
// The polynomial: a fit of 2^f on [-1/2, 1/2] to the least largest relative error with value 1 at 0,
// its coefficients rounded to fp32: within 1.09e-7 (0.92e-7 is the least there is).
constexpr float kLeastZ = -36.f;
struct Rule {
  float max, scale;
  PIC_DEV uint64_t e2(float x0, float x1) const {
    uint64_t z = mul2(add2(f2pack(x0, x1), both(-max)), both(scale));
    float z0, z1;
    f2unpack(z, z0, z1);
    z = f2pack(fmaxf(z0, -38.f), fmaxf(z1, -38.f));
    const uint64_t r = add2(z, both(12582912.f));  // 1.5 2^23: the whole number in the low bits
    const uint64_t f = fma2(add2(r, both(-12582912.f)), both(-1.f), z);  // exact
    // The sums as fma(product, 1, c), the same rounding: a packed product and sum would be
    // contracted into one operation whatever their rounding says.
    auto step = [&](uint64_t p, float c) { return fma2(mul2(p, f), both(1.f), both(c)); };
    uint64_t p = step(both(0.001326472731307149f), 0.009671512991189957f);
    p = step(p, 0.05550733581185341f);
    p = step(p, 0.24022242426872253f);
    p = step(p, 0.6931470036506653f);
    p = step(p, 1.f);
    const uint32_t v0 = lo32(p) + (lo32(r) << 23), v1 = hi32(p) + (hi32(r) << 23);
    return (uint64_t)v1 << 32 | v0;
  }
  // One weight in parts: hi = trunc(2^13 e) and the next 23 bits.
  PIC_DEV uint64_t weight(float x) const;
};
// Sums of weights in two 32-bit parts: hi = trunc(2^13 e), lo the next 23 bits, taken from the
// low bits of a float by adding 2^23 with rounding towards zero (the 2^23's are taken out once).
// (Conversions to 64 bits are issued at a small fraction of the fp32 rate.)
constexpr uint32_t kTwo23 = 0x4b000000u;  // the bits of 2^23
struct Sum {
  uint32_t hi = 0, lo = 0, n = 0;
  PIC_DEV void add(uint64_t e) {
    const uint64_t h = fma2_rz(e, both(8192.f), both(8388608.f));
    const uint64_t r = fma2(e, both(8192.f), fma2(h, both(-1.f), both(8388608.f)));  // exact, in [0, 1)
    const uint64_t l = fma2_rz(r, both(8388608.f), both(8388608.f));
    hi += lo32(h) + hi32(h);
    lo += lo32(l) + hi32(l);
    constexpr uint32_t kOne = 0x2d800000u;  // the bits of 2^-36: a weight
    n += (uint32_t)(lo32(e) >= kOne) + (uint32_t)(hi32(e) >= kOne);
  }
  // Of 8 entries a lane, over the warp (sums of at most 2^21 and 2^31).
  PIC_DEV uint64_t warp_total() {
    n = __reduce_add_sync(0xffffffffu, n);
    return ((uint64_t)__reduce_add_sync(0xffffffffu, hi - 8u * kTwo23) << 23) +
           __reduce_add_sync(0xffffffffu, lo - 8u * kTwo23);
  }
};
PIC_DEV uint64_t Rule::weight(float x) const {
  const uint64_t e = e2(x, x);
  const uint64_t h = fma2_rz(e, both(8192.f), both(8388608.f));
  const uint64_t r = fma2(e, both(8192.f), fma2(h, both(-1.f), both(8388608.f)));
  const uint64_t l = fma2_rz(r, both(8388608.f), both(8388608.f));
  return ((uint64_t)(lo32(h) - kTwo23) << 23) + (lo32(l) - kTwo23);
}

// A CTA's part of a row: chunks [c0, c1) of 256 entries from the aligned address at or below
// the row's start (`lead` entries before it); the first `hold` of them are in shared memory.
template <typename T>
struct Part {
  static constexpr int E = 16 / (int)sizeof(T);  // entries of 16 bytes
  static constexpr int G = 8 / E;                // such pieces of a lane
  const uint4 *base;
  uint4 *held;
  int lead, vocab, c0, c1, hold;
  PIC_DEV int index(int c, int k) const {  // of entry k < 8 of this lane
    return c * kChunk + (k / E * 32 + (int)(threadIdx.x & 31)) * E + k % E - lead;
  }
  PIC_DEV bool edge(int c) const { return c * kChunk < lead || (c + 1) * kChunk > lead + vocab; }
  PIC_DEV void fetch(int c, uint4 *v) const {  // from memory
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int i = index(c, g * E);
      v[g] = make_uint4(0, 0, 0, 0);
      if (i + E > 0 && i < vocab) v[g] = __ldg(base + (size_t)c * (kChunk / E) + g * 32 + (threadIdx.x & 31));
    }
  }
  PIC_DEV void keep(int c, const uint4 *v) const {
    if (c - c0 < hold)
#pragma unroll
      for (int g = 0; g < G; ++g) held[(c - c0) * (kChunk / E) + g * 32 + (threadIdx.x & 31)] = v[g];
  }
  // This lane's entries of a chunk, what is outside the row as -infinity.
  PIC_DEV void entries(int c, const uint4 *v, float *x) const {
#pragma unroll
    for (int g = 0; g < G; ++g)
      if constexpr (E == 4) {
        x[4 * g] = __uint_as_float(v[g].x), x[4 * g + 1] = __uint_as_float(v[g].y);
        x[4 * g + 2] = __uint_as_float(v[g].z), x[4 * g + 3] = __uint_as_float(v[g].w);
      } else {
        unpack8(v[g], x);
      }
    if (edge(c))
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = index(c, k);
        if (i < 0 || i >= vocab) x[k] = -INFINITY;
      }
  }
  PIC_DEV void load(int c, float *x) const {
    uint4 v[G];
    if (c - c0 < hold) {
#pragma unroll
      for (int g = 0; g < G; ++g) v[g] = held[(c - c0) * (kChunk / E) + g * 32 + (threadIdx.x & 31)];
    } else {
      fetch(c, v);
    }
    entries(c, v, x);
  }
};

// What is kept so far: entries before or at (key, index) in the order; x: the key's logit.
struct Last {
  uint32_t key = 0;
  int index = 0x7fffffff;
  float x = -INFINITY;
  PIC_DEV bool keeps(float v, int i) const { return v > x || (v == x && i <= index); }
};

template <typename T>
struct Row {
  Part<T> part;
  Fixed &fx;
  uint64_t *chunk;  // a sum for each of this CTA's chunks
  int rank, C, turn;
  int32_t *status;
  PIC_DEV Row(Fixed &f) : fx(f) {}

  // Two values of each CTA (of its first warp) to all CTAs of the cluster: the slot to read.
  // What else the CTAs have written is not ordered by this (see meet).
  PIC_DEV int exchange(uint64_t a, uint64_t b) {
    const int t = turn % kSlots;
    const uint32_t parity = turn / kSlots & 1, bar = smem_u32(&fx.bar[t]);
    ++turn;
    if ((int)threadIdx.x < C) {  // thread j writes to CTA j
      if (threadIdx.x == 0) mbar_expect_tx(bar, 16 * C);
      send(map_to_rank(smem_u32(&fx.slot[t][rank][0]), threadIdx.x), a, b, map_to_rank(bar, threadIdx.x));
    }
    mbar_wait_no_flag(bar, parity, status, -3, kWaitLimitNs);
    return t;
  }
  // Sums of a and b (the same in all lanes of a warp) over the CTA: in warp 0.
  PIC_DEV void cta_sum(uint64_t &a, uint64_t &b) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) fx.warp[warp][0] = a, fx.warp[warp][1] = b;
    __syncthreads();
    if (warp == 0) {
      a = lane < kWarps ? fx.warp[lane][0] : 0;
      b = lane < kWarps ? fx.warp[lane][1] : 0;
#pragma unroll
      for (int o = kWarps / 2; o; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
      }
    }
  }
  struct Total {
    uint64_t all, before, own, count;  // the row's, ahead of this CTA's part, this part's; entries
  };
  // The values of the CTAs in slot t, lane c the one of CTA c.
  PIC_DEV Total total(int t) const {
    const int lane = threadIdx.x & 31;
    const uint64_t v = lane < C ? fx.slot[t][lane][0] : 0, n = lane < C ? fx.slot[t][lane][1] : 0;
    uint64_t all = v, count = n, before = lane < rank ? v : 0;
#pragma unroll
    for (int o = kMaxCluster / 2; o; o >>= 1) {
      all += __shfl_xor_sync(0xffffffffu, all, o);
      count += __shfl_xor_sync(0xffffffffu, count, o);
      before += __shfl_xor_sync(0xffffffffu, before, o);
    }
    all = __shfl_sync(0xffffffffu, all, 0), count = __shfl_sync(0xffffffffu, count, 0);
    return Total{all, __shfl_sync(0xffffffffu, before, 0), __shfl_sync(0xffffffffu, v, rank), count};
  }
  // work(c, x, n): the sum of chunk c over the warp, n its number of entries (the same in all
  // lanes).  Every chunk's sum stays in `chunk`.
  template <typename F>
  PIC_DEV Total sums(F &&work) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t mine = 0, num = 0;
#pragma unroll 1
    for (int c = part.c0 + warp; c < part.c1; c += kWarps) {
      float x[8];
      part.load(c, x);
      uint32_t n = 0;
      const uint64_t s = work(c, x, n);
      if (lane == 0) chunk[c - part.c0] = s;
      mine += s;
      num += n;
    }
    cta_sum(mine, num);
    return total(exchange(mine, num));
  }
  // The first entry whose running sum of measures exceeds `at` (below the total), by the CTA
  // that holds it: done(index, its measure) in one lane.
  template <typename F, typename D>
  PIC_DEV void find(uint64_t at, const Total &t, F &&measure, D &&done) {
    if (threadIdx.x >= 32 || at < t.before || at >= t.before + t.own) return;
    const int lane = threadIdx.x & 31, n = part.c1 - part.c0;
    uint64_t left = at - t.before;
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
    float x[8];
    part.load(c, x);
    constexpr int E = Part<T>::E;
#pragma unroll
    for (int g = 0; g < Part<T>::G; ++g) {  // (a lane's E entries follow each other)
      uint64_t w[E], s = 0;
#pragma unroll
      for (int k = 0; k < E; ++k) s += w[k] = measure(x[g * E + k], part.index(c, g * E + k));
      const uint64_t in = scan64(s), all = __shfl_sync(0xffffffffu, in, 31);
      if (all <= left) {
        left -= all;
        continue;
      }
      if (in <= left || in - s > left) return;
      left -= in - s;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        if (w[k] > left) return done(part.index(c, g * E + k), w[k]);
        left -= w[k];
      }
      return;
    }
  }
  // Entries that equal v, up to `last`: their number and each chunk's.
  PIC_DEV Total equals(float v, const Last &last) {
    return sums([&](int c, const float *x, uint32_t &n) {
#pragma unroll
      for (int k = 0; k < 8; ++k) n += x[k] == v && last.keeps(x[k], part.index(c, k));
      n = __reduce_add_sync(0xffffffffu, n);
      return (uint64_t)n;
    });
  }

  // ---- the entry up to which a count or a sum is reached
  // work(x, z, index) for the entries with z in [z_min, z_max] that `last` keeps.
  template <typename F>
  PIC_DEV void each(const Rule &rule, const Last &last, float z_min, float z_max, F &&work) {
    const int warp = threadIdx.x >> 5;
#pragma unroll 1
    for (int c = part.c0 + warp; c < part.c1; c += kWarps) {
      float x[8], z[8];
      part.load(c, x);
      bool some = false;
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        f2unpack(mul2(add2(f2pack(x[k], x[k + 1]), both(-rule.max)), both(rule.scale)), z[k], z[k + 1]);
        some |= (z[k] >= z_min && z[k] <= z_max) || (z[k + 1] >= z_min && z[k + 1] <= z_max);
      }
      if (!__any_sync(0xffffffffu, some)) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (z[k] >= z_min && z[k] <= z_max && last.keeps(x[k], part.index(c, k))) work(x[k], z[k], part.index(c, k));
    }
  }
  // The histogram over z of the entries with z >= z_min.
  PIC_DEV void histogram(Bins &bn, const Rule &rule, float z_min) {
    const int warp = threadIdx.x >> 5;
#pragma unroll 1
    for (int c = part.c0 + warp; c < part.c1; c += kWarps) {
      float x[8];
      part.load(c, x);
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        float z[2];
        f2unpack(mul2(add2(f2pack(x[k], x[k + 1]), both(-rule.max)), both(rule.scale)), z[0], z[1]);
        if (!__any_sync(0xffffffffu, z[0] >= z_min || z[1] >= z_min)) continue;
        const uint64_t e = rule.e2(x[k], x[k + 1]);
        const uint64_t h = fma2_rz(e, both(8192.f), both(8388608.f));
        const uint64_t r = fma2(e, both(8192.f), fma2(h, both(-1.f), both(8388608.f)));
        const uint64_t l = fma2_rz(r, both(8388608.f), both(8388608.f));
#pragma unroll
        for (int q = 0; q < 2; ++q)
          if (z[q] >= z_min)
            count_in<true>(bn, (int)(-z[q] * kBinsPerOctave),
                           ((uint64_t)((q ? hi32(h) : lo32(h)) - kTwo23) << 23) + ((q ? hi32(l) : lo32(l)) - kTwo23));
      }
    }
  }
  PIC_DEV void clear(Bins &bn) const {
    uint4 *b = reinterpret_cast<uint4 *>(bn.count);  // and the parts behind
    for (int i = threadIdx.x; i < 3 * kBins / 4; i += kThreads) b[i] = make_uint4(0, 0, 0, 0);
  }
  template <bool kSums>
  PIC_DEV void count_in(Bins &bn, int bin, uint64_t w) const {
    atomicAdd(&bn.count[bin], 1u);
    if constexpr (kSums) {
      const uint32_t lo = (uint32_t)w, old = atomicAdd(&bn.low[bin], lo), hi = (uint32_t)(w >> 32) + (old + lo < old);
      if (hi) atomicAdd(&bn.high[bin], hi);
    }
  }
  PIC_DEV Sum2 bin_sum(const Bins &bn, int i) const { return Sum2{(uint64_t)bn.high[i] << 32 | bn.low[i], bn.count[i]}; }
  // Bins, segments and lists take no barrier of the cluster.  Another CTA reads none of this CTA's
  // bins; what is sent lands in `in` and `list` of the receiver.  A CTA sends segments of a round
  // after it has located the bin of the round before (or, first of all, the sums that follow it),
  // for which it needed what every other CTA sends once it has read that round's segments; the
  // places for a segment's bins and for the list are two each, used in turn, with a location
  // between two uses of one.  An mbarrier counts a phase's bytes only until its receiver, who waits
  // for that phase itself, has also announced them, so none runs a phase ahead.
  // This CTA's sums of each segment of 64 bins to every CTA; lane l gets segment l's of the row.
  PIC_DEV Sum2 segments(Bins &bn) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar = smem_u32(&fx.seg_bar);
    if (threadIdx.x == 0) mbar_expect_tx(bar, (uint32_t)sizeof(Sum2) * kSegs * C);
    __syncthreads();
    for (int g = warp; g < kSegs; g += kWarps) {
      uint64_t s = 0;
      uint32_t n = 0;
#pragma unroll
      for (int k = 0; k < kSegBins; k += 32) {
        const Sum2 b = bin_sum(bn, g * kSegBins + k + lane);
        s += b.sum, n += (uint32_t)b.count;
      }
      s = warp_sum(s), n = __reduce_add_sync(0xffffffffu, n);
      if (lane < C) send(map_to_rank(smem_u32(&bn.in[rank * kSegs + g]), lane), s, n, map_to_rank(bar, lane));
    }
    if (warp == 0) {
      mbar_wait_no_flag(bar, rounds & 1, status, -3, kWaitLimitNs);
      Sum2 t{0, 0};
#pragma unroll 4
      for (int c = 0; c < C; ++c) t.sum += bn.in[c * kSegs + lane].sum, t.count += bn.in[c * kSegs + lane].count;
      bn.seg[lane] = t;
    }
    ++rounds;
    __syncthreads();
    return bn.seg[lane];
  }
  PIC_DEV Total total(const Sum2 &seg) const { return Total{warp_sum(seg.sum), 0, 0, warp_sum(seg.count)}; }
  struct Where {
    int bin;
    uint32_t count, members, first;  // entries ahead of the bin; its own; of them, those of the CTAs before
    uint64_t sum;                    // of those ahead
  };
  // The bin in which the target is reached, behind what sum0 and count0 are; seg: from segments().
  template <bool kCount>
  PIC_DEV Where locate(Bins &bn, const Sum2 &seg, uint64_t target, uint64_t sum0, uint32_t count0) {
    const int tid = threadIdx.x, lane = tid & 31, turn = finds & 1;
    const uint32_t bar = smem_u32(&fx.bin_bar[turn]);
    if (tid == 0) bn.list_n = 0, mbar_expect_tx(bar, (uint32_t)sizeof(Sum2) * kSegBins * C);
    // the first place, in order, up to which the target is reached: ahead of it, it
    auto reach = [&](const Sum2 &v, int *at) {
      const uint64_t s = scan64(v.sum), n = scan64(v.count);
      const unsigned there = __ballot_sync(0xffffffffu, (kCount ? count0 + n : sum0 + s) >= target);
      *at = there ? __ffs(there) - 1 : 31;
      sum0 += __shfl_sync(0xffffffffu, s - v.sum, *at);
      count0 += (uint32_t)__shfl_sync(0xffffffffu, n - v.count, *at);
    };
    int g;
    reach(seg, &g);
    Sum2 *in = bn.in + C * (kSegs + turn * kSegBins);
    {  // this CTA's bins of the segment to every CTA
      const int k = tid % kSegBins, c0 = tid / kSegBins;
      const Sum2 b = bin_sum(bn, g * kSegBins + k);
      for (int c = c0; c < C; c += kThreads / kSegBins)
        send(map_to_rank(smem_u32(&in[rank * kSegBins + k]), c), b.sum, b.count, map_to_rank(bar, c));
    }
    if (tid < 32) {
      mbar_wait_no_flag(bar, finds >> 1 & 1, status, -3, kWaitLimitNs);
      static_assert(kSegBins == 64, "two bins a lane");
      Sum2 a{0, 0}, b{0, 0};  // bins lane, lane + 32
#pragma unroll 4
      for (int c = 0; c < C; ++c) {
        const Sum2 *v = in + c * kSegBins + lane;
        a.sum += v[0].sum, a.count += v[0].count, b.sum += v[32].sum, b.count += v[32].count;
      }
      const uint64_t a_sum = warp_sum(a.sum), a_count = warp_sum(a.count);
      const bool second = (kCount ? count0 + a_count : sum0 + a_sum) < target;
      if (second) a = b, sum0 += a_sum, count0 += (uint32_t)a_count;
      int k;
      reach(a, &k);
      const uint32_t members = (uint32_t)__shfl_sync(0xffffffffu, a.count, k);
      k += second ? 32 : 0;
      uint32_t first = lane < rank ? (uint32_t)in[lane * kSegBins + k].count : 0;
      first = __reduce_add_sync(0xffffffffu, first);
      if (lane == 0) {
        bn.where[0] = g * kSegBins + k, bn.where[1] = count0, bn.where[2] = members, bn.where[3] = first;
        bn.where_sum = sum0;
      }
    }
    ++finds;
    __syncthreads();
    return Where{(int)bn.where[0], bn.where[1], bn.where[2], bn.where[3], bn.where_sum};
  }

  struct Hist {  // what the bins hold
    Sum2 seg;
    bool there;
  };
  // The first entry in the order, of those that `last` keeps, with which their count (kCount) or
  // their sum reaches `target`, into `last`; returns the sum up to it (where weights are
  // counted).  Entries with z < z_min come behind it.  h: a histogram over z that is there
  // already, of all entries, and so of some behind `last`.
  template <bool kCount>
  PIC_DEV uint64_t select(Bins &bn, const Rule &rule, Last &last, uint64_t target, float z_min, Hist &h) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool with_sums = !kCount || h.there;  // (then also the refinements')
    const Last among = h.there ? Last() : last;  // (what is sought is among what `last` keeps either way)
    uint32_t lo = 0, hi = 0xffffffffu;  // its key is one of [lo, hi]
    int shift = -1, zbin = -1;          // shift < 0: bins over z
    uint64_t sum0 = 0;                  // of the entries ahead of the bin
    uint32_t count0 = 0;
    float z_max = 0.f;
    auto bin_of = [&](float x, float z) -> int {
      const int zb = (int)(-z * kBinsPerOctave);
      if (shift < 0) return zb;
      const uint32_t key = key_of(x);
      return zb != zbin || key < lo || key > hi ? -1 : (int)((hi - key) >> shift);
    };
    for (;;) {
      if (!h.there) {
        if (!clean) clear(bn);
        clean = false;
        __syncthreads();
        if (shift < 0 && with_sums && among.x == -INFINITY)
          histogram(bn, rule, z_min);
        else
          each(rule, among, z_min, z_max, [&](float x, float z, int) {
            const int k = bin_of(x, z);
            if (k < 0) return;
            if (with_sums) count_in<true>(bn, k, rule.weight(x));
            else count_in<false>(bn, k, 0);
          });
        __syncthreads();
        h.seg = segments(bn);
      }
      const Where at = locate<kCount>(bn, h.seg, target, sum0, count0);
      sum0 = at.sum, count0 = at.count;
      if (shift < 0) {  // (one 2^-10 of a bin on either side for the rounding of -z bins)
        z_max = fminf(z_max, -((float)at.bin - 0.001f) / kBinsPerOctave);
        z_min = fmaxf(z_min, -((float)at.bin + 1.001f) / kBinsPerOctave);
      }
      const int members = (int)at.members;
      if (members <= kList) {
        // gathered by every CTA: this one's entries behind those of the CTAs before it
        const uint32_t bar = smem_u32(&fx.list_bar[lists & 1]);
        Entry *list = bn.list[lists & 1];
        if (tid == 0) mbar_expect_tx(bar, 16 * (uint32_t)members);
        __syncthreads();
        each(rule, among, z_min, z_max, [&](float x, float z, int i) {
          if (bin_of(x, z) != at.bin) return;
          const uint32_t e = at.first + atomicAdd(&bn.list_n, 1u);
          if (e >= kList) return;
          const uint64_t w = with_sums ? rule.weight(x) : 0;
          const uint32_t dst = smem_u32(&list[e]);
          for (int c = 0; c < C; ++c)
            send(map_to_rank(dst, c), w, (uint64_t)key_of(x) << 32 | ~(uint32_t)i, map_to_rank(bar, c));
        });
        mbar_wait_no_flag(bar, lists++ >> 1 & 1, status, -3, kWaitLimitNs);
        // two threads an entry, each half of the entries ahead of it
        static_assert(kThreads == 2 * kList, "two threads an entry");
        const int i = tid % kList, half = tid / kList;
        uint64_t s = 0, w = 0, place = 0;
        uint32_t n = 0;
        if (i < members) {
          w = list[i].weight, place = list[i].place;
          const int j1 = half ? members : members / 2;
#pragma unroll 4
          for (int j = half ? members / 2 : 0; j < j1; ++j)
            if (list[j].place >= place) s += list[j].weight, ++n;
          if (half) bn.rank[i].sum = s, bn.rank[i].count = n;
        }
        __syncthreads();
        if (!half && i < members) {
          s += sum0 + bn.rank[i].sum, n += count0 + (uint32_t)bn.rank[i].count;
          if (kCount ? n == target : s >= target && s - w < target) bn.pick = place, bn.pick_sum = s;
        }
        __syncthreads();
        const uint32_t key = (uint32_t)(bn.pick >> 32);
        last = Last{key, (int)~(uint32_t)bn.pick, logit_of(key)};
        return bn.pick_sum;
      }
      h.there = false;  // (taken to pieces)
      if (shift == 0) {  // entries of one key: by index
        const uint32_t key = hi - (uint32_t)at.bin;
        const float v = logit_of(key);
        const uint64_t w = rule.weight(v), r = kCount ? target - count0 : (target - sum0 - 1) / w + 1;
        const Total tot = equals(v, among);
        find(r - 1, tot, [&](float x, int i) -> uint64_t { return x == v && among.keeps(x, i); },
             [&](int i, uint64_t) {
               for (int c = 0; c < C; ++c) st_cluster32(map_to_rank(smem_u32(&fx.found), c), (uint32_t)i);
             });
        cluster_sync_all();
        last = Last{key, fx.found, v};
        return sum0 + r * w;
      }
      if (shift < 0) {  // the bin's keys
        zbin = at.bin;
        uint32_t k_lo = 0xffffffffu, k_hi = 0;
        each(rule, among, z_min, z_max, [&](float x, float z, int) {
          if (bin_of(x, z) != at.bin) return;
          k_lo = min(k_lo, key_of(x)), k_hi = max(k_hi, key_of(x));
        });
        k_lo = __reduce_min_sync(0xffffffffu, k_lo), k_hi = __reduce_max_sync(0xffffffffu, k_hi);
        __syncthreads();
        if (lane == 0) fx.warp[warp][0] = k_lo, fx.warp[warp][1] = k_hi;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) k_lo = min(k_lo, (uint32_t)fx.warp[w][0]), k_hi = max(k_hi, (uint32_t)fx.warp[w][1]);
        const int t2 = exchange(k_lo, k_hi);
        lo = 0xffffffffu, hi = 0;
        for (int c = 0; c < C; ++c)
          lo = min(lo, (uint32_t)fx.slot[t2][c][0]), hi = max(hi, (uint32_t)fx.slot[t2][c][1]);
      } else {
        const uint32_t top = hi - ((uint32_t)at.bin << shift);
        lo = max(lo, top - ((1u << shift) - 1));
        hi = top;
      }
      shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
    }
  }
  uint32_t lists = 0, rounds = 0, finds = 0;  // gathered, added up, located so far
  bool clean = true;                          // the bins are zeros
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(Params p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  Fixed &fx = *reinterpret_cast<Fixed *>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) mbar_init(smem_u32(&fx.bar[i]), 1);
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&fx.list_bar[i]), 1), mbar_init(smem_u32(&fx.bin_bar[i]), 1);
    mbar_init(smem_u32(&fx.seg_bar), 1);
    fence_mbar_init();
  }
  // every CTA of the cluster runs before another one writes to its shared memory
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  Row<T> row(fx);
  row.rank = (int)cluster_rank(), row.C = cluster_size(), row.turn = 0, row.status = p.status;
  const int b = blockIdx.x / row.C;
  Part<T> &part = row.part;
  {
    const uintptr_t a = reinterpret_cast<uintptr_t>(static_cast<const T *>(p.logits) + b * p.stride);
    part.base = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
    part.lead = (int)(a & 15) / (int)sizeof(T);
    part.vocab = p.vocab;
    const int chunks = (part.lead + p.vocab + kChunk - 1) / kChunk;
    part.c0 = chunks * row.rank / row.C;
    part.c1 = chunks * (row.rank + 1) / row.C;
    part.hold = p.hold_chunks;
  }
  uint8_t *at = smem + sizeof(Fixed);
  Bins *bins = p.bins ? reinterpret_cast<Bins *>(at) : nullptr;
  if (p.bins) at += bins_bytes(row.C);
  part.held = reinterpret_cast<uint4 *>(at);
  row.chunk = reinterpret_cast<uint64_t *>(at + (size_t)p.hold_chunks * kChunk * sizeof(T));

  // ---- the largest logit, and as much of the row as fits into shared memory
  constexpr int U = 4;  // chunks in flight
  float m = -INFINITY;
#pragma unroll 1
  for (int c = part.c0 + warp; c < part.c1; c += U * kWarps) {
    uint4 v[U][Part<T>::G];
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (c + q * kWarps < part.c1) part.fetch(c + q * kWarps, v[q]);
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (c + q * kWarps < part.c1) {
        part.keep(c + q * kWarps, v[q]);
        float x[8];
        part.entries(c + q * kWarps, v[q], x);
#pragma unroll
        for (int k = 0; k < 8; k += 2) m = max3f(m, x[k], x[k + 1]);  // (a NaN is passed over)
      }
  }
  if (bins) row.clear(*bins);
  // this row's settings
  const float temp = p.temperature ? p.temperature[b] : 1.f, u = p.uniform[b];
  const int top_k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) fx.warp[warp][0] = __float_as_uint(m);
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  auto lanes_max = [&](const uint64_t *v, int n) {  // of v[0], v[2], ...
    m = lane < n ? __uint_as_float((uint32_t)v[2 * lane]) : -INFINITY;
#pragma unroll
    for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = __shfl_sync(0xffffffffu, m, 0);
  };
  if (warp == 0) lanes_max(&fx.warp[0][0], kWarps);
  lanes_max(&fx.slot[row.exchange(__float_as_uint(m), 0)][0][0], row.C);
  const bool writer = row.rank == 0 && tid == 0;
  if (m == -INFINITY) {  // no entry has a weight
    if (writer) {
      p.token[b] = -1;
      if (p.kept) p.kept[b] = 0;
      if (p.logprob) p.logprob[b] = __int_as_float(0x7fffffff);
    }
    return;
  }
  const bool greedy = !(temp > 0.f);
  if (greedy || m == INFINITY) {  // only entries that equal the largest have a weight, 2^36 each
    const typename Row<T>::Total t = row.equals(m, Last());
    uint64_t n = greedy ? 1 : t.all;
    if (top_k > 0) n = min(n, (uint64_t)top_k);
    if (top_p < 1.f) n = min(n, max((share_of(n << 36, top_p, 16777216.f) + ((uint64_t)1 << 36) - 1) >> 36, (uint64_t)1));
    row.find(share_of(n << 36, u, 16777215.f) >> 36, t, [&](float x, int) -> uint64_t { return x == m; },
             [&](int i, uint64_t) {
               p.token[b] = i;
               if (p.kept) p.kept[b] = (int32_t)n;
               if (p.logprob) p.logprob[b] = -logf((float)n);
             });
    return;
  }
  const Rule rule{m, fminf(__fdiv_rn(1.4426950408889634f, temp), 1e30f)};
  const bool by_k = top_k > 0 && top_k < p.vocab, by_p = top_p < 1.f;
  const uint64_t least = max((uint64_t)(fminf(fmaxf(min_p, 0.f), 1.f) * 68719476736.f), (uint64_t)1);
  Last last;
  // The sums of what is kept: of all entries, and (kCut) of those that `last` keeps of a weight
  // of `least` or more.
  auto kept_sums = [&](auto kCut, uint64_t least_) {
    return row.sums([&](int c, const float *x, uint32_t &n) -> uint64_t {
      Sum s;
      if constexpr (kCut) {
        float top = x[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) top = fmaxf(top, x[k]);
        if (!__any_sync(0xffffffffu, top >= last.x)) return 0;
        const float least_e = (float)least_ * 1.4551915228366852e-11f;  // (at most 25 bits: exact)
        unsigned keep = 0;  // one bit an entry
        bool tie = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          keep |= x[k] > last.x ? 1u << k : 0u;
          tie |= x[k] == last.x;
        }
        if (__any_sync(0xffffffffu, tie))
#pragma unroll
          for (int k = 0; k < 8; ++k) keep |= x[k] == last.x && part.index(c, k) <= last.index ? 1u << k : 0u;
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          float e0, e1;
          f2unpack(rule.e2(x[k], x[k + 1]), e0, e1);
          e0 = (keep >> k & 1) && e0 >= least_e ? e0 : 0.f;
          e1 = (keep >> (k + 1) & 1) && e1 >= least_e ? e1 : 0.f;
          s.add(f2pack(e0, e1));
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; k += 2) s.add(rule.e2(x[k], x[k + 1]));
      }
      const uint64_t all = s.warp_total();
      n = s.n;
      return all;
    });
  };
  using No = std::integral_constant<bool, false>;
  using Yes = std::integral_constant<bool, true>;
  typename Row<T>::Total t;
  bool changed = least > 1;
  if (bins && (by_k || by_p)) {
    typename Row<T>::Hist h{{0, 0}, part.vocab <= kSmall * row.C};
    if (h.there) {
      // a small part: the histogram of all entries at once, from which the sums come too
      row.histogram(*bins, rule, kLeastZ);
      row.clean = false;
      __syncthreads();
      h.seg = row.segments(*bins);
      t = row.total(h.seg);
    } else {
      t = kept_sums(No(), 1);
    }
    if (by_k && (uint64_t)top_k < t.count) {
      t.all = row.template select<true>(*bins, rule, last, (uint64_t)top_k, kLeastZ, h);
      changed = true;
      if (by_p && !h.there) t = kept_sums(Yes(), 1);
    }
    if (by_p) {
      const uint64_t target = max(share_of(t.all, top_p, 16777216.f), (uint64_t)1);
      // Entries whose weights are too small to add up to what top-p leaves out: all of them
      // together have less than all - target.
      const float rest = (float)(t.all - target) * (0.999f / (float)p.vocab);
      const float z_min = rest >= 1.f ? fmaxf(__log2f(rest) - 36.01f, kLeastZ) : kLeastZ;
      row.template select<false>(*bins, rule, last, target, h.there ? kLeastZ : z_min, h);
    }
    changed |= by_p || h.there;  // (a histogram leaves no sums of chunks)
  } else if (!changed) {
    t = kept_sums(No(), 1);
  }
  if (changed) t = kept_sums(Yes(), least);
  row.find(share_of(t.all, u, 16777215.f), t,
           [&](float x, int i) -> uint64_t {
             const uint64_t w = last.keeps(x, i) ? rule.weight(x) : 0;
             return w >= least ? w : 0;
           },
           [&](int i, uint64_t w) {
             p.token[b] = i;
             // ln(w / S), near 0 from S - w
             if (p.logprob)
               p.logprob[b] = w > t.all - w ? log1pf(-(float)(t.all - w) / (float)t.all) : logf((float)w / (float)t.all);
           });
  if (writer && p.kept) p.kept[b] = (int32_t)t.count;
}

template <typename T>
static cudaError_t launch(Params p, int batch, cudaStream_t stream) {
  constexpr size_t kSmem = 113 * 1024;  // two CTAs an SM
  auto attempt = [&](int C) {
    const int chunks = (p.vocab + 16 / (int)sizeof(T) - 1 + kChunk - 1) / kChunk;
    const int mine = (chunks + C - 1) / C;
    const size_t fixed = sizeof(Fixed) + (p.bins ? bins_bytes(C) : 0) + (size_t)mine * 8 + 16;
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
  // Parts of up to 4096 entries, but clusters of 16 up to 15 rows and of 12 up to 20 (with a few
  // more rows of so large clusters not all are placed at once), of 8 up to 50, else of 4.  Where rows cost
  // alike, 8 and 4 cross at about 42 rows, with top-p between 50 and 60, and where they cost unlike
  // at more than 60: 50 is a compromise.
  // us of 4, 8, 12 and 16 CTAs: 1 x 50001, top-p, 17.1, 14.4, 14.2 and 12.3; 14 x 50001, mixed, 31.0,
  // 25.7, 26.1 and 17.7; rows of 131072 fp32 at a temperature alone | with top-p | mixed:
  //   16 rows  11.2 10.5  9.0 11.3 | 38.9 31.1 27.1 34.3 | 60.6 38.2 35.6 32.4
  //   20       11.4 11.0  9.1 11.5 | 39.4 33.2 27.4 36.6 | 58.4 43.3 36.3 46.3
  //   24       11.4 11.0 12.7 14.2 | 39.0 33.5 38.2 39.9 | 60.8 44.8 39.0 49.5
  //   32       11.6 11.2 15.6 17.2 | 38.8 34.1 44.0 52.1 | 60.7 46.1 51.6 60.3
  //   39       17.2 15.9 17.4 20.3 | 54.7 46.0 46.7 57.9 | 68.8 53.2 58.2 69.5
  //   44       18.4 18.7 18.9 23.3 | 57.5 52.8 51.1 69.7 | 75.3 55.8 63.9 78.2
  //   50       19.5 21.5 21.7 26.8 | 58.7 56.5 63.5 75.5 | 78.3 69.1 73.0 91.0
  //   56       20.0 22.4 24.2 27.7 | 59.9 58.6 65.0 81.0 | 78.4 67.4 74.0 97.2
  //   64       21.0 23.2 26.2 33.1 | 60.1 61.7 69.4 91.8 | 77.0 69.7 76.2 97.6
  // (the same inputs in turn, from a graph)
  const int most = batch <= 15 ? 16 : batch <= 20 ? 12 : batch <= 50 ? 8 : 4;
  int C = p.vocab > 1 << 22 ? 16 : 1;
  while (C < most && p.vocab > kSmall * C) C = std::min(2 * C, most);
  if (C > 8) {
    if (attempt(C) == cudaSuccess) return cudaSuccess;
    cudaGetLastError();  // (where the device places no such clusters)
    C = 8;
  }
  return attempt(C);
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
           logprob, device_status_ptr()};
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  const cudaError_t e = bf16 ? launch<__nv_bfloat16>(p, batch, stream) : launch<float>(p, batch, stream);
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}

