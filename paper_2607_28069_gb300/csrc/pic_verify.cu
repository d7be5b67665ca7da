// pic_verify_draft: which drafted tokens the target keeps, and the next token.
//
// Rejection sampling of a chain (a token x drawn from q is kept with
// probability min(1, p(x) / q(x)), the first refusal is replaced by a draw from
// max(p - q, 0)), or, where the drafts' probabilities are not given, the
// target's own draw at each node of a tree, followed while a child carries it:
// both leave the tokens distributed as the target's.
//
// A draw is an inverse CDF over up to 2^24 weights.  The weights are taken as
// whole numbers of 2^-36, so their sums are exact in 64 bits in any order: the
// partial sums may be formed by any number of CTAs, and the token drawn does not
// depend on how.
//
// One cluster per request.  Only the rows that the walk visits are read: a row
// is split over the cluster's CTAs in chunks of 1024 entries, one warp per
// chunk; every chunk's sum stays in shared memory, the CTAs' totals are exchanged
// through distributed shared memory, and the CTA that holds the threshold finds
// its chunk and searches that one's entries, which a wide cluster's warps still hold
// in registers and a narrow one's read again.
// Small trees: every token's draw at once, a cluster each, whether the walk gets there
// or not (the random number of a token depends on its depth alone), then the walk.
//
// Measured: 64 chains of 8 over 2^17 entries, 35 of them refused (two rows read, else one: 52
// MB), 14.8 us on changing inputs, the kernel 10.8 on repeated ones.  Not HBM's rate (DRAM 37%
// busy with cold caches): one wave of equal clusters, in which those of a refused request read
// twice the others' bytes, behind two dependent round trips (tokens, their p and q).  A tree level by
// level: 3.9 us for the first and 2.5 for each further one, a chain of the row's loads,
// two cluster barriers and the search; at once, 16 tokens over 50001 entries, 5.6 us.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace verify {

constexpr int kMaxDraft = 64;
constexpr int kMaxVocab = 1 << 24;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kChunk = 1024;
// Requests up to which a cluster has 16 CTAs instead of 8 (us, vocabulary 2^17, 8 and
// 16 CTAs): chain of 8, 4 requests 5.9 and 4.2, 12 6.0 and 5.1, 16 6.0 and 7.4, 64 12.1
// and 22.3; tree of 8, 12 requests 11.1 and 9.6, 24 15.4 and 16.4.
constexpr int kWideBatch = 12;
// Trees whose tokens are all drawn at once (us of the call, level by level and at once;
// random trees, two levels on average): 1 request x 16 tokens x 50001 entries 5.8 and
// 5.4, 4 x 16 10.4 and 6.8, 8 x 16 12.8 and 11.1, 16 x 16 (256 draws) 11.6 and 17.0; x
// 131072 entries 4 x 8 8.4 and 6.8, 8 x 8 10.9 and 9.7, 4 x 16 9.7 and 10.5: with the
// last two, of 2^23 entries each, neither form is the faster one throughout, and from there on
// trees go level by level, which reads less.
constexpr int kNodes = 152;
constexpr long long kNodeEntries = 1 << 23;

struct Params {
  int max_draft, vocab;
  const int32_t *tokens, *parent, *draft_len;
  const float *target, *draft, *uniform;
  long long tb, tt, db, dt;  // strides of target and draft rows
  int32_t *path, *path_len, *next;
  int32_t *status;
};

template <int kCluster>
struct Shared {
  uint64_t chunk[kMaxVocab / kChunk / kCluster];  // sums of this CTA's chunks
  uint64_t tile[32 * 33];       // the weights of the chunk that is searched
  uint64_t warp[kWarps];
  uint64_t totals[2][kCluster]; // every CTA's sum, written by that CTA (by turns)
  int32_t found;                // the token, written by the CTA that holds it
  int32_t refused;
  int32_t parent[kMaxDraft];    // nodes_kernel
};

// A weight as a whole number of 2^-36, trunc(2^36 p) for p clamped to [0, 1]
// (NaN: 0), in two parts of 32 bits: hi = trunc(2^13 p) and lo = trunc(2^23 (2^13 p
// - hi)).  Adding 2^23 with rounding towards zero leaves a whole number in the low
// bits of a float; the sums are taken over the raw bits (mod 2^32) and the 2^23's
// taken out once.  (One conversion to 64 bits per entry instead made the 64 x 2^17
// case 23.9 us: they are issued at a small fraction of the fp32 rate.)
struct Weights {
  uint32_t hi = 0, lo = 0;  // raw sums of up to 256 entries
  PIC_DEV void add(float p) {
    const float a = __saturatef(p);
    const float h = __fmaf_rz(a, 8192.f, 8388608.f);
    const float r = fmaf(a, 8192.f, 8388608.f - h);  // exact, in [0, 1)
    hi += __float_as_uint(h);
    lo += __float_as_uint(__fmaf_rz(r, 8388608.f, 8388608.f));
  }
  PIC_DEV uint64_t sum(uint32_t entries) const {
    constexpr uint32_t kTwo23 = 0x4b000000u;  // the bits of 2^23
    return ((uint64_t)(hi - entries * kTwo23) << 23) + (lo - entries * kTwo23);
  }
};
PIC_DEV void st_cluster64(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
PIC_DEV void st_cluster32(uint32_t addr, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
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

// N entries of a row, 32 apart: of p, or of what p has more than q.  All loads
// go out before the first is used.
template <int N, bool kBoth>
PIC_DEV void load_entries(const float *p, const float *q, int x0, int vocab, float *a) {
  float b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = x0 + 32 * i;
    a[i] = x < vocab ? __ldg(p + x) : 0.f;
    if constexpr (kBoth) b[i] = x < vocab ? __ldg(q + x) : 0.f;
  }
  if constexpr (kBoth)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = __fsub_rn(a[i], b[i]);
}

// A chunk in pieces of N entries a lane (lane l's are l, 32 + l, ...), each given
// to work(a, i), i the number of its first entry.
template <int N, bool kBoth, typename F>
PIC_DEV void walk_chunk(const float *p, const float *q, int c, int vocab, float *a, F &&work) {
  const int x0 = c * kChunk + (threadIdx.x & 31);
#pragma unroll 1
  for (int i = 0; i < 32; i += N) {
    load_entries<N, kBoth>(p, q, x0 + 32 * i, vocab, a);
    work(a, i);
  }
}
PIC_DEV uint64_t warp_sum(uint64_t s) {  // the same in every lane
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
// N of a chunk's entries into the search's tile, which is then searched by one
// warp: the entry of chunk c where the running sum passes `left`.
template <int N>
PIC_DEV void fill_tile(uint64_t *tile, const float *a, int i) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    Weights w;
    w.add(a[k]);
    tile[(i + k) * 33 + (threadIdx.x & 31)] = w.sum(1);
  }
}
PIC_DEV int search_tile(const uint64_t *tile, int c, uint64_t left) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  uint64_t v = 0;  // lane l: entries 32 l .. 32 l + 31
#pragma unroll 8
  for (int k = 0; k < 32; ++k) v += tile[lane * 33 + k];
  uint64_t x = scan64(v);
  const int row = __ffs(__ballot_sync(0xffffffffu, x > left)) - 1;
  left -= __shfl_sync(0xffffffffu, x - v, row);
  x = scan64(tile[row * 33 + lane]);
  return c * kChunk + row * 32 + __ffs(__ballot_sync(0xffffffffu, x > left)) - 1;
}

// One draw by the whole cluster.  Returns false where the row has no weight.
// The token goes to every CTA's sh.found (kAll) or is written to *out by the CTA
// that finds it.  turn: the draws of a kernel alternate between 0 and 1.  number():
// the random number, asked for behind a barrier.
template <int kCluster, bool kBoth, bool kAll, typename F>
PIC_DEV bool draw(Shared<kCluster> &sh, int turn, const float *p, const float *q, int vocab, F &&number,
                  int32_t *out) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)cluster_rank();
  const int chunks = (vocab + kChunk - 1) / kChunk;
  const int c0 = (int)((long long)chunks * rank / kCluster);
  const int c1 = (int)((long long)chunks * (rank + 1) / kCluster);
  // A wide cluster's warps keep their chunk's entries, which are then searched
  // without another read where a warp has a single chunk; a narrow one has the
  // registers for four CTAs an SM instead.
  constexpr bool kKeep = kCluster == 16;
  constexpr int N = kKeep || !kBoth ? 32 : 16;
  uint64_t mine = 0;
  float a[N];
#pragma unroll 1
  for (int c = c0 + warp; c < c1; c += kWarps) {
    Weights w;
    walk_chunk<N, kBoth>(p, q, c, vocab, a, [&](const float *v, int) {
#pragma unroll
      for (int k = 0; k < N; ++k) w.add(v[k]);
    });
    const uint64_t s = warp_sum(w.sum(32));
    if (lane == 0) sh.chunk[c - c0] = s;
    mine += s;
  }
  if (lane == 0) sh.warp[warp] = mine;
  __syncthreads();
  if (tid < kCluster) {  // this CTA's total to every CTA
    uint64_t s = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += sh.warp[w];
    st_cluster64(map_to_rank(smem_u32(&sh.totals[turn][rank]), tid), s);
  }
  cluster_sync_all();
  uint64_t total = 0, before = 0, own = 0;
#pragma unroll
  for (int c = 0; c < kCluster; ++c) {
    const uint64_t t = sh.totals[turn][c];
    if (c < rank) before += t;
    if (c == rank) own = t;
    total += t;
  }
  // floor(total * floor(2^24 u) / 2^24); u outside [0, 1) (NaN: 0)
  const uint64_t n = (uint64_t)fminf(fmaxf(number(), 0.f) * 16777216.f, 16777215.f);
  const uint64_t at = (__umul64hi(total, n) << 40) | ((total * n) >> 24);
  if (before <= at && at < before + own) {  // this CTA holds the threshold
    uint64_t left = at - before;
    const bool single = kKeep && c1 - c0 <= kWarps;  // a chunk a warp
    int c = -1;  // the chunk, where this warp has to search it
    if (single || warp == 0) {
      for (int i = 0;; i += 32) {  // 32 sums at a time
        const uint64_t v = i + lane < c1 - c0 ? sh.chunk[i + lane] : 0, x = scan64(v);
        const unsigned past = __ballot_sync(0xffffffffu, x > left);
        if (past) {
          const int l = __ffs(past) - 1;
          left -= __shfl_sync(0xffffffffu, x - v, l);
          c = c0 + i + l;
          break;
        }
        left -= __shfl_sync(0xffffffffu, x, 31);
      }
      if (single && c != c0 + warp) c = -1;
    }
    if (c >= 0) {
      if (single)
        fill_tile<N>(sh.tile, a, 0);
      else
        walk_chunk<N, kBoth>(p, q, c, vocab, a, [&](const float *v, int i) { fill_tile<N>(sh.tile, v, i); });
      const int x = search_tile(sh.tile, c, left);
      if constexpr (kAll) {
        if (lane < kCluster) st_cluster32(map_to_rank(smem_u32(&sh.found), lane), x);
      } else if (lane == 0) {
        *out = x;
      }
    }
  }
  if constexpr (kAll) cluster_sync_all();
  return total != 0;
}

// The first child of token `at` that carries the token `next`, or -1, by a warp whose lanes
// hold tokens and parents lane and lane + 32.
PIC_DEV int child_of(int at, int next, int n, int tok0, int tok1, int par0, int par1) {
  const int i0 = threadIdx.x & 31, i1 = i0 + 32;
  const bool h0 = i0 < n && i0 > at && tok0 == next && par0 == at && next >= 0;
  const bool h1 = i1 < n && i1 > at && tok1 == next && par1 == at && next >= 0;
  const unsigned m0 = __ballot_sync(0xffffffffu, h0), m1 = __ballot_sync(0xffffffffu, h1);
  return m0 ? __ffs(m0) - 1 : m1 ? __ffs(m1) + 31 : -1;
}

template <int kCluster>
__global__ void __launch_bounds__(kThreads, kCluster == 16 ? 2 : 4) verify_kernel(Params p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared<kCluster> &sh = *reinterpret_cast<Shared<kCluster> *>(smem);
  // every CTA of the cluster runs before another one writes to its shared memory
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31;
  const int b = blockIdx.x / kCluster;
  const bool writer = cluster_rank() == 0 && tid < 32;  // a warp writes the request's outputs
  int32_t *path = p.path + (size_t)b * p.max_draft;
  const float *target = p.target + b * p.tb;
  const float *u = p.uniform + (size_t)b * p.max_draft;
  // lane's tokens lane and lane + 32: read before their number is known
  const int32_t *tok = p.tokens + (size_t)b * p.max_draft;
  const int i0 = lane, i1 = lane + 32;
  const int tok0 = i0 < p.max_draft ? tok[i0] : -1, tok1 = i1 < p.max_draft ? tok[i1] : -1;
  int n = p.draft_len[b];
  const bool bad = n < 0 || n > p.max_draft;
  if (bad) {
    if (writer && lane == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    n = 0;
  }
  int len = 0, next = -1;
  if (n > 0 && p.draft) {
    // ---- a chain of sampled tokens: all tests at once, the first refusal
    const float *draft = p.draft + b * p.db;
    if (tid < 32) {
      auto refused = [&](int i, int x) {
        if (i < 1 || i >= n) return false;
        if (x < 0 || x >= p.vocab) return true;
        return !(__fmul_rn(u[i - 1], __ldg(draft + (i - 1) * p.dt + x)) <
                 __ldg(target + (i - 1) * p.tt + x));
      };
      const bool r0 = refused(i0, tok0), r1 = refused(i1, tok1);
      const unsigned m0 = __ballot_sync(0xffffffffu, r0), m1 = __ballot_sync(0xffffffffu, r1);
      if (lane == 0) sh.refused = m0 ? __ffs(m0) - 1 : m1 ? __ffs(m1) + 31 : n;
    }
    __syncthreads();
    len = sh.refused;
    if (writer)
      for (int i = lane; i < p.max_draft; i += 32) path[i] = i < len ? i : -1;
    if (writer && lane == 0) p.path_len[b] = len;
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    const float *row = target + (len - 1) * p.tt;
    const float last = u[n - 1];
    auto un = [&]() { return last; };
    if (len < n && draw<kCluster, true, false>(sh, 0, row, draft + (len - 1) * p.dt, p.vocab, un, p.next + b))
      return;
    if (!draw<kCluster, false, false>(sh, 1, row, nullptr, p.vocab, un, p.next + b) && writer && lane == 0)
      p.next[b] = -1;
    return;
  }
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (n > 0) {
    // ---- the target's draws down a tree
    int par0 = i0 - 1, par1 = i1 - 1;
    if (p.parent) {
      const int32_t *par = p.parent + (size_t)b * p.max_draft;
      par0 = i0 < p.max_draft ? par[i0] : -1;
      par1 = i1 < p.max_draft ? par[i1] : -1;
    }
    int at = 0;
    if (writer && lane == 0) path[0] = 0;
    for (len = 1;; ++len) {
      const float ul = u[len - 1];
      next = draw<kCluster, false, true>(sh, len & 1, target + at * p.tt, nullptr, p.vocab, [&]() { return ul; },
                                         nullptr)
                 ? sh.found : -1;
      const int child = child_of(at, next, n, tok0, tok1, par0, par1);  // each warp alike
      if (child < 0) break;
      at = child;
      if (writer && lane == 0) path[len] = at;
    }
  }
  if (writer) {
    for (int i = len + lane; i < p.max_draft; i += 32) path[i] = -1;
    if (lane == 0) {
      p.path_len[b] = len;
      p.next[b] = next;
    }
  }
}

// Small trees: the target's draw at every token at once, a cluster each, then (walk_kernel)
// the way down as look-ups.  The draws are left in `path`.  A level after the other costs
// 2.5 us each, this 4.7 to 7 in all.
template <int kCluster>
__global__ void __launch_bounds__(kThreads, kCluster == 16 ? 2 : 4) nodes_kernel(Params p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared<kCluster> &sh = *reinterpret_cast<Shared<kCluster> *>(smem);
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const int tid = threadIdx.x;
  const int item = blockIdx.x / kCluster, b = item / p.max_draft, i = item % p.max_draft;
  const int n = p.draft_len[b];
  if (p.parent && tid < p.max_draft) sh.parent[tid] = p.parent[(size_t)b * p.max_draft + tid];
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (i >= n || n > p.max_draft) return;
  // its depth below token 0 (one that is not below token 0 is never visited)
  auto number = [&]() {
    int d = 0;
    for (int q = i; q > 0; ++d) {
      const int up = p.parent ? sh.parent[q] : q - 1;
      if (up < 0 || up >= q) break;
      q = up;
    }
    return p.uniform[(size_t)b * p.max_draft + d];
  };
  int32_t *out = p.path + (size_t)b * p.max_draft + i;
  if (!draw<kCluster, false, false>(sh, 0, p.target + b * p.tb + i * p.tt, nullptr, p.vocab, number, out) &&
      cluster_rank() == 0 && tid == 0)
    *out = -1;
}

__global__ void __launch_bounds__(kThreads) walk_kernel(Params p, int batch) {  // a warp per request
  pdl_entry();
  const int b = blockIdx.x * kWarps + (int)(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= batch) return;
  const size_t row = (size_t)b * p.max_draft;
  int tok[2], par[2], drawn[2], path[2] = {-1, -1};
  int n = p.draft_len[b];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = lane + 32 * k;
    const bool in = i < p.max_draft;
    tok[k] = in ? p.tokens[row + i] : -1;
    par[k] = !p.parent ? i - 1 : in ? p.parent[row + i] : -1;
    drawn[k] = in ? p.path[row + i] : -1;
  }
  if (n < 0 || n > p.max_draft) {
    if (lane == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    n = 0;
  }
  int len = 0, next = -1;
  for (int at = n > 0 ? 0 : -1; at >= 0;) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (len == lane + 32 * k) path[k] = at;
    ++len;
    const int d0 = __shfl_sync(0xffffffffu, drawn[0], at & 31), d1 = __shfl_sync(0xffffffffu, drawn[1], at & 31);
    next = at < 32 ? d0 : d1;
    at = child_of(at, next, n, tok[0], tok[1], par[0], par[1]);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (lane + 32 * k < p.max_draft) p.path[row + lane + 32 * k] = path[k];
  if (lane == 0) {
    p.path_len[b] = len;
    p.next[b] = next;
  }
}

template <int kCluster>
static cudaError_t launch(void (*kernel)(Params), const Params &p, int clusters, cudaStream_t stream) {
  if (kCluster > 8) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent_cluster(kernel, dim3((unsigned)(clusters * kCluster)), dim3(kThreads),
                                  sizeof(Shared<kCluster>), stream, kCluster, p);
}
// Wide clusters for few (also not where the device places none), else narrow ones.
static cudaError_t launch(void (*wide)(Params), void (*narrow)(Params), const Params &p, int clusters,
                          cudaStream_t stream) {
  if (clusters <= kWideBatch) {
    if (launch<16>(wide, p, clusters, stream) == cudaSuccess) return cudaSuccess;
    cudaGetLastError();
  }
  return launch<8>(narrow, p, clusters, stream);
}

}  // namespace verify
}  // namespace pic

extern "C" pic_status_t pic_verify_draft(int32_t batch, int32_t max_draft, int32_t vocab,
                                         const int32_t *tokens, const int32_t *parent,
                                         const int32_t *draft_len, const float *target_prob,
                                         const int64_t *target_stride, const float *draft_prob,
                                         const int64_t *draft_stride, const float *uniform,
                                         int32_t *path, int32_t *path_len, int32_t *next_token,
                                         pic_stream_t stream) {
  using namespace pic;
  using namespace pic::verify;
  static const char *who = "pic_verify_draft";
  if (batch <= 0 || max_draft <= 0 || vocab <= 0)
    return fail(PIC_ERR_INVALID_ARG, "%s: sizes must be positive", who);
  if (max_draft > kMaxDraft || vocab > kMaxVocab || batch > INT32_MAX / 16)
    return fail(PIC_ERR_UNSUPPORTED, "%s: max_draft %d (at most %d), vocab %d (at most %d)", who,
                max_draft, kMaxDraft, vocab, kMaxVocab);
  if (!tokens || !draft_len || !target_prob || !target_stride || !uniform || !path || !path_len ||
      !next_token || (draft_prob && !draft_stride))
    return fail(PIC_ERR_INVALID_ARG, "%s: NULL tensor", who);
  if (draft_prob && parent)
    return fail(PIC_ERR_INVALID_ARG, "%s: draft_prob needs a chain (parent NULL)", who);
  if (target_stride[0] < 0 || target_stride[1] < 0 ||
      (draft_prob && (draft_stride[0] < 0 || draft_stride[1] < 0)))
    return fail(PIC_ERR_INVALID_ARG, "%s: negative stride", who);
  Params p{max_draft, vocab, tokens, parent, draft_len, target_prob, draft_prob, uniform,
           target_stride[0], target_stride[1], draft_prob ? draft_stride[0] : 0,
           draft_prob ? draft_stride[1] : 0, path, path_len, next_token, device_status_ptr()};
  if (!p.status) return fail(PIC_ERR_CUDA, "%s: no device status word", who);
  cudaError_t e;
  // The draws of all tokens at once read more rows, but not one after the other: taken
  // where their clusters are two waves at most and the rows of all tokens a few
  // microseconds' reading.
  const long long nodes = (long long)batch * max_draft;
  if (!draft_prob && max_draft > 1 && nodes <= kNodes && nodes * vocab < kNodeEntries) {
    e = launch(nodes_kernel<16>, nodes_kernel<8>, p, (int)nodes, stream);
    if (e == cudaSuccess)
      e = launch_dependent(walk_kernel, dim3((batch + kWarps - 1) / kWarps), dim3(kThreads), 0, stream, p, batch);
  } else {
    e = launch(verify_kernel<16>, verify_kernel<8>, p, batch, stream);
  }
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
