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
// its chunk and reads that one again to find the entry.
#include <algorithm>

#include "pic_internal.cuh"

namespace pic {
namespace verify {

constexpr int kMaxDraft = 64;
constexpr int kMaxVocab = 1 << 24;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int kChunk = 1024;
constexpr int kMaxChunks = kMaxVocab / kChunk / kCluster;  // of one CTA

struct Params {
  int max_draft, vocab;
  const int32_t *tokens, *parent, *draft_len;
  const float *target, *draft, *uniform;
  long long tb, tt, db, dt;  // strides of target and draft rows
  int32_t *path, *path_len, *next;
  int32_t *status;
};

struct Shared {
  uint64_t chunk[kMaxChunks];
  uint64_t warp[kWarps];
  uint64_t total;  // of this CTA
  int32_t found;   // the token, written by the CTA that holds it
  int32_t first_refused;
};

// A weight as a whole number of 2^-36; NaN, negative: 0.
PIC_DEV uint64_t weight(float p) {
  return (uint64_t)(fminf(fmaxf(p, 0.f), 1.f) * 68719476736.f);
}
PIC_DEV uint64_t ld_cluster64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
PIC_DEV int ld_cluster32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// The weight of entry x of the row: of p, or of what p has more than q.
PIC_DEV uint64_t entry(const float *p, const float *q, int x) {
  const float a = __ldg(p + x);
  return weight(q ? __fsub_rn(a, __ldg(q + x)) : a);
}

// One draw by the whole cluster; every thread gets the token (-1: no weight).
PIC_DEV int draw(Shared &sh, const float *p, const float *q, int vocab, float u) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int chunks = (vocab + kChunk - 1) / kChunk;
  const int c0 = (int)((long long)chunks * rank / kCluster);
  const int c1 = (int)((long long)chunks * (rank + 1) / kCluster);
  uint64_t mine = 0;
  for (int c = c0 + warp; c < c1; c += kWarps) {
    uint64_t s = 0;
    const int x0 = c * kChunk + lane;
    if ((c + 1) * kChunk <= vocab) {
      // every load of the chunk before the first sum
      float a[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) a[i] = __ldg(p + x0 + 32 * i);
      if (q) {
        float b[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) b[i] = __ldg(q + x0 + 32 * i);
#pragma unroll
        for (int i = 0; i < 32; ++i) a[i] = __fsub_rn(a[i], b[i]);
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) s += weight(a[i]);
    } else {
      for (int x = x0; x < vocab; x += 32) s += entry(p, q, x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) sh.chunk[c - c0] = s;
    mine += s;
  }
  if (lane == 0) sh.warp[warp] = mine;
  __syncthreads();
  if (tid == 0) {
    uint64_t s = 0;
    for (int w = 0; w < kWarps; ++w) s += sh.warp[w];
    sh.total = s;
  }
  cluster_sync_all();
  uint64_t total = 0, before = 0, own = 0;
  uint64_t t[kCluster];
#pragma unroll
  for (int c = 0; c < kCluster; ++c) t[c] = ld_cluster64(map_to_rank(smem_u32(&sh.total), c));
#pragma unroll
  for (int c = 0; c < kCluster; ++c) {
    if (c < (int)rank) before += t[c];
    if (c == (int)rank) own = t[c];
    total += t[c];
  }
  // floor(total * floor(2^24 u) / 2^24); u outside [0, 1) (NaN: 0)
  const uint64_t n = (uint64_t)fminf(fmaxf(u, 0.f) * 16777216.f, 16777215.f);
  const uint64_t at = (__umul64hi(total, n) << 40) | ((total * n) >> 24);
  // the owner of the threshold
  int owner = 0;
  uint64_t run = 0;
#pragma unroll
  for (int c = 0; c < kCluster; ++c) {
    if (run <= at && at < run + t[c]) owner = c;
    run += t[c];
  }
  if (total != 0 && owner == (int)rank && warp == 0) {
    uint64_t left = at - before;  // < own
    int c = 0;
    for (; c < c1 - c0; c += 32) {  // the chunk: 32 sums at a time
      uint64_t v = c + lane < c1 - c0 ? sh.chunk[c + lane] : 0, x = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, x > left);
      if (past) {
        const int l = __ffs(past) - 1;
        left -= __shfl_sync(0xffffffffu, x - v, l);
        c += l;
        break;
      }
      left -= __shfl_sync(0xffffffffu, x, 31);
    }
    const int x0 = (c0 + c) * kChunk + lane * 32;  // 32 consecutive entries a lane
    uint64_t v = 0;
    for (int i = 0; i < 32; ++i)
      if (x0 + i < vocab) v += entry(p, q, x0 + i);
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, x > left);
    if (past && lane == __ffs(past) - 1) {
      uint64_t run2 = x - v;
      int i = 0;
      for (; i < 31; ++i) {
        run2 += entry(p, q, x0 + i);
        if (run2 > left) break;
      }
      sh.found = x0 + i;
    }
  }
  (void)own;
  cluster_sync_all();
  return total ? ld_cluster32(map_to_rank(smem_u32(&sh.found), owner)) : -1;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    verify_kernel(Params p) {
  pdl_entry();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared &sh = *reinterpret_cast<Shared *>(smem);
  const int tid = threadIdx.x, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int b = blockIdx.x / kCluster;
  const bool writer = rank == 0 && tid < 32;  // a warp writes the request's outputs
  int n = p.draft_len[b];
  if (n < 0 || n > p.max_draft) {
    if (writer && lane == 0) dev_fail(p.status, PIC_DEV_BAD_REQUEST, b);
    n = 0;
  }
  int32_t *path = p.path + (size_t)b * p.max_draft;
  const float *target = p.target + b * p.tb;
  const float *u = p.uniform + (size_t)b * p.max_draft;
  const int32_t *tok = p.tokens + (size_t)b * p.max_draft;
  int len = 0, next = -1;
  if (n > 0 && p.draft) {
    // ---- a chain of sampled tokens: all tests at once, the first refusal
    const float *draft = p.draft + b * p.db;
    if (tid < 32) {
      int r = n;  // the first refused token
      for (int i0 = 1; i0 < n && r == n; i0 += 32) {
        const int i = i0 + lane;
        bool ok = true;
        if (i < n) {
          const int x = tok[i];
          ok = false;
          if (x >= 0 && x < p.vocab)
            ok = __fmul_rn(u[i - 1], __ldg(draft + (i - 1) * p.dt + x)) <
                 __ldg(target + (i - 1) * p.tt + x);
        }
        const unsigned no = __ballot_sync(0xffffffffu, !ok);
        if (no) r = i0 + __ffs(no) - 1;
      }
      if (lane == 0) sh.first_refused = r;
    }
    __syncthreads();
    const int r = sh.first_refused;
    len = r;
    const float *row = target + (r - 1) * p.tt;
    if (r < n) next = draw(sh, row, draft + (r - 1) * p.dt, p.vocab, u[n - 1]);
    if (r == n || next < 0) next = draw(sh, row, nullptr, p.vocab, u[n - 1]);
    if (writer)
      for (int i = lane; i < p.max_draft; i += 32) path[i] = i < len ? i : -1;
  } else if (n > 0) {
    // ---- the target's draws down a tree
    const int32_t *par = p.parent ? p.parent + (size_t)b * p.max_draft : nullptr;
    int at = 0;
    if (writer && lane == 0) path[0] = 0;
    for (len = 1;; ++len) {
      next = draw(sh, target + at * p.tt, nullptr, p.vocab, u[len - 1]);
      int child = -1;
      for (int c0 = 0; c0 < n && child < 0; c0 += 32) {  // each warp alike
        const int c = c0 + lane;
        const bool hit = c < n && c > at && next >= 0 && tok[c] == next &&
                         (par ? par[c] : c - 1) == at;
        const unsigned m = __ballot_sync(0xffffffffu, hit);
        if (m) child = c0 + __ffs(m) - 1;
      }
      if (child < 0) break;
      at = child;
      if (writer && lane == 0) path[len] = at;
    }
    if (writer)
      for (int i = len + lane; i < p.max_draft; i += 32) path[i] = -1;
  } else if (writer) {
    for (int i = lane; i < p.max_draft; i += 32) path[i] = -1;
  }
  if (writer && lane == 0) {
    p.path_len[b] = len;
    p.next[b] = next;
  }
  cluster_sync_all();  // the others may still read this CTA's shared memory
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
  if (max_draft > kMaxDraft || vocab > kMaxVocab || batch > INT32_MAX / kCluster)
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
  cudaError_t e = launch_dependent(verify_kernel, dim3((unsigned)(batch * kCluster)), dim3(kThreads),
                                   sizeof(Shared), stream, p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? PIC_OK : cuda_fail(e, who);
}
