// Log probabilities of given tokens with the rows' entropy and most probable tokens, and the
// distance of rows from a teacher's saved logits: one softmax over each row of n x d logits.
//   p_j = exp(scale (z_j - m)) / S      S = sum_j exp(scale (z_j - m))      m = max_j z_j
//   logp = log p_t      H = log S - sum_j p_j scale (z_j - m)      loss = sum_a q_a (log q_a - log p_{i_a})
#include "toc_logits_dev.h"

namespace toc {
namespace logits {
namespace {

constexpr int kEntropy = 1, kTop = 2, kTeach = 4;   // what a kernel is asked for

// Logits in the order that the alternatives have them: the larger first, of equal ones the
// lower column.  A key is never 0 for a column above minus infinity; a NaN has none.
__device__ inline uint64_t key_of(float z, int column) {
  if (!(z > kNone)) return 0;
  const uint32_t b = __float_as_uint(z + 0.0f);   // (-0 as 0)
  return (uint64_t)(b ^ (b >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | (uint32_t)~column;
}
__device__ inline float key_logit(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ inline int key_column(uint64_t key) { return (int)~(uint32_t)key; }

__device__ inline void put_top(const Score &a, int64_t at, uint64_t key, const End &e, float scale) {
  const int column = key ? key_column(key) : -1;
  if (a.ids.bits == 32) ((int32_t *)a.top_ids)[at] = column;
  else ((int64_t *)a.top_ids)[at] = column;
  a.top_logp[at] = key ? log_p(key_logit(key), e, scale) : kNone;
}

// Keys of columns that may be among a row's alternatives; at first the lanes' own.
template <int kLanes>
constexpr int kCand = kLanes > 64 ? 1024 : 512;

template <int kLanes, bool kOn>
struct TopLds {
  uint64_t keys[kOn ? kCand<kLanes> : 1];
  uint64_t best[kLanes / 64];
  uint16_t who[kOn ? kLanes : 1];      // lanes that may hold some
  uint32_t lanes, count;
};

// A row's chunks q0 .. end - 1.
template <typename T>
struct Part {
  const T *z;
  int d, skew, q0, end;

  __device__ inline int column(int q) const { return kCols<T> * q - skew; }
  __device__ inline void numbers(int q, float (&v)[kCols<T>]) const {
    widen<T>(edge_chunk(z, column(q), min(d, column(end)), d), v);
  }
};

__device__ inline uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }

// The alternatives by k searches for the largest key below the last.
template <typename T, int kLanes, typename Put>
__device__ inline void top_searches(const Part<T> &p, int k, int lane, uint64_t *best_lds, Put put) {
  constexpr int N = kCols<T>;
  uint64_t last = ~(uint64_t)0;
  for (int r = 0; r < k; ++r) {
    uint64_t best = 0;
    if (last) {
      for (int q = p.q0 + lane; q < p.end; q += kLanes) {
        float v[N];
        p.numbers(q, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint64_t key = key_of(v[i], p.column(q) + i);
          if (key < last) best = larger(key, best);
        }
      }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) best = larger(best, __shfl_xor((unsigned long long)best, x, 64));
    if (kLanes > 64) {
      __syncthreads();
      if (threadIdx.x % 64 == 0) best_lds[threadIdx.x / 64] = best;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kLanes / 64; ++i) best = larger(best, best_lds[i]);
    }
    if (lane == 0) put(r, best);
    last = best;
  }
}

// A lower bound, and no key lies between it and the k-th largest of a wave's 64 keys: by bits from
// the highest on, of the logits first.  1 if fewer than k keys are not 0.
__device__ inline uint64_t kth_largest(uint64_t key, int k) {
  if (__popcll(__ballot(key != 0)) < k) return 1;
  const uint32_t high = (uint32_t)(key >> 32), low = (uint32_t)key;
  uint32_t t = 0;
  int count = 64;
  for (uint32_t bit = 1u << 31; bit && count != k; bit >>= 1) {
    const int n = __popcll(__ballot(high >= (t | bit)));
    if (n < k) continue;
    t |= bit;
    count = n;
  }
  uint32_t u = 0;
  if (count != k) {
    // more than k at or above t, fewer than k above it: the lowest columns among those at t
    const int more = k - (int)__popcll(__ballot(high > t));
    for (uint32_t bit = 1u << 31; bit; bit >>= 1)
      if ((int)__popcll(__ballot(high == t && low >= (u | bit))) >= more) u |= bit;
  }
  const uint64_t bound = (uint64_t)t << 32 | u;
  uint64_t least = key >= bound ? key : ~(uint64_t)0;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) {
    const uint64_t other = __shfl_xor((unsigned long long)least, x, 64);
    least = other < least ? other : least;
  }
  return least;
}

// The k largest keys of a part, put(r, key) for the r-th of them (0: there
// is none).  The sums' pass over the row leaves each lane's largest logit and its chunk.  Of lanes i,
// i + 64, ... the largest such keys are 64 keys of different columns, so the k-th largest of them is
// a lower bound of the k-th largest of all, and lanes whose own largest logit is below it have none
// of those: the chunks of the other lanes, some k, are dealt out to the group and read again, and
// the keys from the bound on, little more than k, are left in LDS, where each counts those above
// it.  (A lane's chunk stands for its last column: the key is then at most the column's own.)
// Where more than kCand are left, which takes most of the largest logits in the columns of a few
// lanes, k searches follow.
template <typename T, int kLanes, typename Put>
__device__ inline void top_of(const Part<T> &p, int k, int lane, float m, int most, TopLds<kLanes, true> &lds, Put put) {
  constexpr int N = kCols<T>;
  lds.keys[lane] = key_of(m, min(most + N, p.d) - 1);
  if (lane == 0) lds.lanes = lds.count = 0;
  group_sync<kLanes>();
  uint64_t key = lds.keys[lane % 64];
#pragma unroll
  for (int w = 1; w < kLanes / 64; ++w) key = larger(key, lds.keys[w * 64 + lane % 64]);
  const uint64_t bound = kth_largest(key, k);
  if (key_of(m, 0) >= bound) lds.who[atomicAdd(&lds.lanes, 1u)] = (uint16_t)lane;
  group_sync<kLanes>();
  const uint32_t lanes = lds.lanes, deals = (uint32_t)(p.end - p.q0 + kLanes - 1) / kLanes;
  for (uint32_t i = lane; i < lanes * deals; i += kLanes) {
    const int q = p.q0 + (int)lds.who[i % lanes] + (int)(i / lanes) * kLanes;
    if (q >= p.end) continue;
    float v[N];
    p.numbers(q, v);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint64_t key = key_of(v[j], p.column(q) + j);
      if (key < bound) continue;
      const uint32_t at = atomicAdd(&lds.count, 1u);
      if (at < (uint32_t)kCand<kLanes>) lds.keys[at] = key;
    }
  }
  group_sync<kLanes>();
  const int count = (int)lds.count;
  if (count > kCand<kLanes>) {
    top_searches<T, kLanes>(p, k, lane, lds.best, put);
    return;
  }
  for (int i = lane; i < max(count, k); i += kLanes) {
    if (i >= count) {
      put(i, (uint64_t)0);
      continue;
    }
    const uint64_t mine = lds.keys[i];
    int above = 0;
    for (int j = 0; j < count; ++j) above += lds.keys[j] > mine;
    if (above < k) put(above, mine);
  }
}

// kLanes lanes to a row, kPer chunks of a lane asked for at once.
template <typename T, int kLanes, int kPer, int kWhat>
__global__ __launch_bounds__(kThreads<kLanes>) void score_kernel(Rows<T> a, Score o, Teacher t) {
  constexpr int kGroups = kThreads<kLanes> / kLanes;
  constexpr bool kT = kWhat & kEntropy;
  __shared__ Sums sums_lds[kGroups][kLanes / 64];
  __shared__ TopLds<kLanes, (kWhat & kTop) != 0> top_lds[kGroups];
  const int lane = lane_of<kLanes>(), group = group_of<kLanes>();
  const int64_t row = row_of<kLanes>();
  if (row >= a.n) return;
  const T *z = a.Z + row * a.ldz;
  const bool first = lane < 64;          // the wave that has the row's few numbers
  Taught x;
  if ((kWhat & kTeach) && first) x.ask(t, row, a.d, lane);
  const int id = kWhat & kTeach ? -1 : scalar_token(o.ids, row, a.d);
  Batch<T, kLanes, kPer> b;
  const int skew = skew_of(z, a.d);
  const Part<T> p{z, a.d, skew, 0, chunks_in<T>(a.d, skew)};
  b.load(z, skew, p.q0, p.end, a.d, lane);
  float zt = 0.0f;
  if ((kWhat & kTeach) && first) {
    x.gather(t, z);
    x.learn(t, row);
  }
  if (id >= 0) zt = (float)z[id];
  Sums s{kNone, 0.0f, 0.0f};
  int most = 0;
  add_batch<kT>(b, a.c, s, most);
  while (b.next < p.end) {
    b.load(z, skew, b.next, p.end, a.d, lane);
    add_batch<kT>(b, a.c, s, most);
  }
  if ((kWhat & kTeach) && first) x.compare();
  const float m = s.m;
  const End e = end_of(group_sums<kLanes, kT>(s, a.c, sums_lds[group]));
  if (first) {
    if (kWhat & kTeach) {
      if (lane == 0) t.loss[row] = x.loss(e, a.scale);
    } else if (lane == 0) {
      score_row(o, row, id, zt, e, a.scale);
    }
  }
  if constexpr ((kWhat & kTop) != 0)
    top_of<T, kLanes>(p, o.k, lane, m, most, top_lds[group], [&](int r, uint64_t key) {
      put_top(o, row * o.k + r, key, e, a.scale);
    });
}

template <typename T, int kWhat>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, hipStream_t s) {
#define TOC_SCORE(L, K)                                                                          \
  hipLaunchKernelGGL((score_kernel<T, L, K, kWhat>),                                             \
                     grid_of<L>(a.n), dim3(kThreads<L>), 0, s, a, o, t)
  if (a.chunks <= 256) TOC_SCORE(64, 4);
  else if (a.chunks <= 2048) TOC_SCORE(256, 4);
  else if (a.n >= 512) TOC_SCORE(512, 6);
  else TOC_SCORE(1024, 4);
#undef TOC_SCORE
  return launched("score_kernel");
}

template <typename T>
toc_status score(const Rows<T> &a, const Score &o, hipStream_t s) {
  const Teacher t{};
  if (o.k) return o.entropy ? launch<T, kTop | kEntropy>(a, o, t, s) : launch<T, kTop>(a, o, t, s);
  return o.entropy ? launch<T, kEntropy>(a, o, t, s) : launch<T, 0>(a, o, t, s);
}

}  // namespace
}  // namespace logits
}  // namespace toc

using namespace toc;
using namespace toc::logits;

extern "C" {

toc_status toc_logits_workspace_size(int64_t n, int32_t d, int32_t k, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(TOC_EINVAL, "bytes is NULL");
  if (const toc_status st = check_sizes(n, d, TOC_F32)) return st;
  if (k < 0) return fail(TOC_EINVAL, "%d alternatives", k);
  if (k > kMaxTop) return fail(TOC_EUNSUPPORTED, "more than %d alternatives a row", kMaxTop);
  *bytes = 0;
  return TOC_OK;
}

toc_status toc_logprob(int64_t n, int32_t d, int32_t type, const void *Z, int64_t ldz, float scale,
                       const void *ids, int32_t id_bits, float *logp, float *lse, float *entropy,
                       int32_t k, void *top_ids, float *top_logp, void *ws, size_t ws_bytes,
                       void *stream) {
  size_t need = 0;
  toc_status st = toc_logits_workspace_size(n, d, k, &need);
  if (st || (st = check_logits(n, d, type, Z, ldz, scale)) ||
      (st = check_score(n, ids, id_bits, logp, lse, entropy)) ||
      (st = check_vec("top_logp", top_logp, n, k > 0)))
    return st;
  if (k > 0 && n > 0 && !top_ids) return fail(TOC_EINVAL, "top_ids is NULL");
  if ((uintptr_t)top_ids % (uintptr_t)(id_bits / 8))
    return fail(TOC_EINVAL, "top_ids is not aligned to its elements");
  if ((st = check_ws(ws, ws_bytes, need))) return st;
  if (n == 0) return TOC_OK;
  const Score o{Ids{ids, id_bits}, logp, lse, entropy, k, top_ids, top_logp};
  switch (type) {
    case TOC_F32: return score(rows_of<float>(n, d, Z, ldz, scale), o, (hipStream_t)stream);
    case TOC_BF16: return score(rows_of<bf16>(n, d, Z, ldz, scale), o, (hipStream_t)stream);
    default: return score(rows_of<f16>(n, d, Z, ldz, scale), o, (hipStream_t)stream);
  }
}

toc_status toc_distill(int64_t n, int32_t d, int32_t type, const void *Z, int64_t ldz, float scale,
                       int32_t k, const void *top_ids, int32_t id_bits, int64_t ldi, int32_t t_type,
                       const void *top_z, int64_t ldt, float top_scale, const float *top_lse, float *loss,
                       void *ws, size_t ws_bytes, void *stream) {
  size_t need = 0;
  toc_status st = toc_logits_workspace_size(n, d, 0, &need);
  if (st || (st = check_logits(n, d, type, Z, ldz, scale)) ||
      (st = check_teacher(n, type, k, top_ids, id_bits, ldi, t_type, top_z, ldt, top_scale, top_lse)) ||
      (st = check_vec("loss", loss, n, true)) || (st = check_ws(ws, ws_bytes, need)))
    return st;
  if (n == 0) return TOC_OK;
  const Teacher t{Ids{top_ids, id_bits}, ldi, k, t_type, top_z, ldt, top_scale, top_lse, loss};
  const Score o{};
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case TOC_F32: return launch<float, kTeach>(rows_of<float>(n, d, Z, ldz, scale), o, t, s);
    case TOC_BF16: return launch<bf16, kTeach>(rows_of<bf16>(n, d, Z, ldz, scale), o, t, s);
    default: return launch<f16, kTeach>(rows_of<f16>(n, d, Z, ldz, scale), o, t, s);
  }
}

}  // extern "C"
