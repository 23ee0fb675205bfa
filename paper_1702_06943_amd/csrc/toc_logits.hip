// Log probabilities of given tokens with the rows' entropy and most probable tokens, and the
// distance of rows from a teacher's saved logits: one softmax over each row of n x d logits.
//   p_j = exp(scale (z_j - m)) / S      S = sum_j exp(scale (z_j - m))      m = max_j z_j
//   logp = log p_t      H = log S - sum_j p_j scale (z_j - m)      loss = sum_a q_a (log q_a - log p_{i_a})
#include "toc_logits_dev.h"

namespace toc {
namespace logits {
namespace {

constexpr int kEntropy = 1, kTop = 2, kTeach = 4;   // what a kernel is asked for

// The sums of a lane's chunks: the row's chunks are dealt out to the group's lanes in turn.
template <typename T, int kLanes, bool kT>
__device__ inline Sums lane_sums(const T *row, int d, int lane, float c) {
  constexpr int N = kCols<T>;
  Sums a{kNone, 0.0f, 0.0f};
  for (int at = N * lane; at < d; at += N * kLanes) {
    const Place<T, true> l = place<T, true>(at, d);
    float v[N];
    widen_row<T>(settle(fetch(row, l), l), at, d, v);
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, v[i]);
    const float base = from(m);
    a = moved<kT>(a, base, c);
    a.m = m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = (v[i] - base) * c, e = two_to(y);
      a.s += e;
      if (kT) a.t = fmaf(e, fmaxf(y, kFar), a.t);
    }
  }
  return a;
}

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

// The alternatives by k searches of the row for the largest key below the last.
template <typename T, int kLanes>
__device__ inline void top_rounds(const Rows<T> &a, const Score &o, uint32_t row, int lane, const End &e,
                                  uint64_t *lds) {
  constexpr int N = kCols<T>;
  const T *z = a.Z + (int64_t)row * a.ldz;
  uint64_t last = ~(uint64_t)0;
  for (int r = 0; r < o.k; ++r) {
    uint64_t best = 0;
    if (last) {
      for (int at = N * lane; at < a.d; at += N * kLanes) {
        const Place<T, true> l = place<T, true>(at, a.d);
        float v[N];
        widen_row<T>(settle(fetch(z, l), l), at, a.d, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint64_t key = key_of(v[i], at + i);
          if (key < last && key > best) best = key;
        }
      }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) {
      const uint64_t other = __shfl_xor((unsigned long long)best, x, 64);
      best = other > best ? other : best;
    }
    if (kLanes > 64) {
      __syncthreads();
      if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = best;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kLanes / 64; ++i) best = lds[i] > best ? lds[i] : best;
    }
    if (lane == 0) put_top(o, (int64_t)row * o.k + r, best, e, a.scale);
    last = best;
  }
}

template <typename T, int kLanes, int kWhat>
__global__ __launch_bounds__(kBlock) void score_kernel(Rows<T> a, Score o, Teacher t) {
  __shared__ Sums sums[kLanes / 64];
  __shared__ float teach_lds[kLanes / 64 * 4];
  __shared__ uint64_t keys[kLanes / 64];
  const int lane = threadIdx.x;
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T *z = a.Z + (int64_t)row * a.ldz;
    __syncthreads();
    if (kWhat & kTeach) {
      const Taught<kLanes> x = teach<T, kLanes>(t, row, z, a.d, lane, teach_lds);
      const End e = end_of(group_sums<kLanes, false>(lane_sums<T, kLanes, false>(z, a.d, lane, a.c), a.c, sums));
      const float loss = taught_loss<kLanes>(x, e, a.scale, teach_lds + 3 * (kLanes / 64));
      if (lane == 0) t.loss[row] = loss;
      continue;
    }
    constexpr bool kT = kWhat & kEntropy;
    const End e = end_of(group_sums<kLanes, kT>(lane_sums<T, kLanes, kT>(z, a.d, lane, a.c), a.c, sums));
    if (lane == 0) {
      const int id = token(o.ids, row, a.d);
      score_row(o, row, id, id < 0 ? 0.0f : (float)z[id], e, a.scale);
    }
    if (kWhat & kTop) top_rounds<T, kLanes>(a, o, row, lane, e, keys);
  }
}

template <typename T, int kWhat>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20));
  hipLaunchKernelGGL((score_kernel<T, kBlock, kWhat>), grid, dim3(kBlock), 0, s, a, o, t);
  return launched("score_kernel");
}

template <typename T>
toc_status score(const Rows<T> &a, const Score &o, hipStream_t s) {
  const Teacher t{};
  if (o.k) return o.entropy ? launch<T, kTop | kEntropy>(a, o, t, s) : launch<T, kTop>(a, o, t, s);
  return o.entropy ? launch<T, kEntropy>(a, o, t, s) : launch<T, 0>(a, o, t, s);
}

template <typename T>
Rows<T> rows_of(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale) {
  return Rows<T>{(uint32_t)n, d, (const T *)Z, ldz, scale, scale * kLog2e};
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
