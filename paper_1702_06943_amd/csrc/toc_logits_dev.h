// What the operators on rows of logits share (log probabilities of given tokens, distillation
// from a teacher's top logits, and their gradients): the sums of a softmax over a long row,
// what is made of them at the row's end, and the checks of the arguments.
#pragma once

#include "toc_rows_dev.h"

namespace toc {
namespace logits {

using namespace rows;

constexpr int kMaxTop = 64;        // alternatives of a row
constexpr int kMaxTeacher = 256;   // saved logits of a teacher's row
constexpr int kBlock = 256;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kNone = -INFINITY;
// Exponents below this count as this: their power of two is 0 in binary32 all the same, and
// minus infinity times that 0 would be NaN.
constexpr float kFar = -200.0f;

// --- a row's sums --------------------------------------------------------------

// Of some columns of a row: the largest logit m, and with y = scale log2(e) (z - m) the sums
// s of 2^y and t of 2^y y.  The difference comes first and is then scaled: scale z itself
// would be off by 2^-24 of its own size, and an overflow of scale z cannot happen.  No columns,
// or none above minus infinity: m is that, s and t are 0.  A NaN or +infinity makes s NaN.
struct Sums {
  float m, s, t;
};

__device__ inline float two_to(float y) { return __builtin_amdgcn_exp2f(y); }
// What logits are measured from: 0 where all of them are minus infinity.
__device__ inline float from(float m) { return m == kNone ? 0.0f : m; }

// The sums as they are measured from base instead of a.m <= base.
template <bool kT>
__device__ inline Sums moved(Sums a, float base, float c) {
  const float y = fmaxf((a.m - base) * c, kFar), f = two_to(y);
  return Sums{base, a.s * f, kT ? fmaf(a.s, y, a.t) * f : 0.0f};
}

// The sums of a group of kLanes lanes (64: a wave; else the whole workgroup, by way of
// kLanes / 64 words of lds, which are free again after the caller's next barrier).
template <int kLanes, bool kT>
__device__ inline Sums group_sums(Sums a, float c, Sums *lds) {
  float m = a.m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  Sums w = moved<kT>(a, from(m), c);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    w.s += __shfl_xor(w.s, o, 64);
    if (kT) w.t += __shfl_xor(w.t, o, 64);
  }
  w.m = m;
  if (kLanes == 64) return w;
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = w;
  __syncthreads();
  m = lds[0].m;
#pragma unroll
  for (int i = 1; i < kLanes / 64; ++i) m = fmaxf(m, lds[i].m);
  Sums all{m, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kLanes / 64; ++i) {
    const Sums x = moved<kT>(lds[i], from(m), c);
    all.s += x.s;
    if (kT) all.t += x.t;
  }
  return all;
}

// What a group's lanes wrote to LDS is there for all of them.
template <int kLanes>
__device__ inline void group_sync() {
  if (kLanes > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// --- a row's columns -------------------------------------------------------------

// Up to kPer chunks of a lane of a group, of the chunks q .. end - 1 of a row of d columns: lane i
// holds chunks q + i, q + i + kLanes and so on, as they lie in memory.  All loads are asked for
// before any is used.
template <typename T, int kLanes, int kPer>
struct Batch {
  static constexpr int N = kCols<T>;
  Chunk in[kPer];
  int q, end, d, lane;

  // Whether any lane has a chunk k, and whether all have whole ones (the same in all lanes).
  __device__ inline bool any(int k) const { return q + k * kLanes < end; }
  __device__ inline bool whole(int k) const { return q + (k + 1) * kLanes <= min(end, d / N); }
  __device__ inline int column(int k) const { return N * (q + k * kLanes + lane); }

  __device__ inline void load(const T *row, int q_, int end_, int d_, int lane_) {
    q = q_;
    end = end_;
    d = d_;
    lane = lane_;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (!any(k)) continue;
      if (whole(k)) in[k] = *(const Unaligned *)(row + column(k));
      else in[k] = fetch(row, place<T, true>(column(k), d));
    }
  }
  // The numbers of chunk k: minus infinity past the row's end, and in a chunk past `end`.
  __device__ inline void numbers(int k, float (&v)[N]) const {
    if (whole(k)) {
      widen<T>(in[k], v);
      return;
    }
    const int at = column(k), stop = min(d, N * end);
    widen<T>(settle(in[k], place<T, true>(at, d)), v);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = at + i < stop ? v[i] : kNone;
  }
};

// A lane's sums with its batch's numbers added; most: the first column of the first chunk that
// holds its largest logit.
template <bool kT, typename T, int kLanes, int kPer>
__device__ inline void add_batch(const Batch<T, kLanes, kPer> &b, float c, Sums &a, int &most) {
  constexpr int N = kCols<T>;
  float m = a.m;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (!b.any(k)) continue;
    float v[N];
    b.numbers(k, v);
    float x = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) x = fmaxf(x, v[i]);
    if (x > m) most = b.column(k);
    m = fmaxf(m, x);
  }
  const float base = from(m);
  a = moved<kT>(a, base, c);
  a.m = m;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (!b.any(k)) continue;
    float v[N];
    b.numbers(k, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = (v[i] - base) * c, e = two_to(y);
      a.s += e;
      if (kT) a.t = fmaf(e, fmaxf(y, kFar), a.t);
    }
  }
}

// --- a row's end -----------------------------------------------------------------

// What follows from a whole row's sums.
struct End {
  float m, log_s, t_s;   // the largest logit, log s, ln 2 t / s
  bool empty;            // nothing above minus infinity: every probability is 0
};
__device__ inline End end_of(Sums a) {
  End e;
  e.m = a.m;
  e.empty = a.s == 0.0f;
  e.log_s = logf(a.s);
  e.t_s = e.empty ? 0.0f : kLn2 * a.t / a.s;
  return e;
}
__device__ inline float log_p(float z, const End &e, float scale) {
  return e.empty ? kNone : fmaf(scale, z - e.m, -e.log_s);
}
__device__ inline float entropy(const End &e) { return e.empty ? 0.0f : e.log_s - e.t_s; }
__device__ inline float log_sum(const End &e, float scale) {
  return e.empty ? kNone : fmaf(scale, e.m, e.log_s);
}

struct Ids {
  const void *p;   // or NULL: no token anywhere
  int bits;
};
// Token number i, or -1 where it is none of 0..d-1.
__device__ inline int token(const Ids &ids, int64_t i, int d) {
  if (!ids.p) return -1;
  const int64_t id = ids.bits == 32 ? (int64_t)((const int32_t *)ids.p)[i] : ((const int64_t *)ids.p)[i];
  return id >= 0 && id < d ? (int)id : -1;
}

// --- arguments -------------------------------------------------------------------

template <typename T>
struct Rows {
  uint32_t n;
  int d;
  const T *Z;
  int64_t ldz;
  float scale, c;      // c = scale log2(e)
  int chunks;          // of a row
};
template <typename T>
Rows<T> rows_of(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale) {
  return Rows<T>{(uint32_t)n, d, (const T *)Z, ldz, scale, scale * kLog2e, (int)chunks_of<T>(d)};
}

// Log probabilities: what is asked for, each but ids may be NULL.
struct Score {
  Ids ids;
  float *logp, *lse, *entropy;
  int k;               // alternatives, 0: none
  void *top_ids;
  float *top_logp;
};

// A teacher's saved logits, and the rows' losses or NULL.
struct Teacher {
  Ids ids;
  int64_t ldi;
  int k, type;
  const void *t;
  int64_t ldt;
  float scale;
  const float *lse;    // or NULL: the softmax of the saved ones
  float *loss;
};

// The numbers of a row's score, by one lane.  z: the given token's logit, if there is one.
__device__ inline void score_row(const Score &a, uint32_t row, int id, float z, const End &e, float scale) {
  if (a.logp) a.logp[row] = id < 0 ? 0.0f : log_p(z, e, scale);
  if (a.lse) a.lse[row] = log_sum(e, scale);
  if (a.entropy) a.entropy[row] = entropy(e);
}

// A lane's entries of a teacher's row: entry lane + i kLanes.
template <int kLanes>
struct Taught {
  static constexpr int kPer = (kMaxTeacher + kLanes - 1) / kLanes;
  int id[kPer];        // -1: none
  float t[kPer];       // scaled saved logit, then log q
  float z[kPer];       // the row's own logit there
  float q[kPer];
  float sum;           // of q over the row
};

template <int kLanes>
__device__ inline float lanes_sum(float x, float *lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  if (kLanes == 64) return x;
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
  __syncthreads();
  x = 0.0f;
#pragma unroll
  for (int i = 0; i < kLanes / 64; ++i) x += lds[i];
  return x;
}
template <int kLanes>
__device__ inline float lanes_max(float x, float *lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  if (kLanes == 64) return x;
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
  __syncthreads();
  x = lds[0];
#pragma unroll
  for (int i = 1; i < kLanes / 64; ++i) x = fmaxf(x, lds[i]);
  return x;
}

// Reads the entries and makes the teacher's probabilities:
//   q_a = exp(scale T_a - lse), or exp(scale (T_a - max T)) over its sum without lse
// lds: three times kLanes / 64 words, free again after the caller's next barrier.
template <typename T, int kLanes>
__device__ inline Taught<kLanes> teach(const Teacher &a, uint32_t row, const T *zrow, int d, int lane,
                                       float *lds) {
  Taught<kLanes> x;
  float most = kNone;
#pragma unroll
  for (int i = 0; i < x.kPer; ++i) {
    const int e = lane + i * kLanes;
    x.id[i] = -1;
    x.t[i] = kNone;
    x.z[i] = 0.0f;
    if (e < a.k) x.id[i] = token(a.ids, (int64_t)row * a.ldi + e, d);
    if (x.id[i] >= 0) {
      x.z[i] = (float)zrow[x.id[i]];
      const int64_t at = (int64_t)row * a.ldt + e;
      x.t[i] = a.type == TOC_F32 ? ((const float *)a.t)[at]
               : a.type == TOC_BF16 ? (float)((const bf16 *)a.t)[at] : (float)((const f16 *)a.t)[at];
    }
    most = fmaxf(most, x.t[i]);
  }
  float sum = 0.0f, log_sum;
  if (a.lse) {
    log_sum = a.lse[row];
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) x.t[i] = x.id[i] < 0 ? kNone : fmaf(a.scale, x.t[i], -log_sum);
  } else {
    most = from(lanes_max<kLanes>(most, lds));
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) {
      x.t[i] = x.id[i] < 0 ? kNone : a.scale * (x.t[i] - most);
      sum += expf(x.t[i]);
    }
    sum = lanes_sum<kLanes>(sum, lds + kLanes / 64);
    log_sum = logf(sum);
    // (no saved logit above minus infinity: sum is 0, every q 0)
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) x.t[i] = sum == 0.0f ? kNone : x.t[i] - log_sum;
  }
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < x.kPer; ++i) {
    x.q[i] = x.id[i] < 0 ? 0.0f : expf(x.t[i]);
    sum += x.q[i];
  }
  x.sum = lanes_sum<kLanes>(sum, lds + 2 * (kLanes / 64));
  return x;
}

// The row's loss, in every lane: sum of q (log q - log p); an entry with q = 0 adds nothing.
template <int kLanes>
__device__ inline float taught_loss(const Taught<kLanes> &x, const End &e, float scale, float *lds) {
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < x.kPer; ++i)
    if (x.q[i] != 0.0f) sum = fmaf(x.q[i], x.t[i] - log_p(x.z[i], e, scale), sum);
  return lanes_sum<kLanes>(sum, lds);
}

// --- checks ------------------------------------------------------------------------

inline toc_status check_vec(const char *name, const void *p, int64_t n, bool needed) {
  if (needed && n > 0 && !p) return fail(TOC_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % 4) return fail(TOC_EINVAL, "%s is not aligned to its elements", name);
  return TOC_OK;
}

inline toc_status check_logits(int64_t n, int32_t d, int32_t type, const void *Z, int64_t ldz, float scale) {
  toc_status st;
  if ((st = check_sizes(n, d, type)) || (st = check_rows("Z", Z, n, d, ldz, type_size(type)))) return st;
  if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e))
    return fail(TOC_EINVAL, "scale must be positive, and finite times log2(e)");
  return TOC_OK;
}

inline toc_status check_score(int64_t n, const void *ids, int32_t id_bits, const float *logp,
                              const float *lse, const float *entropy) {
  toc_status st;
  if (id_bits != 32 && id_bits != 64)
    return fail(TOC_EINVAL, "token numbers have 32 or 64 bits, not %d", id_bits);
  if (logp && !ids && n > 0) return fail(TOC_EINVAL, "logp without ids");
  if ((uintptr_t)ids % (uintptr_t)(id_bits / 8)) return fail(TOC_EINVAL, "ids is not aligned to its elements");
  if ((st = check_vec("logp", logp, n, false)) || (st = check_vec("lse", lse, n, false)) ||
      (st = check_vec("entropy", entropy, n, false)))
    return st;
  return TOC_OK;
}

inline toc_status check_teacher(int64_t n, int32_t type, int32_t k, const void *ids, int32_t id_bits,
                                int64_t ldi, int32_t t_type, const void *t, int64_t ldt, float t_scale,
                                const float *t_lse) {
  toc_status st;
  if (k < 1) return fail(TOC_EINVAL, "%d saved logits", k);
  if (k > kMaxTeacher) return fail(TOC_EUNSUPPORTED, "more than %d saved logits a row", kMaxTeacher);
  if (id_bits != 32 && id_bits != 64)
    return fail(TOC_EINVAL, "token numbers have 32 or 64 bits, not %d", id_bits);
  if (t_type != type && t_type != TOC_F32)
    return fail(TOC_EINVAL, "the saved logits' type is the rows' or TOC_F32, not %d", t_type);
  if ((st = check_rows("top_ids", ids, n, k, ldi, id_bits / 8)) ||
      (st = check_rows("top_z", t, n, k, ldt, type_size(t_type))) ||
      (st = check_vec("top_lse", t_lse, n, false)))
    return st;
  if (!(t_scale > 0.0f) || !std::isfinite(t_scale))
    return fail(TOC_EINVAL, "top_scale must be positive and finite");
  return TOC_OK;
}

inline toc_status check_ws(const void *ws, size_t ws_bytes, size_t need) {
  if (need && !ws) return fail(TOC_EINVAL, "workspace is NULL");
  if (ws_bytes < need) return fail(TOC_ESIZE, "workspace of %zu bytes below the %zu needed", ws_bytes, need);
  if ((uintptr_t)ws % 16) return fail(TOC_EINVAL, "workspace is not 16-byte aligned");
  return TOC_OK;
}

}  // namespace logits
}  // namespace toc
