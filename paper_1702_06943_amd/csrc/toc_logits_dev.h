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

// Over kLanes lanes (a wave or its rows of 16), the same in all of them: by shifts within rows of 16
// lanes and broadcasts of their last ones, each one operation on the way into the adder (lanes
// without a source take the operation's neutral number); the last lane has the result.
template <int kLanes = 64, typename Op>
__device__ inline uint32_t wave_all(uint32_t x, uint32_t neutral, Op op) {
#define TOC_STEP(ctrl, rows) \
  x = op(x, (uint32_t)__builtin_amdgcn_update_dpp((int)neutral, (int)x, ctrl, rows, 0xf, false))
  TOC_STEP(0x111, 0xf);   // from 1, 2, 4, 8 lanes below
  TOC_STEP(0x112, 0xf);
  TOC_STEP(0x114, 0xf);
  TOC_STEP(0x118, 0xf);
  if (kLanes == 16) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x15f, 0xf, 0xf, false);   // lane 15
  TOC_STEP(0x142, 0xa);   // lane 15 of a row to the next, rows 1 and 3
  TOC_STEP(0x143, 0xc);   // lane 31 to rows 2 and 3
#undef TOC_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ inline uint32_t wave_min(uint32_t x) {
  return wave_all(x, ~0u, [](uint32_t a, uint32_t b) { return min(a, b); });
}
__device__ inline uint32_t wave_max(uint32_t x) {
  return wave_all(x, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ inline uint32_t wave_or(uint32_t x) {
  return wave_all(x, 0u, [](uint32_t a, uint32_t b) { return a | b; });
}
template <int kLanes = 64>
__device__ inline float wave_sum(float x) {
  return __uint_as_float(wave_all<kLanes>(__float_as_uint(x), 0u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
template <int kLanes = 64>
__device__ inline float wave_max(float x) {
  return __uint_as_float(wave_all<kLanes>(__float_as_uint(x), __float_as_uint(kNone), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}

template <bool kT, int kLanes = 64>
__device__ inline Sums wave_sums(Sums a, float c) {
  const float m = wave_max<kLanes>(a.m);
  a = moved<kT>(a, from(m), c);
  return Sums{m, wave_sum<kLanes>(a.s), kT ? wave_sum<kLanes>(a.t) : 0.0f};
}
// The sums of a group of kLanes lanes (16 or 64: of a wave; else the whole workgroup, by way of
// kLanes / 64 words of lds, which are free again after the caller's next barrier).
template <int kLanes, bool kT>
__device__ inline Sums group_sums(Sums a, float c, Sums *lds) {
  a = wave_sums<kT, kLanes == 16 ? 16 : 64>(a, c);
  if (kLanes <= 64) return a;
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = a;
  __syncthreads();
  // every wave's sums again by all waves, one in a lane
  const int lane = (int)threadIdx.x % 64;
  a = Sums{kNone, 0.0f, 0.0f};
  if (lane < kLanes / 64) a = lds[lane];
  return wave_sums<kT>(a, c);
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

// Rows start at any multiple of their elements' size, but loads and stores of 16 bytes are at their
// best at multiples of 16 (8,192 x 32,767 bf16, whose rows start at odd multiples of 2: gradient
// 191 us, 235 with chunks that start where rows do).  So a row's chunks are those of memory: its
// first one starts `skew` columns before the row (nothing is read there: the row's first 16 bytes
// are, and shifted).  Rows too short to gain have skew 0, and those of less than a wave, whose
// chunks would not be alike then.
template <int kLanes, typename T>
__device__ inline int skew_of(const T *z, int d) {
  constexpr int N = kCols<T>;
  return kLanes < 64 || d < 2 * N ? 0 : (int)((uintptr_t)z / sizeof(T) % N);
}
template <typename T>
__device__ inline int chunks_in(int d, int skew) {
  return (d + skew + kCols<T> - 1) / kCols<T>;
}

// A chunk of T, minus infinity but for its columns low .. left - 1.
template <typename T>
__device__ inline Chunk cut(Chunk x, int low, int left) {
  constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80u : 0xfc00u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      x[i] = i >= low && i < left ? x[i] : none;
    } else {
      const uint32_t first = 2 * i >= low && 2 * i < left ? x[i] & 0xffffu : none;
      const uint32_t second = 2 * i + 1 >= low && 2 * i + 1 < left ? x[i] & 0xffff0000u : none << 16;
      x[i] = first | second;
    }
  }
  return x;
}

// A chunk moved up by 0 < by < kCols columns.
template <typename T>
__device__ inline Chunk raise(Chunk c, int by) {
  const int bits = by * 8 * (int)sizeof(T);
  if (bits & 64) c = Chunk{0u, 0u, c[0], c[1]};
  if (bits & 32) c = Chunk{0u, c[0], c[1], c[2]};
  if (sizeof(T) == 2 && (bits & 16))
    c = Chunk{c[0] << 16, c[1] << 16 | c[0] >> 16, c[2] << 16 | c[1] >> 16, c[3] << 16 | c[2] >> 16};
  return c;
}

// A chunk whose first column is `at` (below 0 in a skewed row's first) of a row of d columns: minus
// infinity before the row's first column and from stop <= d on.
template <typename T>
__device__ inline Chunk edge_chunk(const T *row, int at, int stop, int d) {
  const Place<T, true> l = place<T, true>(max(at, 0), d);
  Chunk c = settle(fetch(row, l), l);
  if (at < 0) c = raise<T>(c, -at);
  return cut<T>(c, -at, stop - at);
}

// The columns low .. left - 1 of a chunk to p and on.
template <typename T>
__device__ inline void put_some(T *p, int low, int left, Chunk c) {
#pragma unroll
  for (int i = 0; i < kCols<T>; ++i) {
    if (i < low || i >= left) continue;
    if (sizeof(T) == 4) ((uint32_t *)p)[i] = c[i];
    else ((uint16_t *)p)[i] = (uint16_t)(c[i / 2] >> (16 * (i % 2)));
  }
}

// Chunks q .. end - 1 of a row of d columns, or as many of them as a batch takes, as they lie in
// memory: up to kPer rows of kLanes whole chunks, lane i's the i-th of each, and what is left
// after them where that is less than such a row (`edge`: minus infinity past the row's end and in
// chunks from `end` on).  All loads are asked for before any is used.  What is the same in all
// lanes (the row, q, end, d) is in scalar registers, and a lane's offset is one vector register
// for all its loads.
template <typename T, int kLanes, int kPer>
struct Batch {
  static constexpr int N = kCols<T>;
  Chunk in[kPer], edge;
  int q, rows, next, lane;        // first chunk, rows of whole chunks, first chunk after the batch
  int skew, end;
  bool ragged;                    // whether the lane's wave has a part of an edge

  __device__ inline int column(int k) const { return N * (q + k * kLanes + lane) - skew; }

  __device__ inline void load(const T *row, int skew_, int q_, int end_, int d, int lane_) {
    q = q_;
    end = end_;
    lane = lane_;
    skew = skew_;
    const int whole = min(end, (d + skew) / N);
    rows = min(kPer, (whole - q) / kLanes);
    next = q + rows * kLanes;
    const bool last = whole - next < kLanes;
    const int wave = next + __builtin_amdgcn_readfirstlane(lane);
    ragged = last && wave < end;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      uint32_t at = (uint32_t)(16 * lane);
      if (k == 0 && q == 0 && lane == 0) at = (uint32_t)skew * (uint32_t)sizeof(T);
      if (k < rows) in[k] = *(const Unaligned *)((const char *)(row + (N * (q + k * kLanes) - skew)) + at);
    }
    if (ragged) {
      const int at = N * (next + lane) - skew;
      // (a wave whose chunks are all whole reads them as they are)
      if (wave > 0 && wave + (kLanes < 64 ? kLanes : 64) <= whole) edge = *(const Unaligned *)(row + at);
      else edge = edge_chunk(row, at, min(d, N * end - skew), d);
    }
    if (last) next = end;
  }
  // Puts a skewed row's first chunk right, before its first use.
  __device__ inline void trim() {
    if (q == 0 && skew > 0 && rows > 0 && lane == 0) in[0] = cut<T>(raise<T>(in[0], skew), skew, N);
  }
  // Keeps the compiler from holding the widened numbers, at twice the registers, from one pass over
  // the batch to the next.
  __device__ inline void again() {
    if (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) asm volatile("" : "+v"(in[k]));
    }
  }
  // f(k, chunk) for each of a lane's chunks; the scheduler keeps them apart, so that one chunk's
  // numbers at a time are in registers.
  template <typename F>
  __device__ inline void each(F f) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (k < rows) f(k, in[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (ragged) f(rows, edge);
  }
};

// A lane's sums with its batch's numbers added; most: the first column of the first chunk that
// holds its largest logit.
template <bool kT, typename T, int kLanes, int kPer>
__device__ inline void add_batch(Batch<T, kLanes, kPer> &b, float c, Sums &a, int &most) {
  constexpr int N = kCols<T>;
  float m = a.m;
  b.trim();
  b.each([&](int k, Chunk in) {
    float v[N];
    widen<T>(in, v);
    float x = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) x = fmaxf(x, v[i]);
    if (x > m) most = b.column(k);
    m = fmaxf(m, x);
  });
  const float base = from(m);
  a = moved<kT>(a, base, c);
  a.m = m;
  b.again();
  b.each([&](int, Chunk in) {
    float v[N];
    widen<T>(in, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = (v[i] - base) * c, e = two_to(y);
      a.s += e;
      if (kT) a.t = fmaf(e, fmaxf(y, kFar), a.t);
    }
  });
}

// Workgroups of kBlock threads, or kLanes where those are more; a group of kLanes lanes has one row.
// (Without a loop over rows: hoisted out of one, constants took some thirty registers a lane.)
template <int kLanes>
constexpr int kThreads = kLanes > kBlock ? kLanes : kBlock;
template <int kLanes>
inline dim3 grid_of(int64_t rows) {
  const int64_t blocks = (rows + kThreads<kLanes> / kLanes - 1) / (kThreads<kLanes> / kLanes);
  const int64_t wide = std::min<int64_t>(blocks, 1 << 20);
  return dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}
// From so many short rows on 16 lanes have one.
constexpr uint32_t kShortRows = 4096;
// A thread's group of the workgroup, its row, both the same in all lanes of a wave, and its lane.
template <int kLanes>
__device__ inline int group_of() {
  const int group = (int)threadIdx.x / kLanes;
  return kLanes >= kBlock ? 0 : kLanes == 64 ? __builtin_amdgcn_readfirstlane(group) : group;
}
template <int kLanes>
__device__ inline int64_t row_of() {
  return ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads<kLanes> / kLanes) + group_of<kLanes>();
}
template <int kLanes>
__device__ inline int lane_of() {
  return kLanes >= kBlock ? (int)threadIdx.x : (int)threadIdx.x % kLanes;
}

// --- a row's end -----------------------------------------------------------------

// The scale of the logits.  Two logits' difference, up to twice the largest number, may overflow where
// scale times it, or times a small share of it, does not: a quarter of it is formed (a sum of shares that rounds to
// more than 1 times a half would overflow too) and multiplied by four times the scale, both exact.
// (From a scale of 2^100 on, four times which may overflow, the whole: a share below 2^-100 would be
// needed there.)
struct Scale {
  float whole, part, by;   // whole = part by
  __device__ inline float apart(float z, float from) const { return fmaf(part, z, -part * from); }
};
inline Scale scale_of(float scale) {
  return scale < 0x1p100f ? Scale{scale, 0.25f, 4.0f * scale} : Scale{scale, 1.0f, scale};
}

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
__device__ inline float log_p(float z, const End &e, const Scale &scale) {
  return e.empty ? kNone : fmaf(scale.by, scale.apart(z, e.m), -e.log_s);
}
__device__ inline float entropy(const End &e) { return e.empty ? 0.0f : e.log_s - e.t_s; }
__device__ inline float log_sum(const End &e, const Scale &scale) {
  return e.empty ? kNone : fmaf(scale.whole, e.m, e.log_s);
}

struct Ids {
  const void *p;   // or NULL: no token anywhere
  int bits;
};
// A token number as it is loaded, so that the loads after it do not wait for it; -1 is no token.
struct RawId {
  uint32_t low, high;
};
// The token, or -1 where it is none of 0..d-1.
__device__ inline int token_of(RawId r, int bits, int d) {
  const int64_t id = bits == 32 ? (int64_t)(int32_t)r.low : (int64_t)((uint64_t)r.high << 32 | r.low);
  return id >= 0 && id < d ? (int)id : -1;
}
// p[i] for an i that is the same in all lanes of a wave, by a scalar load, which no wait for a row's
// loads holds up; what it reads is written by no launch that it runs in.
template <typename V>
__device__ inline V scalar(const V *p, int64_t i) {
  return *(const __attribute__((address_space(4))) V *)(p + i);
}
// A row's number: a scalar load where all lanes of a wave have the same row.
template <int kLanes, typename V>
__device__ inline V of_row(const V *p, int64_t i) {
  if constexpr (kLanes >= 64) return scalar(p, i);
  else return p[i];
}
template <int kLanes>
__device__ inline RawId id_of_row(const Ids &ids, int64_t i) {
  RawId r{~0u, ~0u};
  if (!ids.p) return r;
  if (ids.bits == 32) {
    r.low = of_row<kLanes>((const uint32_t *)ids.p, i);
  } else {
    r.low = of_row<kLanes>((const uint32_t *)ids.p, 2 * i);
    r.high = of_row<kLanes>((const uint32_t *)ids.p, 2 * i + 1);
  }
  return r;
}

// --- arguments -------------------------------------------------------------------

template <typename T>
struct Rows {
  uint32_t n;
  int d;
  const T *Z;
  int64_t ldz;
  Scale scale;
  float c;             // scale log2(e)
  int chunks;          // of a row that is not skewed
};
template <typename T>
Rows<T> rows_of(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale) {
  return Rows<T>{(uint32_t)n, d, (const T *)Z, ldz, scale_of(scale), scale * kLog2e, (int)chunks_of<T>(d)};
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
__device__ inline void score_row(const Score &a, int64_t row, int id, float z, const End &e, const Scale &scale) {
  if (a.logp) a.logp[row] = id < 0 ? 0.0f : log_p(z, e, scale);
  if (a.lse) a.lse[row] = log_sum(e, scale);
  if (a.entropy) a.entropy[row] = entropy(e);
}

// A teacher's row, by the first wave of a group while the others go on with theirs: a lane's entries
// are lane, lane + 64 and so on.  The loss is
//   sum q log q - sum q log p = sum q log q - scale (sum q (z - r) + (r - m) sum q) + log S sum q
// with r the largest logit of the row at an entry's column: what the entries give is known before the
// row's own sums are.  Both differences are Scale's.
struct Taught {
  static constexpr int kPer = kMaxTeacher / 64;
  int id[kPer];        // -1: none
  float t[kPer];       // saved logit
  float z[kPer];       // the row's own logit there
  float q[kPer];
  float sum, sum_log;  // of q and of q log q over the row
  float r, sum_z;      // r, and the sum of q (z - r), a part of it

  // The columns and the saved logits as they lie in memory.
  struct Raw {
    RawId id[kPer];
    uint32_t t[kPer];
  };
  __device__ static inline Raw ask(const Teacher &a, int64_t row, int lane) {
    Raw raw;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      raw.id[i] = RawId{~0u, ~0u};
      raw.t[i] = 0;
      const int e = lane + 64 * i;
      if (64 * i >= a.k || e >= a.k) continue;
      const int64_t at = row * a.ldi + e, to = row * a.ldt + e;
      if (a.ids.bits == 32) {
        raw.id[i].low = ((const uint32_t *)a.ids.p)[at];
      } else {
        const uint2 v = ((const uint2 *)a.ids.p)[at];
        raw.id[i] = RawId{v.x, v.y};
      }
      raw.t[i] = a.type == TOC_F32 ? ((const uint32_t *)a.t)[to] : (uint32_t)((const uint16_t *)a.t)[to];
    }
    return raw;
  }
  __device__ inline void read(const Teacher &a, const Raw &raw, int d) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      id[i] = token_of(raw.id[i], a.ids.bits, d);
      t[i] = a.type == TOC_F32 ? __uint_as_float(raw.t[i])
             : a.type == TOC_BF16 ? __uint_as_float(raw.t[i] << 16)
                                  : (float)__builtin_bit_cast(f16, (uint16_t)raw.t[i]);
    }
  }
  template <typename T>
  __device__ inline void gather(const Teacher &a, const T *row) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      z[i] = kNone;
      if (64 * i < a.k && id[i] >= 0) z[i] = (float)row[id[i]];
    }
  }
  // The teacher's probabilities: q_a = exp(scale T_a - lse), or exp(scale (T_a - max T)) over its sum
  // without lse.  An entry that is none has q = 0.
  __device__ inline void learn(const Teacher &a, int64_t row) {
    float log_sum;
    if (a.lse) {
      log_sum = scalar(a.lse, row);
#pragma unroll
      for (int i = 0; i < kPer; ++i) t[i] = id[i] < 0 ? kNone : fmaf(a.scale, t[i], -log_sum);
    } else {
      float most = kNone;
#pragma unroll
      for (int i = 0; i < kPer; ++i) most = fmaxf(most, id[i] < 0 ? kNone : t[i]);
      most = from(wave_max(most));
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        t[i] = id[i] < 0 ? kNone : a.scale * (t[i] - most);
        if (64 * i < a.k) s += expf(t[i]);
      }
      s = wave_sum(s);
      log_sum = logf(s);
      // (no saved logit above minus infinity: s is 0, every q 0)
#pragma unroll
      for (int i = 0; i < kPer; ++i) t[i] = s == 0.0f ? kNone : t[i] - log_sum;
    }
    sum = sum_log = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      q[i] = 0.0f;
      if (64 * i >= a.k) continue;
      q[i] = expf(t[i]);
      sum += q[i];
      if (q[i] != 0.0f) sum_log = fmaf(q[i], t[i], sum_log);
    }
    sum = wave_sum(sum);
    sum_log = wave_sum(sum_log);
  }
  // An entry with q = 0 adds nothing.  (Where entries of a column were put together, the same.)
  __device__ inline void compare(const Scale &scale) {
    r = kNone;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (q[i] != 0.0f) r = fmaxf(r, z[i]);
    r = from(wave_max(r));
    sum_z = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (q[i] != 0.0f) sum_z = fmaf(q[i], scale.apart(z[i], r), sum_z);
    sum_z = wave_sum(sum_z);
  }
  __device__ inline float loss(const End &e, const Scale &scale) const {
    if (sum == 0.0f) return 0.0f;
    if (e.empty) return INFINITY;
    return sum_log - scale.by * fmaf(scale.apart(r, e.m), sum, sum_z) + e.log_s * sum;
  }
};

// --- few long rows ---------------------------------------------------------------

// A row dealt out to `parts` workgroups, `per` chunks to each: their sums (and their largest keys) are
// left in the workspace and put together by a second launch.
struct Split {
  int parts, per;
  Sums *sums;          // n x parts
  uint64_t *keys;      // n x parts x alternatives
};
constexpr int kMaxParts = 64;              // a wave puts them together
constexpr int64_t kMaxPieces = 512;        // rows times parts, where there are parts
constexpr int kPartLanes = 512, kPartPer = 6;

// A row's part of a workgroup of the launches over parts.
struct Piece {
  int64_t row;
  int part, q0, end;
};
__device__ inline Piece piece_of(const Split &s, int chunks) {
  Piece p;
  p.row = (int64_t)(blockIdx.x / (uint32_t)s.parts);
  p.part = (int)(blockIdx.x % (uint32_t)s.parts);
  p.q0 = min(p.part * s.per, chunks);
  p.end = min(p.q0 + s.per, chunks);
  return p;
}
// A whole row's sums from its parts', in every wave.
template <bool kT>
__device__ inline Sums parts_sums(const Split &s, int64_t row, float c) {
  const int lane = (int)threadIdx.x % 64;
  Sums a{kNone, 0.0f, 0.0f};
  if (lane < s.parts) a = s.sums[row * s.parts + lane];
  return wave_sums<kT>(a, c);
}

// The split of n rows of `chunks` chunks, k alternatives, into parts of 1,024 chunks or more; 1
// where rows are short or enough (us):
//   log p     1 x 262,144 f32     whole 17.9   in parts 5.2
//            64 x 262,144 bf16    whole 18.3   in parts 10.3
//            16 x 47,236 bf16     whole 6.1    in parts 6.7
//           200 x 100,000 bf16    whole 10.2   in parts 12.8
//   gradient  1 x 100,000 bf16    whole 13.3   in parts 8.7
//            64 x 65,536 bf16     whole 10.1   in parts 11.5
// The limit of 128 rows goes by the last of log p.  On either side of it, 127 rows in parts and 128 whole:
// log p of 262,144 bf16 18.6, 20.2, of 1,048,576 50, 65; gradient 37.7, 39.7, 131, 146: rows as
// long as these would gain from parts beyond it too.
// Alternatives are looked for in each part, so parts are of 2,048 chunks then, and at most 256 keys come
// together (9 x 88,832 f16, parts of 1,024, 2,048 and 4,096 chunks and whole: 3 alternatives 9.5, 9.5,
// 11.3, 11.6; 20 alternatives 13.3, 12.7, 13.6, 12.9).
inline int parts_of(int64_t n, int64_t chunks, int k) {
  if (n >= 128 || chunks <= 8192) return 1;
  const int64_t most = k ? std::min(chunks / 2048, (int64_t)256 / k) : chunks / 1024;
  return (int)std::max<int64_t>(1, std::min({most, (int64_t)kMaxParts, kMaxPieces / n}));
}
inline Split split_of(int64_t n, int64_t chunks, int k, void *ws) {
  Split s{};
  s.parts = n ? parts_of(n, chunks, k) : 1;
  // (a skewed row has a chunk more)
  s.per = (int)((chunks + 1 + s.parts - 1) / s.parts);
  s.keys = (uint64_t *)ws;
  s.sums = (Sums *)(s.keys + n * s.parts * k);
  return s;
}
// Sums of parts for the gradients, and what is made of a row's parts, in toc_logits.hip.
template <typename T>
toc_status add_parts(const Rows<T> &a, int k, bool entropy, const Split &s, hipStream_t stream);
template <typename T>
toc_status join_parts(const Rows<T> &a, const Score &o, const Teacher &t, const Split &s, hipStream_t stream);

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
