// Log probabilities of given tokens with the rows' entropy and most probable tokens, and the
// distance of rows from a teacher's saved logits: one softmax over each row of n x d logits.
//   p_j = exp(scale (z_j - m)) / S      S = sum_j exp(scale (z_j - m))      m = max_j z_j
//   logp = log p_t      H = log S - sum_j p_j scale (z_j - m)      loss = sum_a q_a (log q_a - log p_{i_a})
// One pass: a lane keeps the sums of its chunks relative to its largest logit so far, lanes, waves and
// parts are put together with the same step.
//   score_kernel  bound by memory where rows are many: 8,192 x 47,236 bf16 131 us, 5.9 TB/s, with
//                 entropy and distance from 64 saved logits alike; with 20 alternatives 152 us.  One row 5.1
//                 us, with 5 alternatives 8.0: the look for them takes some 2.9 us.  18,750 x 900
//                 f16 9.8 us, 3.5 TB/s, bound by a short row's own instructions.
//   part_kernel, join_kernel  few long rows: one of 262,144 f32 5.2 us, 64 of bf16 10.4
#include "toc_logits_dev.h"

namespace toc {
namespace logits {
namespace {

constexpr int kEntropy = 1, kTop = 2, kTeach = 4;   // what a kernel is asked for

// Logits in the order that the alternatives have them: the larger first, of equal ones the
// lower column.  A key is never 0 for a column above minus infinity; a NaN has none.
__device__ inline uint64_t key_of(float z, int column) {
  const uint32_t b = __float_as_uint(z + 0.0f);   // (-0 as 0)
  const uint32_t high = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  const bool real = z > kNone;
  return (uint64_t)(real ? high : 0u) << 32 | (real ? (uint32_t)~column : 0u);
}
__device__ inline float key_logit(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ inline int key_column(uint64_t key) { return (int)~(uint32_t)key; }

__device__ inline void put_top(const Score &a, int64_t at, uint64_t key, const End &e, const Scale &scale) {
  const int column = key ? key_column(key) : -1;
  if (a.ids.bits == 32) ((int32_t *)a.top_ids)[at] = column;
  else ((int64_t *)a.top_ids)[at] = column;
  a.top_logp[at] = key ? log_p(key_logit(key), e, scale) : kNone;
}

// Keys of columns that may be among a row's alternatives, at most.  Of a row of equal logits and fewer
// larger ones than the k <= 64 alternatives up to 8 k + k - 1 = 575 are left: top_of().
constexpr int kCand = 576;

template <int kLanes, bool kOn>
struct TopLds {
  alignas(16) uint64_t keys[!kOn ? 1 : kLanes > kCand ? kLanes : kCand];   // at first one of each lane
  uint64_t best[(kLanes + 63) / 64];
  uint16_t who[kOn ? kLanes : 1];           // lanes that may hold some
  uint64_t bound;
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
    const uint32_t high = wave_max((uint32_t)(best >> 32));
    best = (uint64_t)high << 32 | wave_max((uint32_t)(best >> 32) == high ? (uint32_t)best : 0u);
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

// The k-th largest of a wave's different keys, R in a lane; 1 if fewer than k are not 0.  By the bits
// in which any two differ, until k keys are left.
template <int R>
__device__ inline uint64_t kth_largest(const uint64_t (&key)[R], int k) {
  uint32_t most = 0;
  int count = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    most = max(most, (uint32_t)(key[i] >> 32));
    count += (int)__popcll(__ballot(key[i] != 0));
  }
  if (count < k) return 1;
  most = wave_max(most);
  uint32_t high = 0, low = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    high |= key[i] ? (uint32_t)(key[i] >> 32) ^ most : 0u;
    low |= key[i] ? ~(uint32_t)key[i] : 0u;         // (columns: their own upper bits are 0)
  }
  uint64_t differ = (uint64_t)wave_or(high) << 32 | wave_or(low);
  uint64_t t = ((uint64_t)most << 32 | 0xffffffffu) & ~differ;
  while (differ && count != k) {
    const uint64_t bit = (uint64_t)1 << (63 - __clzll((long long)differ)), trial = t | bit;
    differ ^= bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += (int)__popcll(__ballot(key[i] >= trial));
    if (n < k) continue;
    t = trial;
    count = n;
  }
  // the smallest of the k: its logit, and the highest column with it
  high = low = ~0u;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (key[i] >= t) high = min(high, key[i] ? (uint32_t)(key[i] >> 32) : ~0u);
  high = wave_min(high);
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (key[i] >= t && (uint32_t)(key[i] >> 32) == high) low = min(low, (uint32_t)key[i]);
  return (uint64_t)high << 32 | wave_min(low);
}

// The same for one key in a lane.  Few: one logit after the other; more: each lane counts the logits
// above its own, 64 comparisons that wait for nothing.
__device__ inline uint64_t kth_of_wave(uint64_t key, int k) {
  if ((int)__popcll(__ballot(key != 0)) < k) return 1;
  const uint32_t high = (uint32_t)(key >> 32);
  uint32_t t;
  if (k <= 10) {
    for (uint32_t left = high;;) {
      t = wave_max(left);
      const int n = (int)__popcll(__ballot(left == t));
      if (n >= k) break;
      k -= n;
      left = left == t ? 0u : left;
    }
  } else {
    int above = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) above += (uint32_t)__builtin_amdgcn_readlane((int)high, i) > high;
    t = wave_min(above < k ? high : ~0u);
    k -= (int)__popcll(__ballot(high > t));
  }
  const bool at = high == t;
  if ((int)__popcll(__ballot(at)) == k) return (uint64_t)t << 32 | wave_min(at ? (uint32_t)key : ~0u);
  // of those with the logit t, the k lowest columns
  uint32_t left = at ? (uint32_t)key : 0u, u = 0;
  for (; k > 0; --k) {
    u = wave_max(left);
    left = left == u ? 0u : left;
  }
  return (uint64_t)t << 32 | u;
}

// Of the first n > k keys in LDS moves the k largest, or those that are not 0, to the front, in no
// order, and returns how many they are: by one wave.
template <int R>
__device__ inline int keep_largest(uint64_t *keys, int n, int k, int lane) {
  uint64_t key[R];
#pragma unroll
  for (int i = 0; i < R; ++i) key[i] = 64 * i + lane < n ? keys[64 * i + lane] : 0;
  const uint64_t t = kth_largest(key, k);
  int at = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t all = __ballot(key[i] >= t);
    if (key[i] >= t) keys[at + __popcll(all & (((uint64_t)1 << lane) - 1))] = key[i];
    at += (int)__popcll(all);
  }
  group_sync<64>();
  return at;
}

// put(r, key) for the r-th of the k largest of n <= kMost keys in LDS (0: there is none), by one wave:
// no more than 64 of them, in the order of how many are above each.
template <int kMost, typename Put>
__device__ inline void put_largest(uint64_t *keys, int n, int k, int lane, Put put) {
  const int left = n > 256  ? keep_largest<kMost / 64>(keys, n, k, lane)
                   : n > 64 ? keep_largest<4>(keys, n, k, lane)
                            : n;
  const uint64_t mine = lane < left ? keys[lane] : 0;
  int above = 0;
  for (int i = 0; i < left; i += 8) {
#pragma unroll
    for (int x = 0; x < 8; ++x) {          // (lanes past the last one have 0)
      const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), i + x) << 32 |
                             (uint32_t)__builtin_amdgcn_readlane((int)mine, i + x);
      above += other > mine;
    }
  }
  // (lanes without one have the places after the last)
  const uint64_t without = __ballot(mine == 0);
  if (mine == 0) above = 64 - (int)__popcll(without) + (int)__popcll(without & (((uint64_t)1 << lane) - 1));
  if (above < k) put(above, mine);
}

// The k largest keys of a part, put(r, key) for the r-th of them (0: there is none).  The sums' pass over
// the row leaves each lane's largest logit and its chunk.  Such keys are of different columns, so the
// k-th largest of the largest of some groups of lanes is a lower bound of the k-th largest of all,
// and lanes whose own largest logit is below it have none of those: the chunks of the other lanes,
// some k, are dealt out to the group and read again, and the keys from the bound on, little more
// than k, are left in LDS for the first wave.  (A lane's chunk stands for its last column: the key
// is then at most the column's own.)  A group's lanes are 64 or 256 apart, so that neighbouring chunks
// are of different groups: of equal logits, such as those of a mask of the type's lowest value, the
// groups' keys are the row's first chunks, and no more than the first k chunks' columns and the larger
// logits pass the bound.  (With groups of neighbouring lanes those of some 16 k chunks did: 64 x 47,236
// bf16 with 20 alternatives, all columns but 15 masked, 162 us; now 19, as all lanes with the mask's
// logit are read again, 9.4 without a mask.)  Where more than kCand are left, which takes most of the
// largest logits in the columns of a few lanes, k searches follow.
template <typename T, int kLanes, typename Put>
__device__ inline void top_of(const Part<T> &p, int k, int lane, float m, int most,
                              TopLds<kLanes, true> &lds, Put put) {
  constexpr int N = kCols<T>;
  // groups of lanes with one key each, 256 or 64 of them: the more there are, the nearer the bound
  constexpr int R = (kLanes < 256 ? kLanes : 256) / 64;
  const uint64_t key = key_of(m, min(most + N, p.d) - 1);
  if (kLanes > 64) lds.keys[lane] = key;
  if (lane == 0) lds.lanes = lds.count = 0;
  group_sync<kLanes>();
  if (lane < 64) {
    uint64_t of[R], one = key;
#pragma unroll
    for (int i = 0; i < R; ++i) of[i] = kLanes > 64 ? lds.keys[64 * i + lane] : key;
#pragma unroll
    for (int i = R; i < kLanes / 64; ++i) of[i % R] = larger(of[i % R], lds.keys[64 * i + lane]);
#pragma unroll
    for (int i = 0; i < R; ++i) one = larger(one, of[i]);
    const uint64_t bound = k <= 32 ? kth_of_wave(one, k) : kth_largest(of, k);
    if (lane == 0) lds.bound = bound;
  }
  group_sync<kLanes>();
  const uint64_t bound = lds.bound;
  // (a lane's largest logit may be in a lower column than its key says)
  if (key_of(m, 0) >= bound) lds.who[atomicAdd(&lds.lanes, 1u)] = (uint16_t)lane;
  group_sync<kLanes>();
  const uint32_t lanes = lds.lanes, deals = (uint32_t)(p.end - p.q0 + kLanes - 1) / kLanes;
  for (uint32_t i = lane; i < lanes * deals; i += kLanes) {
    const int q = p.q0 + (int)lds.who[i % lanes] + (int)(i / lanes) * kLanes;
    if (q >= p.end) continue;
    float v[N];
    p.numbers(q, v);
    const int at = p.column(q);
    uint32_t found = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) found |= key_of(v[j], at + j) >= bound ? 1u << j : 0u;
    if (!found) continue;
    uint32_t slot = atomicAdd(&lds.count, (uint32_t)__popc(found));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!(found >> j & 1u)) continue;
      if (slot < (uint32_t)kCand) lds.keys[slot] = key_of(v[j], at + j);
      ++slot;
    }
  }
  group_sync<kLanes>();
  const int count = (int)lds.count;
  if (count > kCand) {
    top_searches<T, kLanes>(p, k, lane, lds.best, put);
    return;
  }
  if (lane < 64) put_largest<kCand>(lds.keys, count, k, lane, put);
}

// kLanes lanes to a row, kPer chunks of a lane asked for at once.
template <typename T, int kLanes, int kPer, int kWhat>
__global__ __launch_bounds__(kThreads<kLanes>, kLanes == 16 ? 6 : 8) void score_kernel(Rows<T> a, Score o,
                                                                                       Teacher t) {
  constexpr int kGroups = kThreads<kLanes> / kLanes;
  constexpr bool kT = kWhat & kEntropy;
  __shared__ Sums sums_lds[kGroups][(kLanes + 63) / 64];
  __shared__ TopLds<kLanes, (kWhat & kTop) != 0> top_lds[kGroups];
  const int lane = lane_of<kLanes>(), group = group_of<kLanes>();
  const int64_t row = row_of<kLanes>();
  if (row >= a.n) return;
  const T *z = a.Z + row * a.ldz;
  const bool first = lane < 64;          // the wave that has the row's few numbers
  Taught::Raw entries;
  RawId given{~0u, ~0u};
  if (kWhat & kTeach) {
    if (first) entries = Taught::ask(t, row, lane);
  } else {
    given = id_of_row<kLanes>(o.ids, row);
    // (what is asked for of a row without a token may need nothing of it)
    if (!o.lse && !o.entropy && !o.k && token_of(given, o.ids.bits, a.d) < 0) {
      if (lane == 0 && o.logp) o.logp[row] = 0.0f;
      return;
    }
  }
  Batch<T, kLanes, kPer> b;
  const int skew = skew_of<kLanes>(z, a.d);
  const Part<T> p{z, a.d, skew, 0, chunks_in<T>(a.d, skew)};
  b.load(z, skew, p.q0, p.end, a.d, lane);
  Taught x;
  float zt = 0.0f;
  const int id = token_of(given, o.ids.bits, a.d);
  if ((kWhat & kTeach) && first) {
    x.read(t, entries, a.d);
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
  if ((kWhat & kTeach) && first) x.compare(a.scale);
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

// The sums, and the k largest keys, of a part of a row.
template <typename T, bool kT, bool kOfTop>
__global__ __launch_bounds__(kPartLanes) void part_kernel(Rows<T> a, int k, Split s) {
  constexpr int kLanes = kPartLanes;
  __shared__ Sums sums_lds[kLanes / 64];
  __shared__ TopLds<kLanes, kOfTop> top_lds;
  const int lane = (int)threadIdx.x;
  const int64_t row = (int64_t)(blockIdx.x / (uint32_t)s.parts);
  const T *z = a.Z + row * a.ldz;
  const int skew = skew_of<kLanes>(z, a.d);
  const Piece piece = piece_of(s, chunks_in<T>(a.d, skew));
  Sums x{kNone, 0.0f, 0.0f};
  int most = 0;
  Batch<T, kLanes, kPartPer> b;
  for (int q = piece.q0; q < piece.end; q = b.next) {
    b.load(z, skew, q, piece.end, a.d, lane);
    add_batch<kT>(b, a.c, x, most);
  }
  const float m = x.m;
  x = group_sums<kLanes, kT>(x, a.c, sums_lds);
  if (lane == 0) s.sums[blockIdx.x] = x;
  if constexpr (kOfTop) {
    const Part<T> p{z, a.d, skew, piece.q0, piece.end};
    top_of<T, kLanes>(p, k, lane, m, most, top_lds,
                      [&](int r, uint64_t key) { s.keys[(int64_t)blockIdx.x * k + r] = key; });
  }
}

// What is asked for of a row from its parts, by one wave.
template <typename T, int kWhat>
__global__ __launch_bounds__(64) void join_kernel(Rows<T> a, Score o, Teacher t, Split s) {
  constexpr int kKeys = 256;
  __shared__ uint64_t keys[kWhat & kTop ? kKeys : 1];
  const int lane = (int)threadIdx.x;
  const int64_t row = blockIdx.x;
  const T *z = a.Z + row * a.ldz;
  Taught x;
  const int id = kWhat & kTeach ? -1 : token_of(id_of_row<64>(o.ids, row), o.ids.bits, a.d);
  float zt = 0.0f;
  if (id >= 0) zt = (float)z[id];
  if (kWhat & kTeach) {
    x.read(t, Taught::ask(t, row, lane), a.d);
    x.gather(t, z);
    x.learn(t, row);
    x.compare(a.scale);
  }
  if (kWhat & kTop)
    for (int i = lane; i < s.parts * o.k; i += 64) keys[i] = s.keys[row * s.parts * o.k + i];
  const End e = end_of(parts_sums<(kWhat & kEntropy) != 0>(s, row, a.c));
  if (lane == 0) {
    if (kWhat & kTeach) t.loss[row] = x.loss(e, a.scale);
    else score_row(o, row, id, zt, e, a.scale);
  }
  if constexpr ((kWhat & kTop) != 0) {
    group_sync<64>();
    put_largest<kKeys>(keys, s.parts * o.k, o.k, lane, [&](int r, uint64_t key) {
      put_top(o, row * o.k + r, key, e, a.scale);
    });
  }
}

template <typename T, int kWhat>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, hipStream_t s) {
  // Lanes of a row and chunks of a lane at once, by the length and the number of rows (log probabilities of
  // bf16 but for the last two, us):
  //    8,192 x 47,236   256 x 4: 139    512 x 6: 134    1,024 x 6: 146
  //        1 x 47,236   512 x 12: 7.7   1,024 x 6: 5.0
  //    3,000 x 16,000   256 x 4: 19.8   512 x 6: 20.9
  //       64 x 16,000   256 x 4: 4.7    512 x 6: 4.2
  //    8,000 x 4,001    64 x 4: 15.5    256 x 4: 17.8
  //       64 x 4,001    64 x 4: 4.5     256 x 4: 3.6
  //   18,750 x 900 f16  16 x 8: 9.8     64 x 4: 11.8
  //    2,000 x 900 f16  16 x 8: 4.0     64 x 4: 3.8
  // More alternatives than 32 need more groups of lanes than 64 lanes have (f16 with 64 of them, us):
  //   18,750 x 900      64 x 4: 187     256 x 4: 108
  //      100 x 900      64 x 4: 91      256 x 4: 12
#define TOC_SCORE(L, K)                                                                              \
  hipLaunchKernelGGL((score_kernel<T, L, K, kWhat>), grid_of<L>(a.n), dim3(kThreads<L>), 0, s, a, o, t)
  if constexpr ((kWhat & (kTop | kTeach)) == 0) {
    if (a.n >= kShortRows && a.chunks + 1 < 16 * 9) {
      TOC_SCORE(16, 8);
      return launched("score_kernel");
    }
  }
  const bool many = a.n >= 512;
  if (a.chunks <= (a.n >= 2048 ? 768 : 256) && !((kWhat & kTop) && o.k > 32)) TOC_SCORE(64, 4);
  else if (a.chunks <= (many ? 2048 : 1024)) TOC_SCORE(256, 4);
  else if (many || a.chunks <= 2048) TOC_SCORE(512, 6);
  else TOC_SCORE(1024, 6);
#undef TOC_SCORE
  return launched("score_kernel");
}

template <typename T>
toc_status distill(const Rows<T> &a, const Teacher &t, void *ws, hipStream_t s) {
  const Score o{};
  const Split split = split_of(a.n, a.chunks, 0, ws);
  if (split.parts == 1) return launch<T, kTeach>(a, o, t, s);
  const toc_status st = add_parts<T>(a, 0, false, split, s);
  return st ? st : join_parts<T>(a, o, t, split, s);
}

template <typename T>
toc_status score(const Rows<T> &a, const Score &o, void *ws, hipStream_t s) {
  const Teacher t{};
  const Split split = split_of(a.n, a.chunks, o.k, ws);
  if (split.parts > 1) {
    const toc_status st = add_parts<T>(a, o.k, o.entropy != nullptr, split, s);
    return st ? st : join_parts<T>(a, o, t, split, s);
  }
  if (o.k) return o.entropy ? launch<T, kTop | kEntropy>(a, o, t, s) : launch<T, kTop>(a, o, t, s);
  return o.entropy ? launch<T, kEntropy>(a, o, t, s) : launch<T, 0>(a, o, t, s);
}

}  // namespace

template <typename T>
toc_status add_parts(const Rows<T> &a, int k, bool entropy, const Split &s, hipStream_t stream) {
  const dim3 grid((unsigned)(a.n * (uint32_t)s.parts)), block(kPartLanes);
  if (k > 0 && entropy) hipLaunchKernelGGL((part_kernel<T, true, true>), grid, block, 0, stream, a, k, s);
  else if (k > 0) hipLaunchKernelGGL((part_kernel<T, false, true>), grid, block, 0, stream, a, k, s);
  else if (entropy) hipLaunchKernelGGL((part_kernel<T, true, false>), grid, block, 0, stream, a, k, s);
  else hipLaunchKernelGGL((part_kernel<T, false, false>), grid, block, 0, stream, a, k, s);
  return launched("part_kernel");
}

template <typename T>
toc_status join_parts(const Rows<T> &a, const Score &o, const Teacher &t, const Split &s, hipStream_t stream) {
  const dim3 grid(a.n), block(64);
  if (t.k > 0) hipLaunchKernelGGL((join_kernel<T, kTeach>), grid, block, 0, stream, a, o, t, s);
  else if (o.k > 0) hipLaunchKernelGGL((join_kernel<T, kEntropy | kTop>), grid, block, 0, stream, a, o, t, s);
  else hipLaunchKernelGGL((join_kernel<T, kEntropy>), grid, block, 0, stream, a, o, t, s);
  return launched("join_kernel");
}

#define TOC_PARTS(T)                                                                         \
  template toc_status add_parts<T>(const Rows<T> &, int, bool, const Split &, hipStream_t);   \
  template toc_status join_parts<T>(const Rows<T> &, const Score &, const Teacher &, const Split &, hipStream_t);
TOC_PARTS(float)
TOC_PARTS(bf16)
TOC_PARTS(f16)
#undef TOC_PARTS

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
  // the most that a call of 1 .. n rows, of the type with the most chunks, takes
  const int64_t most = parts_of(1, chunks_of<float>(d), 0), pieces = std::min(n * most, (int64_t)kMaxPieces);
  *bytes = most > 1 ? (size_t)pieces * (sizeof(Sums) + sizeof(uint64_t) * (size_t)k) : 0;
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
    case TOC_F32: return score(rows_of<float>(n, d, Z, ldz, scale), o, ws, (hipStream_t)stream);
    case TOC_BF16: return score(rows_of<bf16>(n, d, Z, ldz, scale), o, ws, (hipStream_t)stream);
    default: return score(rows_of<f16>(n, d, Z, ldz, scale), o, ws, (hipStream_t)stream);
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
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case TOC_F32: return distill(rows_of<float>(n, d, Z, ldz, scale), t, ws, s);
    case TOC_BF16: return distill(rows_of<bf16>(n, d, Z, ldz, scale), t, ws, s);
    default: return distill(rows_of<f16>(n, d, Z, ldz, scale), t, ws, s);
  }
}

}  // extern "C"
