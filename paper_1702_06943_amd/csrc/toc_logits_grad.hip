// Gradients for the logits of losses made of log probabilities and entropies, and of the distance
// from a teacher's saved logits.  With p_j and H as in the forward pass, row by row:
//   dz_j = scale (gl (1[j = t] - p_j) + gs p_j - ge p_j (log p_j + H))
//   dz_j = scale c (Q p_j - sum of q_a over the entries with i_a = j)
// The probabilities are formed again from the logits: nothing is kept from the forward pass, and what it
// would have given comes along, so that a training step is one read and one write of the logits.
//   grad_kernel       bound by memory: 8,192 x 47,236 bf16 269 us, 5.75 TB/s (a plain map of as many bytes
//                     takes 250), with entropy 271, a teacher's 64 entries 278; 250 x 47,236 f32 20 us, a row a
//                     CU whose read and write are one after the other; 512 x 200,003 bf16 95 us, the
//                     rows read once more, three quarters of that from memory
//   part_grad_kernel  few long rows, after part_kernel: one of 262,144 f32 8.4 us, 64 of bf16 20.9
#include "toc_logits_dev.h"

namespace toc {
namespace logits {
namespace {

template <typename T>
struct Grad {
  T *dZ;
  int64_t lddz;
  const float *dlogp, *dlse, *dentropy;   // each may be NULL: zeros
  const float *dloss;
  bool stream;
};

// A column's gradient but for its target's part is e (a + b y), e = 2^y of the softmax.
struct Slope {
  float a, b;
  bool none;           // 0 throughout: the coefficients are 0, or there are no probabilities
};

// gl, gs, ge: the coefficients of log p, of the sum and of the entropy; with a teacher gs is that of p.
template <bool kTeach>
__device__ inline Slope slope_of(float scale, const Sums &s, const End &e, float gl, float gs, float ge) {
  Slope k;
  if (kTeach) {
    k.none = e.empty || gs == 0.0f;
    k.a = scale * gs / s.s;
    k.b = 0.0f;
  } else {
    k.none = e.empty || (gl == 0.0f && gs == 0.0f && ge == 0.0f);
    k.a = scale * (gs - gl + ge * e.t_s) / s.s;
    k.b = -scale * ge * kLn2 / s.s;
  }
  return k;
}

// A teacher's entries by the chunk of a window of kChunks chunks that holds their column: head[c] is
// 0 or the number, from 1, of the first entry of a list that goes on with next.  Made by one wave.
template <int kChunks>
struct Marks {
  static constexpr int kHeads = (kChunks + 511) / 512 * 512;
  alignas(16) uint16_t head[kHeads];       // (cleared 16 bytes at a time)
  uint16_t next[kMaxTeacher];
  int column[kMaxTeacher];
  float q[kMaxTeacher];
  float weight[kMaxTeacher];   // what an entry's column gets: q, or that of all entries of the column
  float sum;                   // of q over the row

  __device__ inline void keep(const Taught &x, int lane) {
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) {
      column[64 * i + lane] = x.id[i];
      q[64 * i + lane] = x.q[i];
    }
    if (lane == 0) sum = x.sum;
  }
  // Marks the first k entries whose column is in chunks first .. first + kChunks - 1, chunks of n
  // columns.
  __device__ inline void mark(int k, int first, int n, int skew, int lane) {
    for (int i = lane; i < kHeads / 8; i += 64) ((uint4 *)head)[i] = make_uint4(0, 0, 0, 0);
    group_sync<64>();
    bool crowded = false;
    for (int e = lane; e < k; e += 64) {
      const uint32_t c = (uint32_t)((column[e] + skew) / n - first);
      weight[e] = q[e];
      if (column[e] < 0 || c >= (uint32_t)kChunks) continue;
      // (two heads to a word)
      uint32_t *word = (uint32_t *)head + c / 2;
      const uint32_t shift = c % 2 * 16;
      uint32_t old = *word, seen;
      do {
        seen = old;
        old = atomicCAS(word, seen, (seen & ~(0xffffu << shift)) | (uint32_t)(e + 1) << shift);
      } while (old != seen);
      next[e] = (uint16_t)(old >> shift);
      crowded = crowded || next[e] != 0;
    }
    group_sync<64>();
    if (!__any(crowded)) return;
    // Entries of one chunk come in no fixed order.  Those of one column are put together in the first of
    // them and the others count 0, so that the order of the rest does not matter: two along their
    // list, as a sum of two has one value; of more, in the order of the entries.
    for (int e = lane; e < k; e += 64) {
      const uint32_t c = (uint32_t)((column[e] + skew) / n - first);
      if (column[e] < 0 || c >= (uint32_t)kChunks) continue;
      int same = 0;
      float s = q[e];
      for (uint32_t o = head[c]; o != 0; o = next[o - 1]) {
        if (column[o - 1] != column[e] || (int)o - 1 == e) continue;
        ++same;
        s = (int)o - 1 < e ? 0.0f : q[e] + q[o - 1];
      }
      if (same > 1) {
        s = 0.0f;
        bool one = true;
        for (int o = 0; o < k; ++o) {
          if (column[o] != column[e]) continue;
          one = one && o >= e;
          s += q[o];
        }
        s = one ? s : 0.0f;
      }
      weight[e] = s;
    }
  }
};
struct NoMarks {};

// The gradient of a lane's chunks.  hit: what the column `id` gets on top, or with a teacher's entries
// what each gets for its q; window: the first chunk that they are marked from.
template <bool kEntropy, typename T, int kLanes, int kPer, typename M>
__device__ inline void put_batch(Batch<T, kLanes, kPer> &b, float c, float base, Slope k, int id, float hit,
                                 const M &marks, T *dz, int d, bool stream) {
  constexpr int N = kCols<T>;
  b.again();
  b.each([&](int j, Chunk in) {
    float v[N];
    widen<T>(in, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = (v[i] - base) * c;
      v[i] = two_to(y) * (kEntropy ? fmaf(k.b, fmaxf(y, kFar), k.a) : k.a);
    }
    const int at = b.column(j);
    if constexpr (std::is_same<M, NoMarks>::value) {
      if ((uint32_t)(id - at) < (uint32_t)N) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += at + i == id ? hit : 0.0f;
      }
    } else {
      for (uint32_t e = marks.head[j * kLanes + b.lane]; e != 0; e = marks.next[e - 1]) {
        const int column = marks.column[e - 1];
        const float q = marks.weight[e - 1];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = at + i == column ? fmaf(hit, q, v[i]) : v[i];
      }
    }
    T *to = (T *)((char *)(dz + (N * (b.q + j * kLanes) - b.skew)) + (uint32_t)(16 * b.lane));
    const Chunk out = narrow<T>(v);
    // (an edge's lanes past the batch's last chunk have what others write)
    if (j == b.rows && b.q + j * kLanes + b.lane >= b.end) return;
    if ((j < b.rows || at + N <= d) && (j > 0 || at >= 0)) put(to, N, out, stream);
    else put_some(to, -at, d - at, out);
  });
}

// Zeros to chunks q, q + step and so on below end.
template <typename T>
__device__ inline void put_zeros(T *dz, int skew, int q, int end, int step, int d) {
  constexpr int N = kCols<T>;
  const Chunk zero = {0u, 0u, 0u, 0u};
  for (; q < end; q += step) {
    const int at = N * q - skew;
    if (at >= 0 && at + N <= d) put(dz + at, N, zero, false);
    else put_some(dz + at, -at, d - at, zero);
  }
}

// kLanes lanes to a row, kPer chunks to a lane: a row of as many chunks stays in registers between
// its one read and its one write, a longer one is read twice.
template <typename T, int kLanes, int kPer, bool kTeach, bool kEntropy>
__global__ __launch_bounds__(kThreads<kLanes>, kLanes == 1024 && kPer <= 6 ? 8 : 4) void grad_kernel(
    Rows<T> a, Score o, Teacher t, Grad<T> g) {
  constexpr int N = kCols<T>;
  constexpr int kGroups = kThreads<kLanes> / kLanes;
  using M = typename std::conditional<kTeach, Marks<kLanes *(kPer + 1)>, NoMarks>::type;
  __shared__ Sums sums[kGroups][(kLanes + 63) / 64];
  __shared__ M all_marks[kGroups];
  const int lane = lane_of<kLanes>(), group = group_of<kLanes>();
  const int64_t row = row_of<kLanes>();
  if (row >= a.n) return;
  const T *z = a.Z + row * a.ldz;
  T *dz = g.dZ + row * g.lddz;
  M &marks = all_marks[group];
  const bool first = lane < 64;          // the wave that has the row's few numbers
  Taught::Raw entries;
  RawId given{~0u, ~0u};
  float gl = 0.0f, gs = 0.0f, ge = 0.0f;
  if (kTeach) {
    if (first) entries = Taught::ask(t, row, lane);
    gl = of_row<kLanes>(g.dloss, row);
  } else {
    given = id_of_row<kLanes>(o.ids, row);
    if (g.dlogp) gl = of_row<kLanes>(g.dlogp, row);
    if (g.dlse) gs = of_row<kLanes>(g.dlse, row);
    if (g.dentropy) ge = of_row<kLanes>(g.dentropy, row);
  }
  const int skew = skew_of<kLanes>(z, a.d), chunks = chunks_in<T>(a.d, skew);
  const int id = token_of(given, o.ids.bits, a.d);
  if (!kTeach && id < 0) gl = 0.0f;
  // a row that takes no part, and of which nothing is asked for, is not read
  if (kTeach ? gl == 0.0f && !t.loss
             : gl == 0.0f && gs == 0.0f && ge == 0.0f && !o.lse && !o.entropy && !(o.logp && id >= 0)) {
    if (!kTeach && lane == 0 && o.logp) o.logp[row] = 0.0f;
    put_zeros<T>(dz, skew, lane, chunks, kLanes, a.d);
    return;
  }
  Batch<T, kLanes, kPer> b;
  b.load(z, skew, 0, chunks, a.d, lane);
  Taught x;
  float zt = 0.0f;
  if (!kTeach && id >= 0) zt = (float)z[id];
  if constexpr (kTeach) {
    if (first) {
      x.read(t, entries, a.d);
      x.gather(t, z);
      x.learn(t, row);
      marks.keep(x, lane);
      const int rows = (a.d + skew) / N / kLanes;          // the last batch's first chunk
      marks.mark(t.k, rows ? (rows - 1) / kPer * kPer * kLanes : 0, N, skew, lane);
    }
  }
  Sums s{kNone, 0.0f, 0.0f};
  int most = 0;
  add_batch<kEntropy>(b, a.c, s, most);
  while (b.next < chunks) {
    b.load(z, skew, b.next, chunks, a.d, lane);
    add_batch<kEntropy>(b, a.c, s, most);
  }
  // (behind the next barrier dZ, which may be Z, is written: all of Z that is not read again has to be there)
  if (kTeach) {
    if (first) x.compare(a.scale);
  } else {
    asm volatile("" ::"v"(zt));
  }
  s = group_sums<kLanes, kEntropy>(s, a.c, sums[group]);
  const End e = end_of(s);
  if constexpr (kTeach) {
    if (kLanes == 64) group_sync<kLanes>();
    gs = gl == 0.0f ? 0.0f : gl * marks.sum;
    if (lane == 0 && t.loss) t.loss[row] = x.loss(e, a.scale);
  } else if (lane == 0) {
    score_row(o, row, id, zt, e, a.scale);
  }
  const Slope k = slope_of<kTeach>(a.scale.whole, s, e, gl, gs, ge);
  if (k.none) {
    put_zeros<T>(dz, skew, lane, chunks, kLanes, a.d);
    return;
  }
  const float base = from(e.m), hit = kTeach ? -a.scale.whole * gl : a.scale.whole * gl;
  // the last batch is still there; the others from the last on, the likelier to be in a cache
  for (;;) {
    put_batch<kEntropy>(b, a.c, base, k, id, hit, marks, dz, a.d, g.stream);
    const int q = b.q - kLanes * kPer;
    if (q < 0) break;
    b.load(z, skew, q, chunks, a.d, lane);
    b.trim();
    if constexpr (kTeach) {
      group_sync<kLanes>();
      if (first) marks.mark(t.k, q, N, skew, lane);
      group_sync<kLanes>();
    }
  }
}

// A part of a row, from the sums of all its parts.
template <typename T, bool kTeach, bool kEntropy>
__global__ __launch_bounds__(kPartLanes) void part_grad_kernel(Rows<T> a, Score o, Teacher t, Grad<T> g,
                                                               Split split) {
  constexpr int N = kCols<T>, kLanes = kPartLanes;
  using M = typename std::conditional<kTeach, Marks<kLanes *(kPartPer + 1)>, NoMarks>::type;
  __shared__ M marks;
  const int lane = (int)threadIdx.x;
  const int64_t row = (int64_t)(blockIdx.x / (uint32_t)split.parts);
  const T *z = a.Z + row * a.ldz;
  T *dz = g.dZ + row * g.lddz;
  const int skew = skew_of<kLanes>(z, a.d);
  const Piece p = piece_of(split, chunks_in<T>(a.d, skew));
  const bool first = lane < 64;
  int id = -1;
  float gl = 0.0f, gs = 0.0f, ge = 0.0f;
  if constexpr (kTeach) {
    gl = scalar(g.dloss, row);
    if (first) {
      Taught x;
      x.read(t, Taught::ask(t, row, lane), a.d);
      x.learn(t, row);
      marks.keep(x, lane);
    }
  } else {
    id = token_of(id_of_row<64>(o.ids, row), o.ids.bits, a.d);
    if (id >= 0 && g.dlogp) gl = scalar(g.dlogp, row);
    if (g.dlse) gs = scalar(g.dlse, row);
    if (g.dentropy) ge = scalar(g.dentropy, row);
  }
  const Sums s = parts_sums<kEntropy>(split, row, a.c);
  const End e = end_of(s);
  __syncthreads();
  if constexpr (kTeach) gs = gl == 0.0f ? 0.0f : gl * marks.sum;
  const Slope k = slope_of<kTeach>(a.scale.whole, s, e, gl, gs, ge);
  if (k.none) {
    put_zeros<T>(dz, skew, p.q0 + lane, p.end, kLanes, a.d);
    return;
  }
  const float base = from(e.m), hit = kTeach ? -a.scale.whole * gl : a.scale.whole * gl;
  Batch<T, kLanes, kPartPer> b;
  for (int q = p.q0; q < p.end; q = b.next) {
    if constexpr (kTeach) {
      __syncthreads();             // the batch before is done with its marks
      if (first) marks.mark(t.k, q, N, skew, lane);
      __syncthreads();
    }
    b.load(z, skew, q, p.end, a.d, lane);
    b.trim();
    put_batch<kEntropy>(b, a.c, base, k, id, hit, marks, dz, a.d, g.stream);
  }
}

template <typename T, bool kTeach, bool kEntropy>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, const Grad<T> &g, const Split &split,
                  hipStream_t s) {
#define TOC_GRAD(L, K)                                                                             \
  hipLaunchKernelGGL((grad_kernel<T, L, K, kTeach, kEntropy>), grid_of<L>(a.n), dim3(kThreads<L>), 0, s, a, o, t, g)
  if (split.parts > 1) {
    hipLaunchKernelGGL((part_grad_kernel<T, kTeach, kEntropy>), dim3((unsigned)(a.n * (uint32_t)split.parts)),
                       dim3(kPartLanes), 0, s, a, o, t, g, split);
    return launched("part_grad_kernel");
  }
  // Lanes of a row and chunks of a lane: the fewest lanes that hold a row, so that a CU has several rows in turns
  // of reading and writing, where there are that many rows (gradients of log p, bf16 unless said, us):
  //   18,750 x 100         16 x 8: 6.1      64 x 2: 13.1
  //   18,750 x 900 f16     16 x 8: 16.8     64 x 2: 18.9
  //    2,000 x 900 f16     16 x 8: 6.4      64 x 2: 5.3
  //   40,000 x 1,800       64 x 8: 52       256 x 8: 102
  //    2,000 x 4,000       64 x 8: 8.5      256 x 2: 9.5
  //       64 x 4,000       64 x 8: 6.1      256 x 2: 4.3
  //   10,000 x 8,003       256 x 8: 52      1,024 x 2: 99
  //       64 x 16,000      256 x 8: 6.4     512 x 6: 5.8
  //    8,000 x 16,384      256 x 8: 86      512 x 6: 80
  // but by 1,024 x 6 where fewer lanes would have fewer rows in flight, and by 512 x 20 of 16 bits only:
  //    8,192 x 47,236      256 x 24: 315    512 x 12: 302     1,024 x 6: 270
  //    2,000 x 65,536      512 x 20: 85     1,024 x 12: 95
  //    4,000 x 47,236 f32  512 x 24: 309    1,024 x 12: 291
  // Longer rows are read twice, by 1,024 x 6 rather than 1,024 x 16, which holds more of a row but has one a CU:
  //      512 x 200,003     1,024 x 6: 84    1,024 x 16: 89
  const auto fits = [&](int lanes, int per) { return a.chunks + 1 < lanes * (per + 1); };
  if constexpr (!kTeach) {
    if (a.n >= kShortRows && fits(16, 8)) {
      TOC_GRAD(16, 8);
      return launched("grad_kernel");
    }
  }
  if (fits(64, 2)) TOC_GRAD(64, 2);
  else if (a.n >= 1024 && fits(64, 8)) TOC_GRAD(64, 8);
  else if (fits(256, 2)) TOC_GRAD(256, 2);
  else if (a.n >= 512 && fits(256, 8)) TOC_GRAD(256, 8);
  else if (fits(512, 6)) TOC_GRAD(512, 6);
  else if (fits(1024, 6)) TOC_GRAD(1024, 6);
  else if (sizeof(T) == 2 && fits(512, 20)) TOC_GRAD(512, 20);
  else if (fits(1024, 12)) TOC_GRAD(1024, 12);
  else if (fits(1024, 16)) TOC_GRAD(1024, 16);
  else TOC_GRAD(1024, 6);
#undef TOC_GRAD
  return launched("grad_kernel");
}

template <typename T, bool kTeach>
toc_status grad(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale, const Score &o,
                const Teacher &t, void *dZ, int64_t lddz, const float *dlogp, const float *dlse,
                const float *dentropy, const float *dloss, void *ws, void *stream) {
  const Rows<T> a = rows_of<T>(n, d, Z, ldz, scale);
  const Grad<T> g{(T *)dZ, lddz, dlogp, dlse, dentropy, dloss, stream_out(n, d, sizeof(T))};
  const hipStream_t s = (hipStream_t)stream;
  const Split split = split_of(n, a.chunks, 0, ws);
  const bool entropy = !kTeach && (o.entropy || dentropy);
  if (split.parts > 1) {
    // (what is asked for beside dZ before it is written: it may be Z)
    toc_status st = add_parts<T>(a, 0, entropy, split, s);
    if (!st && (o.logp || o.lse || o.entropy || t.loss)) st = join_parts<T>(a, o, t, split, s);
    if (st) return st;
  }
  if constexpr (!kTeach) {
    if (entropy) return launch<T, false, true>(a, o, t, g, split, s);
  }
  return launch<T, kTeach, false>(a, o, t, g, split, s);
}

// dZ in the place of Z has Z's rows.
inline toc_status check_place(int64_t n, const void *Z, int64_t ldz, const void *dZ, int64_t lddz) {
  if (n > 1 && dZ == Z && lddz != ldz) return fail(TOC_EINVAL, "dZ is Z, with another row stride");
  return TOC_OK;
}

}  // namespace
}  // namespace logits
}  // namespace toc

using namespace toc;
using namespace toc::logits;

extern "C" {

toc_status toc_logprob_grad(int64_t n, int32_t d, int32_t type, const void *Z, int64_t ldz, float scale,
                            const void *ids, int32_t id_bits, const float *dlogp, const float *dlse,
                            const float *dentropy, float *logp, float *lse, float *entropy, void *dZ,
                            int64_t lddz, void *ws, size_t ws_bytes, void *stream) {
  size_t need = 0;
  toc_status st = toc_logits_workspace_size(n, d, 0, &need);
  if (st || (st = check_logits(n, d, type, Z, ldz, scale)) ||
      (st = check_score(n, ids, id_bits, logp, lse, entropy)) ||
      (st = check_rows("dZ", dZ, n, d, lddz, type_size(type))) || (st = check_place(n, Z, ldz, dZ, lddz)) ||
      (st = check_vec("dlogp", dlogp, n, false)) || (st = check_vec("dlse", dlse, n, false)) ||
      (st = check_vec("dentropy", dentropy, n, false)))
    return st;
  if (dlogp && !ids && n > 0) return fail(TOC_EINVAL, "dlogp without ids");
  if ((st = check_ws(ws, ws_bytes, need))) return st;
  if (n == 0) return TOC_OK;
  const Score o{Ids{ids, id_bits}, logp, lse, entropy, 0, nullptr, nullptr};
  const Teacher t{};
  switch (type) {
    case TOC_F32:
      return grad<float, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, ws, stream);
    case TOC_BF16:
      return grad<bf16, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, ws, stream);
    default:
      return grad<f16, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, ws, stream);
  }
}

toc_status toc_distill_grad(int64_t n, int32_t d, int32_t type, const void *Z, int64_t ldz, float scale,
                            int32_t k, const void *top_ids, int32_t id_bits, int64_t ldi, int32_t t_type,
                            const void *top_z, int64_t ldt, float top_scale, const float *top_lse,
                            const float *dloss, float *loss, void *dZ, int64_t lddz, void *ws,
                            size_t ws_bytes, void *stream) {
  size_t need = 0;
  toc_status st = toc_logits_workspace_size(n, d, 0, &need);
  if (st || (st = check_logits(n, d, type, Z, ldz, scale)) ||
      (st = check_teacher(n, type, k, top_ids, id_bits, ldi, t_type, top_z, ldt, top_scale, top_lse)) ||
      (st = check_vec("dloss", dloss, n, true)) || (st = check_vec("loss", loss, n, false)) ||
      (st = check_rows("dZ", dZ, n, d, lddz, type_size(type))) || (st = check_place(n, Z, ldz, dZ, lddz)) ||
      (st = check_ws(ws, ws_bytes, need)))
    return st;
  if (n == 0) return TOC_OK;
  const Score o{};
  const Teacher t{Ids{top_ids, id_bits}, ldi, k, t_type, top_z, ldt, top_scale, top_lse, loss};
  switch (type) {
    case TOC_F32:
      return grad<float, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, ws, stream);
    case TOC_BF16:
      return grad<bf16, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, ws, stream);
    default:
      return grad<f16, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, ws, stream);
  }
}

}  // extern "C"
