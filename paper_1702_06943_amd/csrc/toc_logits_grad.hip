// Gradients for the logits of losses made of log probabilities and entropies, and of the distance
// from a teacher's saved logits.  With p_j and H as in the forward pass, row by row:
//   dz_j = scale (gl (1[j = t] - p_j) + gs p_j - ge p_j (log p_j + H))
//   dz_j = scale c (Q p_j - sum of q_a over the entries with i_a = j)
// The probabilities are formed again from the logits: nothing is kept from the forward pass.
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

// The gradient of a lane's chunks; hit: what the column `id` gets on top.
template <typename T, int kLanes, int kPer, bool kEntropy>
__device__ inline void put_batch(Batch<T, kLanes, kPer> &b, float c, float base, Slope k, int id, float hit,
                                 T *dz, int d, bool stream) {
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
    if ((uint32_t)(id - at) < (uint32_t)N) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += at + i == id ? hit : 0.0f;
    }
    T *to = (T *)((char *)(dz + N * (b.q + j * kLanes)) + (uint32_t)(16 * b.lane));
    if (j < b.rows) put(to, N, narrow<T>(v), stream);
    else if (at < d) put(to, d - at, narrow<T>(v), stream);
  });
}

// kLanes lanes to a row, kPer chunks to a lane: a row of as many chunks stays in registers between
// its one read and its one write, a longer one is read twice.
template <typename T, int kLanes, int kPer, bool kTeach, bool kEntropy>
__global__ __launch_bounds__(kThreads<kLanes>) void grad_kernel(Rows<T> a, Score o, Teacher t, Grad<T> g) {
  constexpr int N = kCols<T>;
  constexpr int kGroups = kThreads<kLanes> / kLanes;
  __shared__ Sums sums[kGroups][kLanes / 64];
  __shared__ float q_sum[kGroups];
  __shared__ int ids_lds[kGroups][kTeach ? kMaxTeacher : 1];
  __shared__ float q_lds[kGroups][kTeach ? kMaxTeacher : 1];
  const int lane = lane_of<kLanes>(), group = group_of<kLanes>();
  const int64_t row = row_of<kLanes>();
  if (row >= a.n) return;
  const T *z = a.Z + row * a.ldz;
  T *dz = g.dZ + row * g.lddz;
  const bool first = lane < 64;          // the wave that has the row's few numbers
  Taught x;
  if (kTeach && first) x.ask(t, row, a.d, lane);
  int id = -1;
  float gl = 0.0f, gs = 0.0f, ge = 0.0f;
  if (kTeach) {
    gl = scalar(g.dloss, row);
  } else {
    id = scalar_token(o.ids, row, a.d);
    if (id >= 0 && g.dlogp) gl = scalar(g.dlogp, row);
    if (g.dlse) gs = scalar(g.dlse, row);
    if (g.dentropy) ge = scalar(g.dentropy, row);
  }
  Batch<T, kLanes, kPer> b;
  b.load(z, 0, a.chunks, a.d, lane);
  float zt = 0.0f;
  if (kTeach && first) x.gather(t, z);
  if (!kTeach && id >= 0) zt = (float)z[id];
  Sums s{kNone, 0.0f, 0.0f};
  int most = 0;
  add_batch<kEntropy>(b, a.c, s, most);
  while (b.next < a.chunks) {
    b.load(z, b.next, a.chunks, a.d, lane);
    add_batch<kEntropy>(b, a.c, s, most);
  }
  if (kTeach && first) {
    x.learn(t, row);
    if (lane == 0) q_sum[group] = x.sum;
  }
  // (behind this barrier dZ, which may be Z, is written: all of Z that is not read again is there)
  s = group_sums<kLanes, kEntropy>(s, a.c, sums[group]);
  const End e = end_of(s);
  if (kTeach) {
    if (kLanes == 64) group_sync<kLanes>();
    gs = gl == 0.0f ? 0.0f : gl * q_sum[group];
    if (first && t.loss) {
      const float loss = x.loss(e, a.scale);
      if (lane == 0) t.loss[row] = loss;
    }
  } else if (lane == 0) {
    score_row(o, row, id, zt, e, a.scale);
  }
  Slope k;
  if (kTeach) {
    k.none = e.empty || gs == 0.0f;
    k.a = a.scale * gs / s.s;
    k.b = 0.0f;
  } else {
    k.none = e.empty || (gl == 0.0f && gs == 0.0f && ge == 0.0f);
    k.a = a.scale * (gs - gl + ge * e.t_s) / s.s;
    k.b = -a.scale * ge * kLn2 / s.s;
  }
  if (k.none) {
    for (int q = lane; q < a.chunks; q += kLanes) put(dz + N * q, a.d - N * q, Chunk{0u, 0u, 0u, 0u}, g.stream);
    return;
  }
  const float base = from(e.m);
  const bool held = b.q == 0;
  for (int q = 0; q < a.chunks; q = b.next) {
    if (!held) b.load(z, q, a.chunks, a.d, lane);
    put_batch<T, kLanes, kPer, kEntropy>(b, a.c, base, k, id, a.scale * gl, dz, a.d, g.stream);
  }
  if (kTeach) {
    // the columns with entries, written again: an entry's column by its first one, with the sum of
    // them all
    group_sync<kLanes>();
    if (!first) return;
    int *ids = ids_lds[group];
    float *qs = q_lds[group];
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) {
      ids[lane + 64 * i] = x.id[i];
      qs[lane + 64 * i] = x.q[i];
    }
    group_sync<64>();
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) {
      if (64 * i >= t.k || x.id[i] < 0) continue;
      float q = 0.0f;
      bool one = true;
      for (int j = 0; j < t.k; ++j) {
        if (ids[j] != x.id[i]) continue;
        one = one && j >= lane + 64 * i;
        q += qs[j];
      }
      const float v = fmaf(two_to((x.z[i] - base) * a.c), k.a, -a.scale * gl * q);
      if (one) dz[x.id[i]] = (T)v;
    }
  }
}

template <typename T, bool kTeach, bool kEntropy>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, const Grad<T> &g, hipStream_t s) {
#define TOC_GRAD(L, K)                                                                           \
  hipLaunchKernelGGL((grad_kernel<T, L, K, kTeach, kEntropy>),                                   \
                     grid_of<L>(a.n), dim3(kThreads<L>), 0, s, a, o, t, g)
  if (a.chunks <= 256) TOC_GRAD(64, 4);
  else if (a.chunks <= 2048) TOC_GRAD(256, 8);
  else TOC_GRAD(1024, 6);
#undef TOC_GRAD
  return launched("grad_kernel");
}

template <typename T, bool kTeach>
toc_status grad(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale, const Score &o,
                const Teacher &t, void *dZ, int64_t lddz, const float *dlogp, const float *dlse,
                const float *dentropy, const float *dloss, void *stream) {
  const Rows<T> a = rows_of<T>(n, d, Z, ldz, scale);
  const Grad<T> g{(T *)dZ, lddz, dlogp, dlse, dentropy, dloss, stream_out(n, d, sizeof(T))};
  if constexpr (!kTeach) {
    if (o.entropy || dentropy) return launch<T, false, true>(a, o, t, g, (hipStream_t)stream);
  }
  return launch<T, kTeach, false>(a, o, t, g, (hipStream_t)stream);
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
      (st = check_rows("dZ", dZ, n, d, lddz, type_size(type))) ||
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
      return grad<float, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, stream);
    case TOC_BF16:
      return grad<bf16, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, stream);
    default:
      return grad<f16, false>(n, d, Z, ldz, scale, o, t, dZ, lddz, dlogp, dlse, dentropy, nullptr, stream);
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
      (st = check_rows("dZ", dZ, n, d, lddz, type_size(type))) || (st = check_ws(ws, ws_bytes, need)))
    return st;
  if (n == 0) return TOC_OK;
  const Score o{};
  const Teacher t{Ids{top_ids, id_bits}, ldi, k, t_type, top_z, ldt, top_scale, top_lse, loss};
  switch (type) {
    case TOC_F32:
      return grad<float, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, stream);
    case TOC_BF16:
      return grad<bf16, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, stream);
    default:
      return grad<f16, true>(n, d, Z, ldz, scale, o, t, dZ, lddz, nullptr, nullptr, nullptr, dloss, stream);
  }
}

}  // extern "C"
