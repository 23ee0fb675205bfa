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
};

// A column's gradient before its target's part: e = 2^y of the softmax, y kept above kFar.
struct Slope {
  float a, b;          // dz = e (a + b y)
  bool none;           // the row's coefficients are all zero, or it has no probabilities
};

template <typename T, int kLanes, bool kTeach, bool kEntropy>
__global__ __launch_bounds__(kBlock) void grad_kernel(Rows<T> a, Score o, Teacher t, Grad<T> g) {
  constexpr int N = kCols<T>;
  __shared__ Sums sums[kLanes / 64];
  __shared__ float lds[kLanes / 64 * 4];
  __shared__ int ids[kMaxTeacher];
  __shared__ float qs[kMaxTeacher];
  const int lane = threadIdx.x;
  for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T *z = a.Z + (int64_t)row * a.ldz;
    T *dz = g.dZ + (int64_t)row * g.lddz;
    __syncthreads();
    Taught<kLanes> x;
    int id = -1;
    float zt = 0.0f, gl = 0.0f, gs = 0.0f, ge = 0.0f;
    if (kTeach) {
      x = teach<T, kLanes>(t, row, z, a.d, lane, lds);
      gs = g.dloss[row] * x.sum;
      if (g.dloss[row] == 0.0f) gs = 0.0f;
    } else {
      id = token(o.ids, row, a.d);
      if (id >= 0) zt = (float)z[id];
      if (id >= 0 && g.dlogp) gl = g.dlogp[row];
      if (g.dlse) gs = g.dlse[row];
      if (g.dentropy) ge = g.dentropy[row];
    }
    Sums s{kNone, 0.0f, 0.0f};
    int most = 0;
    Batch<T, kLanes, 4> b;
    for (int q = 0; q < a.chunks; q += kLanes * 4) {
      b.load(z, q, a.chunks, a.d, lane);
      add_batch<kEntropy>(b, a.c, s, most);
    }
    s = group_sums<kLanes, kEntropy>(s, a.c, sums);
    const End e = end_of(s);
    float loss = 0.0f;
    if (kTeach) loss = taught_loss<kLanes>(x, e, a.scale, lds + 3 * (kLanes / 64));
    else __syncthreads();          // the given token's logit is read before dZ, which may be Z, is written
    if (lane == 0) {
      if (kTeach) {
        if (t.loss) t.loss[row] = loss;
      } else {
        score_row(o, row, id, zt, e, a.scale);
      }
    }
    Slope k;
    k.none = e.empty || (gl == 0.0f && gs == 0.0f && ge == 0.0f);
    k.a = a.scale * (gs - gl + ge * e.t_s) / s.s;
    k.b = -a.scale * ge * kLn2 / s.s;
    const float base = from(e.m);
    for (int q = 0; q < a.chunks; q += kLanes * 4) {
      b.load(z, q, a.chunks, a.d, lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!b.any(j)) continue;
        float v[N];
        b.numbers(j, v);
        const int at = b.column(j);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float y = (v[i] - base) * a.c;
          const float p = two_to(y);
          y = fmaxf(y, kFar);
          v[i] = k.none ? 0.0f : p * (kEntropy ? fmaf(k.b, y, k.a) : k.a);
          if (!kTeach && at + i == id && !k.none) v[i] = fmaf(a.scale, gl, v[i]);
        }
        if (at < a.d) store(dz + at, a.d - at, v, false);
      }
    }
    if (kTeach) {
      // the columns with entries, written again: an entry's column by its first one, with the sum of
      // them all
#pragma unroll
      for (int i = 0; i < x.kPer; ++i) {
        if (lane + i * kLanes < t.k) {
          ids[lane + i * kLanes] = x.id[i];
          qs[lane + i * kLanes] = x.q[i];
        }
      }
      __syncthreads();
      if (k.none) continue;
#pragma unroll
      for (int i = 0; i < x.kPer; ++i) {
        if (x.id[i] < 0) continue;
        float q = 0.0f;
        bool first = true;
        for (int b = 0; b < t.k; ++b) {
          if (ids[b] != x.id[i]) continue;
          first = first && b >= lane + i * kLanes;
          q += qs[b];
        }
        const float p = two_to((x.z[i] - base) * a.c);
        const float v = fmaf(p, k.a, -a.scale * g.dloss[row] * q);
        if (first) dz[x.id[i]] = (T)v;
      }
    }
  }
}

template <typename T, bool kTeach>
toc_status launch(const Rows<T> &a, const Score &o, const Teacher &t, const Grad<T> &g, hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20));
  if (!kTeach && (o.entropy || g.dentropy))
    hipLaunchKernelGGL((grad_kernel<T, kBlock, false, true>), grid, dim3(kBlock), 0, s, a, o, t, g);
  else
    hipLaunchKernelGGL((grad_kernel<T, kBlock, kTeach, false>), grid, dim3(kBlock), 0, s, a, o, t, g);
  return launched("grad_kernel");
}

template <typename T, bool kTeach>
toc_status grad(int64_t n, int32_t d, const void *Z, int64_t ldz, float scale, const Score &o,
                const Teacher &t, void *dZ, int64_t lddz, const float *dlogp, const float *dlse,
                const float *dentropy, const float *dloss, void *stream) {
  const Rows<T> a = rows_of<T>(n, d, Z, ldz, scale);
  const Grad<T> g{(T *)dZ, lddz, dlogp, dlse, dentropy, dloss};
  return launch<T, kTeach>(a, o, t, g, (hipStream_t)stream);
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
