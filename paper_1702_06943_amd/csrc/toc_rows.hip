// Embedding lookup with scaling, and dropout: maps of rows to rows, n x d, one output
// chunk per thread step.
//   lookup   out[t, :] = drop(scale E[ids[t], :]), a row of zeros where ids[t] is outside
//            the table; each output row is the row A.W of a tuple whose only pair is
//            ids[t]:scale (Theorem 1), without the compressed image
//   dropout  Y = drop(X): the same kernel, reading row t for output row t
// Bound by memory: an element is read and written once.  Dropout of 65,536 x 2,048 bf16 85 us,
// 6.3 TB/s; lookup of 32,768 x 1,024 bf16 of 47,236 rows 14.8 us, with dropout 17 to 20 (the
// mask's arithmetic, some 10 us of the vector units, does not all hide behind the gather).
#include "toc_rows_dev.h"

namespace toc {
namespace rows {
namespace {

constexpr int kBlock = 256;
struct Same {};           // no token numbers: output row t reads row t

// Chunks of a thread, their loads in flight together.  A lookup's loads wait for its token
// numbers; a plain map has enough in flight with one a thread.  65,536 x 2,048 bf16 dropout
// with 1, 2, 4, 8: 88.5, 95.0, 96.5, 101 us; lookup of 32,768 x 1,024 f32: 50.7, 49.0, 49.8, 51.3.
template <typename Id>
constexpr int kPer = std::is_same<Id, Same>::value ? 1 : 2;

template <typename Id>
__device__ inline int64_t source(const Id *ids, uint32_t row, int64_t n_vocab) {
  const int64_t id = (int64_t)ids[row];
  return id >= 0 && id < n_vocab ? id : -1;
}
__device__ inline int64_t source(const Same *, uint32_t row, int64_t) { return row; }

// Rows row0 .. row0 + n - 1 of the call (src of Same and out start at row0's).
template <typename T, typename Id, bool kDrop>
__global__ __launch_bounds__(kBlock) void rows_kernel(const Id *__restrict__ ids, int64_t n_vocab,
                                                      const T *src, int64_t lds, float scale,
                                                      Mask m, uint32_t row0, uint32_t total,
                                                      int d, Divisor chunks, T *out, int64_t ldo,
                                                      bool stream) {
  constexpr int P = kPer<Id>;
  constexpr bool same = std::is_same<Id, Same>::value;
  const uint32_t o0 = blockIdx.x * (uint32_t)(kBlock * P) + threadIdx.x;
  uint32_t row[P], at[P];
  Place<T, true> l[P];
  int64_t from[P];
  Chunk in[P];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const uint32_t o = o0 + (uint32_t)(k * kBlock);
    row[k] = divide(o < total ? o : 0u, chunks, &at[k]);
    from[k] = o < total ? source(ids, row[k], n_vocab) : (int64_t)-1;
  }
#pragma unroll
  for (int k = 0; k < P; ++k) {
    // (a row of zeros: nothing is read but some row of the table, or none of an empty one)
    l[k] = place<T, true>(from[k] >= 0 ? (int)at[k] * kCols<T> : d, d);
    if (same || n_vocab > 0) in[k] = fetch(src + (from[k] >= 0 ? from[k] : 0) * lds, l[k]);
    else in[k] = Chunk{0u, 0u, 0u, 0u};
  }
#pragma unroll
  for (int k = 0; k < P; ++k) {
    if (o0 + (uint32_t)(k * kBlock) >= total) continue;
    const int c = (int)at[k] * kCols<T>;
    float v[kCols<T>];
    in[k] = settle(in[k], l[k]);
    if (kDrop) drop<T>(in[k], (uint32_t)c, row0 + row[k], m);
    widen<T>(in[k], v);
#pragma unroll
    for (int i = 0; i < kCols<T>; ++i) v[i] *= scale;
    store(out + (int64_t)row[k] * ldo + c, d - c, v, stream);
  }
}

// A launch takes rows as long as their chunks stay below 2^31.
template <typename T, typename Id>
toc_status map_rows(int64_t n, int32_t d, const Id *ids, int64_t n_vocab, const T *src, int64_t lds,
                    float scale, const toc_drop *drop, T *out, int64_t ldo, hipStream_t s) {
  const Mask m = mask_of(drop);
  scale *= m.keep;
  const uint32_t chunks = chunks_of<T>(d);
  const bool stream = stream_out(n, d, sizeof(T));
  const int64_t most = ((int64_t)1 << 30) / chunks;
  constexpr bool same = std::is_same<Id, Same>::value;
  for (int64_t r = 0; r < n; r += most) {
    const int64_t rows = std::min(most, n - r);
    const uint32_t total = (uint32_t)(rows * chunks);
    const dim3 grid((total + kBlock * kPer<Id> - 1) / (kBlock * kPer<Id>));
    const Id *i = same ? ids : ids + r;
    const T *x = same ? src + r * lds : src;
    T *y = out + r * ldo;
    if (m.on)
      hipLaunchKernelGGL((rows_kernel<T, Id, true>), grid, dim3(kBlock), 0, s, i, n_vocab, x, lds, scale,
                         m, (uint32_t)r, total, d, divisor(chunks), y, ldo, stream);
    else
      hipLaunchKernelGGL((rows_kernel<T, Id, false>), grid, dim3(kBlock), 0, s, i, n_vocab, x, lds, scale,
                         m, (uint32_t)r, total, d, divisor(chunks), y, ldo, stream);
  }
  return launched("rows_kernel");
}

template <typename Id>
toc_status map_typed(int32_t type, int64_t n, int32_t d, const void *ids, int64_t n_vocab,
                     const void *src, int64_t lds, float scale, const toc_drop *drop, void *out,
                     int64_t ldo, void *stream) {
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case TOC_F32:
      return map_rows(n, d, (const Id *)ids, n_vocab, (const float *)src, lds, scale, drop, (float *)out, ldo, s);
    case TOC_BF16:
      return map_rows(n, d, (const Id *)ids, n_vocab, (const bf16 *)src, lds, scale, drop, (bf16 *)out, ldo, s);
    default:
      return map_rows(n, d, (const Id *)ids, n_vocab, (const f16 *)src, lds, scale, drop, (f16 *)out, ldo, s);
  }
}

}  // namespace
}  // namespace rows
}  // namespace toc

using namespace toc;
using namespace toc::rows;

extern "C" {

toc_status toc_embed(int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab, int32_t d,
                     int32_t type, const void *E, int64_t lde, float scale, const toc_drop *drop,
                     void *out, int64_t ldo, void *stream) {
  clear_error();
  toc_status st;
  if ((st = check_sizes(n, d, type)) || (st = check_drop(drop)) ||
      (st = check_ids(n, ids, id_bits, n_vocab)) ||
      (st = check_rows("E", E, n_vocab, d, lde, type_size(type))) ||
      (st = check_rows("out", out, n, d, ldo, type_size(type))))
    return st;
  if ((st = check_scale(scale, drop))) return st;
  if (n == 0) return TOC_OK;
  if (id_bits == 32)
    return map_typed<int32_t>(type, n, d, ids, n_vocab, E, lde, scale, drop, out, ldo, stream);
  return map_typed<int64_t>(type, n, d, ids, n_vocab, E, lde, scale, drop, out, ldo, stream);
}

toc_status toc_dropout(int64_t n, int32_t d, int32_t type, const void *X, int64_t ldx,
                       const toc_drop *drop, void *Y, int64_t ldy, void *stream) {
  clear_error();
  toc_status st;
  if (!drop) return fail(TOC_EINVAL, "drop is NULL");
  if ((st = check_sizes(n, d, type)) || (st = check_drop(drop)) ||
      (st = check_rows("X", X, n, d, ldx, type_size(type))) ||
      (st = check_rows("Y", Y, n, d, ldy, type_size(type))))
    return st;
  if (n == 0) return TOC_OK;
  return map_typed<Same>(type, n, d, nullptr, 0, X, ldx, 1.0f, drop, Y, ldy, stream);
}

}  // extern "C"
