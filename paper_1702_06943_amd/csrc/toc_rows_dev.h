// What the row operators share (embedding lookup and gradient, dropout, root-mean-square
// norm): rows of binary32, bfloat16 or binary16 numbers read and written 16 bytes (a chunk of
// 4 or 8 columns) a lane, computed in binary32, and the dropout mask.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "toc_internal.h"

namespace toc {
namespace rows {

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;   // a row's number is one 32-bit counter word

// --- host ------------------------------------------------------------------

inline bool type_ok(int32_t type) { return type == TOC_F32 || type == TOC_BF16 || type == TOC_F16; }
inline int type_size(int32_t type) { return type == TOC_F32 ? 4 : 2; }

// A dropout mask as the kernels take it.  An element is dropped when its 16-bit word is
// below round(65536 p): p is taken to the nearest 2^-16, and 65536 / (65536 - that) makes the
// kept elements' mean the input's exactly at that p.
struct Mask {
  uint32_t k0, k1, s0, s1;   // seed (the key) and mask number, low word first
  uint32_t last;             // the largest word that drops
  uint32_t limit;            // last in both halves, as signed numbers of the same order
  float keep;                // what a kept element is multiplied by; 1 where `on` is not set
  bool on;                   // whether any word drops
};

inline Mask mask_of(const toc_drop *drop) {
  Mask m{};
  m.keep = 1.0f;
  if (!drop) return m;
  const uint32_t below = (uint32_t)std::lrint((double)drop->p * 65536.0);
  if (below == 0) return m;
  m.k0 = (uint32_t)drop->seed;
  m.k1 = (uint32_t)(drop->seed >> 32);
  m.s0 = (uint32_t)drop->mask;
  m.s1 = (uint32_t)(drop->mask >> 32);
  m.last = below - 1;
  m.limit = (m.last ^ 0x8000u) * 0x10001u;
  m.keep = below < 65536u ? (float)(65536.0 / (65536.0 - (double)below)) : 0.0f;
  m.on = true;
  return m;
}

// The checks of one matrix argument of n rows and d columns.
inline toc_status check_rows(const char *name, const void *p, int64_t n, int32_t d, int64_t ld,
                             int size) {
  if (n > 0 && !p) return fail(TOC_EINVAL, "%s is NULL", name);
  if (ld < d)
    return fail(TOC_EINVAL, "row stride %lld of %s below %d columns", (long long)ld, name, d);
  if ((uintptr_t)p % (uintptr_t)size)
    return fail(TOC_EINVAL, "%s is not aligned to its %d-byte elements", name, size);
  return TOC_OK;
}

inline toc_status check_drop(const toc_drop *drop) {
  if (drop && !(drop->p >= 0.0f && drop->p <= 1.0f))
    return fail(TOC_EINVAL, "dropout probability outside 0..1");
  return TOC_OK;
}

// The scale and the kept elements' factor are one product.
inline toc_status check_scale(float scale, const toc_drop *drop) {
  if (!std::isfinite(scale * mask_of(drop).keep))
    return fail(TOC_EINVAL, "scale, times the mask's factor, not finite");
  return TOC_OK;
}

inline toc_status check_sizes(int64_t n, int32_t d, int32_t type) {
  if (n < 0 || d < 1) return fail(TOC_EINVAL, "%lld rows of %d columns", (long long)n, d);
  if (!type_ok(type)) return fail(TOC_EINVAL, "unknown element type %d", type);
  if (n > kMaxRows) return fail(TOC_EUNSUPPORTED, "more than 2^31-1 rows");
  if (d > 1 << 28) return fail(TOC_EUNSUPPORTED, "rows of more than 2^28 columns");
  return TOC_OK;
}

inline toc_status check_ids(int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab) {
  if (id_bits != 32 && id_bits != 64)
    return fail(TOC_EINVAL, "token numbers have 32 or 64 bits, not %d", id_bits);
  if (n > 0 && !ids) return fail(TOC_EINVAL, "ids is NULL");
  if ((uintptr_t)ids % (uintptr_t)(id_bits / 8)) return fail(TOC_EINVAL, "ids is not aligned to its elements");
  if (n_vocab < 0) return fail(TOC_EINVAL, "%lld table rows", (long long)n_vocab);
  if (n_vocab > kMaxRows) return fail(TOC_EUNSUPPORTED, "more than 2^31-1 table rows");
  return TOC_OK;
}

inline toc_status launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TOC_OK : fail(TOC_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Whether a call's output is written past the caches: from 8 MB on it is larger than what the
// next call would find there, and the rows still to be read get their room (us, non-temporal
// and not: lookup of 32,768 x 1,024 f32 27.5, 49.0; norm of 60,000 x 300 f32 53, 67; lookup, two
// norms and two matrix products of 256, 1,024, 4,096, 16,384 rows of 1,024 bf16 31.6, 27.0;
// 35.9, 32.5; 48.8, 49.5; 118.7, 118.8).
inline bool stream_out(int64_t n, int64_t d, int64_t size) { return n * d * size >= (int64_t)8 << 20; }

// Division of o < 2^31 by a divisor known on the host: floor(2^32 / divisor) times o, high
// word, is the quotient or one less.
struct Divisor {
  uint32_t d, inv;
};
inline Divisor divisor(uint32_t d) {
  return Divisor{d, d > 1 ? (uint32_t)(((uint64_t)1 << 32) / d) : 0xffffffffu};
}
__device__ inline uint32_t divide(uint32_t o, Divisor by, uint32_t *rest) {
  uint32_t q = __umulhi(o, by.inv), r = o - q * by.d;
  if (r >= by.d) {
    ++q;
    r -= by.d;
  }
  *rest = r;
  return q;
}

// --- elements ----------------------------------------------------------------

typedef __bf16 bf16;
typedef _Float16 f16;

// Columns of a chunk.  With 8 of binary32, in two loads a lane, neighbouring lanes' loads are
// 32 bytes apart and a large map runs at 5.0 TB/s where 4 columns reach 5.8.
template <typename T>
constexpr int kCols = 16 / (int)sizeof(T);

template <typename T>
inline uint32_t chunks_of(int32_t d) {
  return (uint32_t)((d + kCols<T> - 1) / kCols<T>);
}

// Rows start wherever the caller's strides put them, so a chunk is aligned to its elements
// only; the hardware takes 16-byte loads and stores at such addresses.
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));
typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));

// Where a lane reads its chunk of a row of d columns, from column c on: the last chunk of a
// row is read as the row's last 16 bytes and shifted down, so that all lanes' loads are one
// instruction without a branch.  Rows shorter than a chunk are read by the element; kTiny
// says whether there can be such.
template <typename T, bool kTiny>
struct Place {
  int at, shift;      // first column read; columns to shift down by, kCols: nothing is left
  int tiny;           // 0, or the row's columns
};
template <typename T, bool kTiny>
__device__ inline Place<T, kTiny> place(int c, int d) {
  if (kTiny && d < kCols<T>) return Place<T, kTiny>{0, c < d ? 0 : kCols<T>, d};
  const int shift = min(max(c + kCols<T> - d, 0), kCols<T>);
  return Place<T, kTiny>{shift < kCols<T> ? c - shift : 0, shift, 0};
}

// The chunk as it lies in memory.  Nothing here uses what is loaded, so that the loads of
// several chunks can fly together; settle() comes before its use.
template <typename T, bool kTiny>
__device__ inline Chunk fetch(const T *row, const Place<T, kTiny> &l) {
  if (!kTiny || !l.tiny) return *(const Unaligned *)(row + l.at);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < kCols<T> - 1; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = i < l.tiny ? ((const uint32_t *)row)[i] : 0u;
    else w[i / 2] |= (i < l.tiny ? (uint32_t)((const uint16_t *)row)[i] : 0u) << (16 * (i % 2));
  }
  return Chunk{w[0], w[1], w[2], w[3]};
}

// The lane's own columns first, 0 in those past the row's end.
template <typename T, bool kTiny>
__device__ inline Chunk settle(Chunk c, const Place<T, kTiny> &l) {
  if (l.shift) {
    const int bits = l.shift * 8 * (int)sizeof(T);
    if (bits & 64) c = Chunk{c[2], c[3], 0u, 0u};
    if (bits & 32) c = Chunk{c[1], c[2], c[3], 0u};
    if (sizeof(T) == 2 && (bits & 16))
      c = Chunk{c[0] >> 16 | c[1] << 16, c[1] >> 16 | c[2] << 16, c[2] >> 16 | c[3] << 16, c[3] >> 16};
    if (bits & 128) c = Chunk{0u, 0u, 0u, 0u};
  }
  return c;
}

template <typename T>
__device__ inline void widen(Chunk c, float (&v)[kCols<T>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      v[i] = __uint_as_float(c[i]);
    } else if constexpr (std::is_same<T, bf16>::value) {
      v[2 * i] = __uint_as_float(c[i] << 16);
      v[2 * i + 1] = __uint_as_float(c[i] & 0xffff0000u);
    } else {
      v[2 * i] = (float)__builtin_bit_cast(T, (uint16_t)c[i]);
      v[2 * i + 1] = (float)__builtin_bit_cast(T, (uint16_t)(c[i] >> 16));
    }
  }
}

// N numbers (N: 4 or 8), columns 0..left-1 of them (the others read as 0, and are not
// written): as binary32, a chunk at a time; as T, to nearest even, a NaN staying one.
template <typename T, int N>
__device__ inline void load(const T *p, int left, float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += kCols<T>) {
    float x[kCols<T>];
    if (left - j >= kCols<T>) {
      widen<T>(*(const Unaligned *)(p + j), x);
    } else {
#pragma unroll
      for (int i = 0; i < kCols<T>; ++i) x[i] = i < left - j ? (float)p[j + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kCols<T>; ++i) v[j + i] = x[i];
  }
}

template <typename T>
__device__ inline Chunk narrow(const float *v) {
  typedef float Two __attribute__((ext_vector_type(2)));
  Chunk c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      c[i] = __float_as_uint(v[i]);
    } else {
      typedef T TwoT __attribute__((ext_vector_type(2)));
      const Two x = {v[2 * i], v[2 * i + 1]};
      c[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, TwoT));
    }
  }
  return c;
}

// stream: non-temporal, as stream_out() has it.  (The empty statements keep the compiler from
// making one ordinary store of the two.)
template <typename T>
__device__ inline void put(T *p, int left, Chunk c, bool stream) {
  if (left >= kCols<T>) {
    if (stream) {
      __builtin_nontemporal_store((Unaligned)c, (Unaligned *)p);
    } else {
      asm volatile("");
      *(Unaligned *)p = c;
      asm volatile("");
    }
  } else {
#pragma unroll
    for (int i = 0; i < kCols<T> - 1; ++i) {
      if (i >= left) continue;
      if (sizeof(T) == 4) ((uint32_t *)p)[i] = c[i];
      else ((uint16_t *)p)[i] = (uint16_t)(c[i / 2] >> (16 * (i % 2)));
    }
  }
}

// A lane's N columns in more than one chunk lie 32 bytes from its neighbour's: those stores
// have to meet in the cache (non-temporal, a gradient of 131,072 distinct bf16 rows of 1,024
// into binary32 took 479 us, 316 with these).
template <typename T, int N>
__device__ inline void store(T *p, int left, const float (&v)[N], bool stream) {
#pragma unroll
  for (int j = 0; j < N; j += kCols<T>) put(p + j, left - j, narrow<T>(v + j), stream && N == kCols<T>);
}

struct E4m3 {
  uint8_t b;
};

// N numbers of magnitude at most 448 as e4m3 numbers, rounded to nearest even.
template <int N>
__device__ inline void store(E4m3 *p, int left, const float (&v)[N], bool) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], x, true);
    w[i] = (uint32_t)x;
  }
  if (left >= N) {
    __builtin_memcpy(p, w, N);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < left) p[i].b = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// --- the mask ------------------------------------------------------------------

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011): ten rounds of two 32 x 32 -> 64 bit products on a 128-bit counter.  The counter
// is (eight columns of the row, row, mask number), the key the seed, and the 128 bits are eight
// 16-bit words, one per column: the mask depends on neither strides, launch shape nor type,
// so a gradient makes the one its forward pass used again.  v_mad_u64_u32 gives both words
// of a product at the full rate; with the three-way XOR as one v_bitop3_b32 (truth table
// 0x96) a block takes some 49 instructions, 799 G blocks/s (587 with two XORs, 450 with
// separate high and low products).
__device__ inline uint4 philox(uint32_t eight, uint32_t row, const Mask &m) {
  uint32_t c0 = eight, c1 = row, c2 = m.s0, c3 = m.s1, k0 = m.k0, k1 = m.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96);
    c1 = (uint32_t)b;
    c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Clears the dropped elements of the chunk of row `row` from column c on: cleared and not
// multiplied by 0, so a dropped infinity or NaN is 0.  The caller multiplies by m.keep.  Two
// bytes an element: word i of the block holds the words of the elements in word i of the
// chunk, compared two at a time by the sign of a saturated 16-bit difference.  Four: half of
// the block's words are the chunk's.
template <typename T>
__device__ inline void drop(Chunk &x, uint32_t c, uint32_t row, const Mask &m) {
  const uint4 w = philox(c / 8, row, m);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 4) {
    const bool high = c & 4u;
    const uint32_t lo = high ? u[2] : u[0], hi = high ? u[3] : u[1];
    x[0] = (lo & 0xffffu) > m.last ? x[0] : 0u;
    x[1] = (lo >> 16) > m.last ? x[1] : 0u;
    x[2] = (hi & 0xffffu) > m.last ? x[2] : 0u;
    x[3] = (hi >> 16) > m.last ? x[3] : 0u;
  } else {
    typedef int16_t Two __attribute__((ext_vector_type(2)));
    const Two limit = __builtin_bit_cast(Two, m.limit);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Two word = __builtin_bit_cast(Two, u[i] ^ 0x80008000u);
      const Two kept = __builtin_elementwise_sub_sat(limit, word) >> 15;
      x[i] &= __builtin_bit_cast(uint32_t, kept);
    }
  }
}

}  // namespace rows
}  // namespace toc
