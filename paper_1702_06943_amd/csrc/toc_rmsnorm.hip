// Root-mean-square norm of rows with the residual's addition, and its gradient.
//   h = R + drop(X)       r = 1 / sqrt(mean_j h_j^2 + eps)       y_j = h_j r w_j
// for a row of d columns; 8-bit output: s = max(max_j |y_j|, 2^-100) / 448 and y_j / s as
// e4m3 numbers.  With g_j = dy_j w_j the gradients are
//   dh_j = r g_j - h_j r^3 mean_i(g_i h_i) + dR_j     dX = drop(dh)     dw_j = sum over rows dy_j h_j r
// A row stays in registers between its one read and its one write, as chunks of a group of
// lanes of one wave, or of the lanes of a workgroup.  Where groups walk over rows (long rows,
// and all rows on the way back), w and the group's part of dw stay in registers too.  Sums are
// binary32: a lane's chunks in order, then the lanes in a tree.
//   norm_kernel       bound by memory: 32,768 x 2,048 bf16 with dropout and residual 92 us, 5.8
//                     TB/s; 18,749 x 1,001 f16 rows of a wider matrix into e4m3 25 us, 5.2 TB/s
//   norm_grad_kernel  bound by memory, four or five streams at once: 32,768 x 2,048 bf16 with
//                     dropout 121 us, 5.6 TB/s with dw's parts (the call 127 us, 5.3 without)
//   norm_join_kernel  dw from the workgroups' rows, some 5 us of a call
#include "toc_rows_dev.h"

namespace toc {
namespace rows {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kLeastMax = 0x1p-100f;   // keeps 448 / max finite; a row of zeros gets a scale too

// The larger of a and b; NaN if either is, as the scale of a row that holds one has to be.
__device__ inline float max_nan(float a, float b) { return a > b || a != a ? a : b; }

// Sum over a group of kLanes lanes (kLanes <= 64: of one wave; else the whole workgroup, by
// way of kLanes / 64 words of lds), in every lane.  A caller's next use of the same words
// must lie behind another barrier of the workgroup.
template <int kLanes>
__device__ inline float group_sum(float x, float *lds) {
#pragma unroll
  for (int o = (kLanes < 64 ? kLanes : 64) / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  if (kLanes > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int i = 0; i < kLanes / 64; ++i) x += lds[i];
  }
  return x;
}
// Two sums at once; lds: two of kLanes / 64 pairs, used in turn.
template <int kLanes>
__device__ inline float2 group_sum2(float2 x, float2 *lds) {
#pragma unroll
  for (int o = (kLanes < 64 ? kLanes : 64) / 2; o > 0; o >>= 1) {
    x.x += __shfl_xor(x.x, o, 64);
    x.y += __shfl_xor(x.y, o, 64);
  }
  if (kLanes > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kLanes / 64; ++i) {
      x.x += lds[i].x;
      x.y += lds[i].y;
    }
  }
  return x;
}
template <int kLanes>
__device__ inline float group_max(float x, float *lds) {
#pragma unroll
  for (int o = (kLanes < 64 ? kLanes : 64) / 2; o > 0; o >>= 1) x = max_nan(x, __shfl_xor(x, o, 64));
  if (kLanes > 64) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < kLanes / 64; ++i) x = max_nan(x, lds[i]);
  }
  return x;
}

// A row's mean of d numbers is back times the sum of `by` times each of them.  by is a power of
// two and by d at most 1, so that the sum of d squares (or products) of binary32 numbers
// overflows no earlier than one of them, and has the bits it would have without by.
struct Mean {
  float by, back;
};
inline Mean mean_of(int32_t d) {
  float by = 1.0f;
  while (by * (float)d > 1.0f) by *= 0.5f;
  return Mean{by, 1.0f / (float)d / by};
}

__device__ inline float inv_rms(float sum, Mean mean, float eps) {
  return 1.0f / sqrtf(fmaf(sum, mean.back, eps));
}

template <typename T>
struct NormArgs {
  uint32_t n;
  int d;
  const T *X;
  int64_t ldx;
  const T *R;          // or NULL
  int64_t ldr;
  Mask m;
  const float *w;      // or NULL: ones
  float eps;
  Mean mean;
  T *H;                // or NULL
  int64_t ldh;
  int64_t ldy;
  float *y_scale;
  bool stream;
};

template <int kPer, int N>
__device__ inline void load_w(const float *w, int d, int lane, int lanes, float (&v)[kPer][N]) {
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int c = N * (lane + k * lanes);
#pragma unroll
    for (int i = 0; i < N; ++i) v[k][i] = c + i < d ? 1.0f : 0.0f;
    if (w && c < d) load(w + c, d - c, v[k]);
  }
}

// h = R + drop(X) and its norm; kLanes lanes to a row, kPer chunks to a lane (kCols kLanes kPer
// >= d).
template <typename T, typename Y, int kLanes, int kPer, bool kDrop>
__global__ __launch_bounds__(kLanes > 256 ? kLanes : 256) void norm_kernel(NormArgs<T> a, Y *Yp) {
  constexpr int kBlock = kLanes > 256 ? kLanes : 256;
  constexpr int kGroups = kBlock / kLanes;
  constexpr int N = kCols<T>;
  constexpr bool k8 = std::is_same<Y, E4m3>::value;
  __shared__ float part[2][kLanes > 64 ? kLanes / 64 : 1];
  const int lane = threadIdx.x % kLanes;
  float w[kPer][N];
  load_w(a.w, a.d, lane, kLanes, w);
  Place<T, kLanes == 8> l[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) l[k] = place<T, kLanes == 8>(N * (lane + k * kLanes), a.d);
  // (kLanes >= 64: all lanes of a wave, so all waves of a workgroup, share a row)
  for (uint32_t row = blockIdx.x * kGroups + threadIdx.x / kLanes; row < a.n; row += gridDim.x * kGroups) {
    float h[kPer][N];
    float sum = 0.0f, most = 0.0f;
    const T *x = a.X + (int64_t)row * a.ldx, *res = a.R + (int64_t)row * a.ldr;
    Chunk in[kPer], rin[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      in[k] = fetch(x, l[k]);
    }
    if (a.R) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        rin[k] = fetch(res, l[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      in[k] = settle(in[k], l[k]);
      if (kDrop) drop<T>(in[k], (uint32_t)(N * (lane + k * kLanes)), row, a.m);
      widen<T>(in[k], h[k]);
    }
    if (a.R) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        float v[N];
        rin[k] = settle(rin[k], l[k]);
        widen<T>(rin[k], v);
#pragma unroll
        for (int i = 0; i < N; ++i) h[k][i] = kDrop ? fmaf(h[k][i], a.m.keep, v[i]) : h[k][i] + v[i];
      }
    } else if (kDrop) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) h[k][i] *= a.m.keep;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
#pragma unroll
      for (int i = 0; i < N; ++i) sum = fmaf(h[k][i] * a.mean.by, h[k][i], sum);
      if (k8) {
#pragma unroll
        for (int i = 0; i < N; ++i) most = max_nan(fabsf(h[k][i] * w[k][i]), most);
      }
    }
    // (the row before may still be reading the other reduction's words, never these: a
    // barrier of that other reduction, or of this one, lies between)
    sum = group_sum<kLanes>(sum, part[0]);
    const float r = inv_rms(sum, a.mean, a.eps);
    float s = 1.0f;
    if (k8) {
      most = group_max<kLanes>(most, part[1]) * r;
      most = most < kLeastMax ? kLeastMax : most;
      s = kE4m3Max / most;
      if (lane == 0) a.y_scale[row] = most / kE4m3Max;
    } else if (kLanes > 64) {
      __syncthreads();   // part[0] is free again
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int c = N * (lane + k * kLanes);
      if (c >= a.d) continue;
      if (a.H) store(a.H + (int64_t)row * a.ldh + c, a.d - c, h[k], a.stream);
      float y[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        y[i] = h[k][i] * r * w[k][i];
        if (k8) {
          y[i] *= s;
          // rounding may leave the largest just above 448; NaN stays
          y[i] = y[i] > kE4m3Max ? kE4m3Max : y[i] < -kE4m3Max ? -kE4m3Max : y[i];
        }
      }
      store(Yp + (int64_t)row * a.ldy + c, a.d - c, y, a.stream);
    }
  }
}

template <typename T>
struct GradArgs {
  uint32_t n;
  int d;
  const T *H;
  int64_t ldh;
  const float *w;      // or NULL: ones
  float eps;
  Mean mean;
  const T *dY;
  int64_t lddy;
  const T *dR;         // or NULL
  int64_t lddr;
  Mask m;
  T *dH;               // or NULL
  int64_t lddh;
  T *dX;               // or NULL
  int64_t lddx;
  float *part;         // NULL, or one row of d per workgroup: its part of dw
  bool stream;
};

// dH, dX and the workgroup's part of dw.  r is formed again from h, whose sum of squares comes
// with the sum of g h: it need not be kept from the forward pass.
template <typename T, int kLanes, int kPer, bool kDrop>
__global__ __launch_bounds__(kLanes > 256 ? kLanes : 256) void norm_grad_kernel(GradArgs<T> a) {
  constexpr int kBlock = kLanes > 256 ? kLanes : 256;
  constexpr int kGroups = kBlock / kLanes;
  constexpr int N = kCols<T>;
  __shared__ float2 part[2][kLanes > 64 ? kLanes / 64 : 1];
  const int lane = threadIdx.x % kLanes;
  const uint32_t group = blockIdx.x * kGroups + threadIdx.x / kLanes;
  int turn = 0;
  float w[kPer][N], dw[kPer][N];
  load_w(a.w, a.d, lane, kLanes, w);
  Place<T, kLanes == 8> l[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) l[k] = place<T, kLanes == 8>(N * (lane + k * kLanes), a.d);
#pragma unroll
  for (int k = 0; k < kPer; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) dw[k][i] = 0.0f;
  // The next row's loads are under way while a row is worked on (not in the widest shapes, which
  // have no registers for it: 4,096 x 16,384 bf16 took 186 us with them, 115 without); past the
  // last row they are the last row's again, and without dR they are H's, so that no branch
  // hides how many are.
  constexpr bool kAheadRow = kLanes <= 256 || kPer == 1;
  const T *res = a.dR ? a.dR : a.H;
  const int64_t ldres = a.dR ? a.lddr : a.ldh;
  Chunk hin[kPer], gin[kPer], rin[kPer];
  auto request = [&](uint32_t row) {
    const int64_t at = (int64_t)min(row, a.n - 1);
#pragma unroll
    for (int k = 0; k < kPer; ++k) hin[k] = fetch(a.H + at * a.ldh, l[k]);
#pragma unroll
    for (int k = 0; k < kPer; ++k) gin[k] = fetch(a.dY + at * a.lddy, l[k]);
#pragma unroll
    for (int k = 0; k < kPer; ++k) rin[k] = fetch(res + at * ldres, l[k]);
  };
  if (kAheadRow) request(group);
  for (uint32_t row = group; row < a.n; row += gridDim.x * kGroups) {
    float h[kPer][N], g[kPer][N], dr[kPer][N];
    float2 sum = make_float2(0.0f, 0.0f);   // of h^2 and of g h
    if (!kAheadRow) request(row);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      widen<T>(settle(hin[k], l[k]), h[k]);
      widen<T>(settle(gin[k], l[k]), g[k]);
      if (kAheadRow) widen<T>(settle(rin[k], l[k]), dr[k]);
    }
    if (kAheadRow) request(row + gridDim.x * kGroups);
#pragma unroll
    for (int k = 0; k < kPer; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x = h[k][i] * a.mean.by;
        sum.x = fmaf(x, h[k][i], sum.x);
        sum.y = fmaf(g[k][i] * w[k][i], x, sum.y);
      }
    // (two rows' words: the row before this one's may still be read)
    sum = group_sum2<kLanes>(sum, part[turn]);
    turn ^= 1;
    const float r = inv_rms(sum.x, a.mean, a.eps);
    // dh = r g - (h r) (r mean(g h) r), whose factors stay in range where dh does: r^3 is 0 in
    // binary32 for |h| above 1e15, and infinite in a row of zeros for eps below 1e-26
    const float along = r * (sum.y * a.mean.back) * r;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int c = N * (lane + k * kLanes);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x = h[k][i] * r;
        dw[k][i] = fmaf(g[k][i], x, dw[k][i]);
        h[k][i] = fmaf(g[k][i] * w[k][i], r, -x * along);
      }
      if (c >= a.d) continue;
      if (a.dR) {
        if (!kAheadRow) widen<T>(settle(rin[k], l[k]), dr[k]);
#pragma unroll
        for (int i = 0; i < N; ++i) h[k][i] += dr[k][i];
      }
      if (a.dH) store(a.dH + (int64_t)row * a.lddh + c, a.d - c, h[k], a.stream);
      if (a.dX) {
        if (kDrop) {
#pragma unroll
          for (int i = 0; i < N; ++i) h[k][i] *= a.m.keep;
        }
        Chunk x = narrow<T>(h[k]);
        if (kDrop) drop<T>(x, (uint32_t)c, row, a.m);
        put(a.dX + (int64_t)row * a.lddx + c, a.d - c, x, a.stream);
      }
    }
  }
  if (!a.part) return;
  float *to = a.part + (int64_t)blockIdx.x * a.d;
  if (kGroups == 1) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int c = N * (lane + k * kLanes);
      if (c < a.d) store(to + c, a.d - c, dw[k], false);
    }
    return;
  }
  // the workgroup's groups, in order
  constexpr int kCols = N * kLanes * kPer;
  __shared__ float all[kGroups > 1 ? kGroups * kCols : 1];
#pragma unroll
  for (int k = 0; k < kPer; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) all[threadIdx.x / kLanes * kCols + N * (lane + k * kLanes) + i] = dw[k][i];
  __syncthreads();
  for (int c = threadIdx.x; c < a.d; c += kBlock) {
    float s = all[c];
#pragma unroll
    for (int g = 1; g < kGroups; ++g) s += all[g * kCols + c];
    to[c] = s;
  }
}

// dw (+)= the workgroups' parts, in their order: kJoinParts runs of them at once, then the
// runs.
constexpr int kJoinCols = 16, kJoinParts = 64;
__global__ __launch_bounds__(kJoinCols * kJoinParts) void norm_join_kernel(
    const float *__restrict__ part, int parts, int d, int accumulate, float *__restrict__ dw) {
  __shared__ float sums[kJoinParts][kJoinCols + 1];
  const int col = threadIdx.x % kJoinCols, p = threadIdx.x / kJoinCols;
  const int c = blockIdx.x * kJoinCols + col;
  const int per = (parts + kJoinParts - 1) / kJoinParts;
  float s = 0.0f;
  if (c < d) {
    const int end = min(parts, (p + 1) * per);
#pragma unroll 8
    for (int g = p * per; g < end; ++g) s += part[(int64_t)g * d + c];
  }
  sums[p][col] = s;
  __syncthreads();
#pragma unroll
  for (int n = kJoinParts / 2; n > 0; n /= 2) {
    if (p < n) sums[p][col] += sums[p + n][col];
    __syncthreads();
  }
  if (p == 0 && c < d) dw[c] = accumulate ? dw[c] + sums[0][col] : sums[0][col];
}

// Lanes to a row and chunks to a lane (us: 32,768 x 2,048 bf16 forward by 256 x 1 92, 64 x 4 102;
// 18,749 x 1,001 f16 by 64 x 2 28, 256 x 1 36; 8,192 x 8,192 bf16 with dropout by 512 x 2 88,
// 1,024 x 1 119, backward 135 and 128).  The widest binary32 rows hold 16 numbers of each stream
// a lane, and spill on the way back: 2,000 x 16,384 forward 88, 6.0 TB/s, backward with dropout
// 170, 3.9 TB/s.
struct Shape {
  int lanes, per;
};
constexpr int32_t kMaxCols = 16384;
Shape shape_of(uint32_t chunks, bool grad) {
  if (chunks <= 8) return {8, 1};
  if (chunks <= 32) return {32, 1};
  if (chunks <= 64) return {64, 1};
  if (chunks <= 128) return {64, 2};
  if (chunks <= 256) return {256, 1};
  if (chunks <= 512) return {256, 2};
  if (chunks <= 1024) return grad ? Shape{1024, 1} : Shape{512, 2};
  if (chunks <= 2048) return {1024, 2};
  return {1024, 4};   // binary32 only
}
// F(lanes, per) for each shape that rows of T can take
#define TOC_SHAPES(F) F(8, 1) F(32, 1) F(64, 1) F(64, 2) F(256, 1) F(256, 2) F(1024, 2)

// Workgroups of a launch: as many as the rows need, at most `most`.  Forward, rows of at most
// 256 lanes get a workgroup each (32,768 x 2,048 bf16 with dropout: 93.5 us, 101 with 4,096
// workgroups that walk), longer ones walk (8,192 x 8,192: 93 us, 98.5 with a workgroup each).
// Backward all walk, since each workgroup leaves a row of dw's parts, 512 of them (us for 1,024,
// 768, 512: 32,768 x 2,048 bf16 with dropout 132, 127, 127; 8,192 x 4,096 bf16 63.5, 58.5, 55.5;
// 18,750 x 300 f32 21.4, 21.9, 21.8), short rows 1,024 (100,000 x 64 bf16 15.3, 16.1, 15.9).
// (Few long rows pay for their parts: 1,000 x 4,096 bf16 without dropout 16.0 us, 6.9 without dw.)
int64_t blocks_for(int64_t n, Shape sh, int64_t most) {
  const int64_t groups = sh.lanes > 256 ? 1 : 256 / sh.lanes;
  return std::max<int64_t>(1, std::min((n + groups - 1) / groups, most));
}
int64_t norm_blocks(int64_t n, Shape sh) { return blocks_for(n, sh, sh.lanes > 256 ? 1024 : 1 << 22); }
int64_t grad_blocks(int64_t n, Shape sh) {
  return blocks_for(n, sh, sh.lanes > 256 ? 256 : sh.lanes < 64 ? 1024 : 512);
}

template <typename T, typename Y>
toc_status norm(const NormArgs<T> &a, Y *y, hipStream_t s) {
  const Shape sh = shape_of(chunks_of<T>(a.d), false);
  const dim3 grid((unsigned)norm_blocks(a.n, sh)), block((unsigned)std::max(sh.lanes, 256));
#define TOC_NORM(L, K)                                                                     \
  if (sh.lanes == L && sh.per == K) {                                                      \
    if (a.m.on)                                                                           \
      hipLaunchKernelGGL((norm_kernel<T, Y, L, K, true>), grid, block, 0, s, a, y);        \
    else                                                                                   \
      hipLaunchKernelGGL((norm_kernel<T, Y, L, K, false>), grid, block, 0, s, a, y);       \
  }
  TOC_SHAPES(TOC_NORM)
  TOC_NORM(512, 2)
  if constexpr (sizeof(T) == 4) {
    TOC_NORM(1024, 4)
  }
#undef TOC_NORM
  return launched("norm_kernel");
}

template <typename T>
toc_status norm_grad(const GradArgs<T> &a, hipStream_t s) {
  const Shape sh = shape_of(chunks_of<T>(a.d), true);
  const dim3 grid((unsigned)grad_blocks(a.n, sh)), block((unsigned)std::max(sh.lanes, 256));
#define TOC_GRAD(L, K)                                                                     \
  if (sh.lanes == L && sh.per == K) {                                                      \
    if (a.m.on)                                                                           \
      hipLaunchKernelGGL((norm_grad_kernel<T, L, K, true>), grid, block, 0, s, a);         \
    else                                                                                   \
      hipLaunchKernelGGL((norm_grad_kernel<T, L, K, false>), grid, block, 0, s, a);        \
  }
  TOC_SHAPES(TOC_GRAD)
  TOC_GRAD(1024, 1)
  if constexpr (sizeof(T) == 4) {
    TOC_GRAD(1024, 4)
  }
#undef TOC_GRAD
  return launched("norm_grad_kernel");
}

// Rows of partial dw sums a call leaves in its workspace.
template <typename T>
int64_t grad_parts(int64_t n, int32_t d) {
  return n ? grad_blocks(n, shape_of(chunks_of<T>(d), true)) : 0;
}
int64_t grad_parts(int64_t n, int32_t d, int32_t type) {
  return type == TOC_F32 ? grad_parts<float>(n, d) : grad_parts<bf16>(n, d);
}

template <typename T>
toc_status norm_typed(int64_t n, int32_t d, const void *X, int64_t ldx, const void *R, int64_t ldr,
                      const toc_drop *drop, const float *w, float eps, void *H, int64_t ldh, void *Y,
                      int64_t ldy, bool eight, float *y_scale, void *stream) {
  const NormArgs<T> a{(uint32_t)n, d, (const T *)X, ldx, (const T *)R, ldr, mask_of(drop), w, eps,
                      mean_of(d), (T *)H, ldh, ldy, y_scale, stream_out(n, d, sizeof(T))};
  if (eight) return norm(a, (E4m3 *)Y, (hipStream_t)stream);
  return norm(a, (T *)Y, (hipStream_t)stream);
}

template <typename T>
toc_status grad_typed(int64_t n, int32_t d, const void *H, int64_t ldh, const float *w, float eps,
                      const void *dY, int64_t lddy, const void *dR, int64_t lddr, const toc_drop *drop,
                      void *dH, int64_t lddh, void *dX, int64_t lddx, float *part, void *stream) {
  const GradArgs<T> a{(uint32_t)n, d, (const T *)H, ldh, w, eps, mean_of(d), (const T *)dY, lddy,
                      (const T *)dR, lddr, mask_of(drop), (T *)dH, lddh, (T *)dX, lddx, part,
                      stream_out(n, d, sizeof(T))};
  return norm_grad(a, (hipStream_t)stream);
}

toc_status check_norm(int64_t n, int32_t d, int32_t type, const float *w, float eps) {
  if (const toc_status st = check_sizes(n, d, type)) return st;
  if (d > kMaxCols) return fail(TOC_EUNSUPPORTED, "rows of more than %d columns", kMaxCols);
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail(TOC_EINVAL, "eps must be positive and finite");
  if ((uintptr_t)w % 4) return fail(TOC_EINVAL, "w is not aligned to its elements");
  return TOC_OK;
}

}  // namespace
}  // namespace rows
}  // namespace toc

using namespace toc;
using namespace toc::rows;

extern "C" {

toc_status toc_rmsnorm(int64_t n, int32_t d, int32_t type, const void *X, int64_t ldx, const void *R,
                       int64_t ldr, const toc_drop *drop, const float *w, float eps, void *H,
                       int64_t ldh, int32_t y_type, void *Y, int64_t ldy, float *y_scale,
                       void *stream) {
  clear_error();
  toc_status st;
  if ((st = check_norm(n, d, type, w, eps)) || (st = check_drop(drop))) return st;
  if (y_type != type && y_type != TOC_E4M3)
    return fail(TOC_EINVAL, "the output's type is the input's or TOC_E4M3, not %d", y_type);
  const bool eight = y_type == TOC_E4M3;
  const int size = type_size(type);
  if ((st = check_rows("X", X, n, d, ldx, size)) || (R && (st = check_rows("R", R, n, d, ldr, size))) ||
      (H && (st = check_rows("H", H, n, d, ldh, size))) ||
      (st = check_rows("Y", Y, n, d, ldy, eight ? 1 : size)))
    return st;
  if (eight && n > 0 && !y_scale) return fail(TOC_EINVAL, "y_scale is NULL");
  if ((uintptr_t)y_scale % 4) return fail(TOC_EINVAL, "y_scale is not aligned to its elements");
  if (n == 0) return TOC_OK;
  switch (type) {
    case TOC_F32:
      return norm_typed<float>(n, d, X, ldx, R, ldr, drop, w, eps, H, ldh, Y, ldy, eight, y_scale, stream);
    case TOC_BF16:
      return norm_typed<bf16>(n, d, X, ldx, R, ldr, drop, w, eps, H, ldh, Y, ldy, eight, y_scale, stream);
    default:
      return norm_typed<f16>(n, d, X, ldx, R, ldr, drop, w, eps, H, ldh, Y, ldy, eight, y_scale, stream);
  }
}

toc_status toc_rmsnorm_grad_workspace_size(int64_t n, int32_t d, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(TOC_EINVAL, "bytes is NULL");
  if (const toc_status st = check_norm(n, d, TOC_F32, nullptr, 1.0f)) return st;
  *bytes = (size_t)std::max(grad_parts<float>(n, d), grad_parts<bf16>(n, d)) * (size_t)d * 4;
  return TOC_OK;
}

toc_status toc_rmsnorm_grad(int64_t n, int32_t d, int32_t type, const void *H, int64_t ldh,
                            const float *w, float eps, const void *dY, int64_t lddy, const void *dR,
                            int64_t lddr, const toc_drop *drop, void *dH, int64_t lddh, void *dX,
                            int64_t lddx, float *dw, int32_t accumulate, void *ws, size_t ws_bytes,
                            void *stream) {
  clear_error();
  toc_status st;
  if ((st = check_norm(n, d, type, w, eps)) || (st = check_drop(drop))) return st;
  const int size = type_size(type);
  if ((st = check_rows("H", H, n, d, ldh, size)) || (st = check_rows("dY", dY, n, d, lddy, size)) ||
      (dR && (st = check_rows("dR", dR, n, d, lddr, size))) ||
      (dH && (st = check_rows("dH", dH, n, d, lddh, size))) ||
      (dX && (st = check_rows("dX", dX, n, d, lddx, size))))
    return st;
  if ((uintptr_t)dw % 4) return fail(TOC_EINVAL, "dw is not aligned to its elements");
  if (dw) {
    const size_t need = (size_t)grad_parts(n, d, type) * (size_t)d * 4;
    if (need && !ws) return fail(TOC_EINVAL, "workspace is NULL");
    if (ws_bytes < need) return fail(TOC_ESIZE, "workspace of %zu bytes below the %zu needed", ws_bytes, need);
    if ((uintptr_t)ws % 4) return fail(TOC_EINVAL, "workspace is not 4-byte aligned");
  }
  float *part = dw ? (float *)ws : nullptr;
  if (n > 0) {
    switch (type) {
      case TOC_F32:
        st = grad_typed<float>(n, d, H, ldh, w, eps, dY, lddy, dR, lddr, drop, dH, lddh, dX, lddx, part, stream);
        break;
      case TOC_BF16:
        st = grad_typed<bf16>(n, d, H, ldh, w, eps, dY, lddy, dR, lddr, drop, dH, lddh, dX, lddx, part, stream);
        break;
      default:
        st = grad_typed<f16>(n, d, H, ldh, w, eps, dY, lddy, dR, lddr, drop, dH, lddh, dX, lddx, part, stream);
    }
    if (st) return st;
  }
  if (!dw) return TOC_OK;
  hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((d + kJoinCols - 1) / kJoinCols)),
                     dim3(kJoinCols * kJoinParts), 0, (hipStream_t)stream, part,
                     (int)grad_parts(n, d, type), d, accumulate, dw);
  return launched("norm_join_kernel");
}

}  // extern "C"
