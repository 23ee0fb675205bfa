// Gradient of the embedding lookup by sorted token numbers:
//   dE[v, :] (+)= scale * sum of drop(G)[t, :] over the tokens t with ids[t] = v
// the left product G^T.A (Theorem 2) of tuples that hold one pair each, in a fixed order:
//   sort   (number, token) pairs stably by number, 9 bits or fewer a pass: each tile's count
//          of every digit (count_kernel), then each tile places its pairs (scatter_kernel);
//          numbers outside the table sort last, as number V
//   sum    the sorted list cut into chunks of equal length, so that a frequent number costs
//          no more than others: a group of lanes walks a chunk, its chunks of dE's row in
//          registers, and writes a row when its number ends.  A number that crosses chunks
//          leaves one partial row in each
//   join   partial rows added in the chunks' order
//   zero   rows of numbers that do not occur (unless accumulating)
// Bound by memory: G is read once and every row of dE written once.
#include "toc_rows_dev.h"

namespace toc {
namespace rows {
namespace {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64;
constexpr int kMaxBits = 9;                  // digit bits a pass
constexpr int64_t kMaxTiles = 256;
constexpr int kSumBlock = 256;
constexpr int kAhead = 8;                    // entries whose rows' loads fly together
constexpr int kZeroBlock = 256, kZeroPer = 4;
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr int32_t kMaxGradCols = 1 << 20;

// The sort's shape, the chunks and where the workspace's parts lie (bytes).
struct Plan {
  int bits, passes;       // digit bits of a pass
  int64_t tile, tiles;    // entries of a tile
  int64_t chunk, chunks;  // entries of a chunk
  size_t key[2], pos[2], count, present, part, end;
};

size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

Plan plan_of(int64_t n, int64_t n_vocab, int32_t d) {
  Plan p{};
  int width = 1;                             // bits of the numbers 0..V
  while (width < 32 && ((int64_t)1 << width) <= n_vocab) ++width;
  p.passes = (width + kMaxBits - 1) / kMaxBits;
  p.bits = (width + p.passes - 1) / p.passes;
  p.tiles = std::max<int64_t>(1, std::min(kMaxTiles, (n + 2047) / 2048));
  p.tile = ((n + p.tiles - 1) / p.tiles + kSortBlock - 1) / kSortBlock * kSortBlock;
  p.chunk = std::max<int64_t>(16, std::min<int64_t>((n + 4095) / 4096, 64));
  p.chunk = std::max(p.chunk, (n + (1 << 22) - 1) >> 22);
  p.chunks = (n + p.chunk - 1) / p.chunk;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = align16(at + bytes);
    return here;
  };
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take((size_t)n * 4);
    p.pos[i] = take((size_t)n * 4);
  }
  p.count = take((size_t)p.tiles << (p.bits + 2));
  p.present = take((size_t)n_vocab);
  p.part = take((size_t)p.chunks * 2 * (size_t)d * 4);
  p.end = at;
  return p;
}

template <typename Id>
__device__ inline uint32_t key_at(const Id *ids, uint32_t i, uint32_t n_vocab) {
  const int64_t id = (int64_t)ids[i];
  return id >= 0 && id < (int64_t)n_vocab ? (uint32_t)id : n_vocab;
}
__device__ inline uint32_t key_at(const uint32_t *keys, uint32_t i, uint32_t) { return keys[i]; }

// Workgroups 0..tiles-1: the tile's count of each digit.  The others (first pass only) clear
// `present`, which the first scatter fills.
template <typename Id>
__global__ __launch_bounds__(kSortBlock) void count_kernel(const Id *__restrict__ ids, uint32_t n,
                                                           uint32_t n_vocab, uint32_t tile,
                                                           uint32_t tiles, int shift, int bits,
                                                           uint32_t *__restrict__ count,
                                                           uint8_t *__restrict__ present) {
  __shared__ uint32_t c[1 << kMaxBits];
  if (blockIdx.x >= tiles) {
    // (the workspace keeps `present` 16-byte aligned and rounded up)
    const uint32_t words = (n_vocab + 3u) / 4u;
    for (uint32_t i = (blockIdx.x - tiles) * kSortBlock + threadIdx.x; i < words;
         i += (gridDim.x - tiles) * kSortBlock)
      ((uint32_t *)present)[i] = 0u;
    return;
  }
  const uint32_t digits = 1u << bits;
  for (uint32_t i = threadIdx.x; i < digits; i += kSortBlock) c[i] = 0u;
  __syncthreads();
  const uint32_t end = min(n, (blockIdx.x + 1) * tile);
  for (uint32_t i = blockIdx.x * tile + threadIdx.x; i < end; i += kSortBlock)
    atomicAdd(&c[key_at(ids, i, n_vocab) >> shift & (digits - 1)], 1u);
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < digits; i += kSortBlock)
    count[(size_t)blockIdx.x * digits + i] = c[i];
}

// Places a tile's entries.  A digit's entries of this tile start after all entries of lower
// digits and this digit's of earlier tiles; inside the tile each wave owns a run of entries,
// and a wave's 64 entries are ranked by comparing digits across its lanes, so equal digits
// keep their order.
template <typename Id, bool kFirst>
__global__ __launch_bounds__(kSortBlock) void scatter_kernel(
    const Id *__restrict__ ids, const uint32_t *__restrict__ pos, uint32_t n, uint32_t n_vocab,
    uint32_t tile, uint32_t tiles, int shift, int bits, const uint32_t *__restrict__ count,
    uint32_t *__restrict__ key_out, uint32_t *__restrict__ pos_out, uint8_t *__restrict__ present) {
  __shared__ uint32_t at[kSortWaves][1 << kMaxBits];
  __shared__ uint32_t wave_sum[kSortWaves];
  const uint32_t digits = 1u << bits;
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (uint32_t i = threadIdx.x; i < kSortWaves * (1u << kMaxBits); i += kSortBlock) (&at[0][0])[i] = 0u;
  uint32_t before = 0, total = 0;
  if (threadIdx.x < digits) {
#pragma unroll 8
    for (uint32_t t = 0; t < tiles; ++t) {
      const uint32_t x = count[(size_t)t * digits + threadIdx.x];
      before += t < blockIdx.x ? x : 0u;
      total += x;
    }
  }
  uint32_t incl = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(incl, o, 64);
    if ((int)lane >= o) incl += x;
  }
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  uint32_t base = incl - total + before;
  for (uint32_t w = 0; w < wave; ++w) base += wave_sum[w];
  const uint32_t per = tile / kSortWaves;
  const uint64_t first = (uint64_t)blockIdx.x * tile + (uint64_t)wave * per;
  const uint32_t i0 = (uint32_t)min(first, (uint64_t)n), i1 = (uint32_t)min(first + per, (uint64_t)n);
  for (uint32_t i = i0 + lane; i < i1; i += 64)
    atomicAdd(&at[wave][key_at(ids, i, n_vocab) >> shift & (digits - 1)], 1u);
  __syncthreads();
  if (threadIdx.x < digits) {
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t x = at[w][threadIdx.x];
      at[w][threadIdx.x] = base;
      base += x;
    }
  }
  __syncthreads();
  for (uint32_t s = i0; s < i1; s += 64) {
    const uint32_t i = s + lane;
    const bool in = i < i1;
    const uint32_t key = in ? key_at(ids, i, n_vocab) : 0u;
    const uint32_t digit = key >> shift & (digits - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
      const uint64_t ones = __ballot(digit >> b & 1u);
      same &= digit >> b & 1u ? ones : ~ones;
    }
    const uint32_t rank = (uint32_t)__popcll(same & (((uint64_t)1 << lane) - 1));
    if (in) {
      const uint32_t to = at[wave][digit] + rank;
      key_out[to] = key;
      pos_out[to] = kFirst ? i : pos[i];
      if (kFirst && key < n_vocab) present[key] = 1;
    }
    // all lanes have read their digit's place before its first entry's lane moves it on
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && rank == 0) at[wave][digit] += (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <typename T>
struct SumArgs {
  const uint32_t *key, *pos;
  uint32_t n, n_vocab, chunk, chunks;
  int d, lanes;
  const T *G;
  int64_t ldg;
  float scale;
  Mask m;
  float *part;
  int accumulate;
};

template <typename TO, int N>
__device__ inline void write_row(TO *p, int left, float (&v)[N], float scale, int accumulate) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] *= scale;
  if (accumulate) {
    float old[N];
    load((const TO *)p, left, old);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += old[i];
  }
  store(p, left, v);
}

// Chunk blockIdx.x * (256 / lanes) + group, columns from kCols lanes blockIdx.y.
template <typename T, typename TO, bool kDrop>
__global__ __launch_bounds__(kSumBlock) void sum_kernel(SumArgs<T> a, TO *__restrict__ dE, int64_t lde) {
  const uint32_t chunk = blockIdx.x * (uint32_t)(kSumBlock / a.lanes) + threadIdx.x / a.lanes;
  constexpr int N = kCols<T>;
  const int c = (int)(blockIdx.y * a.lanes + threadIdx.x % a.lanes) * N, left = a.d - c;
  if (chunk >= a.chunks || left <= 0) return;
  const uint32_t e0 = chunk * a.chunk, e1 = min(a.n, e0 + a.chunk);
  const uint32_t after = e1 < a.n ? a.key[e1] : kNone;
  uint32_t cur = a.key[e0];
  bool from_before = e0 > 0 && a.key[e0 - 1] == cur;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.0f;
  auto flush = [&](bool goes_on) {
    if (cur >= a.n_vocab) return;
    if (from_before || goes_on)
      store(a.part + ((int64_t)chunk * 2 + (from_before ? 0 : 1)) * a.d + c, left, acc);
    else
      write_row(dE + (int64_t)cur * lde + c, left, acc, a.scale, a.accumulate);
  };
  for (uint32_t e = e0; e < e1; e += kAhead) {
    uint32_t k[kAhead], p[kAhead];
    Chunk in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      k[u] = e + u < e1 ? a.key[e + u] : kNone;
      p[u] = e + u < e1 ? a.pos[e + u] : 0u;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) in[u] = fetch(a.G + (int64_t)p[u] * a.ldg + c, k[u] < a.n_vocab ? left : 0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (e + u >= e1) break;
      if (k[u] != cur) {
        flush(false);
        cur = k[u];
        from_before = false;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.0f;
      }
      float v[N];
      if (kDrop) drop<T>(in[u], (uint32_t)c, p[u], a.m);
      widen<T>(in[u], v);
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += v[i];
    }
  }
  flush(after == cur);
}

// The row of a number that begins in chunk blockIdx.x and goes on in later ones: its part at
// that chunk's end, then those at the next chunks' starts, their sum split over the
// workgroup's groups of lanes.
template <typename T, typename TO>
__global__ __launch_bounds__(kSumBlock) void join_kernel(SumArgs<T> a, TO *__restrict__ dE, int64_t lde) {
  constexpr int N = kCols<T>;
  __shared__ float sums[kSumBlock][N];
  const uint32_t chunk = blockIdx.x;
  const uint32_t e0 = chunk * a.chunk, e1 = min(a.n, e0 + a.chunk);
  if (e1 >= a.n) return;
  const uint32_t key = a.key[e1 - 1];
  if (key >= a.n_vocab || a.key[e1] != key) return;
  if (a.key[e0] == key && e0 > 0 && a.key[e0 - 1] == key) return;   // it began earlier
  uint32_t lo = e1, hi = a.n;                                        // the first entry above key
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (a.key[mid] > key) hi = mid;
    else lo = mid + 1;
  }
  const uint32_t parts = (lo - 1) / a.chunk - chunk;                 // starts of later chunks
  const uint32_t groups = kSumBlock / a.lanes, group = threadIdx.x / a.lanes;
  const int c = (int)(blockIdx.y * a.lanes + threadIdx.x % a.lanes) * N, left = a.d - c;
  const uint32_t per = (parts + groups - 1) / groups;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.0f;
  if (left > 0) {
    if (group == 0) load((const float *)a.part + ((int64_t)chunk * 2 + 1) * a.d + c, left, acc);
    const uint32_t q1 = min(parts, (group + 1) * per);
#pragma unroll 4
    for (uint32_t q = group * per; q < q1; ++q) {
      float v[N];
      load((const float *)a.part + ((int64_t)(chunk + 1 + q) * 2) * a.d + c, left, v);
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += v[i];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) sums[threadIdx.x][i] = acc[i];
  __syncthreads();
  if (group != 0 || left <= 0) return;
  for (uint32_t g = 1; g < groups; ++g)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] += sums[g * a.lanes + threadIdx.x][i];
  write_row(dE + (int64_t)key * lde + c, left, acc, a.scale, a.accumulate);
}

// Rows row0 .. of dE whose number does not occur.  present: NULL when none does.
template <typename TO>
__global__ __launch_bounds__(kZeroBlock) void zero_kernel(const uint8_t *__restrict__ present, uint32_t total,
                                                          int d, Divisor chunks, TO *__restrict__ dE,
                                                          int64_t lde) {
  const float zero[kCols<TO>] = {};
#pragma unroll
  for (int k = 0; k < kZeroPer; ++k) {
    const uint32_t o = blockIdx.x * (uint32_t)(kZeroBlock * kZeroPer) + k * kZeroBlock + threadIdx.x;
    if (o >= total) return;
    uint32_t at;
    const uint32_t row = divide(o, chunks, &at);
    if (present && present[row]) continue;
    const int c = (int)at * kCols<TO>;
    store(dE + (int64_t)row * lde + c, d - c, zero);
  }
}

template <typename TO>
void zero_rows(int64_t n_vocab, int32_t d, const uint8_t *present, TO *dE, int64_t lde, hipStream_t s) {
  const uint32_t chunks = chunks_of<TO>(d);
  const int64_t most = ((int64_t)1 << 30) / chunks;
  for (int64_t r = 0; r < n_vocab; r += most) {
    const uint32_t total = (uint32_t)(std::min(most, n_vocab - r) * chunks);
    hipLaunchKernelGGL(zero_kernel<TO>, dim3((total + kZeroBlock * kZeroPer - 1) / (kZeroBlock * kZeroPer)),
                       dim3(kZeroBlock), 0, s, present ? present + r : nullptr, total, d, divisor(chunks),
                       dE + r * lde, lde);
  }
}

// Lanes that walk a chunk: a power of two that holds a row's chunks, at most a wave.
int lanes_of(uint32_t chunks) {
  int lanes = 8;
  while ((uint32_t)lanes < chunks && lanes < 64) lanes *= 2;
  return lanes;
}

template <typename Id>
void sort_ids(const Plan &p, int64_t n, const Id *ids, int64_t n_vocab, uint8_t *ws, hipStream_t s) {
  uint32_t *count = (uint32_t *)(ws + p.count);
  uint8_t *present = ws + p.present;
  for (int pass = 0; pass < p.passes; ++pass) {
    const uint32_t *kin = (const uint32_t *)(ws + p.key[(pass + 1) % 2]);
    const uint32_t *pin = (const uint32_t *)(ws + p.pos[(pass + 1) % 2]);
    uint32_t *kout = (uint32_t *)(ws + p.key[pass % 2]), *pout = (uint32_t *)(ws + p.pos[pass % 2]);
    const uint32_t tile = (uint32_t)p.tile, tiles = (uint32_t)p.tiles;
    const int shift = pass * p.bits;
    if (pass == 0) {
      const unsigned clear = (unsigned)std::min<int64_t>(256, (n_vocab + 4 * kSortBlock - 1) / (4 * kSortBlock));
      hipLaunchKernelGGL(count_kernel<Id>, dim3(tiles + clear), dim3(kSortBlock), 0, s, ids, (uint32_t)n,
                         (uint32_t)n_vocab, tile, tiles, shift, p.bits, count, present);
      hipLaunchKernelGGL((scatter_kernel<Id, true>), dim3(tiles), dim3(kSortBlock), 0, s, ids,
                         (const uint32_t *)nullptr, (uint32_t)n, (uint32_t)n_vocab, tile, tiles, shift,
                         p.bits, count, kout, pout, present);
    } else {
      hipLaunchKernelGGL(count_kernel<uint32_t>, dim3(tiles), dim3(kSortBlock), 0, s, kin, (uint32_t)n,
                         (uint32_t)n_vocab, tile, tiles, shift, p.bits, count, present);
      hipLaunchKernelGGL((scatter_kernel<uint32_t, false>), dim3(tiles), dim3(kSortBlock), 0, s, kin, pin,
                         (uint32_t)n, (uint32_t)n_vocab, tile, tiles, shift, p.bits, count, kout, pout,
                         present);
    }
  }
}

template <typename T, typename TO>
toc_status grad(const Plan &p, int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab, int32_t d,
                const T *G, int64_t ldg, float scale, const toc_drop *drop, TO *dE, int64_t lde,
                int32_t accumulate, uint8_t *ws, hipStream_t s) {
  if (n == 0) {
    if (!accumulate) zero_rows(n_vocab, d, nullptr, dE, lde, s);
    return launched("zero_kernel");
  }
  if (id_bits == 32) sort_ids(p, n, (const int32_t *)ids, n_vocab, ws, s);
  else sort_ids(p, n, (const int64_t *)ids, n_vocab, ws, s);
  const Mask m = mask_of(drop);
  const int last = (p.passes - 1) % 2;
  SumArgs<T> a{(const uint32_t *)(ws + p.key[last]), (const uint32_t *)(ws + p.pos[last]), (uint32_t)n,
               (uint32_t)n_vocab, (uint32_t)p.chunk, (uint32_t)p.chunks, d, lanes_of(chunks_of<T>(d)), G, ldg, scale * m.keep,
               m, (float *)(ws + p.part), accumulate};
  const unsigned slices = (unsigned)((chunks_of<T>(d) + a.lanes - 1) / a.lanes);
  const unsigned per = (unsigned)(kSumBlock / a.lanes);
  const dim3 grid((unsigned)((p.chunks + per - 1) / per), slices);
  if (!accumulate) zero_rows(n_vocab, d, ws + p.present, dE, lde, s);
  if (a.m.on)
    hipLaunchKernelGGL((sum_kernel<T, TO, true>), grid, dim3(kSumBlock), 0, s, a, dE, lde);
  else
    hipLaunchKernelGGL((sum_kernel<T, TO, false>), grid, dim3(kSumBlock), 0, s, a, dE, lde);
  if (p.chunks > 1)
    hipLaunchKernelGGL((join_kernel<T, TO>), dim3((unsigned)p.chunks, slices), dim3(kSumBlock), 0, s, a, dE, lde);
  return launched("embed gradient kernels");
}

template <typename T>
toc_status grad_typed(const Plan &p, int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab,
                      int32_t d, const void *G, int64_t ldg, float scale, const toc_drop *drop,
                      bool f32, void *dE, int64_t lde, int32_t accumulate, void *ws, void *stream) {
  const hipStream_t s = (hipStream_t)stream;
  if (f32)
    return grad(p, n, ids, id_bits, n_vocab, d, (const T *)G, ldg, scale, drop, (float *)dE, lde, accumulate,
                (uint8_t *)ws, s);
  return grad(p, n, ids, id_bits, n_vocab, d, (const T *)G, ldg, scale, drop, (T *)dE, lde, accumulate,
              (uint8_t *)ws, s);
}

toc_status check_grad(int64_t n, int64_t n_vocab, int32_t d) {
  if (const toc_status st = check_sizes(n, d, TOC_F32)) return st;
  if (d > kMaxGradCols) return fail(TOC_EUNSUPPORTED, "rows of more than %d columns", kMaxGradCols);
  if (n_vocab < 0) return fail(TOC_EINVAL, "%lld table rows", (long long)n_vocab);
  if (n_vocab > kMaxRows) return fail(TOC_EUNSUPPORTED, "more than 2^31-1 table rows");
  return TOC_OK;
}

}  // namespace
}  // namespace rows
}  // namespace toc

using namespace toc;
using namespace toc::rows;

extern "C" {

toc_status toc_embed_grad_workspace_size(int64_t n, int64_t n_vocab, int32_t d, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(TOC_EINVAL, "bytes is NULL");
  if (const toc_status st = check_grad(n, n_vocab, d)) return st;
  *bytes = n ? plan_of(n, n_vocab, d).end : 0;
  return TOC_OK;
}

toc_status toc_embed_grad(int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab, int32_t d,
                          int32_t type, const void *G, int64_t ldg, float scale, const toc_drop *drop,
                          int32_t de_type, void *dE, int64_t lde, int32_t accumulate, void *ws,
                          size_t ws_bytes, void *stream) {
  clear_error();
  toc_status st;
  if ((st = check_sizes(n, d, type)) || (st = check_drop(drop)) || (st = check_ids(n, ids, id_bits, n_vocab)) ||
      (st = check_grad(n, n_vocab, d)))
    return st;
  if (de_type != type && de_type != TOC_F32)
    return fail(TOC_EINVAL, "the gradient's type is the rows' or TOC_F32, not %d", de_type);
  if ((st = check_rows("G", G, n, d, ldg, type_size(type))) ||
      (st = check_rows("dE", dE, n_vocab, d, lde, type_size(de_type))))
    return st;
  if ((st = check_scale(scale, drop))) return st;
  const Plan p = plan_of(n, n_vocab, d);
  if (n > 0 && !ws) return fail(TOC_EINVAL, "workspace is NULL");
  if (n > 0 && ws_bytes < p.end) return fail(TOC_ESIZE, "workspace of %zu bytes below the %zu needed", ws_bytes, p.end);
  if ((uintptr_t)ws % 16) return fail(TOC_EINVAL, "workspace is not 16-byte aligned");
  if (n_vocab == 0) return TOC_OK;
  const bool f32 = de_type == TOC_F32;
  switch (type) {
    case TOC_F32:
      return grad_typed<float>(p, n, ids, id_bits, n_vocab, d, G, ldg, scale, drop, f32, dE, lde, accumulate, ws, stream);
    case TOC_BF16:
      return grad_typed<bf16>(p, n, ids, id_bits, n_vocab, d, G, ldg, scale, drop, f32, dE, lde, accumulate, ws, stream);
    default:
      return grad_typed<f16>(p, n, ids, id_bits, n_vocab, d, G, ldg, scale, drop, f32, dE, lde, accumulate, ws, stream);
  }
}

}  // extern "C"
