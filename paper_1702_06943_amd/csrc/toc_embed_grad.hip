// Gradient of the embedding lookup by sorted token numbers:
//   dE[v, :] (+)= scale * sum of drop(G)[t, :] over the tokens t with ids[t] = v
// the left product G^T.A (Theorem 2) of tuples that hold one pair each, in a fixed order:
//   sort   (number, token) pairs stably by number, 9 bits or fewer a pass; numbers outside
//          the table sort last, as number V.  Up to 128 pairs by every workgroup of the sums
//          for itself (one launch in all), up to 4,096 in one workgroup's LDS, else in tiles:
//          each tile's count of every digit, then each tile places its pairs
//   sum    the sorted list cut into spans of equal length, so that a frequent number costs
//          no more than others: a group of lanes walks a span, its chunk of dE's row in
//          registers, and writes a row when its number ends.  A number that crosses spans
//          of one workgroup is put together in LDS, one that crosses workgroups leaves a
//          partial row in each
//   join   partial rows added in order
//   zero   rows of numbers that do not occur (unless accumulating), by workgroups of the
//          sort's and the sums' launches: the sort leaves most of the chip idle
// Bound by memory, G read once and every row of dE written once, plus the sort's launches, each
// a chain of a few loads: 131,072 x 1,024 bf16 tokens of 47,236 numbers into binary32 rows take
// 133 us, of them the sort 36 (with 69 MB of zeros), the sums 90 (4.4 TB/s of reads and writes), the
// joining 8; 18,750 x 300 f32 37 us, of them the sort 23, the sums 12, the joining 4.  Accumulating,
// a row's old numbers are read where its number ends, and that wait empties the loads under
// way: 131,072 x 1,024 bf16 into bf16 121 us (109 without), 40,000 distinct rows 80 (52).
#include "toc_rows_dev.h"

namespace toc {
namespace rows {
namespace {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64;
constexpr int kMaxBits = 9;                  // digit bits a pass
constexpr int kMaxDigits = 1 << kMaxBits;
constexpr int kTileKeys = 2;                 // pairs of a thread, in registers
constexpr uint32_t kTile = kTileKeys * kSortBlock;
constexpr int kSmallKeys = 4;
constexpr uint32_t kSmall = kSmallKeys * kSortBlock;
// Above, the tiles' counts are summed by scan_kernel, one launch a pass more; at 64 tiles a
// scatter workgroup's own sums take 16 loads a thread.
constexpr uint32_t kFewTiles = 64;
constexpr int kSumBlock = 512;
constexpr uint32_t kMinSpan = 8, kMaxSpan = 32;   // entries of a span
constexpr int kAhead = 8;                    // entries whose rows' loads fly together
// Pairs that each workgroup of the sums sorts itself (us in one launch and with a sort before:
// 20 x 100 bf16 7, 13; 75 x 333 f16 9, 13.5; 128 x 1,024 bf16 14.1, 16.5; 256 x 1,024 24.3, 16.9).
constexpr uint32_t kTiny = 128;
constexpr int kJoinBlock = 256;
constexpr uint32_t kZeroRows = 256;          // most rows of dE that a workgroup looks up at a time
constexpr uint32_t kZeroChunks = 4096;       // ... of about so many chunks
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr int32_t kMaxGradCols = 1 << 20;

// The sort's shape, and where the workspace's parts lie (bytes).
struct Plan {
  int bits, passes;       // digit bits of a pass
  bool tiny, small;
  uint32_t tiles;
  size_t orig, key[2], pos[2], count, total, slot, part, end;
};

size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

// Lanes that walk a span, a power of two of a wave at most: the most lanes of which a row's
// chunks leave no more than a sixth idle, or else those that leave the fewest.
int lanes_of(uint32_t chunks) {
  int best = 64;
  uint32_t best_used = 0;                    // of 64ths, rounded
  for (int lanes = 64; lanes >= 8; lanes /= 2) {
    const uint32_t room = (chunks + lanes - 1) / lanes * lanes;
    const uint32_t used = (uint32_t)((uint64_t)chunks * 60 / room);
    if (used >= 50) return lanes;
    if (used > best_used) {
      best_used = used;
      best = lanes;
    }
  }
  return best;
}

constexpr int64_t kSumLanes = 4096 * 64;
// Entries of a span: the more, the fewer parts of rows are put together, as long as the chip
// has some 4,096 waves (us for 8, 16, 32: 131,072 x 1,024 bf16 161, 151, 148; 131,072 x 512 f16
// of 300 numbers 80, 68, 58; 100,000 x 64 f32 35.9, 36.6, 43.8; 4,000 x 256 bf16 21.5, 25.2, 31.3).
// Up to kTiny pairs: so many that one workgroup walks them all.
uint32_t span_of(int64_t n, uint32_t chunks) {
  if (n <= (int64_t)kTiny) {
    const uint32_t groups = (uint32_t)(kSumBlock / lanes_of(chunks));
    return std::max<uint32_t>(kMinSpan, ((uint32_t)n + groups * kMinSpan - 1) / (groups * kMinSpan) * kMinSpan);
  }
  const int64_t lanes = lanes_of(chunks), slices = (chunks + lanes - 1) / lanes;
  uint32_t span = kMaxSpan;
  while (span > kMinSpan && n / span * lanes * slices < kSumLanes) span /= 2;
  return span;
}

// Entries of the sorted list that a workgroup of sum_kernel walks.
template <typename T>
uint32_t block_span(int64_t n, int32_t d) {
  return (uint32_t)(kSumBlock / lanes_of(chunks_of<T>(d))) * span_of(n, chunks_of<T>(d));
}

// The most workgroups along the list that a call of at most n tokens has.  They halve where the
// span doubles, so the last count of tokens before each doubling is looked at too: a workspace is
// enough for smaller calls.
template <typename T>
int64_t most_blocks(int64_t n, int32_t d) {
  auto blocks = [d](int64_t m) {
    const int64_t span = block_span<T>(m, d);
    return (m + span - 1) / span;
  };
  const int64_t chunks = chunks_of<T>(d), lanes = lanes_of(chunks), wide = (chunks + lanes - 1) / lanes * lanes;
  int64_t most = blocks(n);
  for (int64_t next = 2 * kMinSpan; next <= kMaxSpan; next *= 2)
    most = std::max(most, blocks(std::min(n, next * ((kSumLanes + wide - 1) / wide) - 1)));
  return most;
}

Plan plan_of(int64_t n, int64_t n_vocab, int32_t d) {
  Plan p{};
  int width = 1;                             // bits of the numbers 0..V
  while (width < 32 && ((int64_t)1 << width) <= n_vocab) ++width;
  p.passes = (width + kMaxBits - 1) / kMaxBits;
  p.bits = (width + p.passes - 1) / p.passes;
  p.tiny = n <= (int64_t)kTiny;
  p.small = !p.tiny && n <= (int64_t)kSmall;
  p.tiles = p.tiny || p.small ? 0 : (uint32_t)((n + kTile - 1) / kTile);
  const int64_t blocks = std::max(most_blocks<float>(n, d), most_blocks<bf16>(n, d));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = align16(at + bytes);
    return here;
  };
  // (tiny sorts keep nothing here; their calls ask for it all the same, by one rule for all)
  const bool one = p.tiny || p.small;
  p.orig = take(one ? 0 : (size_t)n * 4);
  for (int i = 0; i < 2; ++i) {
    // (a small sort keeps all passes but the last in LDS)
    p.key[i] = i == 0 || !one ? take((size_t)n * 4) : p.key[0];
    p.pos[i] = i == 0 || !one ? take((size_t)n * 4) : p.pos[0];
  }
  p.count = take(((size_t)p.tiles << p.bits) * 4);
  p.total = take(p.tiles > kFewTiles ? (size_t)4 << p.bits : 0);
  p.slot = take(one ? 0 : (size_t)n_vocab * 4);
  p.part = take(blocks > 1 ? (size_t)blocks * 2 * (size_t)d * 4 : 0);
  p.end = at;
  return p;
}

// A token number, or V for one outside the table.
template <typename Id>
__device__ inline uint32_t key_of(const Id *ids, uint32_t i, uint32_t n_vocab) {
  const int64_t id = (int64_t)ids[i];
  return id >= 0 && id < (int64_t)n_vocab ? (uint32_t)id : n_vocab;
}

// The token numbers of a call as they are, for the workgroups that sort up to kTiny of them;
// ids NULL in other calls.
struct TinyIds {
  const void *ids;
  int bits;
  uint32_t n_vocab;
};
__device__ inline uint32_t key_of(const TinyIds &t, uint32_t i) {
  return t.bits == 32 ? key_of((const int32_t *)t.ids, i, t.n_vocab)
                      : key_of((const int64_t *)t.ids, i, t.n_vocab);
}

// --- zero ----------------------------------------------------------------------

// Rows row0 .. row0 + rows - 1 of dE, `per` of them at a time by a workgroup.  keys NULL: all
// of them are written.  Else those whose number does not occur: count_kernel left in slot[v]
// some token of number v if there is one, and whatever else a slot holds is no such token,
// since the token's own number is looked up again (so the slots need no clearing).  Of at most
// kTiny tokens (tiny.ids) every workgroup looks at all.
template <typename TO>
struct ZeroArgs {
  TO *dE;
  int64_t lde;
  int d;
  Divisor chunks;
  const uint32_t *slot, *keys;
  TinyIds tiny;
  uint32_t n;
  int64_t row0, rows;
  uint32_t per, blocks;
  bool stream;
};

template <int kBlock, typename TO>
__device__ inline void zero_rows(const ZeroArgs<TO> &z, uint32_t block) {
  __shared__ uint32_t absent[kZeroRows], n_absent;
  __shared__ uint8_t occurs[kZeroRows];
  const Chunk zero = {0u, 0u, 0u, 0u};
  for (int64_t r0 = (int64_t)block * z.per; r0 < z.rows; r0 += (int64_t)z.blocks * z.per) {
    if (threadIdx.x == 0) n_absent = 0u;
    if (threadIdx.x < kZeroRows) occurs[threadIdx.x] = 0;
    __syncthreads();
    if (z.tiny.ids) {
      if (threadIdx.x < z.n) {
        const int64_t r = (int64_t)key_of(z.tiny, threadIdx.x) - (z.row0 + r0);
        if (r >= 0 && r < (int64_t)z.per) occurs[r] = 1;
      }
      __syncthreads();
    }
    if (threadIdx.x < z.per && r0 + threadIdx.x < z.rows) {
      const int64_t row = z.row0 + r0 + threadIdx.x;
      const uint32_t t = z.keys ? z.slot[row] : kNone;
      // (their order in the list does not matter)
      if (!occurs[threadIdx.x] && !(t < z.n && (int64_t)z.keys[t] == row))
        absent[atomicAdd(&n_absent, 1u)] = threadIdx.x;
    }
    __syncthreads();
    const uint32_t total = n_absent * z.chunks.d;
    for (uint32_t o = threadIdx.x; o < total; o += kBlock) {
      uint32_t at;
      const uint32_t i = divide(o, z.chunks, &at);
      const int c = (int)at * kCols<TO>;
      put(z.dE + (z.row0 + r0 + absent[i]) * z.lde + c, z.d - c, zero, z.stream);
    }
    __syncthreads();
  }
}

template <typename TO>
__global__ __launch_bounds__(256) void zero_kernel(ZeroArgs<TO> z) {
  zero_rows<256>(z, blockIdx.x);
}

// --- sort ------------------------------------------------------------------------

// Exclusive sums of x over the first `digits` threads (a multiple of 64, or fewer than 64);
// lds: a word per wave.
__device__ inline uint32_t digits_before(uint32_t x, uint32_t *lds) {
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(incl, o, 64);
    if ((int)lane >= o) incl += y;
  }
  if (lane == 63) lds[wave] = incl;
  __syncthreads();
  uint32_t base = incl - x;
  for (uint32_t w = 0; w < wave && w < kMaxDigits / 64; ++w) base += lds[w];
  return base;
}

// For each of a wave's K * 64 entries, in their order, how many before it have its digit;
// at: the wave's count of each digit, 0 before and the wave's counts after.  64 entries are
// compared across the lanes, a ballot a bit.
template <int K>
__device__ inline void wave_ranks(const uint32_t (&digit)[K], const bool (&in)[K], int bits,
                                  uint16_t *at, uint32_t (&rank)[K]) {
  const uint64_t below = ((uint64_t)1 << (threadIdx.x % 64)) - 1;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    uint64_t same = __ballot(in[k]);
    for (int b = 0; b < bits; ++b) {
      const uint64_t ones = __ballot(digit[k] >> b & 1u);
      same &= digit[k] >> b & 1u ? ones : ~ones;
    }
    rank[k] = in[k] ? at[digit[k]] + (uint32_t)__popcll(same & below) : 0u;
    // every lane has its digit's count before the digit's first lane moves it on
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in[k] && !(same & below)) at[digit[k]] += (uint16_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The waves' counts of digit threadIdx.x become the counts of the waves before; returns all.
__device__ inline uint32_t waves_before(uint16_t (*at)[kMaxDigits]) {
  uint32_t run = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    const uint32_t x = at[w][threadIdx.x];
    at[w][threadIdx.x] = (uint16_t)run;
    run += x;
  }
  return run;
}

// Workgroup 0: all passes over n <= kSmall pairs in LDS.  The others write zeros to all of dE
// (rows of numbers that occur are written later): they end with the sort, or soon after.
template <typename TO, typename Id>
__global__ __launch_bounds__(kSortBlock) void small_kernel(const Id *__restrict__ ids, uint32_t n,
                                                           uint32_t n_vocab, int bits, int passes,
                                                           uint32_t *__restrict__ key_out,
                                                           uint32_t *__restrict__ pos_out,
                                                           ZeroArgs<TO> z) {
  __shared__ uint16_t at[kSortWaves][kMaxDigits];
  __shared__ uint32_t base[kMaxDigits], sums[kSortWaves];
  __shared__ uint32_t keys[kSmall];
  __shared__ uint16_t from[kSmall];
  if (blockIdx.x > 0) {
    zero_rows<kSortBlock>(z, blockIdx.x - 1);
    return;
  }
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, digits = 1u << bits;
  // a wave's entries; few enough are spread over all waves
  const uint32_t per = (n + kSortWaves * 64 - 1) / (kSortWaves * 64);
  uint32_t key[kSmallKeys], pos[kSmallKeys], digit[kSmallKeys], rank[kSmallKeys], i[kSmallKeys];
  bool in[kSmallKeys];
#pragma unroll
  for (int k = 0; k < kSmallKeys; ++k) {
    i[k] = (wave * per + k) * 64 + lane;
    in[k] = (uint32_t)k < per && i[k] < n;
    key[k] = in[k] ? key_of(ids, i[k], n_vocab) : 0u;
    pos[k] = i[k];
  }
  for (int pass = 0; pass < passes; ++pass) {
    for (uint32_t j = threadIdx.x; j < kSortWaves * kMaxDigits; j += kSortBlock) (&at[0][0])[j] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallKeys; ++k) digit[k] = key[k] >> (pass * bits) & (digits - 1);
    wave_ranks(digit, in, bits, at[wave], rank);
    __syncthreads();
    const uint32_t count = threadIdx.x < digits ? waves_before(at) : 0u;
    const uint32_t before = digits_before(count, sums);
    if (threadIdx.x < digits) base[threadIdx.x] = before;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallKeys; ++k) {
      if (!in[k]) continue;
      const uint32_t to = base[digit[k]] + at[wave][digit[k]] + rank[k];
      if (pass + 1 == passes) {
        key_out[to] = key[k];
        pos_out[to] = pos[k];
      } else {
        keys[to] = key[k];
        from[to] = (uint16_t)pos[k];
      }
    }
    if (pass + 1 == passes) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallKeys; ++k) {
      if (!in[k]) continue;
      key[k] = keys[i[k]];
      pos[k] = from[i[k]];
    }
  }
}

// The tile's count of each digit.  First pass (Id a token number): also the pairs' numbers
// into orig, and a token of each number into slot (NULL when accumulating).
template <typename Id, bool kFirst>
__global__ __launch_bounds__(kSortBlock) void count_kernel(const Id *__restrict__ ids, uint32_t n,
                                                           uint32_t n_vocab, int shift, int bits,
                                                           uint32_t *__restrict__ count,
                                                           uint32_t *__restrict__ orig,
                                                           uint32_t *__restrict__ slot) {
  __shared__ uint32_t c[kMaxDigits];
  const uint32_t digits = 1u << bits;
  if (threadIdx.x < digits) c[threadIdx.x] = 0u;
  uint32_t key[kTileKeys];
#pragma unroll
  for (int k = 0; k < kTileKeys; ++k) {
    const uint32_t i = blockIdx.x * kTile + k * kSortBlock + threadIdx.x;
    key[k] = i >= n ? kNone : kFirst ? key_of(ids, i, n_vocab) : (uint32_t)ids[i];
    if (kFirst && i < n) {
      orig[i] = key[k];
      if (slot && key[k] < n_vocab) slot[key[k]] = i;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kTileKeys; ++k)
    if (key[k] != kNone) atomicAdd(&c[key[k] >> shift & (digits - 1)], 1u);
  __syncthreads();
  if (threadIdx.x < digits) count[(size_t)blockIdx.x * digits + threadIdx.x] = c[threadIdx.x];
}

// Digit blockIdx.x: its tiles' counts become the counts of the tiles before; total: of all.
__global__ __launch_bounds__(256) void scan_kernel(uint32_t *__restrict__ count, uint32_t tiles, int bits,
                                                   uint32_t *__restrict__ total) {
  __shared__ uint32_t sums[kSortWaves];
  uint32_t carry = 0;
  for (uint32_t t0 = 0; t0 < tiles; t0 += 256) {
    const uint32_t t = t0 + threadIdx.x;
    const size_t at = ((size_t)t << bits) + blockIdx.x;
    const uint32_t x = t < tiles ? count[at] : 0u;
    const uint32_t before = digits_before(x, sums);
    if (t < tiles) count[at] = carry + before;
    const uint32_t all = sums[0] + sums[1] + sums[2] + sums[3];
    __syncthreads();                         // sums are free again
    carry += all;
  }
  if (threadIdx.x == 0) total[blockIdx.x] = carry;
}

// Workgroups 0 .. tiles-1 place a tile's pairs: a digit's pairs of the tile come after all
// pairs of lower digits and the digit's of earlier tiles, waves and lanes.  total: NULL, or
// scan_kernel's, and count then holds the counts before; pos NULL: the pairs are in their
// first order.  The other workgroups write zeros.
template <typename TO>
__global__ __launch_bounds__(kSortBlock) void scatter_kernel(
    const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos, uint32_t n,
    uint32_t tiles, int shift, int bits, const uint32_t *__restrict__ count,
    const uint32_t *__restrict__ total, uint32_t *__restrict__ key_out, uint32_t *__restrict__ pos_out,
    ZeroArgs<TO> z) {
  __shared__ uint16_t at[kSortWaves][kMaxDigits];
  __shared__ uint32_t base[kMaxDigits], sums[kSortWaves];
  __shared__ uint32_t before[kSortBlock], all[kSortBlock];
  if (blockIdx.x >= tiles) {
    zero_rows<kSortBlock>(z, blockIdx.x - tiles);
    return;
  }
  const uint32_t digits = 1u << bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  uint32_t key[kTileKeys], from[kTileKeys], digit[kTileKeys], rank[kTileKeys];
  bool in[kTileKeys];
#pragma unroll
  for (int k = 0; k < kTileKeys; ++k) {
    const uint32_t i = blockIdx.x * kTile + (wave * kTileKeys + k) * 64 + lane;
    in[k] = i < n;
    key[k] = in[k] ? keys[i] : 0u;
    from[k] = in[k] && pos ? pos[i] : i;
    digit[k] = key[k] >> shift & (digits - 1);
  }
  uint32_t b = 0, a = 0;
  if (total) {
    if (threadIdx.x < digits) {
      b = count[(size_t)blockIdx.x * digits + threadIdx.x];
      a = total[threadIdx.x];
    }
  } else {
    // the counts of a digit split over kSortBlock / digits threads
    const uint32_t d = threadIdx.x & (digits - 1), parts = kSortBlock >> bits;
#pragma unroll 8
    for (uint32_t t = threadIdx.x >> bits; t < tiles; t += parts) {
      const uint32_t x = count[(size_t)t * digits + d];
      b += t < blockIdx.x ? x : 0u;
      a += x;
    }
    before[threadIdx.x] = b;
    all[threadIdx.x] = a;
  }
  for (uint32_t j = threadIdx.x; j < kSortWaves * kMaxDigits; j += kSortBlock) (&at[0][0])[j] = 0;
  __syncthreads();
  if (!total && threadIdx.x < digits) {
    b = a = 0;
    for (uint32_t j = threadIdx.x; j < kSortBlock; j += digits) {
      b += before[j];
      a += all[j];
    }
  }
  wave_ranks(digit, in, bits, at[wave], rank);
  const uint32_t lower = digits_before(threadIdx.x < digits ? a : 0u, sums);   // (a barrier)
  if (threadIdx.x < digits) {
    waves_before(at);
    base[threadIdx.x] = lower + b;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kTileKeys; ++k) {
    if (!in[k]) continue;
    const uint32_t to = base[digit[k]] + at[wave][digit[k]] + rank[k];
    key_out[to] = key[k];
    pos_out[to] = from[k];
  }
}

// --- sums --------------------------------------------------------------------------

template <typename T>
struct SumArgs {
  const uint32_t *key, *pos;     // the sorted list; not there where tiny.ids is
  TinyIds tiny;
  uint32_t n, n_vocab, blocks;   // workgroups along the list
  Divisor slices;                // and along the columns
  int d, lanes, shift;           // lanes = 1 << shift
  uint32_t span;                 // entries of a group of lanes
  const T *G;
  int64_t ldg;
  float scale;
  Mask m;
  float *part;                   // two rows a workgroup: its first number's, its last number's
  int accumulate;
  bool stream;                   // dE's rows go past the caches
};

template <typename TO, int N>
__device__ inline void write_row(TO *p, int left, float (&v)[N], float scale, int accumulate,
                                 bool stream) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] *= scale;
  if (accumulate) {
    float old[N];
    load((const TO *)p, left, old);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += old[i];
  }
  store(p, left, v, stream);
}

// Workgroup b of the first a.blocks slices: slice b mod slices of kLanes chunks of the columns
// (neighbours read and write the same rows), entries of the list (b / slices groups + g) span
// onwards for group g.  The other workgroups write zeros.  A group's
// lanes hold its entries' numbers and tokens between them, so that the rows' loads wait for
// nothing but each other: kAhead of them are always under way.  Up to kTiny tokens are ranked
// here, each against all the others, in every workgroup.
template <typename T, typename TO, int kLanes, bool kDrop>
__global__ __launch_bounds__(kSumBlock) void sum_kernel(SumArgs<T> a, TO *__restrict__ dE, int64_t lde,
                                                        ZeroArgs<TO> z) {
  constexpr int N = kCols<T>;
  constexpr uint32_t kGroups = kSumBlock / kLanes;
  constexpr int kHold = ((int)kMaxSpan + kLanes - 1) / kLanes;
  __shared__ float heads[kSumBlock][N];          // each group's part of a number from before
  __shared__ uint8_t through[kGroups];           // ... which goes on after the group
  uint32_t slice;
  const uint32_t block = divide(blockIdx.x, a.slices, &slice);
  if (block >= a.blocks) {
    zero_rows<kSumBlock>(z, blockIdx.x - a.blocks * a.slices.d);
    return;
  }
  __shared__ __attribute__((aligned(16))) uint32_t tiny_in[kTiny];
  __shared__ uint32_t tiny_key[kTiny], tiny_pos[kTiny];
  const bool tiny = a.tiny.ids != nullptr;
  if (tiny) {
    const uint32_t t = threadIdx.x;
    const uint32_t key = t < a.n ? key_of(a.tiny, t) : kNone;
    if (t < kTiny) tiny_in[t] = key;
    __syncthreads();
    if (t < a.n) {
      uint32_t rank = 0;                         // (entries past n are above all numbers)
      for (uint32_t j = 0; j < a.n; j += 4) {
        const Chunk other = *(const Chunk *)&tiny_in[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) rank += other[i] < key || (other[i] == key && j + i < t) ? 1u : 0u;
      }
      tiny_key[rank] = key;
      tiny_pos[rank] = t;
    }
    __syncthreads();
  }
  auto key_at = [&](uint32_t e) { return tiny ? tiny_key[e] : a.key[e]; };
  uint32_t group = threadIdx.x / kLanes;
  if (kLanes == 64) group = __builtin_amdgcn_readfirstlane(group);
  const int lane = threadIdx.x % kLanes;
  const int c = (int)(slice * kLanes + lane) * N, left = a.d - c;
  const Place<T, kLanes == 8> l = place<T, kLanes == 8>(c, a.d);
  const uint32_t e0 = (uint32_t)min(((uint64_t)block * kGroups + group) * a.span, (uint64_t)a.n);
  const uint32_t entries = min(a.n - e0, a.span);
  uint32_t keys[kHold], tokens[kHold];
#pragma unroll
  for (int j = 0; j < kHold; ++j) {
    const uint32_t e = lane + j * kLanes;
    keys[j] = e < entries ? key_at(e0 + e) : kNone;
    tokens[j] = e >= entries ? 0u : tiny ? tiny_pos[e0 + e] : a.pos[e0 + e];
  }
  const uint32_t prev = e0 > 0 && entries ? key_at(e0 - 1) : kNone;
  const uint32_t next = e0 + entries < a.n ? key_at(e0 + entries) : kNone;
  // entry u's number or token, in all lanes of the group (all of them take part)
  auto of = [&](const uint32_t(&held)[kHold], int u) -> uint32_t {
    if constexpr (kLanes == 64) return __builtin_amdgcn_readlane(held[0], u);
    else {
      uint32_t x = held[0];
#pragma unroll
      for (int j = 1; j < kHold; ++j) x = u < j * kLanes ? x : held[j];
      return __shfl(x, u % kLanes, kLanes);
    }
  };
  Chunk in[kAhead];
  uint32_t at[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    at[u] = of(tokens, u);
    in[u] = fetch(a.G + (int64_t)at[u] * a.ldg, l);
  }
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.0f;
  uint32_t cur = of(keys, 0);
  const uint32_t start = cur;
  const bool begun = entries && prev == cur;     // the first number is from before
  bool from_before = begun;
  auto step = [&](int u, int j) {
    const uint32_t key = of(keys, u);
    if (u >= (int)entries) return;
    if (key != cur) {
      if (from_before) {
#pragma unroll
        for (int i = 0; i < N; ++i) heads[threadIdx.x][i] = acc[i];
      } else if (left > 0) {                     // (cur < V: a larger number sorts after it)
        write_row(dE + (int64_t)cur * lde + c, left, acc, a.scale, a.accumulate, a.stream);
      }
      cur = key;
      from_before = false;
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    }
    Chunk x = settle(in[j], l);
    float v[N];
    if (kDrop) drop<T>(x, (uint32_t)c, at[j], a.m);
    widen<T>(x, v);
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] += v[i];
  };
  // (the loads under way are the same on every path through the loop, so that a step waits
  // for its own and not for all, but where write_row() accumulates)
  int u0 = 0;
#pragma unroll 1
  for (; u0 + kAhead < (int)a.span; u0 += kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      step(u0 + j, j);
      at[j] = of(tokens, u0 + j + kAhead);
      in[j] = fetch(a.G + (int64_t)at[j] * a.ldg, l);
    }
  }
#pragma unroll
  for (int j = 0; j < kAhead; ++j) step(u0 + j, j);
  const bool goes_on = entries && next == cur;
  if (from_before) {
#pragma unroll
    for (int i = 0; i < N; ++i) heads[threadIdx.x][i] = acc[i];
  } else if (entries && !goes_on && cur < a.n_vocab && left > 0) {
    write_row(dE + (int64_t)cur * lde + c, left, acc, a.scale, a.accumulate, a.stream);
  }
  if (lane == 0) through[group] = from_before && goes_on;
  __syncthreads();
  if (left <= 0 || !entries) return;
  // A group whose last number begins in it and goes on adds the parts of the groups that
  // follow; group 0 does so for a number from before the workgroup.
  if (group == 0 && begun && start < a.n_vocab) {
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = heads[threadIdx.x][i];
    for (uint32_t g = 0; g + 1 < kGroups && through[g]; ++g)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += heads[(g + 1) * kLanes + lane][i];
    store(a.part + (int64_t)block * 2 * a.d + c, left, v, false);
  }
  if (goes_on && !from_before && cur < a.n_vocab) {
    uint32_t g = group + 1;
    bool open = true;                            // whether the number reaches group g
    for (; g < kGroups && open; ++g) {
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += heads[g * kLanes + lane][i];
      open = through[g];
    }
    if (open) store(a.part + ((int64_t)block * 2 + 1) * a.d + c, left, acc, false);
    else write_row(dE + (int64_t)cur * lde + c, left, acc, a.scale, a.accumulate, a.stream);
  }
}

// The row of a number that begins in a workgroup's entries and goes on after them: its part
// there, then those of the workgroups that follow, split over this one's groups of lanes.
template <typename T, typename TO>
__global__ __launch_bounds__(kJoinBlock) void join_kernel(SumArgs<T> a, uint32_t span,
                                                          TO *__restrict__ dE, int64_t lde) {
  constexpr int N = kCols<T>;
  __shared__ float sums[kJoinBlock][N];
  uint32_t slice;
  const uint32_t block = divide(blockIdx.x, a.slices, &slice);
  const uint32_t e0 = block * span, e1 = e0 + span;          // (the last one has no later)
  const uint32_t key = a.key[e1 - 1], next = a.key[e1], head = a.key[e0];
  const uint32_t prev = e0 > 0 ? a.key[e0 - 1] : kNone;
  if (key >= a.n_vocab || next != key || (head == key && prev == key)) return;
  // one part in each later workgroup up to the first whose last entry is another number
  uint32_t parts = 0;
  for (bool more = true; more;) {
    const uint32_t b = block + 1 + parts + threadIdx.x % 64;
    const uint64_t end = ((uint64_t)b + 1) * span;
    const bool full = b < a.blocks && end < a.n && a.key[end - 1] == key && a.key[end] == key;
    const uint64_t stop = ~__ballot(full);
    more = stop == 0;
    parts += more ? 64 : (uint32_t)__builtin_ctzll(stop) + 1;
  }
  const uint32_t groups = kJoinBlock >> a.shift, group = threadIdx.x >> a.shift;
  const int c = (int)(slice * a.lanes + (threadIdx.x & (a.lanes - 1))) * N, left = a.d - c;
  const uint32_t per = (parts + groups - 1) / groups;
  float acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.0f;
  if (left > 0) {
    if (group == 0) load((const float *)a.part + ((int64_t)block * 2 + 1) * a.d + c, left, acc);
    const uint32_t q1 = min(parts, (group + 1) * per);
#pragma unroll 4
    for (uint32_t q = group * per; q < q1; ++q) {
      float v[N];
      load((const float *)a.part + ((int64_t)(block + 1 + q) * 2) * a.d + c, left, v);
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
  write_row(dE + (int64_t)key * lde + c, left, acc, a.scale, a.accumulate, a.stream);
}

// --- launches -----------------------------------------------------------------------

// dE's rows that a call has to write zeros to, handed out to its launches.
template <typename TO>
struct Zeros {
  ZeroArgs<TO> z;
  int64_t left;

  // keys: the tokens' numbers if the slots tell the rows that occur, or NULL
  Zeros(TO *dE, int64_t lde, int64_t n_vocab, int32_t d, const uint32_t *slot, const uint32_t *keys,
        const TinyIds &tiny, int64_t n)
      : left(n_vocab) {
    const uint32_t chunks = chunks_of<TO>(d);
    z = ZeroArgs<TO>{dE, lde, d, divisor(chunks), slot, keys, tiny, (uint32_t)n, 0, 0,
                     std::max(1u, std::min(kZeroRows, kZeroChunks / chunks)), 0,
                     stream_out(n_vocab, d, sizeof(TO))};
  }
  // Rows for the next `most` chunks, about, and workgroups for them.
  ZeroArgs<TO> take(int64_t most) {
    ZeroArgs<TO> t = z;
    t.rows = std::min(left, most / t.chunks.d + 1);
    t.blocks = (uint32_t)std::min<int64_t>((t.rows + t.per - 1) / t.per, 1 << 17);
    z.row0 += t.rows;
    left -= t.rows;
    return t;
  }
  ZeroArgs<TO> rest() { return take(left * z.chunks.d); }
};

// Chunks that a sort launch writes beside its own work, which takes some 5 us and little of the
// chip: 24 MB, or 48 MB where the sums read more than 64 MB and would be held up by what is
// left to them (us with 0, 24, 48 MB: 18,750 x 300 f32 42.8, 37.2, 40.0; 65,536 x 1,024 bf16
// 80.4, 75.4, 71.0; 131,072 x 1,024 144.5, 136.2, 134.0).
int64_t beside(int64_t read_bytes) { return (read_bytes > 64 << 20 ? 2 : 1) * ((int64_t)3 << 19); }

template <typename TO, typename Id>
void sort_tiles(const Plan &p, uint32_t n, const Id *ids, uint32_t n_vocab, bool slots, uint8_t *ws,
                Zeros<TO> &zeros, int64_t zero_chunks, hipStream_t s) {
  uint32_t *count = (uint32_t *)(ws + p.count), *orig = (uint32_t *)(ws + p.orig);
  uint32_t *total = p.tiles > kFewTiles ? (uint32_t *)(ws + p.total) : nullptr;
  uint32_t *slot = slots ? (uint32_t *)(ws + p.slot) : nullptr;
  for (int pass = 0; pass < p.passes; ++pass) {
    const uint32_t *kin = pass ? (const uint32_t *)(ws + p.key[(pass + 1) % 2]) : orig;
    const uint32_t *pin = pass ? (const uint32_t *)(ws + p.pos[(pass + 1) % 2]) : nullptr;
    uint32_t *kout = (uint32_t *)(ws + p.key[pass % 2]), *pout = (uint32_t *)(ws + p.pos[pass % 2]);
    const int shift = pass * p.bits;
    if (pass == 0)
      hipLaunchKernelGGL((count_kernel<Id, true>), dim3(p.tiles), dim3(kSortBlock), 0, s, ids, n, n_vocab,
                         shift, p.bits, count, orig, slot);
    else
      hipLaunchKernelGGL((count_kernel<uint32_t, false>), dim3(p.tiles), dim3(kSortBlock), 0, s, kin, n,
                         n_vocab, shift, p.bits, count, (uint32_t *)nullptr, (uint32_t *)nullptr);
    if (total)
      hipLaunchKernelGGL(scan_kernel, dim3(1u << p.bits), dim3(256), 0, s, count, p.tiles, p.bits, total);
    const ZeroArgs<TO> z = zeros.take(zero_chunks);
    hipLaunchKernelGGL(scatter_kernel<TO>, dim3(p.tiles + z.blocks), dim3(kSortBlock),
                       0, s, kin, pin, n, p.tiles, shift, p.bits, count, total, kout, pout, z);
  }
}

template <typename T, typename TO, typename Id>
toc_status grad(const Plan &p, int64_t n, const Id *ids, int64_t n_vocab, int32_t d, const T *G,
                int64_t ldg, float scale, const toc_drop *drop, TO *dE, int64_t lde, bool accumulate,
                uint8_t *ws, hipStream_t s) {
  const TinyIds tiny{p.tiny && n > 0 ? ids : nullptr, 8 * (int)sizeof(Id), (uint32_t)n_vocab};
  const bool tiled = !p.tiny && !p.small;
  Zeros<TO> zeros(dE, lde, accumulate ? 0 : n_vocab, d, tiled ? (const uint32_t *)(ws + p.slot) : nullptr,
                  tiled ? (const uint32_t *)(ws + p.orig) : nullptr, tiny, n);
  if (n == 0) {
    const ZeroArgs<TO> z = zeros.rest();
    if (z.blocks) hipLaunchKernelGGL(zero_kernel<TO>, dim3(z.blocks), dim3(256), 0, s, z);
    return launched("zero_kernel");
  }
  if (p.small) {
    const ZeroArgs<TO> z = zeros.rest();
    hipLaunchKernelGGL((small_kernel<TO, Id>), dim3(1 + z.blocks), dim3(kSortBlock), 0, s, ids, (uint32_t)n,
                       (uint32_t)n_vocab, p.bits, p.passes, (uint32_t *)(ws + p.key[0]),
                       (uint32_t *)(ws + p.pos[0]), z);
  } else if (tiled) {
    sort_tiles(p, (uint32_t)n, ids, (uint32_t)n_vocab, !accumulate, ws, zeros,
               beside(n * d * (int64_t)sizeof(T)), s);
  }
  const Mask m = mask_of(drop);
  const int last = p.small || p.tiny ? 0 : (p.passes - 1) % 2;
  const uint32_t span = block_span<T>(n, d);
  const int lanes = lanes_of(chunks_of<T>(d));
  const uint32_t slices = (chunks_of<T>(d) + lanes - 1) / lanes;
  SumArgs<T> a{(const uint32_t *)(ws + p.key[last]), (const uint32_t *)(ws + p.pos[last]), tiny, (uint32_t)n,
               (uint32_t)n_vocab, (uint32_t)((n + span - 1) / span), divisor(slices), d, lanes,
               __builtin_ctz(lanes), span_of(n, chunks_of<T>(d)), G, ldg, scale * m.keep, m,
               (float *)(ws + p.part), accumulate,
               stream_out(accumulate ? std::min(n, n_vocab) : n_vocab, d, sizeof(TO))};
  const ZeroArgs<TO> z = zeros.rest();
  const dim3 grid(a.blocks * slices + z.blocks);
#define TOC_SUM(L)                                                                                      \
  if (lanes == L) {                                                                                      \
    if (m.on)                                                                                            \
      hipLaunchKernelGGL((sum_kernel<T, TO, L, true>), grid, dim3(kSumBlock), 0, s, a, dE, lde, z);      \
    else                                                                                                 \
      hipLaunchKernelGGL((sum_kernel<T, TO, L, false>), grid, dim3(kSumBlock), 0, s, a, dE, lde, z);     \
  }
  TOC_SUM(8) TOC_SUM(16) TOC_SUM(32) TOC_SUM(64)
#undef TOC_SUM
  if (a.blocks > 1)
    hipLaunchKernelGGL((join_kernel<T, TO>), dim3((a.blocks - 1) * slices), dim3(kJoinBlock), 0, s, a, span, dE,
                       lde);
  return launched("embed gradient kernels");
}

template <typename T, typename TO>
toc_status grad_ids(const Plan &p, int64_t n, const void *ids, int32_t id_bits, int64_t n_vocab,
                    int32_t d, const void *G, int64_t ldg, float scale, const toc_drop *drop, void *dE,
                    int64_t lde, int32_t accumulate, void *ws, void *stream) {
  if (id_bits == 32)
    return grad(p, n, (const int32_t *)ids, n_vocab, d, (const T *)G, ldg, scale, drop, (TO *)dE, lde,
                accumulate != 0, (uint8_t *)ws, (hipStream_t)stream);
  return grad(p, n, (const int64_t *)ids, n_vocab, d, (const T *)G, ldg, scale, drop, (TO *)dE, lde,
              accumulate != 0, (uint8_t *)ws, (hipStream_t)stream);
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
  if (n > 0 && ws_bytes < p.end)
    return fail(TOC_ESIZE, "workspace of %zu bytes below the %zu needed", ws_bytes, p.end);
  if ((uintptr_t)ws % 16) return fail(TOC_EINVAL, "workspace is not 16-byte aligned");
  if (n_vocab == 0) return TOC_OK;
  const bool f32 = de_type == TOC_F32;
#define TOC_GRAD(T, TO) \
  grad_ids<T, TO>(p, n, ids, id_bits, n_vocab, d, G, ldg, scale, drop, dE, lde, accumulate, ws, stream)
  switch (type) {
    case TOC_F32:
      return TOC_GRAD(float, float);
    case TOC_BF16:
      return f32 ? TOC_GRAD(bf16, float) : TOC_GRAD(bf16, bf16);
    default:
      return f32 ? TOC_GRAD(f16, float) : TOC_GRAD(f16, f16);
  }
#undef TOC_GRAD
}

}  // extern "C"
