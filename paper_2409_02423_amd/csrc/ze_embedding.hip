// ze_embedding.hip -- gfx950 kernels and C ABI of the embedding in include/ze.h: the lookup of this rank's rows, and their gradient.
//
// The gradient is a sum over the tokens that have a row, in the order of the tokens.  They are sorted by row (a stable counting sort, eight bits of the
// row's number at a time), the sorted list is cut into pieces of the same length, and each wavefront adds up one piece, for 64 vectors of the
// columns: a row whose tokens lie within a piece is done, parts of rows that go on are kept and joined by a second kernel, in which a workgroup shares out a
// row of many parts.  So there are no sums by atomics, their order depends on the ids alone, and a token that the whole batch has (a pad token that is
// an ordinary row) takes 1.1 to 2.2 times the time of as many tokens of many rows: 8192 tokens of 6144 bf16 values 121 us for 110, 16384 of 256 87 for 56,
// 16384 of 1024 146 for 66, 65536 of 1024 163 for 91.
//
// Memory bounds both on large tensors, the chain of launches the gradient of small ones.  8192 tokens on one of four ranks, 12608 rows of 6144
// bf16 values: lookup 23.8 us at 4.9 TB/s, of which six sevenths are written; fp32 gradient 11.9 (sort) + 62.7 (sums and zeros, 5.4 TB/s) + 6.0 (joins).
// 65536 tokens of 1024 values: 50 (sort, six launches) + 38.6 + 6.9.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ze.h"
#include "ze_common.h"

namespace {

constexpr int kThreads = 256;

// ---- lookup ------------------------------------------------------------------------------

struct LookupArgs {
  const void* ids;
  const char* table;
  char* out;
  size_t tokens, stride_table, stride_out;   // bytes
  long long first, rows;
  int cols, vectors;       // vectors of 16 bytes in a row, the last one moved to end where the row does
  int lanes_log2;          // lanes that share a row
  float scale;
};

constexpr int kLookupSteps = 4;   // vectors of a lane

// A row's lanes ask for all that they have of it before they use any.  Ids come from the same few cache lines for all workgroups of a token, rows that are not this
// rank's cost their stores alone.

template <int DT, class ID>
__global__ void __launch_bounds__(kThreads) lookup_kernel(LookupArgs a) {
  constexpr int kN = kVec<DT>;
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const size_t n = (size_t)blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  if (n >= a.tokens) return;
  const long long local = row_of_id(static_cast<const ID*>(a.ids)[n], a.first, a.rows);
  const bool here = local >= 0;
  const char* row = a.table + (here ? (size_t)local : 0) * a.stride_table;
  char* out = a.out + n * a.stride_out;
  const int from = (int)blockIdx.y * kLookupSteps * lanes + lane;
  if (a.cols < kN) {   // narrower than a vector
    if (lane != 0) return;
    Raw<DT> raw;
#pragma unroll
    for (int i = 0; i < raw.kWords; ++i) raw.w[i] = 0;
    if (here) raw.load(row, 0, a.cols);
    float v[kN];
    raw.unpack(v);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = here ? v[j] * a.scale : 0.0f;
    raw.pack(v);
    raw.store(out, 0, a.cols);
    return;
  }
  Raw<DT> raw[kLookupSteps];
  uint32_t at[kLookupSteps];
#pragma unroll
  for (int i = 0; i < kLookupSteps; ++i) {
    const int vector = from + i * lanes, start = vector * kN;
    at[i] = (start + kN <= a.cols ? start : a.cols - kN) * kBytes<DT>;
    if (here && vector < a.vectors) raw[i].load(row, at[i]);
  }
#pragma unroll
  for (int i = 0; i < kLookupSteps; ++i) {
    if (from + i * lanes >= a.vectors) continue;
    float v[kN];
    raw[i].unpack(v);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = here ? v[j] * a.scale : 0.0f;
    raw[i].pack(v);
    raw[i].store(out, at[i]);
  }
}

// ---- tokens sorted by row ------------------------------------------------------------------

constexpr int kSortThreads = 1024, kSortItems = 8, kSortTile = kSortThreads * kSortItems, kWaves = kSortThreads / 64, kDigitBits = 8, kBins = 1 << kDigitBits;
// A digit's numbers of the wavefronts, one behind the other; 17 words from digit to digit, so that digits fall into different banks of LDS.
constexpr int kCounts = kBins * (kWaves + 1);
__device__ __forceinline__ int count_at(uint32_t digit, int wave) { return (int)digit * (kWaves + 1) + wave; }
constexpr int kEach = kBins * kWaves / kSortThreads;
static_assert(kEach == 4 && kWaves == 16, "four lanes for each digit");

// An item's place among those with its digit in its wavefront's part of a tile (items that follow one another, 64 at a time, `rounds` times), and at the end the
// number of each digit in each wavefront's part.
template <int ITEMS>
__device__ __forceinline__ void rank_items(const uint32_t (&digit)[ITEMS], int rounds, int bits, uint32_t (&rank)[ITEMS], uint32_t (&counts)[kCounts]) {
  const int wave = threadIdx.x / 64;
  for (int i = threadIdx.x; i < (kWaves + 1) << bits; i += kSortThreads) counts[i] = 0;
  // the lanes with the same digit: each bit is one comparison, and takes the lanes that differ in it out
  uint32_t low[ITEMS], high[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (i >= rounds) break;
    low[i] = high[i] = 0xFFFFFFFFu;
    for (int b = 0; b < bits; ++b) {
      const uint32_t mine = 0u - (digit[i] >> b & 1u);
      const uint64_t with = __builtin_amdgcn_ballot_w64(mine != 0);
      low[i] &= ~((uint32_t)with ^ mine);
      high[i] &= ~((uint32_t)(with >> 32) ^ mine);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (i >= rounds) break;
    uint32_t* const count = &counts[count_at(digit[i], wave)];
    const uint32_t before = __builtin_amdgcn_mbcnt_hi(high[i], __builtin_amdgcn_mbcnt_lo(low[i], 0));
    rank[i] = *count + before;
    // (a wavefront's reads and writes of LDS happen in order: all lanes have read before one of them writes)
    if (before == 0) *count = rank[i] + __builtin_popcount(low[i]) + __builtin_popcount(high[i]);
  }
  __syncthreads();
}

// Numbers of digits in wavefronts' parts -> how many items come before each: digit by digit, and within one wavefront by wavefront.
__device__ __forceinline__ void sum_counts(uint32_t (&counts)[kCounts], int bits, uint32_t (&buffer)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, at = count_at(threadIdx.x / 4, threadIdx.x % 4 * kEach);
  const bool there = threadIdx.x < 4 << bits;
  uint32_t v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = there ? counts[at + i] : 0;
    sum += v[i];
  }
  const uint32_t up_to = sum_up_to(sum);
  if (lane == 63) buffer[wave] = up_to;
  __syncthreads();
  uint32_t before = up_to - sum;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) before += w < wave ? buffer[w] : 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (there) counts[at + i] = before;
    before += v[i];
  }
  __syncthreads();
}

// A token's key: its row of the table, or `rows` where it has none.
template <class ID>
__device__ __forceinline__ uint32_t key_of(const void* ids, size_t n, long long first, long long rows) {
  const long long row = row_of_id(static_cast<const ID*>(ids)[n], first, rows);
  return row >= 0 ? (uint32_t)row : (uint32_t)rows;
}

struct SortArgs {
  const void* ids;
  uint32_t tokens;
  long long first, rows;
  int passes, bits;                // bits of the keys that a pass sorts by
  uint32_t *keys, *places;         // sorted: rows of the table, tokens
  uint32_t *other_keys, *other_places;
  uint32_t* table;                 // [256][tiles]
  uint8_t* named;                  // a byte for each row: whether a token has it (NULL: it is not asked for)
  uint32_t tiles;
};

// (The same byte, and the same value, from several tokens.)
__device__ __forceinline__ void name_row(const SortArgs& a, uint32_t row) { a.named[row] = 1; }
__device__ __forceinline__ void name_none(const SortArgs& a, uint32_t thread, uint32_t threads) {
  uint32_t* const words = reinterpret_cast<uint32_t*>(a.named);   // (up to whole words)
  for (uint32_t i = thread; i < ((uint32_t)a.rows + 3) / 4; i += threads) words[i] = 0;
}

// Up to one tile: one workgroup takes all passes in LDS.  The tokens that have a row are brought together first (on one of four ranks they are
// a quarter), so that the rest costs what they cost.  What bounds it is the chain of steps that wait for one another.  8192 tokens of which a quarter has a
// row, 14 bits in two passes: 11.9 us; 512 tokens, 10 bits in two passes: 4.1 us.
template <class ID, int ITEMS>
__global__ void __launch_bounds__(kSortThreads) sort_kernel(SortArgs a) {
  __shared__ uint32_t keys[kSortThreads * ITEMS], counts[kCounts], buffer[kWaves];
  __shared__ uint16_t places[kSortThreads * ITEMS];
  static_assert(ITEMS <= 8, "two numbers for each lane of a wavefront");
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t key[ITEMS], place[ITEMS], digit[ITEMS], rank[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint32_t n = i * kSortThreads + threadIdx.x;
    key[i] = n < a.tokens ? key_of<ID>(a.ids, n, a.first, a.rows) : (uint32_t)a.rows;
  }
  if (a.named) name_none(a, threadIdx.x, kSortThreads);   // (the barriers below stand between this and the names)
  uint64_t has[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    has[i] = __builtin_amdgcn_ballot_w64(key[i] < (uint32_t)a.rows);
    if (lane == 0) counts[i * kWaves + wave] = __builtin_popcountll(has[i]);
  }
  __syncthreads();
  // each wavefront sums up the numbers for itself
  const int entry = 2 * lane;
  const uint32_t first = entry < ITEMS * kWaves ? counts[entry] : 0, second = entry < ITEMS * kWaves ? counts[entry + 1] : 0, up_to = sum_up_to(first + second);
  const uint32_t there = (uint32_t)__builtin_amdgcn_readlane((int)up_to, 63), below = up_to - first - second;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = i * kWaves + wave;
    const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(at & 1 ? below + first : below), at / 2);
    const uint32_t to = before + __builtin_amdgcn_mbcnt_hi((uint32_t)(has[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has[i], 0));
    if (key[i] < (uint32_t)a.rows) {
      keys[to] = key[i];
      places[to] = (uint16_t)(i * kSortThreads + threadIdx.x);
      if (a.named) name_row(a, key[i]);
    }
  }
  for (uint32_t i = there + threadIdx.x; i < a.tokens; i += kSortThreads) a.keys[i] = (uint32_t)a.rows;   // tokens without a row come last
  __syncthreads();
  const int rounds = (int)((there + kSortThreads - 1) / kSortThreads);
  for (int pass = 0; pass < a.passes; ++pass) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i >= rounds) break;
      const uint32_t at = wave * (64 * rounds) + i * 64 + lane;
      // (those behind the last stay there: they are the last ones with the greatest of digits)
      key[i] = at < there ? keys[at] : 0xFFFFFFFFu;
      place[i] = at < there ? places[at] : 0;
      digit[i] = key[i] >> (a.bits * pass) & ((1u << a.bits) - 1);
    }
    rank_items(digit, rounds, a.bits, rank, counts);
    sum_counts(counts, a.bits, buffer);
    const bool last = pass + 1 == a.passes;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i >= rounds) break;
      const uint32_t to = counts[count_at(digit[i], wave)] + rank[i];
      if (to >= there) continue;
      if (last) {
        a.keys[to] = key[i];
        a.places[to] = place[i];
      } else {
        keys[to] = key[i];
        places[to] = (uint16_t)place[i];
      }
    }
    __syncthreads();
  }
}

// More than a tile: for each pass the digits' numbers in each tile, their sums, and the items to their places.  65536 tokens, 14 bits in two passes:
// (4.7 + 4.6 + 15.9) us each, most of it steps that wait for one another; 16384 tokens 3.9 + 1.6 + 15.9.
template <class ID>
__device__ __forceinline__ uint32_t item_key(const SortArgs& a, const uint32_t* in, uint32_t at) {
  return in ? in[at] : key_of<ID>(a.ids, at, a.first, a.rows);
}

template <class ID>
__global__ void __launch_bounds__(kSortThreads) count_kernel(SortArgs a, int pass, const uint32_t* in) {
  __shared__ uint32_t counts[kBins];
  if (threadIdx.x < kBins) counts[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = blockIdx.x * kSortTile + i * kSortThreads + threadIdx.x;
    // (numbers alone: the order in which they are counted does not matter)
    if (at < a.tokens) atomicAdd(&counts[item_key<ID>(a, in, at) >> (a.bits * pass) & ((1u << a.bits) - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < 1u << a.bits) a.table[(size_t)threadIdx.x * a.tiles + blockIdx.x] = counts[threadIdx.x];
  if (a.named && pass == 0) name_none(a, blockIdx.x * kSortThreads + threadIdx.x, gridDim.x * kSortThreads);
}

// In one workgroup: each entry of the table becomes the sum of those before it.
__global__ void __launch_bounds__(kSortThreads) sums_kernel(uint32_t* table, uint32_t entries) {
  __shared__ uint32_t buffer[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t before = 0;
  for (uint32_t base = 0; base < entries; base += kSortThreads * 4) {
    uint32_t v[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t at = base + threadIdx.x * 4 + i;
      v[i] = at < entries ? table[at] : 0;
      sum += v[i];
    }
    const uint32_t up_to = sum_up_to(sum);
    if (lane == 63) buffer[wave] = up_to;
    __syncthreads();
    uint32_t mine = before + up_to - sum;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) mine += buffer[w];
      before += buffer[w];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t at = base + threadIdx.x * 4 + i;
      if (at < entries) table[at] = mine;
      mine += v[i];
    }
  }
}

template <class ID>
__global__ void __launch_bounds__(kSortThreads) scatter_kernel(SortArgs a, int pass, const uint32_t* in, const uint32_t* in_places, uint32_t* out, uint32_t* out_places) {
  __shared__ uint32_t counts[kCounts];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t key[kSortItems], place[kSortItems], digit[kSortItems], rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = blockIdx.x * kSortTile + wave * (64 * kSortItems) + i * 64 + lane;
    const bool there = at < a.tokens;
    key[i] = there ? item_key<ID>(a, in, at) : 0xFFFFFFFFu;
    place[i] = there ? (in_places ? in_places[at] : at) : 0;
    digit[i] = key[i] >> (a.bits * pass) & ((1u << a.bits) - 1);   // those behind the last token: the greatest, behind all others in the last tile
  }
  rank_items(digit, kSortItems, a.bits, rank, counts);
  // sums over the wavefronts of each digit: four lanes have a digit's sixteen numbers
  const int at_digit = count_at(threadIdx.x / 4, threadIdx.x % 4 * kEach);
  uint32_t v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = counts[at_digit + i];   // (digits past the last have none, but what they hold is not used)
    sum += v[i];
  }
  uint32_t up_to = sum;
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const uint32_t other = __shfl_up(up_to, d, 4);
    if ((lane & 3) >= d) up_to += other;
  }
  if (threadIdx.x < 4u << a.bits) {
    uint32_t before = a.table[(size_t)(threadIdx.x / 4) * a.tiles + blockIdx.x] + up_to - sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      counts[at_digit + i] = before;
      before += v[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = blockIdx.x * kSortTile + wave * (64 * kSortItems) + i * 64 + lane;
    if (at >= a.tokens) continue;
    const uint32_t to = counts[count_at(digit[i], wave)] + rank[i];
    out[to] = key[i];
    out_places[to] = place[i];
    if (a.named && pass + 1 == a.passes && key[i] < (uint32_t)a.rows) name_row(a, key[i]);
  }
}

// ---- sums over each row's tokens -----------------------------------------------------------

constexpr int kMostPiece = 64;

struct SumArgs {
  const uint32_t *keys, *places;   // sorted
  uint32_t tokens, rows;
  const char* dout;
  size_t stride_dout;              // bytes
  char* dtable;
  size_t stride_dtable;            // bytes
  float* kept;                     // [pieces][2][vectors][values of a vector]
  int cols, vectors;
  int piece;                       // tokens, up to kMostPiece
  uint32_t pieces;
  float scale;
  int accumulate;
  unsigned sum_groups;             // workgroups that add up; those behind them write zeros
  const uint8_t* named;            // a byte for each row: whether a token has it (NULL: none has)
};

// A vector of sums into its row of the gradient, or the row as it was plus them.
template <int DT, int DO>
__device__ __forceinline__ void store_sums(const SumArgs& a, uint32_t row, int vector, const float (&sum)[kVec<DT>], const Raw<DO, kVec<DT>>& old) {
  constexpr int kN = kVec<DT>;
  float v[kN];
  if (a.accumulate) {
    old.unpack(v);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] += a.scale * sum[j];
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = a.scale * sum[j];
  }
  Raw<DO, kN> raw;
  raw.pack(v);
  raw.store(a.dtable + (size_t)row * a.stride_dtable, (uint32_t)vector * kN * kBytes<DO>, a.cols - vector * kN);
}
template <int DT, int DO>
__device__ __forceinline__ void load_old(const SumArgs& a, uint32_t row, int vector, Raw<DO, kVec<DT>>& old) {
  constexpr int kN = kVec<DT>;
  old.load(a.dtable + (size_t)row * a.stride_dtable, (uint32_t)vector * kN * kBytes<DO>, a.cols - vector * kN);
}

template <int DT>
__device__ __forceinline__ float* kept_at(const SumArgs& a, uint32_t piece, int which, int vector) {
  return a.kept + (((size_t)piece * 2 + which) * a.vectors + vector) * kVec<DT>;
}

template <int N>
__device__ __forceinline__ void keep(float* to, const float (&v)[N]) {
  typedef float f4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<f4*>(to + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// One piece of the sorted list, in 64 vectors of the columns (wavefronts beside one another take those beside one another, of the same tokens).  A run of
// tokens with the same row that begins and ends in the piece is stored; the part of one that comes from the piece before is kept as the piece's first, that
// of one which goes on (and began here) as its second.  What is read of eight tokens is asked for at once: their rows, and with `accumulate` the
// gradient's rows that are done among them.
template <int DT, int DO>
__device__ __forceinline__ void add_piece(const SumArgs& a, uint32_t piece, int vector) {
  constexpr int kN = kVec<DT>, kAhead = 8;
  const int lane = threadIdx.x & 63;
  const uint32_t from = piece * (uint32_t)a.piece, left = a.tokens - from, count = left < (uint32_t)a.piece ? left : (uint32_t)a.piece;
  // keys and tokens of the piece, one a lane, and the keys beside it
  const uint32_t mine = from + ((uint32_t)lane < count ? (uint32_t)lane : count - 1);
  const uint32_t keys = a.keys[mine], places = a.places[mine];
  const uint32_t before = from > 0 ? a.keys[from - 1] : 0xFFFFFFFFu, behind = from + count < a.tokens ? a.keys[from + count] : 0xFFFFFFFFu;
  const bool there = vector < a.vectors;
  const uint32_t at = (uint32_t)vector * kN * kBytes<DT>;
  const int valid = there ? a.cols - vector * kN : 0;
  float sum[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) sum[j] = 0.0f;
  bool began = (uint32_t)__builtin_amdgcn_readlane((int)keys, 0) != before;   // the present run, in this piece
  for (uint32_t i = 0; i < count; i += kAhead) {
    Raw<DT> raw[kAhead];
    Raw<DO, kN> old[kAhead];
    uint32_t key[kAhead];
    bool ends[kAhead], own[kAhead];   // the run at the token, or its part in this piece; and it began here
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t q = i + u < count ? i + u : count - 1;
      key[u] = i + u < count ? (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)q) : a.rows;
      const uint32_t next = q + 1 == count ? behind : (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)q + 1);
      ends[u] = next != key[u] || q + 1 == count;
      own[u] = began;
      if (key[u] >= a.rows) continue;   // without a row
      raw[u].load(a.dout + (size_t)(uint32_t)__builtin_amdgcn_readlane((int)places, (int)q) * a.stride_dout, there ? at : 0, valid);
      if (a.accumulate && there && began && next != key[u]) load_old<DT, DO>(a, key[u], vector, old[u]);
      began = began || ends[u];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (key[u] >= a.rows) return;   // tokens without a row come last
      float v[kN];
      raw[u].unpack(v);
#pragma unroll
      for (int j = 0; j < kN; ++j) sum[j] += v[j];
      if (!ends[u]) continue;
      if (there) {
        if (!own[u]) keep(kept_at<DT>(a, piece, 0, vector), sum);
        else if (i + u + 1 == count && behind == key[u]) keep(kept_at<DT>(a, piece, 1, vector), sum);
        else store_sums<DT, DO>(a, key[u], vector, sum, old[u]);
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) sum[j] = 0.0f;
    }
  }
}

constexpr int kZeroRows = 4;   // of a workgroup

template <int DT, int DO>
__global__ void __launch_bounds__(kThreads) sum_kernel(SumArgs a) {
  if (blockIdx.x < a.sum_groups) {
    const uint32_t chunks = (a.vectors + 63) / 64, units = a.pieces * chunks;
    for (uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + threadIdx.x / 64); unit < units; unit += a.sum_groups * (kThreads / 64))
      add_piece<DT, DO>(a, unit / chunks, (int)(unit % chunks * 64 + (threadIdx.x & 63)));
    return;
  }
  // zeros for the rows that no token has
  constexpr int kN = kVec<DO>;
  Raw<DO> zero;
#pragma unroll
  for (int i = 0; i < zero.kWords; ++i) zero.w[i] = 0;
  for (uint32_t row0 = (blockIdx.x - a.sum_groups) * kZeroRows; row0 < a.rows; row0 += (gridDim.x - a.sum_groups) * kZeroRows) {
    const uint32_t named = a.named ? *reinterpret_cast<const uint32_t*>(a.named + row0) : 0;
    for (int r = 0; r < kZeroRows; ++r) {
      if (row0 + r >= a.rows || named >> 8 * r & 1) continue;
      char* const row = a.dtable + (size_t)(row0 + r) * a.stride_dtable;
      for (int x = threadIdx.x * kN; x < a.cols; x += kThreads * kN) {
        if (x + kN <= a.cols) zero.template store<true>(row, (uint32_t)x * kBytes<DO>);
        else zero.store(row, (uint32_t)x * kBytes<DO>, a.cols - x);
      }
    }
  }
}

// The rows whose tokens do not lie within a piece (few, where ids are many: the launch is most of the time): the sums that were kept of them, from the piece
// that they begin in.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
constexpr uint32_t kShortRun = 32;   // pieces behind its first that a wavefront adds up alone

// The last piece of the run that goes on from a piece into the next, or the piece itself where none does, or one that began before.
__device__ __forceinline__ uint32_t last_of_run(const SumArgs& a, uint32_t piece, uint32_t& key) {
  const uint32_t from = piece * (uint32_t)a.piece, next = from + (uint32_t)a.piece;
  if (piece + 1 >= a.pieces) return piece;
  key = a.keys[next - 1];
  if (key >= a.rows || a.keys[next] != key) return piece;
  // a run that fills the piece and comes from the one before it began there
  if (a.keys[from] == key && from > 0 && a.keys[from - 1] == key) return piece;
  // The pieces' first keys are sorted: those of the run come before all others.  64 are compared at once, next to one another and then as far apart as
  // those that are left ask for.
  uint32_t low = piece, high = a.pieces, step = 1;   // low has the key, high (or the end) has not
  for (;;) {
    const uint32_t q = low + ((threadIdx.x & 63) + 1) * step;
    const uint64_t same = __builtin_amdgcn_ballot_w64(q < high && a.keys[q * (size_t)a.piece] == key);
    const uint32_t many = ~same ? (uint32_t)__builtin_ctzll(~same) : 64;
    if (many < 64 && low + (many + 1) * step < high) high = low + (many + 1) * step;
    low += many * step;
    if (high - low <= 1) return low;
    step = (high - low - 1 + 63) / 64;
  }
}

// sum += the first sums that were kept of the pieces from..to-1, in their order
template <int DT>
__device__ __forceinline__ void add_kept(const SumArgs& a, uint32_t from, uint32_t to, int vector, float (&sum)[kVec<DT>]) {
  constexpr int kN = kVec<DT>, kAhead = 8;
  typedef float f4 __attribute__((ext_vector_type(4)));
  for (uint32_t q = from; q < to; q += kAhead) {
    f4 v[kAhead][kN / 4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int j = 0; j < kN / 4; ++j) v[u][j] = reinterpret_cast<const f4*>(kept_at<DT>(a, q + u < to ? q + u : to - 1, 0, vector))[j];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (q + u < to) {
#pragma unroll
        for (int j = 0; j < kN; ++j) sum[j] += v[u][j / 4][j % 4];
      }
  }
}

// A wavefront for each piece and 64 vectors of the columns; a workgroup has pieces that follow one another.  A run of many pieces (one at most begins among
// them: kShortRun is more than they are) is shared out among all wavefronts, each of which adds up pieces that follow one another, and their
// sums are added in that order: what bounds it are loads that wait for one another, eight parts at a time.  All tokens of one row, us a call, with one wavefront for
// a run and with eight: 16384 tokens of 256 bf16 values 244 and 87, 65536 of 1024 292 and 163.  Sixteen took 82 and 122, and 84.8 for 81.2 where no run is
// long (8192 tokens of 6144).
template <int DT, int DO>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(SumArgs a) {
  constexpr int kN = kVec<DT>;
  static_assert(kShortRun >= kJoinWaves, "one long run in a workgroup");
  __shared__ uint32_t lasts[kJoinWaves];   // of a long run that begins in the wavefront's piece, or 0
  __shared__ float sums[kJoinWaves][kN][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t groups = (a.pieces + kJoinWaves - 1) / kJoinWaves, units = groups * ((a.vectors + 63) / 64);
  for (uint32_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const uint32_t first = unit % groups * kJoinWaves, piece = first + wave;
    const int vector = (int)(unit / groups * 64) + lane;
    const bool there = vector < a.vectors;
    uint32_t key = 0;
    const uint32_t last = last_of_run(a, piece, key);
    const bool many = last - piece > kShortRun;
    if (lane == 0) lasts[wave] = many ? last : 0;
    Raw<DO, kN> old;
    float sum[kN];
    if (last > piece && there) {
      if (a.accumulate) load_old<DT, DO>(a, key, vector, old);
      const float* p = kept_at<DT>(a, piece, 1, vector);
#pragma unroll
      for (int j = 0; j < kN; ++j) sum[j] = p[j];
      if (!many) {
        add_kept<DT>(a, piece + 1, last + 1, vector, sum);
        store_sums<DT, DO>(a, key, vector, sum, old);
      }
    }
    __syncthreads();
    const uint32_t mine = lasts[lane % kJoinWaves];
    const uint64_t with = __builtin_amdgcn_ballot_w64(mine > 0) & ((1u << kJoinWaves) - 1);
    if (with) {   // (the same in all wavefronts)
      const int owner = __builtin_ctzll(with);
      const uint32_t begin = first + owner + 1, count = (uint32_t)__builtin_amdgcn_readlane((int)mine, owner) + 1 - begin;
      const uint32_t from = begin + (uint32_t)((uint64_t)count * wave / kJoinWaves), to = begin + (uint32_t)((uint64_t)count * (wave + 1) / kJoinWaves);
      float part[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) part[j] = 0.0f;
      if (there) add_kept<DT>(a, from, to, vector, part);
#pragma unroll
      for (int j = 0; j < kN; ++j) sums[wave][j][lane] = part[j];
      __syncthreads();
      if (wave == owner && there) {
#pragma unroll 4
        for (int w = 0; w < kJoinWaves; ++w)
#pragma unroll
          for (int j = 0; j < kN; ++j) sum[j] += sums[w][j][lane];
        store_sums<DT, DO>(a, key, vector, sum, old);
      }
    }
    __syncthreads();
  }
}

// ---- host ----------------------------------------------------------------------------------

struct Plan {
  uint32_t tiles, pieces;
  int piece, passes, bits, vectors;
  size_t keys, places, other_keys, other_places, table, named, kept, bytes;
};

Plan plan_for(const struct ze_form& f) {
  Plan p = {};
  p.vectors = (int)parts(f.cols, 16 / dtype_bytes(f.dtype));
  p.tiles = (uint32_t)parts(f.tokens, kSortTile);
  int bits = 1;
  while (f.rows >> bits) ++bits;   // of keys up to `rows`
  p.passes = (bits + kDigitBits - 1) / kDigitBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  // Short pieces where there are few of them, so that none waits for a second load; else longer ones, which keep less.  In turn, sums + joins in us: 512
  // tokens of 256 fp32 values, pieces of 8 5.3 + 3.3, of 16 7.5 + 3.3; 8192 tokens of 6144 bf16 values, 8 71.4 + 9.6, 16 67.7 + 6.2.
  p.piece = parts(f.tokens, 16) * parts((size_t)p.vectors, 64) <= 2048 ? 8 : f.tokens <= 16384 ? 16 : f.tokens <= 65536 ? 32 : kMostPiece;
  p.pieces = (uint32_t)parts(f.tokens, (size_t)p.piece);
  Places places;
  p.keys = places.take(f.tokens * 4);
  p.places = places.take(f.tokens * 4);
  if (p.tiles > 1) {
    p.other_keys = places.take(f.tokens * 4);
    p.other_places = places.take(f.tokens * 4);
    p.table = places.take((size_t)p.tiles * kBins * 4);
  }
  p.named = places.take(up(f.rows, 4));
  p.kept = places.take((size_t)p.pieces * 2 * p.vectors * (16 / dtype_bytes(f.dtype)) * 4);
  p.bytes = places.at;
  return p;
}

template <class ID>
void sort_tokens(const SortArgs& a, const Plan& p, char* work, hipStream_t s) {
  if (p.tiles == 1) {
    const dim3 one(1), threads(kSortThreads);
    if (a.tokens <= kSortThreads) hipLaunchKernelGGL((sort_kernel<ID, 1>), one, threads, 0, s, a);
    else if (a.tokens <= kSortThreads * 4) hipLaunchKernelGGL((sort_kernel<ID, 4>), one, threads, 0, s, a);
    else hipLaunchKernelGGL((sort_kernel<ID, kSortItems>), one, threads, 0, s, a);
    return;
  }
  const uint32_t *in = nullptr, *in_places = nullptr;
  for (int pass = 0; pass < p.passes; ++pass) {
    const bool own = (p.passes - pass) % 2 == 1;   // the last pass writes what is read
    uint32_t *out = own ? a.keys : a.other_keys, *out_places = own ? a.places : a.other_places;
    hipLaunchKernelGGL(count_kernel<ID>, dim3(p.tiles), dim3(kSortThreads), 0, s, a, pass, in);
    hipLaunchKernelGGL(sums_kernel, dim3(1), dim3(kSortThreads), 0, s, a.table, p.tiles << a.bits);
    hipLaunchKernelGGL(scatter_kernel<ID>, dim3(p.tiles), dim3(kSortThreads), 0, s, a, pass, in, in_places, out, out_places);
    in = out;
    in_places = out_places;
  }
}

template <int DT, int DO>
void launch_sums(const SumArgs& a, size_t rows, hipStream_t s) {
  const size_t units = (size_t)a.pieces * parts((size_t)a.vectors, 64);
  constexpr size_t kMostGroups = (size_t)1 << 21;   // of a kind
  const size_t groups = parts(units, kThreads / 64), zeros = a.accumulate ? 0 : parts(rows, kZeroRows);
  SumArgs b = a;
  b.sum_groups = (unsigned)(groups < kMostGroups ? groups : kMostGroups);
  hipLaunchKernelGGL((sum_kernel<DT, DO>), dim3((unsigned)(b.sum_groups + (zeros < kMostGroups ? zeros : kMostGroups))), dim3(kThreads), 0, s, b);
  const size_t joins = parts((size_t)a.pieces, kJoinWaves) * parts((size_t)a.vectors, 64);
  if (a.pieces > 1) hipLaunchKernelGGL((join_kernel<DT, DO>), dim3((unsigned)(joins < kMostGroups ? joins : kMostGroups)), dim3(kJoinThreads), 0, s, b);
}

}  // namespace

extern "C" {

int ze_embedding(const struct ze_form* form, const void* d_ids, const void* d_table, void* d_out, void* stream) {
  const int rc = check_form(form);
  if (rc != ZC_OK) return rc;
  const struct ze_form& f = *form;
  if (!good_output(f.stride_dtokens, f.cols)) return ZC_ERR_ARG;
  if (f.tokens == 0 || f.cols == 0) return ZC_OK;
  if (!d_ids || (!d_table && f.rows) || !d_out) return ZC_ERR_NULL;
  const size_t e = dtype_bytes(f.dtype);
  if (!aligned_ids(d_ids, f.id_dtype) || !aligned(d_table, e) || !aligned(d_out, e)) return ZC_ERR_ALIGN;
  LookupArgs a;
  a.ids = d_ids;
  a.table = static_cast<const char*>(d_table);
  a.out = static_cast<char*>(d_out);
  a.tokens = f.tokens;
  a.stride_table = stride_of(f.stride_table, f.cols) * e;
  a.stride_out = stride_of(f.stride_dtokens, f.cols) * e;
  a.first = f.first;
  a.rows = (long long)f.rows;
  a.cols = (int)f.cols;
  a.vectors = (int)parts(f.cols, 16 / e);
  a.scale = f.scale;
  a.lanes_log2 = 0;
  while (a.lanes_log2 < 6 && (1 << a.lanes_log2) < a.vectors) ++a.lanes_log2;
  const dim3 grid((unsigned)parts(f.tokens, kThreads >> a.lanes_log2), (unsigned)parts((size_t)a.vectors, (size_t)kLookupSteps << a.lanes_log2));
  const hipStream_t s = static_cast<hipStream_t>(stream);
#define LAUNCH(DT)                                                                                           \
  do {                                                                                                       \
    if (f.id_dtype == ZE_I64) hipLaunchKernelGGL((lookup_kernel<DT, long long>), grid, dim3(kThreads), 0, s, a); \
    else hipLaunchKernelGGL((lookup_kernel<DT, int>), grid, dim3(kThreads), 0, s, a);                        \
  } while (0)
  if (f.dtype == ZC_F32) LAUNCH(kF32);
  else if (f.dtype == ZC_BF16) LAUNCH(kBF16);
  else LAUNCH(kF16);
#undef LAUNCH
  return finish_launch();
}

size_t ze_embedding_work_bytes(const struct ze_form* form) {
  if (check_form(form) != ZC_OK || form->tokens == 0 || form->cols == 0 || form->rows == 0) return 0;
  return plan_for(*form).bytes;
}

int ze_embedding_backward(const struct ze_form* form, const void* d_ids, const void* d_dout, void* d_dtable, int accumulate, void* d_work, size_t work_bytes,
                          void* stream) {
  const int rc = check_form(form);
  if (rc != ZC_OK) return rc;
  const struct ze_form& f = *form;
  if (f.grad_dtype != f.dtype && f.grad_dtype != ZC_F32) return ZC_ERR_DTYPE;
  if (!good_output(f.stride_dtable, f.cols) || (accumulate != 0 && accumulate != 1)) return ZC_ERR_ARG;
  if (f.rows == 0 || f.cols == 0 || (f.tokens == 0 && accumulate)) return ZC_OK;
  if ((f.tokens && (!d_ids || !d_dout || !d_work)) || !d_dtable) return ZC_ERR_NULL;
  const size_t e = dtype_bytes(f.dtype), eo = dtype_bytes(f.grad_dtype);
  if (!aligned_ids(d_ids, f.id_dtype) || !aligned(d_dout, e) || !aligned(d_dtable, eo) || !aligned(d_work, 256)) return ZC_ERR_ALIGN;
  const Plan p = plan_for(f);
  if (f.tokens && work_bytes < p.bytes) return ZC_ERR_CAPACITY;
  char* const work = static_cast<char*>(d_work);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const auto in_work = [&](size_t at) { return reinterpret_cast<uint32_t*>(work + at); };
  if (f.tokens) {
    SortArgs a;
    a.ids = d_ids;
    a.tokens = (uint32_t)f.tokens;
    a.first = f.first;
    a.rows = (long long)f.rows;
    a.passes = p.passes;
    a.bits = p.bits;
    a.keys = in_work(p.keys);
    a.places = in_work(p.places);
    a.other_keys = in_work(p.other_keys);
    a.other_places = in_work(p.other_places);
    a.table = in_work(p.table);
    a.tiles = p.tiles;
    a.named = accumulate ? nullptr : reinterpret_cast<uint8_t*>(work + p.named);
    if (f.id_dtype == ZE_I64) sort_tokens<long long>(a, p, work, s);
    else sort_tokens<int>(a, p, work, s);
  }
  SumArgs a = {};
  a.keys = in_work(p.keys);
  a.places = in_work(p.places);
  a.tokens = (uint32_t)f.tokens;
  a.rows = (uint32_t)f.rows;
  a.dout = static_cast<const char*>(d_dout);
  a.stride_dout = stride_of(f.stride_tokens, f.cols) * e;
  a.dtable = static_cast<char*>(d_dtable);
  a.stride_dtable = stride_of(f.stride_dtable, f.cols) * eo;
  a.kept = reinterpret_cast<float*>(work + p.kept);
  a.cols = (int)f.cols;
  a.vectors = p.vectors;
  a.piece = p.piece;
  a.pieces = p.pieces;
  a.scale = f.scale;
  a.accumulate = accumulate;
  a.named = f.tokens && !accumulate ? reinterpret_cast<const uint8_t*>(work + p.named) : nullptr;
#define LAUNCH(DT)                                                     \
  do {                                                                 \
    if (f.grad_dtype == ZC_F32) launch_sums<DT, kF32>(a, f.rows, s);   \
    else launch_sums<DT, DT>(a, f.rows, s);                            \
  } while (0)
  if (f.dtype == ZC_F32) LAUNCH(kF32);
  else if (f.dtype == ZC_BF16) LAUNCH(kBF16);
  else LAUNCH(kF16);
#undef LAUNCH
  return finish_launch();
}

}  // extern "C"
