// ze_embedding.hip -- gfx950 kernels and C ABI of the embedding in include/ze.h: the lookup of this rank's rows, and their gradient.
//
// The gradient is a sum over the tokens that have a row, in the order of the tokens.  They are sorted by row (a stable counting sort, eight bits of the
// row's number at a time), the sorted list is cut into pieces of the same length, and each wavefront adds up one piece, for 64 vectors of the
// columns: a row whose tokens lie within a piece is done, parts of rows that go on are kept and joined by a second kernel.  So a token that half of the batch has
// takes no longer than others, there are no atomics, and the sums' order depends on the ids alone.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ze.h"
#include "ze_host.h"

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

template <int DT, class ID>
__global__ void __launch_bounds__(kThreads) lookup_kernel(LookupArgs a) {
  constexpr int kN = kVec<DT>;
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const size_t n = (size_t)blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  if (n >= a.tokens) return;
  const long long local = (long long)static_cast<const ID*>(a.ids)[n] - a.first;
  const bool here = local >= 0 && local < a.rows;
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

constexpr int kSortThreads = 1024, kSortItems = 8, kSortTile = kSortThreads * kSortItems, kWaves = kSortThreads / 64, kBins = 256;
// A digit's numbers of the wavefronts, one behind the other; 17 words from digit to digit, so that digits fall into different banks of LDS.
constexpr int kCounts = kBins * (kWaves + 1);
__device__ __forceinline__ int count_at(uint32_t digit, int wave) { return (int)digit * (kWaves + 1) + wave; }
constexpr int kEach = kBins * kWaves / kSortThreads;
static_assert(kEach == 4 && kWaves == 16, "four lanes for each digit");

// An item's place among those with its digit in its wavefront's part of a tile (512 items that follow one another, 64 at a time), and at the end the number of
// each digit in each wavefront's part.
__device__ __forceinline__ void rank_items(const uint32_t (&digit)[kSortItems], uint32_t (&rank)[kSortItems], uint32_t (&counts)[kCounts]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  for (int i = threadIdx.x; i < kCounts; i += kSortThreads) counts[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    uint64_t same = ~(uint64_t)0;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const bool bit = digit[i] >> b & 1;
      const uint64_t with = __builtin_amdgcn_ballot_w64(bit);
      same &= bit ? with : ~with;
    }
    uint32_t* const count = &counts[count_at(digit[i], wave)];
    const uint32_t before = __builtin_popcountll(same & (((uint64_t)1 << lane) - 1));
    rank[i] = *count + before;
    // (a wavefront's reads and writes of LDS happen in order: all lanes have read before one of them writes)
    if (before == 0) *count = rank[i] + __builtin_popcountll(same);
  }
  __syncthreads();
}

// Numbers of digits in wavefronts' parts -> how many items come before each: digit by digit, and within one wavefront by wavefront.
__device__ __forceinline__ void sum_counts(uint32_t (&counts)[kCounts], uint32_t (&buffer)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, at = count_at(threadIdx.x / 4, threadIdx.x % 4 * kEach);
  uint32_t v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = counts[at + i];
    sum += v[i];
  }
  uint32_t up_to = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t other = __shfl_up(up_to, d);
    if (lane >= d) up_to += other;
  }
  if (lane == 63) buffer[wave] = up_to;
  __syncthreads();
  uint32_t before = up_to - sum;
  for (int w = 0; w < wave; ++w) before += buffer[w];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    counts[at + i] = before;
    before += v[i];
  }
  __syncthreads();
}

// A token's key: its row of the table, or `rows` where it has none.
template <class ID>
__device__ __forceinline__ uint32_t key_of(const void* ids, size_t n, long long first, long long rows) {
  const long long local = (long long)static_cast<const ID*>(ids)[n] - first;
  return local >= 0 && local < rows ? (uint32_t)local : (uint32_t)rows;
}

struct SortArgs {
  const void* ids;
  uint32_t tokens;
  long long first, rows;
  int passes;                      // of 8 bits
  uint32_t *keys, *places;         // sorted: rows of the table, tokens
  uint32_t *other_keys, *other_places;
  uint32_t* table;                 // [256][tiles]
  uint32_t tiles;
};

// Up to one tile: one workgroup takes all passes in LDS.  (8192 tokens, two passes: see the head of this file.)
template <class ID>
__global__ void __launch_bounds__(kSortThreads) sort_kernel(SortArgs a) {
  __shared__ uint32_t keys[kSortTile], counts[kCounts], buffer[kWaves];
  __shared__ uint16_t places[kSortTile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t key[kSortItems], place[kSortItems], digit[kSortItems], rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    place[i] = wave * (64 * kSortItems) + i * 64 + lane;
    // those behind the last token stay behind it: they are the last ones with the greatest of keys
    key[i] = place[i] < a.tokens ? key_of<ID>(a.ids, place[i], a.first, a.rows) : (uint32_t)a.rows;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) digit[i] = key[i] >> (8 * pass) & 255u;
    rank_items(digit, rank, counts);
    sum_counts(counts, buffer);
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const uint32_t to = counts[count_at(digit[i], wave)] + rank[i];
      keys[to] = key[i];
      places[to] = (uint16_t)place[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const int at = wave * (64 * kSortItems) + i * 64 + lane;
      key[i] = keys[at];
      place[i] = places[at];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = wave * (64 * kSortItems) + i * 64 + lane;
    if (at < a.tokens) {
      a.keys[at] = key[i];
      a.places[at] = place[i];
    }
  }
}

// More than a tile: for each pass the digits' numbers in each tile, their sums, and the items to their places.
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
    if (at < a.tokens) atomicAdd(&counts[item_key<ID>(a, in, at) >> (8 * pass) & 255u], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kBins) a.table[(size_t)threadIdx.x * a.tiles + blockIdx.x] = counts[threadIdx.x];
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
    uint32_t up_to = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t other = __shfl_up(up_to, d);
      if (lane >= d) up_to += other;
    }
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
    digit[i] = key[i] >> (8 * pass) & 255u;   // those behind the last token: 255, behind all others in the last tile
  }
  rank_items(digit, rank, counts);
  // sums over the wavefronts of each digit: four lanes have a digit's sixteen numbers
  const int at_digit = count_at(threadIdx.x / 4, threadIdx.x % 4 * kEach);
  uint32_t v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    v[i] = counts[at_digit + i];
    sum += v[i];
  }
  uint32_t up_to = sum;
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    const uint32_t other = __shfl_up(up_to, d, 4);
    if ((lane & 3) >= d) up_to += other;
  }
  uint32_t before = a.table[(size_t)(threadIdx.x / 4) * a.tiles + blockIdx.x] + up_to - sum;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    counts[at_digit + i] = before;
    before += v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const uint32_t at = blockIdx.x * kSortTile + wave * (64 * kSortItems) + i * 64 + lane;
    if (at >= a.tokens) continue;
    const uint32_t to = counts[count_at(digit[i], wave)] + rank[i];
    out[to] = key[i];
    out_places[to] = place[i];
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
};

// A vector of sums into its row of the gradient, or its row plus them.
template <int DT, int DO>
__device__ __forceinline__ void store_sums(const SumArgs& a, uint32_t row, int vector, const float (&sum)[kVec<DT>]) {
  constexpr int kN = kVec<DT>;
  char* const to = a.dtable + (size_t)row * a.stride_dtable;
  const int valid = a.cols - vector * kN;
  const uint32_t at = (uint32_t)vector * kN * kBytes<DO>;
  float v[kN];
  if (a.accumulate) {
    Raw<DO, kN> old;
    old.load(to, at, valid);
    old.unpack(v);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] += a.scale * sum[j];
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] = a.scale * sum[j];
  }
  Raw<DO, kN> raw;
  raw.pack(v);
  raw.store(to, at, valid);
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

// One piece of the sorted list, in 64 vectors of the columns.  A run of tokens with the same row that begins and ends in the piece is stored; the part of one that
// comes from the piece before is kept as the piece's first, that of one which goes on (and began here) as its second.
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
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t q = i + u < count ? i + u : count - 1;
      const uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)q);
      const char* row = a.dout + (size_t)(uint32_t)__builtin_amdgcn_readlane((int)places, (int)q) * a.stride_dout;
      if (key < a.rows && i + u < count) raw[u].load(row, there ? at : 0, valid);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u >= count) break;
      const uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)(i + u));
      if (key >= a.rows) return;   // tokens without a row come last
      float v[kN];
      raw[u].unpack(v);
#pragma unroll
      for (int j = 0; j < kN; ++j) sum[j] += v[j];
      const bool last = i + u + 1 == count;
      const uint32_t next = last ? behind : (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)(i + u + 1));
      if (next == key && !last) continue;
      if (there) {
        if (!began) keep(kept_at<DT>(a, piece, 0, vector), sum);
        else if (next == key) keep(kept_at<DT>(a, piece, 1, vector), sum);
        else store_sums<DT, DO>(a, key, vector, sum);
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) sum[j] = 0.0f;
      began = true;
    }
  }
}

// First row at or behind which the sorted keys are `key` or more.
__device__ __forceinline__ uint32_t first_of(const uint32_t* keys, uint32_t count, uint32_t key) {
  uint32_t lo = 0, hi = count;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

constexpr int kZeroRows = 16;   // of a workgroup

template <int DT, int DO>
__global__ void __launch_bounds__(kThreads) sum_kernel(SumArgs a) {
  if (blockIdx.x < a.sum_groups) {
    const uint32_t chunks = (a.vectors + 63) / 64, units = a.pieces * chunks;
    for (uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + threadIdx.x / 64); unit < units; unit += a.sum_groups * (kThreads / 64))
      add_piece<DT, DO>(a, unit / chunks, (int)(unit % chunks * 64 + (threadIdx.x & 63)));
    return;
  }
  // zeros for the rows that no token has
  __shared__ uint32_t ends[kZeroRows + 1];
  constexpr int kN = kVec<DO>;
  Raw<DO> zero;
#pragma unroll
  for (int i = 0; i < zero.kWords; ++i) zero.w[i] = 0;
  for (uint32_t row0 = (blockIdx.x - a.sum_groups) * kZeroRows; row0 < a.rows; row0 += (gridDim.x - a.sum_groups) * kZeroRows) {
    if (threadIdx.x <= kZeroRows) ends[threadIdx.x] = first_of(a.keys, a.tokens, row0 + threadIdx.x);
    __syncthreads();
    for (int r = 0; r < kZeroRows; ++r) {
      if (row0 + r >= a.rows || ends[r] != ends[r + 1]) continue;
      char* const row = a.dtable + (size_t)(row0 + r) * a.stride_dtable;
      for (int x = threadIdx.x * kN; x < a.cols; x += kThreads * kN) zero.store(row, (uint32_t)x * kBytes<DO>, a.cols - x);
    }
    __syncthreads();
  }
}

// The rows whose tokens do not lie within a piece: the sums that were kept of them, from the piece that they begin in.
template <int DT, int DO>
__device__ __forceinline__ void join_from(const SumArgs& a, uint32_t piece, int vector) {
  constexpr int kN = kVec<DT>, kAhead = 4;
  typedef float f4 __attribute__((ext_vector_type(4)));
  const uint32_t from = piece * (uint32_t)a.piece, next = from + (uint32_t)a.piece;
  if (piece + 1 >= a.pieces) return;
  const uint32_t key = a.keys[next - 1];
  if (key >= a.rows || a.keys[next] != key) return;
  // a run that fills the piece and comes from the one before it began there
  if (a.keys[from] == key && from > 0 && a.keys[from - 1] == key) return;
  if (vector >= a.vectors) return;
  float sum[kN];
  const float* p = kept_at<DT>(a, piece, 1, vector);
#pragma unroll
  for (int j = 0; j < kN; ++j) sum[j] = p[j];
  const uint32_t to = first_of(a.keys, a.tokens, key + 1);               // behind the run's last token
  const uint32_t last = (to - 1) / (uint32_t)a.piece;                    // its piece
  for (uint32_t q = piece + 1; q <= last; q += kAhead) {
    f4 v[kAhead][kN / 4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int j = 0; j < kN / 4; ++j) v[u][j] = reinterpret_cast<const f4*>(kept_at<DT>(a, q + u <= last ? q + u : last, 0, vector))[j];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (q + u <= last) {
#pragma unroll
        for (int j = 0; j < kN; ++j) sum[j] += v[u][j / 4][j % 4];
      }
  }
  store_sums<DT, DO>(a, key, vector, sum);
}

template <int DT, int DO>
__global__ void __launch_bounds__(kThreads) join_kernel(SumArgs a) {
  const uint32_t chunks = (a.vectors + 63) / 64, units = a.pieces * chunks;
  for (uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + threadIdx.x / 64); unit < units; unit += gridDim.x * (kThreads / 64))
    join_from<DT, DO>(a, unit / chunks, (int)(unit % chunks * 64 + (threadIdx.x & 63)));
}

// ---- host ----------------------------------------------------------------------------------

struct Plan {
  uint32_t tiles, pieces;
  int piece, passes, vectors;
  size_t keys, places, other_keys, other_places, table, kept, bytes;
};

Plan plan_for(const struct ze_form& f) {
  Plan p = {};
  p.vectors = (int)parts(f.cols, 16 / dtype_bytes(f.dtype));
  p.tiles = (uint32_t)parts(f.tokens, kSortTile);
  p.passes = f.rows < 1u << 8 ? 1 : f.rows < 1u << 16 ? 2 : f.rows < 1u << 24 ? 3 : 4;   // keys up to `rows`
  p.piece = f.tokens <= 16384 ? 16 : f.tokens <= 65536 ? 32 : kMostPiece;
  p.pieces = (uint32_t)parts(f.tokens, (size_t)p.piece);
  Places places;
  p.keys = places.take(f.tokens * 4);
  p.places = places.take(f.tokens * 4);
  if (p.tiles > 1) {
    p.other_keys = places.take(f.tokens * 4);
    p.other_places = places.take(f.tokens * 4);
    p.table = places.take((size_t)p.tiles * kBins * 4);
  }
  p.kept = places.take((size_t)p.pieces * 2 * p.vectors * (16 / dtype_bytes(f.dtype)) * 4);
  p.bytes = places.at;
  return p;
}

template <class ID>
void sort_tokens(const SortArgs& a, const Plan& p, char* work, hipStream_t s) {
  if (p.tiles == 1) {
    hipLaunchKernelGGL(sort_kernel<ID>, dim3(1), dim3(kSortThreads), 0, s, a);
    return;
  }
  const uint32_t *in = nullptr, *in_places = nullptr;
  for (int pass = 0; pass < p.passes; ++pass) {
    const bool own = (p.passes - pass) % 2 == 1;   // the last pass writes what is read
    uint32_t *out = own ? a.keys : a.other_keys, *out_places = own ? a.places : a.other_places;
    hipLaunchKernelGGL(count_kernel<ID>, dim3(p.tiles), dim3(kSortThreads), 0, s, a, pass, in);
    hipLaunchKernelGGL(sums_kernel, dim3(1), dim3(kSortThreads), 0, s, a.table, p.tiles * kBins);
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
  if (a.pieces > 1) hipLaunchKernelGGL((join_kernel<DT, DO>), dim3(b.sum_groups), dim3(kThreads), 0, s, b);
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
    a.keys = in_work(p.keys);
    a.places = in_work(p.places);
    a.other_keys = in_work(p.other_keys);
    a.other_places = in_work(p.other_places);
    a.table = in_work(p.table);
    a.tiles = p.tiles;
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
