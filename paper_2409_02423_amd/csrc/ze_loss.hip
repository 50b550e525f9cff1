// ze_loss.hip -- gfx950 kernels and C ABI of the softmax cross entropy in include/ze.h.
//
// Forward: one matrix product of hidden states and output matrix whose tiles of logits stay in registers; each wavefront leaves the greatest
// logit and the sum of exponentials of its part of a row, a second kernel joins them.  Backward, for a piece of the vocabulary at a time: the same product again,
// whose tiles become g = dloss (softmax - onehot) in the workspace, and two products that read it, along the vocabulary for the hidden states'
// gradient and across it for the matrix's.  Tokens without a label are left out before anything else: the products work on a list of those that have
// one, so what the others hold has no part in any result.
//
// The products bound all of it, but for a few tokens, where reading the matrix does.  8192 tokens, 12608 rows of 6144 bf16 values: forward 964 us of
// product (1317 TFLOP/s; a library's bare product of that size takes 957) and 15 of the rest; backward 1014 + 938 + 860 and 44 (3 to 5 % more on other cards).  The matrix
// units are 60 to 73 % busy at the clock that their power leaves.  Four tokens: 34.0 us, 4.6 TB/s.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ze.h"
#include "ze_common.h"
#include "ze_product.h"

namespace {

constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

// ---- the tokens that have a label --------------------------------------------------------

struct Head {          // of a workspace, made on the GPU
  int rows;            // tokens with a label
  float most;          // the greatest finite |dloss| of theirs
};
constexpr size_t kHeadBytes = 256;

// Rows are numbered as the tokens with a label come; `padded` places each (a multiple of 256), those behind the last row empty.
struct List {
  Head* head;
  int* row_of;         // of each token: its row, or -1
  int* token_of;       // of each row: its token, or -1
  int* label_of;       // of each row: its label among this rank's, or -1
  float* target;       // forward: -inf, until the label's logit is known
  float *lse, *dloss;  // backward: the token's
  size_t padded;
};

constexpr int kThreads = 256;

// A copy of rows of `cols` values whose rows start at multiples of 128 bytes and end in zeros.  Row r of the copy is row token_of[r] of `in`, or of
// zeros where that is negative; without a list row r, of `rows`.
struct PackArgs {
  const char* in;
  size_t stride;        // bytes
  const int* token_of;
  size_t rows;          // of `in`, without a list
  char* out;
  size_t out_stride;    // bytes, a multiple of 128
  int cols;
};

// Of row r of the copy, 16 bytes at `at`.
template <int DT>
__device__ __forceinline__ void pack_piece(const PackArgs& a, size_t r, long long source, uint32_t at) {
  constexpr int kN = kVec<DT>;
  Raw<DT> raw;
  const int valid = source < 0 ? 0 : a.cols - (int)(at / kBytes<DT>);
  const char* in = a.in + (source < 0 ? 0 : (size_t)source) * a.stride;
  if (valid >= kN) {
    raw.load(in, at);
  } else {
#pragma unroll
    for (int i = 0; i < raw.kWords; ++i) raw.w[i] = 0;
    if (valid > 0) raw.load(in, at, valid);
  }
  raw.store(a.out + r * a.out_stride, at);
}
__device__ __forceinline__ long long source_of(const PackArgs& a, size_t r) { return a.token_of ? (long long)a.token_of[r] : r < a.rows ? (long long)r : -1; }

template <int DT>
__device__ __forceinline__ void pack_row(const PackArgs& a, size_t r) {
  const long long source = source_of(a, r);
  for (uint32_t at = threadIdx.x * 16; at < a.out_stride; at += kThreads * 16) pack_piece<DT>(a, r, source, at);
}

// The same of rows of one step each (a row's ends), `many` rows from `first` on: eight lanes a row.
template <int DT>
__device__ __forceinline__ void pack_ends(const PackArgs& a, size_t first, size_t many) {
  const size_t r = first + threadIdx.x / 8;
  if (r < many) pack_piece<DT>(a, r, source_of(a, r), threadIdx.x % 8 * 16);
}

template <int DT>
__global__ void __launch_bounds__(kThreads) pack_kernel(PackArgs a, size_t from) {
  pack_row<DT>(a, from + blockIdx.x);
}

__device__ __forceinline__ void zero_row(char* row, size_t bytes) {
  const size_t head = (16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15;
  if (bytes <= head) {
    for (size_t i = threadIdx.x * 2; i < bytes; i += kThreads * 2) *reinterpret_cast<uint16_t*>(row + i) = 0;
    return;
  }
  const size_t body = (bytes - head) / 16;
  for (size_t i = threadIdx.x; i < body; i += kThreads) reinterpret_cast<i32x4*>(row + head)[i] = i32x4{0, 0, 0, 0};
  for (size_t i = threadIdx.x * 2; i < head; i += kThreads * 2) *reinterpret_cast<uint16_t*>(row + i) = 0;
  for (size_t i = head + body * 16 + threadIdx.x * 2; i < bytes; i += kThreads * 2) *reinterpret_cast<uint16_t*>(row + i) = 0;
}

constexpr int kListThreads = 1024, kListRounds = 8;

// The rows' ends that the products need beside the list, of the table and of the hidden states (none where out is NULL).
struct EndsArgs {
  PackArgs of[2];
  unsigned groups;     // of the first, kListThreads / 8 rows each
};

// One workgroup makes the list.  A token's row is the number of those before it: counted in the lanes before its own, the wavefronts before its own, and
// the rounds before its own, 8 x 1024 tokens at a time.  The others copy the rows' ends meanwhile (a launch less: 301 tokens, 5003 rows of 1025 fp32 values
// 3.0 us in all).  8192 tokens take 6.1 us, with what the backward call copies of each 8.0: the steps that wait for one another, not what is read.
template <class ID, int DT>
__global__ void __launch_bounds__(kListThreads) list_kernel(const ID* ids, int tokens, long long first, long long rows, const float* lse, const float* dloss, List list,
                                                            EndsArgs ends) {
  if (blockIdx.x > 0) {
    const unsigned group = blockIdx.x - 1;
    const PackArgs& a = ends.of[group < ends.groups ? 0 : 1];
    pack_ends<DT>(a, (size_t)(group < ends.groups ? group : group - ends.groups) * (kListThreads / 8), a.rows);
    return;
  }
  __shared__ int counts[kListRounds * 16 + 1];
  __shared__ float greatest[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  int before = 0;
  float most = 0.0f;
  for (int base = 0; base < tokens; base += kListRounds * kListThreads) {
    long long id[kListRounds];
    float of_lse[kListRounds], of_dloss[kListRounds];
#pragma unroll
    for (int i = 0; i < kListRounds; ++i) {
      const int n = base + i * kListThreads + tid;
      id[i] = n < tokens ? (long long)ids[n] : -1;
      if (lse) {
        of_lse[i] = n < tokens ? lse[n] : 0.0f;
        of_dloss[i] = n < tokens ? dloss[n] : 0.0f;
      }
    }
    uint64_t there[kListRounds];
#pragma unroll
    for (int i = 0; i < kListRounds; ++i) {
      there[i] = __builtin_amdgcn_ballot_w64(id[i] >= 0);
      if (lane == 0) counts[i * 16 + wave] = __builtin_popcountll(there[i]);
    }
    __syncthreads();
    if (wave == 0) {
      const int a = counts[2 * lane], b = counts[2 * lane + 1], sum = (int)sum_up_to((uint32_t)(a + b));
      counts[2 * lane] = sum - a - b;
      counts[2 * lane + 1] = sum - b;
      if (lane == 63) counts[kListRounds * 16] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kListRounds; ++i) {
      const int n = base + i * kListThreads + tid;
      if (n >= tokens) continue;
      const int row = before + counts[i * 16 + wave] + __builtin_popcountll(there[i] & (((uint64_t)1 << lane) - 1));
      const bool has = id[i] >= 0;
      list.row_of[n] = has ? row : -1;
      if (!has) continue;
      list.token_of[row] = n;
      list.label_of[row] = (int)row_of_id(id[i], first, rows);
      if (list.target) list.target[row] = -kInf;
      if (lse) {
        const float size = fabsf(of_dloss[i]);
        list.lse[row] = of_lse[i];
        list.dloss[row] = of_dloss[i];
        if (size < kInf) most = fmaxf(most, size);
      }
    }
    before += counts[kListRounds * 16];
    __syncthreads();
  }
  for (size_t row = (size_t)before + tid; row < list.padded; row += kListThreads) {
    list.token_of[row] = -1;
    list.label_of[row] = -1;
    if (lse) list.lse[row] = list.dloss[row] = 0.0f;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  if (lane == 0) greatest[wave] = most;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 16; ++w) most = fmaxf(most, greatest[w]);
    list.head->rows = before;
    list.head->most = most;
  }
}

// ---- rows where the products can read them -----------------------------------------------

// The rows with a label, packed; and zeros for the gradients of the hidden states of tokens without one.  (One pass over them, 31.5 us for 8192 x 6144 bf16 values, 6.4 TB/s: the
// matrix's gradient runs over them across k, where a list of places would be one for each row of each step.  After it the hidden states themselves are not read any
// more, and the rows that are read are not those that get zeros: so the gradients may take their place.)
template <int DT>
__global__ void __launch_bounds__(kThreads) pack_hidden_kernel(PackArgs a, size_t from, const int* row_of, size_t tokens, char* dhidden, size_t dhidden_stride) {
  const size_t r = from + blockIdx.x;
  pack_row<DT>(a, r);
  if (dhidden && r < tokens && row_of[r] < 0) zero_row(dhidden + r * dhidden_stride, (size_t)a.cols * kBytes<DT>);
}

__global__ void __launch_bounds__(kThreads) zero_rows_kernel(char* out, size_t stride, size_t bytes, size_t from) {
  zero_row(out + (from + blockIdx.x) * stride, bytes);
}

// Values of a row in two 16 x 16 products beside one another: a lane has v at x and w at x + 16, four of each.  Half precision: lanes of
// neighbouring groups exchange theirs, so that each has eight that follow one another and a row's 64 bytes go out at once (as four times eight bytes for each
// of the two they took the caches twice as many requests).  Values at `cols` and behind it are left out.
template <int DT>
__device__ __forceinline__ void store_pair(char* row, int x, int cols, const float (&v)[4], const float (&w)[4]) {
  Raw<DT, 4> a, b;
  a.pack(v);
  b.pack(w);
  if constexpr (DT == kF32) {
    a.store(row, x * 4, cols - x);
    b.store(row, (x + 16) * 4, cols - x - 16);
  } else {
    const auto low = __builtin_amdgcn_permlane16_swap(a.w[0], b.w[0], false, false), high = __builtin_amdgcn_permlane16_swap(a.w[1], b.w[1], false, false);
    Raw<DT> both;
    both.w[0] = low[0];
    both.w[1] = high[0];
    both.w[2] = low[1];
    both.w[3] = high[1];
    const int group = (threadIdx.x & 63) / 16, to = x - 4 * group + 16 * (group & 1) + 8 * (group / 2);
    both.store(row, to * 2, cols - to);
  }
}

__device__ __forceinline__ bool any_lane(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

// ---- forward -----------------------------------------------------------------------------

struct Part {
  float most, sum;
};

struct LogitsArgs {
  Matrix table, hidden;        // the piece's rows; the rows with a label
  Ends table_ends, hidden_ends;
  const Head* head;
  const int* label_of;
  int nx, ny, steps;           // tiles, and steps of k
  int v0, rows;                // the piece's first row and number of rows
  float scale;
  Part* parts;                 // [rows with a label][stride], this piece's first
  size_t parts_stride;
  float* target;
};

// The tiles of the products of hidden states and rows of the table, whose ends may be apart: of the rows that have a label, as many for each XCD, however many
// tokens have none.
template <int DT, class S, class ARGS, class Use>
__device__ __forceinline__ void logits_of_tiles(const ARGS& a, int there, const Use& use) {
  using Both = Operands<DT, S, kAlong, kAlong>;
  products<Both>(
      Tiles(a.nx, (there + S::BY - 1) / S::BY), a.steps, a.table_ends.at != nullptr, [&](Both& both, int tx, int ty) { both.start(a.table, a.hidden, tx, ty); },
      [&](Both& both, int tx, int ty) {
        both.start(Matrix{a.table_ends.at, a.table_ends.bytes, a.table_ends.stride, nullptr},
                   Matrix{a.hidden_ends.at, a.hidden_ends.bytes, a.hidden_ends.stride, a.hidden_ends.places},
                   tx, ty);
      },
      use);
}

// The greatest logit and the sum of exponentials in each wavefront's part of a row.  In a tile that is all there is of them: 4 x 16 columns to
// a lane group, so a row's maximum takes NX x 4 comparisons in a lane and two across lanes.
template <int DT, class S>
__device__ __forceinline__ void use_logits(const LogitsArgs& a, int there, f32x4 (&sum)[S::NX][S::NY], int tx, int ty) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wx = wave % S::WX, wy = wave / S::WX;
  const int x_wave = __builtin_amdgcn_readfirstlane(tx * S::BX + wx * (S::BX / S::WX));
  const bool edge = x_wave + S::BX / S::WX > a.rows;
  const int x0 = tx * S::BX + wx * (S::BX / S::WX) + lane / 16 * 4, y0 = ty * S::BY + wy * (S::BY / S::WY) + (lane & 15);
  int labels[S::NY];   // asked for at once (there are places for whole tiles of rows)
#pragma unroll
  for (int j = 0; j < S::NY; ++j) labels[j] = a.label_of[y0 + 16 * j];
  have_come(labels);
#pragma unroll
  for (int j = 0; j < S::NY; ++j) {
    rest_of_sums<S>(sum, j);
    const int y = y0 + 16 * j;
    if (y >= there) continue;
    const int label = labels[j] - a.v0;
    f32x4 l[S::NX];
#pragma unroll
    for (int i = 0; i < S::NX; ++i) l[i] = a.scale * sum[i][j];
    if (edge) {
#pragma unroll
      for (int i = 0; i < S::NX; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) l[i][r] = x0 + 16 * i + r < a.rows ? l[i][r] : -kInf;
    }
    if (any_lane((unsigned)(label - x_wave) < (unsigned)(S::BX / S::WX))) {   // few parts of rows have a label
#pragma unroll
      for (int i = 0; i < S::NX; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (x0 + 16 * i + r == label && label < a.rows) a.target[y] = l[i][r];
    }
    float most = -kInf;
#pragma unroll
    for (int i = 0; i < S::NX; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) most = fmaxf(most, l[i][r]);
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    const float from = most == -kInf ? 0.0f : most;   // nothing there: exp(-inf) = 0 each
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < S::NX; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) total += __builtin_amdgcn_exp2f((l[i][r] - from) * kLog2E);
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    if (lane < 16) a.parts[y * a.parts_stride + tx * S::WX + wx] = Part{most, total};
  }
}
template <int DT, class S>
__global__ void __launch_bounds__(S::kThreads) logits_kernel(LogitsArgs a) {
  const int there = a.head->rows;
  logits_of_tiles<DT, S>(a, there, [&](f32x4 (&sum)[S::NX][S::NY], int tx, int ty) { use_logits<DT, S>(a, there, sum, tx, ty); });
}

template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)));
}
// The greatest of the 64 lanes' values, in every lane.  All 64 have to be active.
__device__ __forceinline__ float wave_max(float v) {
  v = dpp_max<0xB1>(v);    // quad_perm 1 0 3 2
  v = dpp_max<0x4E>(v);    // quad_perm 2 3 0 1
  v = dpp_max<0x141>(v);   // row_half_mirror
  v = dpp_max<0x140>(v);   // row_mirror
  return fmaxf(fmaxf(read_lane(v, 0), read_lane(v, 16)), fmaxf(read_lane(v, 32), read_lane(v, 48)));
}

// Joins parts of a sum of exponentials: the sums are taken to the greater of the two logits.  (Where that is -inf there is nothing in either.)
__device__ __forceinline__ void join(float& most, float& total, float other_most, float other) {
  const float to = fmaxf(most, other_most), from = to == -kInf ? 0.0f : to;
  total = total * __builtin_amdgcn_exp2f((most - from) * kLog2E) + other * __builtin_amdgcn_exp2f((other_most - from) * kLog2E);
  most = to;
}

// Joins a row's parts: a wavefront for each token, eight parts of a lane asked for at once.  8192 tokens of 100 parts 4.7 us, four of 788 4.6: a chain of loads.
__global__ void __launch_bounds__(kThreads) stats_kernel(const int* row_of, size_t tokens, const Part* parts, size_t stride, size_t count, const float* target,
                                                         float* stats) {
  const size_t n = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  const int lane = threadIdx.x & 63;
  if (n >= tokens) return;
  const int row = row_of[n];
  float most = -kInf, total = 0.0f, label = 0.0f;
  if (row >= 0) {
    label = target[row];
    const Part* p = parts + (size_t)row * stride;
    constexpr int kAhead = 8;
    for (size_t i = lane; i < count; i += 64 * kAhead) {
      Part part[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) part[u] = i + 64 * u < count ? p[i + 64 * u] : Part{-kInf, 0.0f};
      float to = most;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) to = fmaxf(to, part[u].most);
      const float from = to == -kInf ? 0.0f : to;
      total *= __builtin_amdgcn_exp2f((most - from) * kLog2E);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) total += part[u].sum * __builtin_amdgcn_exp2f((part[u].most - from) * kLog2E);
      most = to;
    }
    const float to = wave_max(most), from = to == -kInf ? 0.0f : to;
    total = wave_sum(total * __builtin_amdgcn_exp2f((most - from) * kLog2E));
    most = to;
  }
  if (lane == 0) {
    stats[n] = most;
    stats[tokens + n] = total;
    stats[2 * tokens + n] = label;
  }
}

template <class ID>
__global__ void __launch_bounds__(kThreads) join_kernel(size_t tokens, int ranks, const float* stats, const ID* ids, float* loss, float* lse) {
  const size_t n = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (n >= tokens) return;
  if (ids[n] < 0) {
    if (loss) loss[n] = 0.0f;
    lse[n] = 0.0f;
    return;
  }
  float most = -kInf, total = 0.0f, target = -kInf;
#pragma unroll 4
  for (int r = 0; r < ranks; ++r) {
    const float* of = stats + (size_t)r * 3 * tokens + n;
    join(most, total, of[0], of[tokens]);
    target = fmaxf(target, of[2 * tokens]);
  }
  const float l = (most == -kInf ? 0.0f : most) + logf(total);
  lse[n] = l;
  if (loss) loss[n] = l - target;
}

// ---- backward ----------------------------------------------------------------------------

// What g is multiplied by before it is rounded, beside 1 / max |dloss|.
template <int DT> constexpr float kLift = DT == kF16 ? 32768.0f : 1.0f;

struct GradientArgs {
  Matrix table, hidden;
  Ends table_ends, hidden_ends;
  const Head* head;
  const int* label_of;
  const float *lse, *dloss;
  int nx, ny, steps;
  int v0, rows, rows_padded;   // of the piece; padded to whole steps
  float scale;
  char* g;                     // [rows with a label, to a whole step], the piece's first column
  size_t g_stride;             // bytes
};

// g of a tile, zeros behind the piece's last row and behind the last row with a label, up to whole steps of the products that read it.
template <int DT, class S>
__device__ __forceinline__ void use_gradient(const GradientArgs& a, int there, float most, f32x4 (&sum)[S::NX][S::NY], int tx, int ty) {
  const int padded = (there + kStep<DT> - 1) / kStep<DT> * kStep<DT>;
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wx = wave % S::WX, wy = wave / S::WX;
  const int x_wave = __builtin_amdgcn_readfirstlane(tx * S::BX + wx * (S::BX / S::WX));
  const bool edge = x_wave + S::BX / S::WX > a.rows || (ty + 1) * S::BY > there;
  const int x0 = tx * S::BX + wx * (S::BX / S::WX) + lane / 16 * 4, y0 = ty * S::BY + wy * (S::BY / S::WY) + (lane & 15);
  int labels[S::NY];   // asked for at once (there are places for whole tiles of rows)
  float of_lse[S::NY], of_dloss[S::NY];
#pragma unroll
  for (int j = 0; j < S::NY; ++j) {
    labels[j] = a.label_of[y0 + 16 * j];
    of_lse[j] = a.lse[y0 + 16 * j];
    of_dloss[j] = a.dloss[y0 + 16 * j];
  }
  have_come(labels);
  have_come(of_lse);
  have_come(of_dloss);
#pragma unroll
  for (int j = 0; j < S::NY; ++j) {
    rest_of_sums<S>(sum, j);
    const int y = y0 + 16 * j;
    if (y >= padded) continue;
    const int label = labels[j] - a.v0;
    const float lse = of_lse[j], factor = most > 0.0f ? of_dloss[j] / most * kLift<DT> : of_dloss[j];
    char* const row = a.g + (size_t)y * a.g_stride;
    const bool has = any_lane((unsigned)(label - x_wave) < (unsigned)(S::BX / S::WX));   // few parts of rows have a label
#pragma unroll
    for (int i = 0; i < S::NX; i += 2) {
      float v[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int x = x0 + 16 * (i + k);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[k][r] = factor * __builtin_amdgcn_exp2f(fmaf(a.scale, sum[i + k][j][r], -lse) * kLog2E);
        if (has) {
#pragma unroll
          for (int r = 0; r < 4; ++r) v[k][r] -= x + r == label ? factor : 0.0f;
        }
        if (edge) {
#pragma unroll
          for (int r = 0; r < 4; ++r) v[k][r] = x + r < a.rows && y < there ? v[k][r] : 0.0f;
        }
      }
      store_pair<DT>(row, x0 + 16 * i, a.rows_padded, v[0], v[1]);
    }
  }
}
template <int DT, class S>
__global__ void __launch_bounds__(S::kThreads) gradient_kernel(GradientArgs a) {
  const int there = a.head->rows;
  const float most = a.head->most;
  logits_of_tiles<DT, S>(a, there, [&](f32x4 (&sum)[S::NX][S::NY], int tx, int ty) { use_gradient<DT, S>(a, there, most, sum, tx, ty); });
}

// out[y][x] from a tile's sums.
struct OutArgs {
  Matrix mx, my;
  const Head* head;
  int nx, ny, steps;
  int cols, rows;              // of the output: x, and y where they are not the rows with a label
  float scale;
  char* out;                   // of type DT
  size_t out_stride;           // bytes
  const int* token_of;         // of each y: its row of the output
  float* kept;                 // fp32 sums, [splits][rows with a label, to whole tiles][kept_stride]
  size_t kept_stride;
  int add, last;               // whether there are kept sums of pieces before this one, and whether this is the last one
  int sharers, most_splits;    // see splits_of
};

// How many workgroups share the steps of a tile: where the rows with a label make few tiles, as many as there are sharers for.  (Only the GPU knows how
// many rows those are; the sums that are kept are added up in the order of the shares.)
template <class S>
__device__ __forceinline__ int splits_of(int rows, int nx, int sharers, int most) {
  const int tiles = nx * ((rows + S::BY - 1) / S::BY), splits = tiles ? sharers / tiles : 1;
  return splits < 1 ? 1 : splits < most ? splits : most;
}

// The matrix's gradient: x along the columns, y the piece's rows, k the rows with a label.
template <int DT, class S>
__device__ __forceinline__ void use_table_gradient(const OutArgs& a, float factor, f32x4 (&sum)[S::NX][S::NY], int tx, int ty) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wx = wave % S::WX, wy = wave / S::WX;
  const int x0 = tx * S::BX + wx * (S::BX / S::WX) + lane / 16 * 4, y0 = ty * S::BY + wy * (S::BY / S::WY) + (lane & 15);
#pragma unroll
  for (int j = 0; j < S::NY; ++j) {
    rest_of_sums<S>(sum, j);
    const int y = y0 + 16 * j;
    if (y >= a.rows) continue;
    char* const row = a.out + (size_t)y * a.out_stride;
#pragma unroll
    for (int i = 0; i < S::NX; i += 2) {
      float v[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[k][r] = factor * sum[i + k][j][r];
      store_pair<DT>(row, x0 + 16 * i, a.cols, v[0], v[1]);
    }
  }
}
template <int DT, class S>
__global__ void __launch_bounds__(S::kThreads) table_gradient_kernel(OutArgs a) {
  using Both = Operands<DT, S, kAcross, kAcross>;
  const int there = a.head->rows;
  const float factor = a.scale * (a.head->most / kLift<DT>);
  const auto start = [&](Both& both, int tx, int ty) { both.start(a.mx, a.my, tx, ty); };
  products<Both>(Tiles(a.nx, a.ny), (there + kStep<DT> - 1) / kStep<DT>, false, start, start,
                 [&](f32x4 (&sum)[S::NX][S::NY], int tx, int ty) { use_table_gradient<DT, S>(a, factor, sum, tx, ty); });
}

// The hidden states' gradient: x along the columns, y the rows with a label, k the piece's rows, which several workgroups may share.
template <int DT, class S>
__device__ __forceinline__ void use_hidden_gradient(const OutArgs& a, int there, int ny, int split, bool finish, float factor, f32x4 (&sum)[S::NX][S::NY], int tx, int ty) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wx = wave % S::WX, wy = wave / S::WX;
  const int x0 = tx * S::BX + wx * (S::BX / S::WX) + lane / 16 * 4, y0 = ty * S::BY + wy * (S::BY / S::WY) + (lane & 15);
  int tokens[S::NY];   // asked for at once (there are places for whole tiles of rows)
#pragma unroll
  for (int j = 0; j < S::NY; ++j) tokens[j] = a.token_of[y0 + 16 * j];
  have_come(tokens);
#pragma unroll
  for (int j = 0; j < S::NY; ++j) {
    rest_of_sums<S>(sum, j);
    const int y = y0 + 16 * j;
    if (y >= there) continue;
    char* const row = finish ? a.out + (size_t)tokens[j] * a.out_stride : nullptr;
    float* const kept = a.kept + ((size_t)split * ny * S::BY + y) * a.kept_stride;
#pragma unroll
    for (int i = 0; i < S::NX; i += 2) {
      float v[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int x = x0 + 16 * (i + k);
        f32x4 s = sum[i + k][j];
        if (a.add && x < a.cols) s += *reinterpret_cast<const f32x4*>(kept + x);   // (kept rows are a multiple of 4 wide)
        if (!finish && x < a.cols) *reinterpret_cast<f32x4*>(kept + x) = s;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[k][r] = factor * s[r];
      }
      if (finish) store_pair<DT>(row, x0 + 16 * i, a.cols, v[0], v[1]);
    }
  }
}
template <int DT, class S>
__global__ void __launch_bounds__(S::kThreads) hidden_gradient_kernel(OutArgs a) {
  using Both = Operands<DT, S, kAcross, kAlong>;
  const int there = a.head->rows, splits = splits_of<S>(there, a.nx, a.sharers, a.most_splits), ny = (there + S::BY - 1) / S::BY;
  const float factor = a.scale * (a.head->most / kLift<DT>);
  const bool finish = a.last && splits == 1;
  // the steps, shared out: where there are several parts of them a workgroup has one tile, and so one part
  const Tiles tiles(a.nx, ny * splits);
  if (tiles.count == 0) return;
  int tx, ty;
  tiles.at(0, tx, ty);
  const int split = splits == 1 ? 0 : ty / ny;
  const int from = (int)((long long)a.steps * split / splits), to = (int)((long long)a.steps * (split + 1) / splits);
  Matrix mx = a.mx, my = a.my;
  const size_t skip = (size_t)from * kStep<DT> * mx.stride;
  mx.at += skip < mx.bytes ? skip : mx.bytes;
  mx.bytes -= skip < mx.bytes ? skip : mx.bytes;
  my.at += (size_t)from * kStepBytes;
  my.bytes -= (size_t)from * kStepBytes;
  const auto start = [&](Both& both, int tx, int ty) { both.start(mx, my, tx, ty - split * ny); };
  products<Both>(tiles, to - from, false, start, start, [&](f32x4 (&sum)[S::NX][S::NY], int tx, int ty) {
    use_hidden_gradient<DT, S>(a, there, ny, split, finish, factor, sum, tx, ty - split * ny);
  });
}

// The sums that several workgroups have kept of each place, one after the other.
template <int DT, class S>
__global__ void __launch_bounds__(kThreads) hidden_finish_kernel(OutArgs a) {
  const int there = a.head->rows, splits = splits_of<S>(there, a.nx, a.sharers, a.most_splits), x = (blockIdx.x * kThreads + threadIdx.x) * 4;
  if (splits == 1 || x >= a.cols) return;
  const size_t split = (size_t)((there + S::BY - 1) / S::BY) * S::BY * a.kept_stride;
  const float factor = a.scale * (a.head->most / kLift<DT>);
  for (int y = blockIdx.y; y < there; y += gridDim.y) {
    const float* kept = a.kept + (size_t)y * a.kept_stride + x;
    f32x4 s = *reinterpret_cast<const f32x4*>(kept);
    constexpr int kAhead = 4;
    for (int i = 1; i < splits; i += kAhead) {
      f32x4 more[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) more[u] = *reinterpret_cast<const f32x4*>(kept + (i + u < splits ? i + u : i) * split);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u < splits) s += more[u];
    }
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = factor * s[r];
    Raw<DT, 4> raw;
    raw.pack(v);
    raw.store(a.out + (size_t)a.token_of[y] * a.out_stride, x * kBytes<DT>, a.cols - x);
  }
}

// ---- host: how a call is laid out ----------------------------------------------------------

using Large = Shape<256, 256, 2, 2, 2, true>;   // half precision
using Half = Shape<256, 128, 2, 2, 2, true>;    // the same
using Deep = Shape<256, 128, 2, 2, 3, true>;    // a half one for many steps: three under way
using Medium = Shape<128, 128, 2, 2, 2>;
using Small = Shape<64, 64, 2, 2, 4>;
// Logits of up to 16 tokens: what counts is how many compute units read the table, and how much of it they have under way (4 tokens, 12608 rows of 6144 bf16
// values 34.0 us, 4.6 TB/s, where a plain copy reaches 4.8).
using Thin = Shape<32, 16, 2, 1, 8>;
enum { kLarge, kHalf, kMedium, kSmall, kThin, kShapes };
struct Size {
  int x, y;         // of a tile
  int part;         // columns of a wavefront
  int at_once;      // workgroups of a compute unit
  int cost;         // of a value, in hundredths of that in a large tile where there are many tiles
};
template <class S>
constexpr Size size_of(int at_once, int cost) {
  return Size{S::BX, S::BY, S::BX / S::WX, at_once, cost};
}
constexpr Size kSizes[kShapes] = {size_of<Large>(1, 100), size_of<Half>(1, 115), size_of<Medium>(2, 145), size_of<Small>(2, 220), size_of<Thin>(3, 0)};
constexpr int kComputeUnits = 256;
constexpr size_t kMostTiles = (size_t)1 << 22;   // of one launch

size_t tiles(int shape, size_t nx, size_t ny) { return parts(nx, kSizes[shape].x) * parts(ny, kSizes[shape].y); }

// Workgroups of a launch: one for each tile, or, where a workgroup goes on from tile to tile, for each compute unit.
template <class S>
unsigned groups_for(size_t tiles) {
  return (unsigned)(S::kByHand && tiles > kComputeUnits ? kComputeUnits : tiles);
}

// The shape that takes the least time: as many tiles one after the other as the busiest compute unit has, times what one costs.  Small tiles where a y is
// no longer than one of them: then x is read, and little else.  Forward calls with all tiles of one shape, us:
//
//     tokens x rows x cols             large   half   medium   small
//     8192 x 12288 x 6144 bf16           993   1121     1188    1868
//     2048 x 4000 x 1024 bf16             43     32       32      45
//     1024 x 4000 x 1024 bf16             42     30       26      29
//     512 x 12608 x 2048 bf16             64     44       46      60
//     256 x 1000 x 1024 bf16              40     29       23      19
//     4096 x 8192 x 4096 fp32                          1922    2119
//     300 x 16000 x 1024 fp32                           133     101
//
// The rule takes the least of each line.
int shape_for(int dtype, size_t nx, size_t ny) {
  if (ny <= (size_t)kSizes[kSmall].y) return kSmall;
  int best = kSmall;
  size_t least = ~(size_t)0;
  for (int s = dtype == ZC_F32 ? kMedium : kLarge; s <= kSmall; ++s) {
    // (fp32 products are bound by the matrix instructions in every shape, by those alone in the larger one)
    const size_t cost = dtype != ZC_F32 ? kSizes[s].cost : s == kMedium ? 100 : 115;
    const size_t time = parts(tiles(s, nx, ny), kComputeUnits) * kSizes[s].x * kSizes[s].y * cost;
    if (time < least) {
      least = time;
      best = s;
    }
  }
  return best;
}

#define ZE_BY_SHAPE_AND(HALF, SHAPE, DT, LAUNCH)    \
  do {                                              \
    if ((SHAPE) == kMedium) LAUNCH(DT, Medium);     \
    else if ((SHAPE) == kSmall) LAUNCH(DT, Small);  \
    else if constexpr (DT != kF32) {                \
      if ((SHAPE) == kHalf) LAUNCH(DT, HALF);       \
      else LAUNCH(DT, Large);                       \
    }                                               \
  } while (0)
#define ZE_BY_SHAPE(SHAPE, DT, LAUNCH) ZE_BY_SHAPE_AND(Half, SHAPE, DT, LAUNCH)
#define ZE_BY_SHAPE_OF_HIDDEN(SHAPE, DT, LAUNCH) ZE_BY_SHAPE_AND(Deep, SHAPE, DT, LAUNCH)
#define ZE_BY_SHAPE_OF_LOGITS(SHAPE, DT, LAUNCH)    \
  do {                                              \
    if ((SHAPE) == kThin) LAUNCH(DT, Thin);         \
    else ZE_BY_SHAPE(SHAPE, DT, LAUNCH);            \
  } while (0)
#define ZE_BY_TYPE(TYPE, CALL)             \
  do {                                     \
    if ((TYPE) == ZC_F32) CALL(kF32);      \
    else if ((TYPE) == ZC_BF16) CALL(kBF16); \
    else CALL(kF16);                       \
  } while (0)

// A call's workspace and the way it takes.
struct Plan {
  size_t e, padded;                  // bytes of a value; tokens, to whole tiles
  size_t cols_padded;                // to whole steps
  int steps;                         // whole ones
  bool ends;                         // whether rows have an end behind them
  size_t stride_hidden, stride_table;   // bytes
  bool pack_hidden, pack_table;
  size_t piece;                      // rows of the table at a time
  int shape;                         // of the logits
  size_t parts;                      // forward: of a row
  int hidden_shape, sharers, most_splits;   // backward
  size_t list[7], packed_hidden, packed_table, table_ends, hidden_ends, part, g, kept, bytes;
};

constexpr size_t kMostPacked = (size_t)64 << 20;   // bytes of the table that are copied at a time

bool readable(const void* p, size_t stride_bytes) {
  return aligned(p, 4) && stride_bytes % 4 == 0;
}

// Whether the operands are copied to where a product can read them decides what the workspace holds.
Plan plan_with(const struct ze_form& f, bool backward, size_t piece, bool pack_hidden, bool pack_table) {
  Plan p = {};
  p.pack_hidden = pack_hidden;
  p.pack_table = pack_table;
  p.e = dtype_bytes(f.dtype);
  p.padded = up(f.tokens, 256);
  p.cols_padded = up(f.cols, kStepBytes / p.e);
  p.stride_hidden = stride_of(f.stride_tokens, f.cols) * p.e;
  p.stride_table = stride_of(f.stride_table, f.cols) * p.e;
  if (backward) {
    const size_t most = ((size_t)128 << 20) / (f.tokens ? f.tokens : 1);
    p.piece = piece ? up(piece < f.rows ? piece : f.rows, 256) : most > 4096 ? most / 256 * 256 : 4096;
  } else {
    p.piece = f.rows;
  }
  const size_t limit = kMostTiles / parts(p.padded, 64) / 4 * 256;    // tiles of a launch, were they small ones
  if (p.piece > limit) p.piece = limit;
  if (pack_table) {
    const size_t most = kMostPacked / (p.cols_padded * p.e) / 256 * 256;
    if (p.piece > most) p.piece = most > 256 ? most : 256;
  }
  if (p.piece > f.rows) p.piece = f.rows;
  if (backward && !piece && p.piece && p.piece < f.rows) {   // pieces of the same size
    const size_t n = parts(f.rows, p.piece);
    const size_t even = up(parts(f.rows, n), 256);
    if (even < p.piece) p.piece = even;
  }
  p.shape = shape_for(f.dtype, p.piece, f.tokens);
  if (!backward && f.tokens <= Thin::BY) p.shape = kThin;
  // (The ends are added first also where a copy has them behind the rest: the sums do not depend on where the tensors lie, as long as a copied table
  // comes in the pieces that it would be taken in where it lies.  Of more than kMostPacked bytes it may come in more, whose tiles may have another shape.)
  p.steps = (int)(f.cols * p.e / kStepBytes);
  p.ends = f.cols * p.e % kStepBytes != 0;
  Places places;
  places.take(kHeadBytes);
  for (int i = 0; i < 7; ++i) p.list[i] = places.take(p.padded * 4);
  p.packed_hidden = places.take(backward || pack_hidden ? p.padded * p.cols_padded * p.e : 0);
  p.packed_table = places.take(pack_table ? p.piece * p.cols_padded * p.e : 0);
  p.table_ends = places.take(p.ends ? f.rows * kStepBytes : 0);
  p.hidden_ends = places.take(p.ends && !backward && !pack_hidden ? f.tokens * kStepBytes : 0);
  if (!backward) {
    const size_t part = kSizes[p.shape].part;
    p.parts = p.piece ? parts(f.rows, p.piece) * parts(up(p.piece, 256), part) : 0;
    p.part = places.take(f.tokens * p.parts * sizeof(Part));
  } else {
    const size_t padded = up(p.piece, kStepBytes / p.e);
    p.g = places.take(p.padded * padded * p.e);
    const size_t steps = padded * p.e / kStepBytes;
    p.hidden_shape = shape_for(f.dtype, f.cols, f.tokens);
    // Where a tile's steps are shared out, few tiles are as good as many.  Large ones then keep twice the sums that half ones do, which pays once there are
    // many steps for each compute unit.  Backward calls without the matrix's gradient, bf16, large / half tiles in us, with all tokens labelled and
    // with half of them:
    //
    //     tokens x rows x cols     steps of all large tiles / compute units
    //     1024 x 2000 x 2048         4          54.7 / 48.5      47.3 / 41.2
    //     1024 x 8000 x 2048        16          93.1 / 88.4      79.3 / 72.1
    //     1024 x 16000 x 2048       31         140.0 / 138.7    108.5 / 104.2
    //     1024 x 32003 x 2048       63         234.9 / 242.1    139.2 / 139.7
    //     512 x 32003 x 4096        63         234.7 / 257.6    191.9 / 185.9
    //     2047 x 32003 x 2048      125         438.5 / 470.3    240.4 / 243.8
    //
    // Below 32 half ones were as fast or faster in all of 120 calls, up to 1.16 times; from 125 on large ones in all of 10.
    constexpr size_t kManySteps = 48;
    if (f.dtype != ZC_F32 && f.tokens > (size_t)kSizes[kSmall].y && p.hidden_shape != kLarge && tiles(kHalf, f.cols, f.tokens) * (steps / 8) >= kComputeUnits)
      p.hidden_shape = tiles(kLarge, f.cols, f.tokens) * steps >= kManySteps * kComputeUnits ? kLarge : kHalf;
    const Size& size = kSizes[p.hidden_shape];
    p.sharers = size.at_once * kComputeUnits;   // as many as run at once
    p.most_splits = (int)(steps < 16 ? 1 : steps / 8);
    if (p.piece < f.rows || p.most_splits > 1) {
      // splits x rows is greatest where all sharers have a tile, or all rows one
      const size_t rows = up(f.tokens, size.y), shared = parts((size_t)p.sharers, parts(f.cols, size.x)) * size.y;
      p.kept = places.take((rows > shared ? rows : shared) * up(f.cols, 4) * 4);
    }
  }
  p.bytes = places.at;
  return p;
}

// The plan for tensors where they lie; NULL: for the place that asks for most.
Plan plan_for(const struct ze_form& f, bool backward, size_t piece, const void* d_hidden, const void* d_table) {
  const size_t e = dtype_bytes(f.dtype), stride = stride_of(f.stride_tokens, f.cols) * e;
  // a list of rows tells places apart by 32 bits
  const bool pack_hidden = !d_hidden || !readable(d_hidden, stride) || f.tokens * (stride > kStepBytes ? stride : kStepBytes) > 0xF0000000u;
  // Rows that overlap reach behind the piece's last row, where the products over it count on zeros.
  const size_t apart = stride_of(f.stride_table, f.cols);
  return plan_with(f, backward, piece, pack_hidden, !d_table || !readable(d_table, apart * e) || apart < f.cols);
}
size_t work_bytes_for(const struct ze_form& f, bool backward, size_t piece, const void* d_hidden, const void* d_table) {
  const size_t bytes = plan_for(f, backward, piece, d_hidden, d_table).bytes;
  if (d_hidden && d_table) return bytes;
  // (A table that is not copied may be taken in larger pieces.)
  const size_t other = plan_with(f, backward, piece, true, false).bytes;
  return bytes > other ? bytes : other;
}

List list_in(const Plan& p, char* work, bool backward) {
  const auto at = [&](int i) { return work + p.list[i]; };
  List l;
  l.head = reinterpret_cast<Head*>(work);
  l.row_of = reinterpret_cast<int*>(at(0));
  l.token_of = reinterpret_cast<int*>(at(1));
  l.label_of = reinterpret_cast<int*>(at(2));
  l.target = backward ? nullptr : reinterpret_cast<float*>(at(3));
  l.lse = reinterpret_cast<float*>(at(4));
  l.dloss = reinterpret_cast<float*>(at(5));
  l.padded = p.padded;
  return l;
}

template <int DT>
void launch_list(const struct ze_form& f, const void* d_labels, const float* d_lse, const float* d_dloss, const List& list, const EndsArgs& ends, hipStream_t s) {
  const unsigned groups = 1 + ends.groups + (ends.of[1].out ? (unsigned)parts(ends.of[1].rows, kListThreads / 8) : 0);
  if (f.id_dtype == ZE_I64)
    hipLaunchKernelGGL((list_kernel<long long, DT>), dim3(groups), dim3(kListThreads), 0, s, static_cast<const long long*>(d_labels), (int)f.tokens, f.first,
                       (long long)f.rows, d_lse, d_dloss, list, ends);
  else
    hipLaunchKernelGGL((list_kernel<int, DT>), dim3(groups), dim3(kListThreads), 0, s, static_cast<const int*>(d_labels), (int)f.tokens, f.first, (long long)f.rows,
                       d_lse, d_dloss, list, ends);
}

constexpr size_t kMostGroups = (size_t)1 << 23;   // of one launch: a grid has fewer than 2^32 lanes

// The rows `v0` to `v0 + count` of the table where a product can read them.
template <int DT>
Matrix table_piece(const struct ze_form& f, const Plan& p, const void* d_table, size_t v0, size_t count, char* work, hipStream_t s) {
  Matrix m;
  m.places = nullptr;
  const char* at = static_cast<const char*>(d_table) + v0 * p.stride_table;
  if (!p.pack_table) {
    m.at = at;
    m.stride = p.stride_table;
    m.bytes = up((count - 1) * m.stride + f.cols * p.e, 4);   // (a word that holds a value may be read)
    return m;
  }
  PackArgs a = {at, p.stride_table, nullptr, count, work + p.packed_table, p.cols_padded * p.e, (int)f.cols};
  for (size_t from = 0; from < count; from += kMostGroups) {
    const size_t groups = count - from < kMostGroups ? count - from : kMostGroups;
    hipLaunchKernelGGL(pack_kernel<DT>, dim3((unsigned)groups), dim3(kThreads), 0, s, a, from);
  }
  m.at = a.out;
  m.stride = a.out_stride;
  m.bytes = count * a.out_stride;
  return m;
}

// The copies of rows' ends that a call makes.
EndsArgs ends_to_copy(const struct ze_form& f, const Plan& p, const void* d_hidden, const void* d_table, char* work, bool hidden) {
  EndsArgs a = {};
  if (!p.ends || f.rows == 0) return a;
  const size_t skip = (size_t)p.steps * kStepBytes;
  const int cols = (int)(f.cols - skip / p.e);
  a.of[0] = PackArgs{static_cast<const char*>(d_table) + skip, p.stride_table, nullptr, f.rows, work + p.table_ends, kStepBytes, cols};
  a.groups = (unsigned)parts(f.rows, kListThreads / 8);
  if (hidden) a.of[1] = PackArgs{static_cast<const char*>(d_hidden) + skip, p.stride_hidden, nullptr, f.tokens, work + p.hidden_ends, kStepBytes, cols};
  return a;
}
// Those of the table's rows from v0 on.
Ends table_ends(const Plan& p, size_t v0, size_t count, const char* work) {
  if (!p.ends) return Ends{nullptr, 0, 0, nullptr};
  return Ends{work + p.table_ends + v0 * kStepBytes, count * kStepBytes, kStepBytes, nullptr};
}
// Those of rows that have been copied, ends and all.
Ends ends_in(const Plan& p, const Matrix& m) {
  if (!p.ends) return Ends{nullptr, 0, 0, nullptr};
  const size_t skip = (size_t)p.steps * kStepBytes;
  return Ends{m.at + skip, m.bytes - skip, m.stride, nullptr};
}

template <int DT>
void forward(const struct ze_form& f, const Plan& p, const void* d_hidden, const void* d_table, const List& list, char* work, float* d_stats, hipStream_t s) {
  LogitsArgs a;
  a.head = list.head;
  a.label_of = list.label_of;
  a.scale = f.scale;
  a.target = list.target;
  a.parts_stride = p.parts;
  a.steps = p.steps;
  if (p.piece) {
    if (p.pack_hidden) {
      PackArgs pack = {static_cast<const char*>(d_hidden), p.stride_hidden, list.token_of, 0, work + p.packed_hidden, p.cols_padded * p.e, (int)f.cols};
      for (size_t from = 0; from < p.padded; from += kMostGroups) {
        const size_t groups = p.padded - from < kMostGroups ? p.padded - from : kMostGroups;
        hipLaunchKernelGGL(pack_kernel<DT>, dim3((unsigned)groups), dim3(kThreads), 0, s, pack, from);
      }
      a.hidden = Matrix{pack.out, p.padded * pack.out_stride, pack.out_stride, nullptr};
      a.hidden_ends = ends_in(p, a.hidden);
    } else {
      a.hidden = Matrix{static_cast<const char*>(d_hidden), up((f.tokens - 1) * p.stride_hidden + f.cols * p.e, 4), p.stride_hidden, list.token_of};
      a.hidden_ends = Ends{p.ends ? work + p.hidden_ends : nullptr, f.tokens * kStepBytes, kStepBytes, list.token_of};
    }
  }
  size_t part = 0;
  for (size_t v0 = 0; v0 < f.rows; v0 += p.piece) {
    const size_t count = f.rows - v0 < p.piece ? f.rows - v0 : p.piece;
    a.table = table_piece<DT>(f, p, d_table, v0, count, work, s);
    a.table_ends = table_ends(p, v0, count, work);
    a.v0 = (int)v0;
    a.rows = (int)count;
    a.parts = reinterpret_cast<Part*>(work + p.part) + part;
#define LAUNCH(D, S)                                                                                                                  \
  do {                                                                                                                                \
    a.nx = (int)parts(count, S::BX);                                                                                                  \
    a.ny = (int)parts(f.tokens, S::BY);                                                                                               \
    part += (size_t)a.nx * S::WX;                                                                                                     \
    hipLaunchKernelGGL((logits_kernel<D, S>), dim3(groups_for<S>((size_t)a.nx * a.ny)), dim3(S::kThreads), 0, s, a);                             \
  } while (0)
    ZE_BY_SHAPE_OF_LOGITS(p.shape, DT, LAUNCH);
#undef LAUNCH
  }
  const size_t groups = parts(f.tokens, kThreads / 64);
  hipLaunchKernelGGL(stats_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, list.row_of, f.tokens, reinterpret_cast<const Part*>(work + p.part), p.parts, part,
                     list.target, d_stats);
}

template <int DT>
void backward(const struct ze_form& f, const Plan& p, const void* d_hidden, const void* d_table, const List& list, char* work, void* d_dhidden, void* d_dtable,
              hipStream_t s) {
  const size_t dhidden_stride = stride_of(f.stride_dtokens, f.cols) * p.e, dtable_stride = stride_of(f.stride_dtable, f.cols) * p.e;
  // the rows with a label, to a whole step of the product over them
  PackArgs pack = {static_cast<const char*>(d_hidden), p.stride_hidden, list.token_of, 0, work + p.packed_hidden, p.cols_padded * p.e, (int)f.cols};
  for (size_t from = 0; from < p.padded; from += kMostGroups) {
    const size_t groups = p.padded - from < kMostGroups ? p.padded - from : kMostGroups;
    hipLaunchKernelGGL(pack_hidden_kernel<DT>, dim3((unsigned)groups), dim3(kThreads), 0, s, pack, from, list.row_of, f.tokens, static_cast<char*>(d_dhidden),
                       dhidden_stride);
  }
  const Matrix hidden = {pack.out, p.padded * pack.out_stride, pack.out_stride, nullptr};
  for (size_t v0 = 0; v0 < f.rows; v0 += p.piece) {
    const size_t count = f.rows - v0 < p.piece ? f.rows - v0 : p.piece, padded = up(count, kStep<DT>);
    const Matrix table = table_piece<DT>(f, p, d_table, v0, count, work, s);
    GradientArgs g;
    g.table = table;
    g.hidden = hidden;
    g.table_ends = table_ends(p, v0, count, work);
    g.hidden_ends = ends_in(p, hidden);
    g.head = list.head;
    g.label_of = list.label_of;
    g.lse = list.lse;
    g.dloss = list.dloss;
    g.steps = p.steps;
    g.v0 = (int)v0;
    g.rows = (int)count;
    g.rows_padded = (int)padded;
    g.scale = f.scale;
    g.g = work + p.g;
    g.g_stride = padded * p.e;
#define LAUNCH(D, S)                                                                                           \
  do {                                                                                                         \
    g.nx = (int)parts(count, S::BX);                                                                           \
    g.ny = (int)parts(f.tokens, S::BY);                                                                        \
    hipLaunchKernelGGL((gradient_kernel<D, S>), dim3(groups_for<S>((size_t)g.nx * g.ny)), dim3(S::kThreads), 0, s, g);    \
  } while (0)
    ZE_BY_SHAPE(p.shape, DT, LAUNCH);
#undef LAUNCH
    const Matrix gradient = {g.g, p.padded * padded * p.e, padded * p.e, nullptr};
    OutArgs a = {};
    a.head = list.head;
    a.scale = f.scale;
    a.cols = (int)f.cols;
    if (d_dtable) {
      a.mx = hidden;
      a.my = gradient;
      a.rows = (int)count;
      a.out = static_cast<char*>(d_dtable) + v0 * dtable_stride;
      a.out_stride = dtable_stride;
#define LAUNCH(D, S)                                                                                               \
  do {                                                                                                             \
    a.nx = (int)parts(f.cols, S::BX);                                                                              \
    a.ny = (int)parts(count, S::BY);                                                                               \
    hipLaunchKernelGGL((table_gradient_kernel<D, S>), dim3(groups_for<S>((size_t)a.nx * a.ny)), dim3(S::kThreads), 0, s, a);  \
  } while (0)
      ZE_BY_SHAPE(shape_for(f.dtype, f.cols, count), DT, LAUNCH);
#undef LAUNCH
    }
    if (d_dhidden) {
      a.mx = table;
      a.my = gradient;
      a.steps = (int)(padded / kStep<DT>);
      a.out = static_cast<char*>(d_dhidden);
      a.out_stride = dhidden_stride;
      a.token_of = list.token_of;
      a.kept = reinterpret_cast<float*>(work + p.kept);
      a.kept_stride = up(f.cols, 4);
      a.sharers = p.sharers;
      a.most_splits = p.most_splits;
      a.add = v0 > 0;
      a.last = v0 + count == f.rows;
#define LAUNCH(D, S)                                                                                                                       \
  do {                                                                                                                                     \
    a.nx = (int)parts(f.cols, S::BX);                                                                                                      \
    const size_t all = a.nx * parts(f.tokens, S::BY), groups = p.most_splits > 1 && all < (size_t)p.sharers ? (size_t)p.sharers : all;     \
    hipLaunchKernelGGL((hidden_gradient_kernel<D, S>), dim3(groups_for<S>(groups)), dim3(S::kThreads), 0, s, a);                                \
    if (a.last && p.most_splits > 1)                                                                                                       \
      hipLaunchKernelGGL((hidden_finish_kernel<D, S>), dim3((unsigned)parts(f.cols, kThreads * 4), (unsigned)(f.tokens < 512 ? f.tokens : 512)), \
                         dim3(kThreads), 0, s, a);                                                                                         \
  } while (0)
      ZE_BY_SHAPE_OF_HIDDEN(p.hidden_shape, DT, LAUNCH);
#undef LAUNCH
    }
  }
}

// Rows of zeros.
void launch_zeros(void* out, size_t rows, size_t stride, size_t bytes, hipStream_t s) {
  for (size_t from = 0; from < rows; from += kMostGroups) {
    const size_t groups = rows - from < kMostGroups ? rows - from : kMostGroups;
    hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, static_cast<char*>(out), stride, bytes, from);
  }
}

int check_loss_form(const struct ze_form* f) {
  const int rc = check_form(f);
  if (rc != ZC_OK) return rc;
  return f->cols == 0 ? ZC_ERR_SIZE : ZC_OK;
}

}  // namespace

extern "C" {

size_t ze_loss_work_bytes(const struct ze_form* form, const void* d_hidden, const void* d_table) {
  if (check_loss_form(form) != ZC_OK || form->tokens == 0) return 0;
  return work_bytes_for(*form, false, 0, d_hidden, form->rows ? d_table : d_hidden);
}

int ze_vocab_loss(const struct ze_form* form, const void* d_hidden, const void* d_table, const void* d_labels, float* d_stats, void* d_work, size_t work_bytes,
                  void* stream) {
  const int rc = check_loss_form(form);
  if (rc != ZC_OK) return rc;
  if (form->tokens == 0) return ZC_OK;
  if (!d_hidden || (!d_table && form->rows) || !d_labels || !d_stats || !d_work) return ZC_ERR_NULL;
  const size_t e = dtype_bytes(form->dtype);
  if (!aligned(d_hidden, e) || !aligned(d_table, e) || !aligned_ids(d_labels, form->id_dtype) || !aligned(d_stats, 4) || !aligned(d_work, 256)) return ZC_ERR_ALIGN;
  const Plan p = plan_for(*form, false, 0, d_hidden, form->rows ? d_table : d_hidden);
  if (work_bytes < p.bytes) return ZC_ERR_CAPACITY;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  char* const work = static_cast<char*>(d_work);
  const List list = list_in(p, work, false);
  const EndsArgs ends = ends_to_copy(*form, p, d_hidden, d_table, work, !p.pack_hidden);
#define CALL(DT)                                                             \
  do {                                                                       \
    launch_list<DT>(*form, d_labels, nullptr, nullptr, list, ends, s);       \
    forward<DT>(*form, p, d_hidden, d_table, list, work, d_stats, s);        \
  } while (0)
  ZE_BY_TYPE(form->dtype, CALL);
#undef CALL
  return finish_launch();
}

int ze_join_loss(size_t tokens, int ranks, int id_dtype, const float* d_stats, const void* d_labels, float* d_loss, float* d_lse, void* stream) {
  if (id_dtype != ZE_I32 && id_dtype != ZE_I64) return ZC_ERR_ARG;
  if (ranks < 1) return ZC_ERR_K;
  if (tokens > ZE_MAX_TOKENS) return ZC_ERR_SIZE;
  if (tokens == 0) return ZC_OK;
  if (!d_stats || !d_labels || !d_lse) return ZC_ERR_NULL;
  if (!aligned(d_stats, 4) || !aligned_ids(d_labels, id_dtype) || !aligned(d_loss, 4) || !aligned(d_lse, 4)) return ZC_ERR_ALIGN;
  const dim3 grid((unsigned)parts(tokens, kThreads));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (id_dtype == ZE_I64)
    hipLaunchKernelGGL(join_kernel<long long>, grid, dim3(kThreads), 0, s, tokens, ranks, d_stats, static_cast<const long long*>(d_labels), d_loss, d_lse);
  else
    hipLaunchKernelGGL(join_kernel<int>, grid, dim3(kThreads), 0, s, tokens, ranks, d_stats, static_cast<const int*>(d_labels), d_loss, d_lse);
  return finish_launch();
}

size_t ze_loss_backward_work_bytes(const struct ze_form* form, const void* d_hidden, const void* d_table, size_t piece) {
  if (check_loss_form(form) != ZC_OK || form->tokens == 0 || form->rows == 0) return 0;
  return work_bytes_for(*form, true, piece, d_hidden, d_table);
}

int ze_vocab_loss_backward(const struct ze_form* form, const void* d_hidden, const void* d_table, const void* d_labels, const float* d_lse, const float* d_dloss,
                           void* d_dhidden, void* d_dtable, size_t piece, void* d_work, size_t work_bytes, void* stream) {
  const int rc = check_loss_form(form);
  if (rc != ZC_OK) return rc;
  if (!good_output(form->stride_dtokens, form->cols) || !good_output(form->stride_dtable, form->cols)) return ZC_ERR_ARG;
  const size_t e = dtype_bytes(form->dtype);
  if (!aligned(d_dhidden, e) || !aligned(d_dtable, e)) return ZC_ERR_ALIGN;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (form->tokens == 0 || form->rows == 0) {   // sums of nothing
    if (d_dhidden) launch_zeros(d_dhidden, form->tokens, stride_of(form->stride_dtokens, form->cols) * e, form->cols * e, s);
    if (d_dtable) launch_zeros(d_dtable, form->rows, stride_of(form->stride_dtable, form->cols) * e, form->cols * e, s);
    return finish_launch();
  }
  if (!d_hidden || !d_table || !d_labels || !d_lse || !d_dloss || !d_work) return ZC_ERR_NULL;
  if (!aligned(d_hidden, e) || !aligned(d_table, e) || !aligned_ids(d_labels, form->id_dtype) || !aligned(d_lse, 4) || !aligned(d_dloss, 4) || !aligned(d_work, 256))
    return ZC_ERR_ALIGN;
  const Plan p = plan_for(*form, true, piece, d_hidden, d_table);
  if (work_bytes < p.bytes) return ZC_ERR_CAPACITY;
  char* const work = static_cast<char*>(d_work);
  const List list = list_in(p, work, true);
  const EndsArgs ends = ends_to_copy(*form, p, d_hidden, d_table, work, false);
#define CALL(DT)                                                                           \
  do {                                                                                     \
    launch_list<DT>(*form, d_labels, d_lse, d_dloss, list, ends, s);                       \
    backward<DT>(*form, p, d_hidden, d_table, list, work, d_dhidden, d_dtable, s);         \
  } while (0)
  ZE_BY_TYPE(form->dtype, CALL);
#undef CALL
  return finish_launch();
}

}  // extern "C"
