// ze_product.h -- the matrix product inside the vocabulary's operators: out[y][x] = sum over k of X[x][k] Y[y][k], a tile of it for each
// workgroup, left in registers for what the operator makes of it.
//
// Both operands come through LDS, in steps of 128 bytes of k (64 half-precision values, 32 fp32): loads go there directly, past the registers, and a
// step's loads are under way while kStages - 1 steps before it are worked on.  An operand lies in memory either along k (rows of x or y, kAlong) or
// across it (rows of k, kAcross: then half-precision values are turned around as they are read from LDS), so none of the products needs a
// transposed copy.  Sums are fp32, in one fixed order of k.
#ifndef ZE_PRODUCT_H
#define ZE_PRODUCT_H

#include "zt_device.h"

namespace {

#define ZE_LDS __attribute__((address_space(3)))

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;   // of k
template <int DT> constexpr int kStep = kStepBytes / kBytes<DT>;   // values of k

enum Lies { kAlong, kAcross };

// Sums of 16 x 16 products over half a step: 32 half-precision values of k in one instruction, 16 fp32 values in four.
template <int DT>
__device__ __forceinline__ f32x4 multiply(i32x4 x, i32x4 y, f32x4 sum) {
  if constexpr (DT == kBF16) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), sum, 0, 0, 0);
  } else if constexpr (DT == kF16) {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), sum, 0, 0, 0);
  } else {
    const f32x4 fx = __builtin_bit_cast(f32x4, x), fy = __builtin_bit_cast(f32x4, y);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(fx[j], fy[j], sum, 0, 0, 0);
    return sum;
  }
}

// An operand in memory: every row starts at a multiple of 16 bytes.  Nothing is read at or behind `bytes`: what would be is zero.
struct Matrix {
  const char* at;
  size_t bytes, stride;   // stride in bytes
  const int* places;      // kAlong: NULL, or the row that stands for each row (the matrix then has less than 2^32 bytes)
};

constexpr uint32_t kNowhere = 0xFFFFFF00u;   // behind the end of every buffer

// One operand of a tile that is SIZE rows of x (or y) wide, for a workgroup of THREADS lanes.
//
// In LDS a piece of 16 bytes is the smallest thing that a load can put somewhere; which place a lane's piece goes to is fixed, so it is the piece's address
// in memory that is chosen.  kAlong: a row's eight pieces are exchanged by the row's number, so that 16 lanes that read the same piece of 16 rows
// touch all banks.  kAcross: pieces of 16 values along the row are exchanged by k, for the same reason.
template <int DT, Lies LIES, int SIZE, int THREADS>
struct Operand {
  static constexpr int kE = kBytes<DT>, kTileBytes = SIZE * kStepBytes, kLoads = kTileBytes / (THREADS * 16), kRow = SIZE * kE;
  static_assert(kLoads * THREADS * 16 == kTileBytes, "whole loads");
  static constexpr int kParts = SIZE / 16 < 8 ? SIZE / 16 : 8;   // kAcross, half precision: 16 values of a row, places that are exchanged
  static constexpr int kAddresses = LIES == kAlong ? 2 : DT == kF32 ? 4 : kParts;
  static_assert(DT != kF32 || SIZE >= 64, "exchanged places");

  uint32_t from[kLoads];   // bytes from the tile's start
  const char* at;          // the tile's start, at the present step
  size_t left, step;
  int lane_at[kAddresses];

  static __device__ __forceinline__ int swap_along(int row) { return (row >> 1) & 7; }
  static __device__ __forceinline__ int swap_across(int k) {
    if constexpr (DT == kF32) return (k >> 2) & 3;
    else return ((k & 3) | ((k >> 3) & 3) << 2) & (SIZE / 16 - 1);
  }

  // The tile's `first` row of x; the wavefront's part of it starts at `wave_first`.
  __device__ __forceinline__ void start(const Matrix& m, size_t first, int wave_first) {
    const int tid = threadIdx.x, lane = tid & 63, group = lane >> 4;
    if constexpr (LIES == kAlong) {
      step = kStepBytes;
      const bool listed = m.places != nullptr;
      const size_t skip = listed ? 0 : first * m.stride;
      at = m.at + skip;
      left = skip < m.bytes ? m.bytes - skip : 0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = j * (THREADS / 8) + tid / 8, piece = (tid & 7) ^ swap_along(row);
        if (listed) {
          const int place = m.places[first + row];
          from[j] = place < 0 ? kNowhere : (uint32_t)place * (uint32_t)m.stride + piece * 16;
        } else {
          from[j] = row * (uint32_t)m.stride + piece * 16;
        }
      }
      const int row = wave_first + (lane & 15);
#pragma unroll
      for (int h = 0; h < 2; ++h) lane_at[h] = row * kStepBytes + ((group + 4 * h) ^ swap_along(lane & 15)) * 16;
    } else {
      step = m.stride * kStep<DT>;
      at = m.at + first * kE;
      left = first * kE < m.bytes ? m.bytes - first * kE : 0;
      constexpr int kUnit = DT == kF32 ? 4 : 2;   // pieces of 16 values
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int byte = (j * THREADS + tid) * 16, k = byte / kRow, place = byte % kRow / 16;
        from[j] = k * (uint32_t)m.stride + (((place / kUnit) ^ swap_across(k)) * kUnit + place % kUnit) * 16;
      }
      // lane i of 16 asks for four values at 4 (i & 3) of row i >> 2 and gets the four rows' values at i; fp32: each lane its own value
      const int k = DT == kF32 ? group * 4 : group * 8 + (lane & 15) / 4;
#pragma unroll
      for (int p = 0; p < kAddresses; ++p)
        lane_at[p] = k * kRow + ((wave_first / 16 + p) ^ swap_across(k)) * (16 * kE) + (DT == kF32 ? (lane & 15) * 4 : (lane & 3) * 8);
    }
  }

  // The next step's loads into `tile`; zeros where there is none.  (Every wavefront counts on kLoads loads of its own.)
  __device__ __forceinline__ void load(ZE_LDS char* tile, bool any) {
    const uint32_t records = !any ? 0u : left > 0xFFFFFE00u ? 0xFFFFFE00u : (uint32_t)left;
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, (int)records, 0x00027000);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (ZE_LDS void*)(tile + (j * THREADS + wave * 64) * 16), 16, (int)from[j], 0, 0, 0);
    at += step;
    left -= step < left ? step : left;
  }

  // What a lane puts into a product: row 16 t + its number of the wavefront's part, its group's quarter of half h of the step.
  __device__ __forceinline__ i32x4 read(const ZE_LDS char* tile, int t, int h) const {
    if constexpr (LIES == kAlong) {
      return *(const ZE_LDS i32x4*)(tile + lane_at[h] + t * 16 * kStepBytes);
    } else if constexpr (DT != kF32) {
      typedef short v4 __attribute__((ext_vector_type(4)));
      typedef int i32x2 __attribute__((ext_vector_type(2)));
      ZE_LDS char* p = (ZE_LDS char*)(tile + lane_at[t % kAddresses] + t / kAddresses * (kAddresses * 16 * kE) + h * 32 * kRow);
      const i32x2 low = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ZE_LDS v4*)p));
      const i32x2 high = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ZE_LDS v4*)(p + 4 * kRow)));
      return i32x4{low[0], low[1], high[0], high[1]};
    } else {
      const ZE_LDS char* p = tile + lane_at[t % kAddresses] + t / kAddresses * (kAddresses * 16 * kE) + h * 16 * kRow;
      i32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const ZE_LDS int*)(p + j * kRow);
      return v;
    }
  }
};

// How a product is shared out: a tile of BX x BY for each workgroup, of which each of WX x WY wavefronts has a part.
template <int BX_, int BY_, int WX_, int WY_, int STAGES_>
struct Shape {
  static constexpr int BX = BX_, BY = BY_, WX = WX_, WY = WY_, kStages = STAGES_, kThreads = WX * WY * 64;
  static constexpr int NX = BX / WX / 16, NY = BY / WY / 16;   // 16 x 16 products of a wavefront
};

// waits until at most `loads` of the wavefront's loads into LDS are under way and all its reads of LDS have come
template <int LOADS>
__device__ __forceinline__ void wait_for_loads() {
  static_assert(LOADS < 64, "");
  __builtin_amdgcn_s_waitcnt(0x0070 | (LOADS & 15) | (LOADS >> 4) << 14);
}
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The tile's sums: sum[i][j][r] is that of x = the wavefront's first + 16 i + 4 (lane / 16) + r, y = the wavefront's first + 16 j + lane % 16.
template <int DT, class S, Lies LX, Lies LY>
__device__ __forceinline__ void product(const Matrix& mx, const Matrix& my, size_t first_x, size_t first_y, int steps, f32x4 (&sum)[S::NX][S::NY]) {
  constexpr int kTile = (S::BX + S::BY) * kStepBytes, kMore = S::kStages > 2 ? kTile : 16;
  // An array for each stage: what is loaded into one is seen to leave the others alone.
  __shared__ __attribute__((aligned(1024))) char stage0[kTile], stage1[kTile], stage2[kMore], stage3[kMore];
  ZE_LDS char* const stages[4] = {(ZE_LDS char*)stage0, (ZE_LDS char*)stage1, (ZE_LDS char*)stage2, (ZE_LDS char*)stage3};
  static_assert(S::kStages == 2 || S::kStages == 4, "arrays");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Operand<DT, LX, S::BX, S::kThreads> ox;
  Operand<DT, LY, S::BY, S::kThreads> oy;
  constexpr int kLoads = ox.kLoads + oy.kLoads;
  ox.start(mx, first_x, wave % S::WX * (S::BX / S::WX));
  oy.start(my, first_y, wave / S::WX * (S::BY / S::WY));
#pragma unroll
  for (int i = 0; i < S::NX; ++i)
#pragma unroll
    for (int j = 0; j < S::NY; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const auto load = [&](ZE_LDS char* tile, bool any) {
    ox.load(tile, any);
    oy.load(tile + S::BX * kStepBytes, any);
  };
  i32x4 x[2][S::NX], y[2][S::NY];
  const auto read = [&](const ZE_LDS char* tile, int h) {
#pragma unroll
    for (int i = 0; i < S::NX; ++i) x[h][i] = ox.read(tile, i, h);
#pragma unroll
    for (int j = 0; j < S::NY; ++j) y[h][j] = oy.read(tile + S::BX * kStepBytes, j, h);
  };
  const auto add = [&](int h) {
#pragma unroll
    for (int j = 0; j < S::NY; ++j)
#pragma unroll
      for (int i = 0; i < S::NX; ++i) sum[i][j] = multiply<DT>(x[h][i], y[h][j], sum[i][j]);
  };

#pragma unroll
  for (int s = 0; s < S::kStages; ++s) load(stages[s], s < steps);
  wait_for_loads<(S::kStages - 1) * kLoads>();
  meet();
  read(stages[0], 0);
  // Half of a step is multiplied while the other half, or the next step's first, is read.  Between the halves all wavefronts have read
  // the step for good, so that its place takes the loads of the step kStages behind it.  (Steps behind the last are zeros.)
  for (int t = 0; t < steps; t += S::kStages) {
#pragma unroll
    for (int s = 0; s < S::kStages; ++s) {
      read(stages[s], 1);
      add(0);
      wait_for_loads<(S::kStages - 2) * kLoads>();
      meet();
      load(stages[s], t + s + S::kStages < steps);
      read(stages[(s + 1) % S::kStages], 0);
      add(1);
    }
  }
  // nothing may be under way into LDS when the workgroup ends or uses it for something else
  wait_for_loads<0>();
}

// Which tile a workgroup has, of nx x ny: neighbours in a band of eight rows of tiles follow one another in an XCD (workgroups go to the
// eight of them in turn), so that what they share is read into its cache once.
__device__ __forceinline__ void tile_of(int nx, int ny, int& x, int& y) {
  const int total = nx * ny, each = total / 8, more = total % 8, xcd = blockIdx.x & 7;
  const int at = xcd * each + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
  constexpr int kBand = 8;
  const int band = at / (kBand * nx), in = at - band * (kBand * nx), rows = ny - band * kBand < kBand ? ny - band * kBand : kBand;
  y = band * kBand + in % rows;
  x = in / rows;
}

}  // namespace
#endif  // ZE_PRODUCT_H
