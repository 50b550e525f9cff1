// ze_product.h -- the matrix product inside the vocabulary's operators: out[y][x] = sum over k of X[x][k] Y[y][k], a tile of it for each
// workgroup, left in registers for what the operator makes of it.
//
// Both operands come through LDS, in steps of 128 bytes of k (64 half-precision values, 32 fp32): loads go there directly, past the registers, and a
// step's loads are under way while kStages - 1 steps before it are worked on.  An operand lies in memory either along k (rows of x or y, kAlong) or
// across it (rows of k, kAcross: then half-precision values are turned around as they are read from LDS), so none of the products needs a
// transposed copy.  Sums are fp32, in one fixed order of k.
//
// Large bf16 products run at 1250 (where g is stored) to 1480 TFLOP/s (a library's product of 8192 x 8192 matrices: 1432), fp32 ones at 125 to 144 (154): the power that the
// matrix units draw bounds the first, their rate the second.
#ifndef ZE_PRODUCT_H
#define ZE_PRODUCT_H

#include <type_traits>
#include <utility>

#include "zt_device.h"

namespace {

#define ZE_LDS __attribute__((address_space(3)))

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;   // of k
template <int DT> constexpr int kStep = kStepBytes / kBytes<DT>;   // values of k

enum Lies { kAlong, kAcross };

// Sums of 16 x 16 products over half a step: 32 half-precision values of k in one instruction, 16 fp32 values in four, of which this is one.
template <int DT> constexpr int kInstructions = DT == kF32 ? 4 : 1;
template <int DT>
__device__ __forceinline__ f32x4 multiply(i32x4 x, i32x4 y, int part, f32x4 sum) {
  if constexpr (DT == kBF16) {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), sum, 0, 0, 0);
  } else if constexpr (DT == kF16) {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), sum, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, x)[part], __builtin_bit_cast(f32x4, y)[part], sum, 0, 0, 0);
  }
}

// An operand in memory: every row starts at a multiple of 4 bytes.  Nothing is read at or behind `bytes`, a multiple of 4: what would be is zero.
struct Matrix {
  const char* at;
  size_t bytes, stride;   // stride in bytes
  const int* places;      // kAlong: NULL, or the row that stands for each row (the matrix then has less than 2^32 bytes)
};

// A row's end behind its last whole step: one step more, which ends in zeros, of rows of its own (kAlong).  at = NULL where there is none.
struct Ends {
  const char* at;
  size_t bytes, stride;
  const int* places;
};

// Loads have come.  (Where one may stay unused the compiler waits for it wherever its register is needed next: in the steps of the next tile.)
template <class T, int N>
__device__ __forceinline__ void have_come(T (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

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
  static constexpr int kAddresses = LIES == kAlong ? 2 : DT == kF32 && kParts > 4 ? 4 : kParts;

  uint32_t from[kLoads];   // bytes from the tile's start
  const char* at;          // the tile's start, at the present step
  long long left, step;    // bytes from there to the matrix's end (or less than none), and from step to step
  int lane_at[kAddresses];

  static __device__ __forceinline__ int swap_along(int row) { return (row >> 1) & 7; }
  static __device__ __forceinline__ int swap_across(int k) {
    if constexpr (DT == kF32) return (k >> 2) & 3 & (SIZE / 16 - 1);
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
      left = (long long)m.bytes - (long long)skip;
      const int row0 = tid / 8;
      if (listed) {
        // (asked for at once; one after the other, 8192 x 12608 x 6144 bf16 took 973 us for 963)
        int place[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) place[j] = m.places[first + row0 + j * (THREADS / 8)];
        have_come(place);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) from[j] = place[j] < 0 ? kNowhere : (uint32_t)place[j] * (uint32_t)m.stride + ((tid & 7) ^ swap_along(row0 + j * (THREADS / 8))) * 16;
      } else {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int row = row0 + j * (THREADS / 8);
          from[j] = row * (uint32_t)m.stride + ((tid & 7) ^ swap_along(row)) * 16;
        }
      }
      const int row = wave_first + (lane & 15);
#pragma unroll
      for (int h = 0; h < 2; ++h) lane_at[h] = row * kStepBytes + ((group + 4 * h) ^ swap_along(lane & 15)) * 16;
    } else {
      step = (long long)m.stride * kStep<DT>;
      at = m.at + first * kE;
      left = (long long)m.bytes - (long long)(first * kE);
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

  // The next step's loads into `tile`; zeros where there is none (every wavefront counts on kLoads loads of its own).  One after the other, between
  // other work, or all at once.
  struct Step {
    __amdgpu_buffer_rsrc_t buffer;
    ZE_LDS char* tile;      // the wavefront's part
  };
  __device__ __forceinline__ Step next(ZE_LDS char* tile, bool any) {
    const int high = (int)(left >> 32);
    const uint32_t records = !any || high < 0 ? 0u : high > 0 ? 0xFFFFFE00u : (uint32_t)left;
    const Step s = {__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, (int)records, 0x00027000),
                    tile + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 1024};
    at += step;
    left -= step;
    return s;
  }
  __device__ __forceinline__ void load_one(const Step& s, int j) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(s.buffer, (ZE_LDS void*)(s.tile + j * THREADS * 16), 16, (int)from[j], 0, 0, 0);
  }
  __device__ __forceinline__ void load(ZE_LDS char* tile, bool any) {
    const Step s = next(tile, any);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_one(s, j);
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
template <int BX_, int BY_, int WX_, int WY_, int STAGES_, bool BY_HAND = false>
struct Shape {
  static constexpr bool kByHand = BY_HAND;   // half precision alone
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

template <int DT_, class S_, Lies LX, Lies LY>
struct Operands {
  static constexpr int DT = DT_;
  using S = S_;
  Operand<DT, LX, S::BX, S::kThreads> x;
  Operand<DT, LY, S::BY, S::kThreads> y;
  static constexpr int kLoadsX = decltype(x)::kLoads, kLoads = kLoadsX + decltype(y)::kLoads, kTile = (S::BX + S::BY) * kStepBytes, kY = S::BX * kStepBytes;

  __device__ __forceinline__ void start(const Matrix& mx, const Matrix& my, int tx, int ty) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    x.start(mx, (size_t)tx * S::BX, wave % S::WX * (S::BX / S::WX));
    y.start(my, (size_t)ty * S::BY, wave / S::WX * (S::BY / S::WY));
  }
  __device__ __forceinline__ void load(ZE_LDS char* tile, bool any) {
    x.load(tile, any);
    y.load(tile + kY, any);
  }
  __device__ __forceinline__ i32x4 read_x(const ZE_LDS char* tile, int i, int h) const { return x.read(tile, i, h); }
  __device__ __forceinline__ i32x4 read_y(const ZE_LDS char* tile, int j, int h) const { return y.read(tile + kY, j, h); }
};

// Nothing is moved across this by the compiler.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// sum = x y + sum, in accumulation registers.  (As an instruction by name: left to itself the compiler moves half of 256 sums to and from other
// registers in every step.  It knows nothing of the time that it takes, see products_of_four.)
template <int DT>
__device__ __forceinline__ void multiply_in_place(i32x4 x, i32x4 y, f32x4& sum) {
  if constexpr (DT == kBF16) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(sum) : "v"(x), "v"(y));
  else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(sum) : "v"(x), "v"(y));
}

// The tiles of a workgroup, of nx x ny: neighbours in a band of eight rows of tiles follow one another in an XCD (workgroups go to the
// eight of them in turn), so that what they share is read into its cache once.
struct Tiles {
  int nx, ny, first, stride, count;
  __device__ __forceinline__ Tiles(int nx, int ny) : nx(nx), ny(ny) {
    const int total = nx * ny, each = total / 8, more = total % 8, xcd = blockIdx.x & 7, n = blockIdx.x >> 3;
    const int mine = each + (xcd < more);                  // the XCD's
    stride = ((int)gridDim.x - xcd + 7) >> 3;              // its workgroups
    count = n < mine ? (mine - n + stride - 1) / stride : 0;
    first = xcd * each + (xcd < more ? xcd : more) + n;
  }
  __device__ __forceinline__ void at(int k, int& x, int& y) const {
    constexpr int kBand = 8;
    const int at = first + k * stride, band = at / (kBand * nx), in = at - band * (kBand * nx), rows = ny - band * kBand < kBand ? ny - band * kBand : kBand;
    y = band * kBand + in % rows;
    x = in / rows;
  }
};

// Four wavefronts with 128 x 128 sums each, one for each SIMD: a value that is read from LDS goes into eight products, which leaves a quarter of LDS's time
// (eight wavefronts of 128 x 64 fill all of it).  Nothing but the order of instructions hides anything here, so it is written down: of a step's
// 128 products, two follow each read of the next half step, and five each load.  At kMeet, all of the step has been read; its place takes the loads of the step
// after the next from there on, spread so that the cache answers them about as fast as they are asked for (all at once behind the meeting, a
// load took 516 cycles on average; a bf16 product of 8192 x 8192 x 8192 830 us, so 748 to 764).  Behind a tile's last step come the next tile's first: they are
// under way while `use` has the tile's sums.
template <class Both, class Start, class StartEnds, class Use, class S = typename Both::S>
__device__ __forceinline__ void products_of_four(const Tiles& tiles, int steps, bool has_ends, const Start& start, const StartEnds& start_ends, const Use& use) {
  constexpr int DT = Both::DT;
  constexpr int kStages = S::kStages;
  __shared__ __attribute__((aligned(1024))) char stage0[Both::kTile], stage1[Both::kTile], stage2[kStages > 2 ? Both::kTile : 16];
  ZE_LDS char* const stages[3] = {(ZE_LDS char*)stage0, (ZE_LDS char*)stage1, (ZE_LDS char*)stage2};
  constexpr int NX = S::NX, NY = S::NY, kReads = NX + NY, kHalf = NX * NY, kReadEvery = 2, kMeet = kReads * kReadEvery + NX, kSpread = (2 * kHalf - kMeet) / Both::kLoads;
  static_assert((kStages == 2 || kStages == 3) && kReads * kReadEvery <= kMeet && kMeet + (Both::kLoads - 1) * kSpread < 2 * kHalf && kReads * kReadEvery <= kHalf, "order");
  Both both;
  f32x4 sum[NX][NY];
  i32x4 x[2][NX], y[2][NY];
  const auto read = [&](auto q, const ZE_LDS char* tile, auto h) __attribute__((always_inline)) {
    if constexpr (q < NX) x[h][q] = both.read_x(tile, q, h);
    else y[h][q - NX] = both.read_y(tile, q - NX, h);
  };
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;
  const auto read_all = [&](const ZE_LDS char* tile, auto h) __attribute__((always_inline)) {
    each_of([&](auto q) __attribute__((always_inline)) { read(q, tile, h); }, std::make_integer_sequence<int, kReads>{});
  };
  const auto step = [&](ZE_LDS char* here, const ZE_LDS char* there, bool any) __attribute__((always_inline)) {
    const auto from_x = both.x.next(here, any);
    const auto from_y = both.y.next(here + Both::kY, any);
    each_of([&](auto p) __attribute__((always_inline)) {
      constexpr int h = p / kHalf, m = p % kHalf;
      in_order();
      if constexpr (p == kMeet) {
        wait_for_loads<(kStages - 2) * Both::kLoads>();
        meet();
        in_order();
      }
      if constexpr (h == 0 && m % kReadEvery == 0 && m / kReadEvery < kReads) read(std::integral_constant<int, m / kReadEvery>{}, here, Second{});
      if constexpr (h == 1 && m % kReadEvery == 1 && m / kReadEvery < kReads) read(std::integral_constant<int, m / kReadEvery>{}, there, First{});
      if constexpr (p >= kMeet && (p - kMeet) % kSpread == 0 && (p - kMeet) / kSpread < Both::kLoads) {
        constexpr int q = (p - kMeet) / kSpread;
        if constexpr (q < Both::kLoadsX) both.x.load_one(from_x, q);
        else both.y.load_one(from_y, q - Both::kLoadsX);
      }
      in_order();
      multiply_in_place<DT>(x[h][m % NX], y[h][m / NX], sum[m % NX][m / NX]);
    }, std::make_integer_sequence<int, 2 * kHalf>{});
  };

  for (int k = 0; k < tiles.count; ++k) {
    int tx, ty;
    tiles.at(k, tx, ty);
#pragma unroll
    for (int i = 0; i < NX; ++i)
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        asm volatile("" : "+a"(sum[i][j]));
      }
    asm volatile("s_nop 1");   // (a register that has just been written is not yet a product's)
    if (k == 0 || has_ends || steps == 0) {   // nothing of this tile is under way
      if (has_ends) {
        start_ends(both, tx, ty);
        both.load(stages[0], true);
        wait_for_loads<0>();
        meet();
        each_of([&](auto h) __attribute__((always_inline)) {
          read_all(stages[0], h);
          each_of([&](auto m) __attribute__((always_inline)) { multiply_in_place<DT>(x[h][m % NX], y[h][m / NX], sum[m % NX][m / NX]); },
                  std::make_integer_sequence<int, kHalf>{});
        }, std::make_integer_sequence<int, 2>{});
        meet();
      }
      start(both, tx, ty);
      each_of([&](auto s) __attribute__((always_inline)) { both.load(stages[s], s < steps); }, std::make_integer_sequence<int, kStages>{});
      wait_for_loads<(kStages - 1) * Both::kLoads>();
      meet();
      read_all(stages[0], First{});
    }
    for (int t = 0; t < steps; t += kStages) {
      const bool last = t + kStages >= steps, next = last && k + 1 < tiles.count && !has_ends;
      if (next) {
        int nx, ny;
        tiles.at(k + 1, nx, ny);
        start(both, nx, ny);
      }
      each_of([&](auto s) __attribute__((always_inline)) {
        step(stages[s], stages[(s + 1) % kStages], last ? next && s < steps : t + kStages + s < steps);
      }, std::make_integer_sequence<int, kStages>{});
      // a sum may be read eleven issues after its product, wherever the compiler reads it behind the loop
      asm volatile("s_nop 7\n\ts_nop 3");
      in_order();
    }
    use(sum, tx, ty);
    if (has_ends || steps == 0) {   // LDS is free for another beginning
      wait_for_loads<0>();
      meet();
    }
  }
  wait_for_loads<0>();
}

// The sums of a workgroup's tiles, one tile after the other: use(sum, tx, ty), where sum[i][j][r] is that of x = the wavefront's first + 16 i + 4 (lane / 16) + r,
// y = the wavefront's first + 16 j + lane % 16.  start(both, tx, ty) puts the operands to a tile's start; start_ends, if there are any, to a step that is added first
// (the rows' ends).
template <class Both, class Start, class StartEnds, class Use, class S = typename Both::S>
__device__ __forceinline__ void products(const Tiles& tiles, int steps, bool has_ends, const Start& start, const StartEnds& start_ends, const Use& use) {
  if constexpr (S::kByHand) {
    products_of_four<Both>(tiles, steps, has_ends, start, start_ends, use);
  } else {
    if (tiles.count == 0) return;   // (as many workgroups as tiles, or more)
    int tx, ty;
    tiles.at(0, tx, ty);
    constexpr int DT = Both::DT, kTile = Both::kTile, kMore = S::kStages > 2 ? kTile : 16, kMost = S::kStages > 4 ? kTile : 16;
    // An array for each stage: what is loaded into one is seen to leave the others alone.
    __shared__ __attribute__((aligned(1024))) char stage0[kTile], stage1[kTile], stage2[kMore], stage3[kMore], stage4[kMost], stage5[kMost], stage6[kMost], stage7[kMost];
    ZE_LDS char* const stages[8] = {(ZE_LDS char*)stage0, (ZE_LDS char*)stage1, (ZE_LDS char*)stage2, (ZE_LDS char*)stage3,
                                    (ZE_LDS char*)stage4, (ZE_LDS char*)stage5, (ZE_LDS char*)stage6, (ZE_LDS char*)stage7};
    static_assert(S::kStages == 2 || S::kStages == 4 || S::kStages == 8, "arrays");
    Both both;
    f32x4 sum[S::NX][S::NY];
#pragma unroll
    for (int i = 0; i < S::NX; ++i)
#pragma unroll
      for (int j = 0; j < S::NY; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    i32x4 x[2][S::NX], y[2][S::NY];
    const auto read = [&](const ZE_LDS char* tile, int h) {
#pragma unroll
      for (int i = 0; i < S::NX; ++i) x[h][i] = both.read_x(tile, i, h);
#pragma unroll
      for (int j = 0; j < S::NY; ++j) y[h][j] = both.read_y(tile, j, h);
    };
    const auto add = [&](int h) {   // (a sum's next product does not follow at once, where there are others)
#pragma unroll
      for (int part = 0; part < kInstructions<DT>; ++part)
#pragma unroll
        for (int j = 0; j < S::NY; ++j)
#pragma unroll
          for (int i = 0; i < S::NX; ++i) sum[i][j] = multiply<DT>(x[h][i], y[h][j], part, sum[i][j]);
    };

    if (has_ends) {
      start_ends(both, tx, ty);
      both.load(stages[0], true);
      wait_for_loads<0>();
      meet();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        read(stages[0], h);
        add(h);
      }
      wait_for_loads<0>();
      meet();
    }
    start(both, tx, ty);
#pragma unroll
    for (int s = 0; s < S::kStages; ++s) both.load(stages[s], s < steps);
    wait_for_loads<(S::kStages - 1) * Both::kLoads>();
    meet();
    read(stages[0], 0);
    // Half of a step is multiplied while the other half, or the next step's first, is read.  Between the halves all wavefronts have read
    // the step for good, so that its place takes the loads of the step kStages behind it, before anything else is done: left to the compiler they
    // came last.  (Steps behind the last are zeros.)
    for (int t = 0; t < steps; t += S::kStages) {
#pragma unroll
      for (int s = 0; s < S::kStages; ++s) {
        read(stages[s], 1);
        add(0);
        wait_for_loads<(S::kStages - 2) * Both::kLoads>();
        meet();
        both.load(stages[s], t + s + S::kStages < steps);
        in_order();
        read(stages[(s + 1) % S::kStages], 0);
        add(1);
      }
    }
    // nothing may be under way into LDS when the workgroup ends
    wait_for_loads<0>();
    use(sum, tx, ty);
  }
}

// Before the sums of row j are used: they and those behind them stay where they are until then.  (Where sums fill half of all registers, they cannot all be
// taken out at once.)
template <class S>
__device__ __forceinline__ void rest_of_sums(f32x4 (&sum)[S::NX][S::NY], int j) {
  if constexpr (S::kByHand) {
#pragma unroll
    for (int i = 0; i < S::NX; ++i)
#pragma unroll
      for (int k = 0; k < S::NY; ++k)
        if (k >= j) asm volatile("" : "+a"(sum[i][k]));
    in_order();
  }
}

}  // namespace
#endif  // ZE_PRODUCT_H
