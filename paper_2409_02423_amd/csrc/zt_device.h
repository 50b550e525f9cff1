// zt_device.h -- what the training-step kernels share: vectors of values at any address, conversions,
// sums over a wavefront and a workgroup, launch helpers.
#ifndef ZT_DEVICE_H
#define ZT_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/zt.h"

namespace {

constexpr int kF32 = ZC_F32, kBF16 = ZC_BF16, kF16 = ZC_F16;

template <int DT> constexpr int kBytes = DT == kF32 ? 4 : 2;
// Values of a 16-byte vector: what a lane loads and stores at once.
template <int DT> constexpr int kVec = 16 / kBytes<DT>;

#define ZT_GLOBAL __attribute__((address_space(1)))

// N consecutive values as they lie in memory, at any address that is aligned to a value: rows of an odd number of values and slices of a
// bucket start anywhere.  Global accesses of any alignment are one instruction on gfx950; one that touches a second cache line
// costs that line.
template <int DT, int N = kVec<DT>>
struct Raw {
  static constexpr int kWords = N * kBytes<DT> / 4, kPart = kWords < 4 ? kWords : 4;
  typedef uint32_t part_t __attribute__((ext_vector_type(kPart)));
  typedef part_t part_at_t __attribute__((aligned(kBytes<DT>)));
  uint32_t w[kWords];

  // All of them, `at` bytes behind `base`; base is the same in every lane, which leaves the addressing to the load itself.
  // ONCE: what is not read or written again soon (nontemporal) leaves the caches to what is.
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const char* base, uint32_t at) {
#pragma unroll
    for (int i = 0; i < kWords / kPart; ++i) {
      const ZT_GLOBAL part_at_t* p = reinterpret_cast<const ZT_GLOBAL part_at_t*>((const ZT_GLOBAL char*)base + at) + i;
      const part_t v = ONCE ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
      for (int j = 0; j < kPart; ++j) w[i * kPart + j] = v[j];
    }
  }
  // The first `valid`, the rest zero; nothing is read behind them.  What is missing is read as the last one there, so that the loads
  // do not wait for one another.
  __device__ __forceinline__ void load(const char* base, uint32_t at, int valid) {
    if (valid >= N) {
      load(base, at);
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
    if (valid <= 0) return;
    const ZT_GLOBAL char* p = (const ZT_GLOBAL char*)base + at;
    uint32_t one[N - 1];
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
      const int j = i < valid ? i : valid - 1;
      if constexpr (DT == kF32) one[i] = reinterpret_cast<const ZT_GLOBAL uint32_t*>(p)[j];
      else one[i] = reinterpret_cast<const ZT_GLOBAL uint16_t*>(p)[j];
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
      const uint32_t v = i < valid ? one[i] : 0;
      if constexpr (DT == kF32) w[i] = v;
      else w[i / 2] |= v << (i % 2 * 16);
    }
  }
  template <bool ONCE = false>
  __device__ __forceinline__ void store(char* base, uint32_t at) const {
#pragma unroll
    for (int i = 0; i < kWords / kPart; ++i) {
      part_t v;
#pragma unroll
      for (int j = 0; j < kPart; ++j) v[j] = w[i * kPart + j];
      ZT_GLOBAL part_at_t* p = reinterpret_cast<ZT_GLOBAL part_at_t*>((ZT_GLOBAL char*)base + at) + i;
      if constexpr (ONCE) __builtin_nontemporal_store(part_at_t(v), p);
      else *p = v;
    }
  }
  // Those from `from` to `to`.
  __device__ __forceinline__ void store(char* base, uint32_t at, int from, int to) const {
    ZT_GLOBAL char* p = (ZT_GLOBAL char*)base + at;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (DT == kF32) {
        if (i >= from && i < to) reinterpret_cast<ZT_GLOBAL uint32_t*>(p)[i] = w[i];
      } else {
        if (i >= from && i < to) reinterpret_cast<ZT_GLOBAL uint16_t*>(p)[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
      }
    }
  }
  // The first `valid`.
  __device__ __forceinline__ void store(char* base, uint32_t at, int valid) const {
    if (valid >= N) store(base, at);
    else store(base, at, 0, valid);
  }
  // Exact.
  __device__ __forceinline__ float get(int i) const {
    if constexpr (DT == kF32) return __builtin_bit_cast(float, w[i]);
    else if constexpr (DT == kBF16) return __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> (i % 2 * 16)));
  }
  __device__ __forceinline__ void unpack(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = get(i);
  }
  // To the nearest, ties to even; NaN stays NaN.
  __device__ __forceinline__ void pack(const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (DT == kF32) {
        w[i] = __builtin_bit_cast(uint32_t, v[i]);
      } else if constexpr (DT == kBF16) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{v[2 * i], v[2 * i + 1]}), b2));
      } else {
        w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[2 * i + 1]) << 16;
      }
    }
  }
};

// ---- sums ------------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true);
  return v + __builtin_bit_cast(float, other);
}
template <int CTRL>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float read_lane(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sum over each row of 16 lanes, in every lane of it: neighbours, pairs, then the row's mirrors.
template <class T>
__device__ __forceinline__ T row_sum(T v) {
  v = dpp_add<0xB1>(v);    // quad_perm 1 0 3 2
  v = dpp_add<0x4E>(v);    // quad_perm 2 3 0 1
  v = dpp_add<0x141>(v);   // row_half_mirror
  return dpp_add<0x140>(v);   // row_mirror
}
// Sum over the 64 lanes, in every lane.  All 64 have to be active.
template <class T>
__device__ __forceinline__ T wave_sum(T v) {
  v = row_sum(v);
  return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}

constexpr int kMostWaves = 16;   // of a workgroup

// Sums of K values over a workgroup of up to 16 wavefronts, the same in every lane.  The caller takes two buffers in turn: between two
// uses of one there is a barrier, that of the other's use, which each wavefront passes after it has read the one.
template <int K, class T>
__device__ __forceinline__ void group_sum(T (&v)[K], T (&buffer)[K][kMostWaves]) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, waves = blockDim.x / 64;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const T s = wave_sum(v[k]);
    if (lane == 0) buffer[k][wave] = s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = row_sum((lane & 15) < waves ? buffer[k][lane & 15] : T(0));
}

// ---- host ------------------------------------------------------------------------------

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool known_dtype(int dtype) { return dtype == ZC_F32 || dtype == ZC_BF16 || dtype == ZC_F16; }
size_t dtype_bytes(int dtype) { return dtype == ZC_F32 ? 4 : 2; }
int finish_launch() { return hipGetLastError() == hipSuccess ? ZC_OK : ZC_ERR_LAUNCH; }

}  // namespace
#endif  // ZT_DEVICE_H
