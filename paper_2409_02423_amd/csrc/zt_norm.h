// zt_norm.h -- what the forward and the backward kernel of the residual join share: how rows lie over lanes, sums over a row, the
// checks of a form.
#ifndef ZT_NORM_H
#define ZT_NORM_H

#include <math.h>

#include <initializer_list>

#include "zt_device.h"

namespace {

// How a row lies over lanes.  A workgroup takes whole rows, one at a time, or with WAVE each of its wavefronts does; a lane has NV
// vectors of 16 bytes of a row, neighbouring lanes neighbouring ones.  NV = 0 is the form for rows that registers do not hold: as many
// vectors as it takes, operands loaded where they are used and the row's fp32 values in LDS.
template <int DT, int NV, bool WAVE>
struct Lanes {
  static constexpr int V = kVec<DT>;
  int lane, lanes, cols;
  uint32_t first, step;   // rows of this workgroup or wavefront
  __device__ __forceinline__ explicit Lanes(int columns) : cols(columns) {
    lane = WAVE ? threadIdx.x & 63 : threadIdx.x;
    lanes = WAVE ? 64 : blockDim.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    first = WAVE ? blockIdx.x * waves + wave : blockIdx.x;
    step = WAVE ? gridDim.x * waves : gridDim.x;
  }
  __device__ __forceinline__ int col(int i) const { return (lane + i * lanes) * V; }
  // Values of vector i that are in the row; 0 or less for none.
  __device__ __forceinline__ int valid(int i) const { return cols - col(i); }
  __device__ __forceinline__ bool leads() const { return lane == 0; }
  // f(i) for each of a lane's vectors.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) f(i);
    } else {
      const int count = (cols + lanes * V - 1) / (lanes * V);
#pragma unroll 1
      for (int i = 0; i < count; ++i) f(i);
    }
  }
  __device__ __forceinline__ void store(char* row, int i, const float (&v)[V]) const {
    Raw<DT> r;
    r.pack(v);
    r.store(row, (uint32_t)col(i) * kBytes<DT>, valid(i));
  }
  // What lies behind the row's end counts as zero.
  __device__ __forceinline__ void clear_rest(float (&v)[V], int i) const {
    const int n = valid(i);
    if (n < V) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= n) v[j] = 0.0f;
    }
  }
};

// A row of one operand, or of weights: a lane's vectors, loaded at once and held, or each loaded where it is used (NV = 0).  An
// operand that is absent is the same value everywhere.
template <int DT, int NV, bool WAVE>
struct Operand {
  Raw<DT> held[NV > 0 ? NV : 1];
  const char* row;
  float otherwise;
  __device__ __forceinline__ void open(const Lanes<DT, NV, WAVE>& at, const char* p, float absent = 0.0f) {
    row = p;
    otherwise = absent;
    if constexpr (NV > 0) at.each([&](int i) { held[i] = fetch(at, i); });
  }
  __device__ __forceinline__ Raw<DT> fetch(const Lanes<DT, NV, WAVE>& at, int i) const {
    Raw<DT> r;
    if (row) {
      r.load(row, (uint32_t)at.col(i) * kBytes<DT>, at.valid(i));
    } else {
      float v[kVec<DT>];
#pragma unroll
      for (int j = 0; j < kVec<DT>; ++j) v[j] = otherwise;
      r.pack(v);
    }
    return r;
  }
  __device__ __forceinline__ void get(const Lanes<DT, NV, WAVE>& at, int i, float (&v)[kVec<DT>]) const {
    if constexpr (NV > 0) held[i].unpack(v);
    else fetch(at, i).unpack(v);
  }
};

// A row's fp32 values: in registers, or in LDS (NV = 0), where a lane reads only what it has written.
template <int DT, int NV, bool WAVE>
struct Values {
  static constexpr int V = kVec<DT>;
  float held[NV > 0 ? NV : 1][V];
  float4* lds;
  __device__ __forceinline__ Values() {
    if constexpr (NV == 0) {
      __shared__ float4 row[ZT_MAX_COLS / 4];
      lds = row;
    }
  }
  __device__ __forceinline__ void get(const Lanes<DT, NV, WAVE>& at, int i, float (&v)[V]) const {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if constexpr (NV > 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[j + q] = held[i][j + q];
      } else {
        const float4 f = at.valid(i) > 0 ? lds[(at.col(i) + j) / 4] : float4{0.0f, 0.0f, 0.0f, 0.0f};
        v[j] = f.x;
        v[j + 1] = f.y;
        v[j + 2] = f.z;
        v[j + 3] = f.w;
      }
    }
  }
  __device__ __forceinline__ void set(const Lanes<DT, NV, WAVE>& at, int i, const float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if constexpr (NV > 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) held[i][j + q] = v[j + q];
      } else if (at.valid(i) > 0) {
        lds[(at.col(i) + j) / 4] = float4{v[j], v[j + 1], v[j + 2], v[j + 3]};
      }
    }
  }
};
static_assert(ZT_MAX_COLS % 8 == 0, "a row's last vector in LDS");

// Sums of K values over a row's lanes, the same in each of them.
template <int K, bool WAVE>
struct Sums {
  float (*buffers)[K][kMostWaves];
  int next = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    if constexpr (WAVE) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    } else {
      group_sum(v, buffers[next]);
      next ^= 1;
    }
  }
};

// ---- host ------------------------------------------------------------------------------

constexpr unsigned kCUs = 256;
constexpr size_t kMaxStride = (size_t)1 << 40;

// NV vectors a lane (0: the form for wide rows); a workgroup of `lanes` for a row, at most `most`, or with most = 64 four wavefronts for four rows.
struct Layout {
  int vectors, lanes, most;
};
size_t row_vectors(size_t cols, int dtype) { return (cols * dtype_bytes(dtype) + 15) / 16; }
int lanes_for(size_t vectors, int each) { return (int)(((vectors + each - 1) / each + 63) / 64 * 64); }

int check_form(const zt_residual* f) {
  if (!f) return ZC_ERR_NULL;
  if (!known_dtype(f->dtype)) return ZC_ERR_DTYPE;
  if ((f->kind != ZT_RMS && f->kind != ZT_LAYER) || (f->post != 0 && f->post != 1) || f->gate < ZT_GATE_NONE || f->gate > ZT_GATE_FULL ||
      !(fabsf(f->residual_scale) < INFINITY) || !(f->eps >= 0.0f && f->eps < INFINITY))
    return ZC_ERR_ARG;
  if (f->cols > ZT_MAX_COLS || f->rows > ZT_MAX_ROWS) return ZC_ERR_SIZE;
  return ZC_OK;
}
size_t stride_of(size_t stride, size_t cols) { return stride ? stride : cols; }
// Strides of what is read may be anything, those of what is written leave rows apart.
bool good_strides(std::initializer_list<size_t> read, std::initializer_list<size_t> written, size_t cols) {
  for (size_t s : read)
    if (s > kMaxStride) return false;
  for (size_t s : written)
    if (s > kMaxStride || (s != 0 && s < cols)) return false;
  return true;
}
bool all_aligned(std::initializer_list<const void*> pointers, size_t to) {
  for (const void* p : pointers)
    if (!aligned(p, to)) return false;
  return true;
}
const char* bytes_of(const void* p) { return static_cast<const char*>(p); }

}  // namespace
#endif  // ZT_NORM_H
