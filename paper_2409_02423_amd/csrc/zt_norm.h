// zt_norm.h -- what the forward and the backward kernel of the residual join share: how rows lie over lanes, sums over a row, the
// checks of a form.
#ifndef ZT_NORM_H
#define ZT_NORM_H

#include <math.h>

#include <initializer_list>

#include "zt_device.h"

namespace {

// How a row lies over lanes.  A workgroup takes whole rows, one at a time; a lane has NV vectors of 16 bytes of a row, neighbouring
// lanes neighbouring ones.  NV = 0 is the form for rows that registers do not hold: as many
// vectors as it takes, operands loaded where they are used and the row's fp32 values in LDS.  NV = kShort16, kShort32 and kShort64 are those for rows of
// 16, 32 and 64 vectors at most, which as many lanes take each, four, two or one to a wavefront and 16, 8 or 4 to a workgroup; they may be shorter than a vector.
//
// So that every load is a whole one, a row's last vector is moved to end where the row does.  What it then shares with the one ahead of
// it is not its own: it is loaded but counts for nothing and is not stored.  (Loading the last values one by one, in a branch of
// their own, held up each row's first sum: 8192 x 4099 values in fp32 150 us forward, now 111.)  Which lane has which column does not depend on where
// tensors lie, nor do the results, bit for bit.  (Vectors that start where memory is aligned to them made 8192 x 4099 in bf16 12 % faster, at that price.)
constexpr int kShort16 = -1, kShort32 = -2, kShort64 = -3;
template <int NV> constexpr int kShortLanes = NV == kShort16 ? 16 : NV == kShort32 ? 32 : NV == kShort64 ? 64 : 0;   // of a row, where a workgroup has several
template <int NV> constexpr int kHeld = NV > 0 ? NV : 1;   // vectors that registers hold, if any

template <int DT, int NV>
struct Lanes {
  static constexpr int V = kVec<DT>;
  mutable int lane;
  int lanes, cols;
  uint32_t first, step;   // rows
  __device__ __forceinline__ explicit Lanes(int columns) : cols(columns) {
    if constexpr (NV < 0) {
      lanes = kShortLanes<NV>;
      lane = threadIdx.x % kShortLanes<NV>;
      first = (blockIdx.x * blockDim.x + threadIdx.x) / kShortLanes<NV>;
      if constexpr (NV == kShort64) first = __builtin_amdgcn_readfirstlane(first);
      step = gridDim.x * blockDim.x / kShortLanes<NV>;
    } else {
      lane = threadIdx.x;
      lanes = blockDim.x;
      first = blockIdx.x;
      step = gridDim.x;
    }
  }
  // Place of a lane's vector i in the order of lanes, and the column that it is loaded from.
  __device__ __forceinline__ int place(int i) const { return (lane + i * lanes) * V; }
  __device__ __forceinline__ int col(int i) const { return max(0, min(place(i), cols - V)); }
  // Its own values are those from `from` to `to`.
  __device__ __forceinline__ int from(int i) const { return min(place(i) - col(i), V); }
  __device__ __forceinline__ int to() const { return NV < 0 && cols < V ? cols : V; }
  __device__ __forceinline__ bool whole(int i) const { return place(i) <= cols - V; }
  __device__ __forceinline__ bool any(int i) const { return place(i) < cols; }
  // What follows works its places out anew: kept for all vectors and rows they take registers that wide rows need.
  __device__ __forceinline__ void forget() const { asm volatile("" : "+v"(lane)); }
  // f(i) for each of a lane's vectors.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (NV != 0) {
#pragma unroll
      for (int i = 0; i < kHeld<NV>; ++i) f(i);
    } else {
      const int count = (cols + lanes * V - 1) / (lanes * V);
#pragma unroll 1
      for (int i = 0; i < count; ++i) f(i);
    }
  }
  __device__ __forceinline__ Raw<DT> load(const char* row, int i) const {
    Raw<DT> r;
    if (NV >= 0 || cols >= V) r.load(row, (uint32_t)col(i) * kBytes<DT>);
    else r.load(row, 0, cols);
    return r;
  }
  // Nontemporal: rows together are far more than the caches next to the lanes hold.  What is not a lane's own is dropped by the
  // store's bounds and not branched around: behind a branch it is not known how many stores there were, and the next wait for a load,
  // which counts them, is for all of them (backward, 8192 x 4100 values in bf16, 110 us; now 80).
  __device__ __forceinline__ void store(char* row, int i, const float (&v)[V]) const {
    Raw<DT> r;
    r.pack(v);
    if constexpr (NV > 0) {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      constexpr int kNontemporal = 2, kNowhere = -16;
      const auto to_row = __builtin_amdgcn_make_buffer_rsrc(row, 0, cols * kBytes<DT>, 0x00027000);
      const int at = place(i) * kBytes<DT>;
      __builtin_amdgcn_raw_buffer_store_b128(u32x4{r.w[0], r.w[1], r.w[2], r.w[3]}, to_row, whole(i) ? at : kNowhere, 0, kNontemporal);
      const int own = cols % V;
      if (own != 0) {      // the last vector's, which are the last of its values: in parts of 8, 4 and 2 bytes
        const bool mine = !whole(i) && any(i);
        if constexpr (DT == kF32) {
          if (own & 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2{r.w[2], r.w[3]}, to_row, mine ? at + (own & 1) * 4 : kNowhere, 0, 0);
          if (own & 1) __builtin_amdgcn_raw_buffer_store_b32(own & 2 ? r.w[1] : r.w[3], to_row, mine ? at : kNowhere, 0, 0);
        } else {
          if (own & 4) __builtin_amdgcn_raw_buffer_store_b64(u32x2{r.w[2], r.w[3]}, to_row, mine ? at + (own & 3) * 2 : kNowhere, 0, 0);
          if (own & 2) __builtin_amdgcn_raw_buffer_store_b32(own & 4 ? r.w[1] : r.w[3], to_row, mine ? at + (own & 1) * 2 : kNowhere, 0, 0);
          const uint32_t last = own & 4 ? (own & 2 ? r.w[0] : r.w[1]) : (own & 2 ? r.w[2] : r.w[3]);
          if (own & 1) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(last >> 16), to_row, mine ? at : kNowhere, 0, 0);
        }
      }
    } else {
      if (whole(i)) r.template store<true>(row, (uint32_t)col(i) * kBytes<DT>);
      else if (any(i)) r.store(row, (uint32_t)col(i) * kBytes<DT>, from(i), to());
    }
  }
  // What is not its own counts as zero.
  __device__ __forceinline__ void clear_rest(float (&v)[V], int i) const {
    if (NV > 0 ? cols < NV * lanes * V : !whole(i)) {
      const int begin = from(i), end = to();
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = j < begin || j >= end ? 0.0f : v[j];
    }
  }
};

// A row of one operand, or of weights: a lane's vectors, loaded at once and held, or each loaded where it is used.  An operand that is
// absent is the same value everywhere.
template <int DT, int NV, bool HOLD = (NV != 0)>
struct Operand {
  Raw<DT> held[kHeld<NV>];
  const char* row;
  float otherwise;
  __device__ __forceinline__ void open(const Lanes<DT, NV>& at, const char* p, float absent = 0.0f) {
    row = p;
    otherwise = absent;
    if constexpr (HOLD) at.each([&](int i) { held[i] = fetch(at, i); });
  }
  __device__ __forceinline__ Raw<DT> fetch(const Lanes<DT, NV>& at, int i) const {
    Raw<DT> r;
    const char* p = row;
    if constexpr (!HOLD) asm volatile("" : "+s"(p));   // loaded anew each time: the compiler would keep what registers have no room for
    if (p) {
      r = at.load(p, i);
    } else {
      float v[kVec<DT>];
#pragma unroll
      for (int j = 0; j < kVec<DT>; ++j) v[j] = otherwise;
      r.pack(v);
    }
    return r;
  }
  __device__ __forceinline__ void get(const Lanes<DT, NV>& at, int i, float (&v)[kVec<DT>]) const {
    if constexpr (HOLD) held[i].unpack(v);
    else fetch(at, i).unpack(v);
  }
};

// A row's fp32 values: in registers, or in LDS, where a lane reads only what it has written (of MOST lanes at most).
template <int DT, int NV, int MOST, bool HOLD = (NV != 0)>
struct Values {
  static constexpr int V = kVec<DT>;
  float held[kHeld<NV>][V];
  float4* lds;
  __device__ __forceinline__ Values() {
    if constexpr (!HOLD) {
      __shared__ float4 row[NV > 0 ? MOST * NV * V / 4 : ZT_MAX_COLS / 4];
      lds = row;
    }
  }
  __device__ __forceinline__ void get(const Lanes<DT, NV>& at, int i, float (&v)[V]) const {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if constexpr (HOLD) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[j + q] = held[i][j + q];
      } else {
        const float4 f = lds[(at.place(i) + j) / 4];
        v[j] = f.x;
        v[j + 1] = f.y;
        v[j + 2] = f.z;
        v[j + 3] = f.w;
      }
    }
  }
  __device__ __forceinline__ void set(const Lanes<DT, NV>& at, int i, const float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if constexpr (HOLD) {
#pragma unroll
        for (int q = 0; q < 4; ++q) held[i][j + q] = v[j + q];
      } else {
        lds[(at.place(i) + j) / 4] = float4{v[j], v[j + 1], v[j + 2], v[j + 3]};
      }
    }
  }
};
static_assert(ZT_MAX_COLS % (1024 * 8) == 0, "the last vectors of a workgroup's lanes in LDS");

// Sums of K values over a row's lanes, the same in each of them.
template <int K, int NV>
struct Sums {
  float (*buffers)[K][kMostWaves];
  int next = 0;
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    if constexpr (NV < 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] = NV == kShort64 ? wave_sum(v[k]) : row_sum(v[k]);
        if constexpr (NV == kShort32) v[k] += __shfl_xor(v[k], 16);
      }
    } else {
      group_sum(v, buffers[next]);
      next ^= 1;
    }
  }
};

// ---- host ------------------------------------------------------------------------------

constexpr unsigned kCUs = 256;
constexpr size_t kMaxStride = (size_t)1 << 40;

// NV vectors a lane (0: the form for wide rows, below: those for short ones); a workgroup of `lanes`, at most `most`, for a row, or `rows` short ones.
struct Layout {
  int vectors, lanes, most, rows = 1;
};
int vector_values(int dtype) { return dtype == ZC_F32 ? 4 : 8; }
size_t row_vectors(size_t cols, int dtype) { return (cols + vector_values(dtype) - 1) / vector_values(dtype); }
// Short rows share a workgroup, and those that would leave most of a wavefront idle a wavefront, too. us in bf16 with a workgroup of one
// wavefront for each row and with this, forward and backward: 262144 x 7 values 3066 and 38, 6226 and 80 (values of rows shorter than a vector were loaded one by
// one by the only lane that had any); x 64 96 and 29, 252 and 53; 131072 x 129 65 and 37, 152 and 62; x 200 60 and 39, 148 and 65; 65536 x 257 49 and 44, 86 and 69;
// x 400 40 and 41, 78 and 65; x 512 48 and 47, 86 and 81.
bool short_rows(size_t vectors) { return vectors <= 64; }
Layout short_layout(size_t vectors) { return vectors <= 16 ? Layout{kShort16, 256, 256, 16} : vectors <= 32 ? Layout{kShort32, 256, 256, 8} : Layout{kShort64, 256, 256, 4}; }
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
