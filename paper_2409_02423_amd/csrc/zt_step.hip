// zt_step.hip -- gfx950 kernels and C ABI of the optimizer's side of include/zt.h: the global gradient norm over many tensors,
// clipping, the clipped AdamW step on a shard.
//
// All of them are bound by memory.  A list of tensors is cut into chunks of kChunk values of one tensor; the list travels in the
// kernel's arguments, so nothing is copied to the GPU ahead of a launch, and lists longer than kMostTensors take several
// launches.  The sum of squares is left as one double per workgroup of the first pass (ZT_SLOTS of them), which every workgroup of the
// second pass adds up for itself, in the same order, while its values are under way: no launch in between, and no atomics.
//
// What they reach, in bytes read and written: sum of squares 6.2 TB/s (2.3e8 fp32 values in 147 us), clipping 6.6 (272 us), AdamW 5.8 to 6.2
// (1.5e8 parameters with fp32 gradients and a bf16 copy, 720 to 770 us by card).  The second pass has one tile or chunk for each workgroup and no loop (AdamW
// in a loop with 2048 workgroups 1007 us, without 830), and asks for its values as ones that do not come again (nontemporal: 808 in that measurement,
// scaling 212 to 188); the first does not, so that what fits the last-level cache is there for the second (2.5e7 fp32 values, both passes, 47 us with
// nontemporal loads in the first, 38 without).
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "../../include/zt.h"
#include "zt_device.h"

namespace {

constexpr int kMostTensors = 112;      // of one launch: 3.5 KB of its arguments
constexpr int kChunk = 8192;           // values
constexpr size_t kMostChunks = (size_t)1 << 31;   // of one list
constexpr size_t kMostGroups = (size_t)1 << 23;   // of one launch: a grid has fewer than 2^32 lanes
constexpr size_t kMaxValues = (size_t)1 << 40;    // of a tensor

// (All of it in words of four bytes and more.  With the types in bytes the compiler took the address of a pointer apart into the list's start + t and
// 7 t; a scalar load leaves out the lowest two bits of each, and the pointer was another one's.)
struct TensorList {
  const char* in[kMostTensors];
  char* out[kMostTensors];
  unsigned long long n[kMostTensors];
  uint32_t first[kMostTensors + 1];    // chunks of the tensors before this one
  uint32_t types[kMostTensors];        // of the input, and above its 8 bits of the output
  int count;
};
static_assert(sizeof(TensorList) + 64 <= 4096, "a launch's arguments");

// Which tensor a chunk is of: a lane has the ends of two, and all of them are compared with the chunk at once.  (A search through the
// list waits for each of its steps: 48 tensors with 5.0e7 bf16 values took 31 us to sum up, one tensor with as many 20.)
struct Ends {
  uint32_t end[2];
  __device__ __forceinline__ explicit Ends(const TensorList& list) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) end[i] = lane + 64 * i < list.count ? list.first[lane + 64 * i + 1] : 0xFFFFFFFFu;
  }
  __device__ __forceinline__ int tensor_of(uint32_t chunk) const {
    return __builtin_popcountll(__builtin_amdgcn_ballot_w64(end[0] <= chunk)) + __builtin_popcountll(__builtin_amdgcn_ballot_w64(end[1] <= chunk));
  }
};
static_assert(kMostTensors <= 128, "two tensors a lane");

// A chunk of a list: where its values are and how many the tensor has from there on.
struct Place {
  const char* in;
  size_t left;
  int type;
  __device__ __forceinline__ Place(const TensorList& list, const Ends& ends, uint32_t chunk) {
    const int t = ends.tensor_of(chunk);
    const size_t at = (size_t)(chunk - list.first[t]) * kChunk;
    type = (int)(list.types[t] & 255u);
    in = list.in[t] + at * (type == kF32 ? 4 : 2);
    left = list.n[t] - at;
  }
};

// ---- sum of squares --------------------------------------------------------------------

constexpr int kSumThreads = 1024;

// The squares of a chunk; what `then` does is done while the values are under way.
template <int DT, class F>
__device__ __forceinline__ void add_chunk(const Place& c, double (&sum)[2], F&& then) {
  constexpr int kSteps = kChunk / kSumThreads / kVec<DT>;
  Raw<DT> raw[kSteps];
  const bool full = c.left >= (size_t)kChunk;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int at = (threadIdx.x + i * kSumThreads) * kVec<DT>;
    if (full) raw[i].load(c.in, at * kBytes<DT>);
    else raw[i].load(c.in, at * kBytes<DT>, (int)c.left - at);
  }
  then();
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int j = 0; j < kVec<DT>; ++j) {
      const double v = raw[i].get(j);      // 24 significant bits: the square is exact
      sum[j & 1] = __builtin_fma(v, v, sum[j & 1]);
    }
}

__global__ void __launch_bounds__(kSumThreads) sum_squares_kernel(TensorList list, int accumulate, double* slots) {
  __shared__ double buffer[1][kMostWaves];
  double sum[2] = {0.0, 0.0};
  const uint32_t chunks = list.first[list.count];
  uint32_t chunk = blockIdx.x;
  if (chunk < chunks) {
    const Ends ends(list);
    Place place(list, ends, chunk);
    for (; chunk < chunks; chunk += gridDim.x) {
      const Place now = place;
      const auto look_ahead = [&] {
        if (chunk + gridDim.x < chunks) place = Place(list, ends, chunk + gridDim.x);
      };
      switch (now.type) {
        case kF32: add_chunk<kF32>(now, sum, look_ahead); break;
        case kBF16: add_chunk<kBF16>(now, sum, look_ahead); break;
        default: add_chunk<kF16>(now, sum, look_ahead); break;
      }
    }
  }
  double total[1] = {sum[0] + sum[1]};
  group_sum(total, buffer);
  if (threadIdx.x == 0) slots[blockIdx.x] = accumulate ? slots[blockIdx.x] + total[0] : total[0];
}

// ---- the norm and the factor -----------------------------------------------------------

constexpr int kThreads = 256;
static_assert(ZT_SLOTS % kThreads == 0, "slots per lane");

// Total of the slots, the same in every lane of every workgroup.
__device__ __forceinline__ double slots_total(const double* slots, double (&buffer)[1][kMostWaves]) {
  double v[1] = {0.0};
#pragma unroll
  for (int i = 0; i < ZT_SLOTS / kThreads; ++i) v[0] += slots[threadIdx.x + i * kThreads];
  group_sum(v, buffer);
  return v[0];
}

__device__ __forceinline__ float clip_factor(double norm, float scale, float max_norm) {
  return norm <= (double)max_norm ? scale : (float)((double)scale * ((double)max_norm / norm));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* slots, float scale, float* norm) {
  __shared__ double buffer[1][kMostWaves];
  const double total = slots_total(slots, buffer);
  if (threadIdx.x == 0) norm[0] = (float)((double)scale * sqrt(total));
}

// ---- clipping --------------------------------------------------------------------------

// One chunk: its loads go out first, and the factor is made while they are under way.
template <int DI, int DO, bool FULL, class F>
__device__ __forceinline__ void scale_chunk(const char* in, char* out, int left, F&& make_factor) {
  // Values per lane and step: 16 bytes of the wider type.  (Eight where one type is fp32, whose stores then leave gaps: 5.0e7 bf16 gradients
  // into an fp32 bucket 78 us, so 47.)
  constexpr int kN = DI == kF32 || DO == kF32 ? 4 : 8;
  constexpr int kSteps = kChunk / kThreads / kN;
  Raw<DI, kN> raw[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int at = (threadIdx.x + i * kThreads) * kN;
    if constexpr (FULL) raw[i].template load<true>(in, at * kBytes<DI>);
    else raw[i].load(in, at * kBytes<DI>, left - at);
  }
  const float factor = make_factor();
  if (DI == DO && in == out && factor == 1.0f) return;   // in place, and nothing to change
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int at = (threadIdx.x + i * kThreads) * kN;
    float v[kN];
    raw[i].unpack(v);
#pragma unroll
    for (int j = 0; j < kN; ++j) v[j] *= factor;
    Raw<DO, kN> result;
    result.pack(v);
    if constexpr (FULL) result.template store<true>(out, at * kBytes<DO>);
    else result.store(out, at * kBytes<DO>, left - at);
  }
}
template <int DI, int DO, class F>
__device__ __forceinline__ void scale_chunk(const char* in, char* out, size_t at, size_t n, F&& make_factor) {
  in += at * kBytes<DI>;
  out += at * kBytes<DO>;
  if (n - at >= (size_t)kChunk) scale_chunk<DI, DO, true>(in, out, 0, make_factor);
  else scale_chunk<DI, DO, false>(in, out, (int)(n - at), make_factor);
}

__global__ void __launch_bounds__(kThreads) clip_kernel(TensorList list, uint32_t from, const double* slots, float scale, float max_norm, float* norm_out) {
  __shared__ double buffer[1][kMostWaves];
  const auto make_factor = [&] {
    const double norm = (double)scale * sqrt(slots_total(slots, buffer));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) norm_out[0] = (float)norm;
    return clip_factor(norm, scale, max_norm);
  };
  const uint32_t chunk = from + blockIdx.x;
  if (chunk >= list.first[list.count]) {   // an empty list: the norm alone
    make_factor();
    return;
  }
  const int t = Ends(list).tensor_of(chunk);
  const size_t at = (size_t)(chunk - list.first[t]) * kChunk, n = list.n[t];
  const char* in = list.in[t];
  char* out = list.out[t];
  const uint32_t types = list.types[t];
  switch ((types & 255u) * 3 + (types >> 8)) {
    case kF32 * 3 + kF32: scale_chunk<kF32, kF32>(in, out, at, n, make_factor); break;
    case kF32 * 3 + kBF16: scale_chunk<kF32, kBF16>(in, out, at, n, make_factor); break;
    case kF32 * 3 + kF16: scale_chunk<kF32, kF16>(in, out, at, n, make_factor); break;
    case kBF16 * 3 + kF32: scale_chunk<kBF16, kF32>(in, out, at, n, make_factor); break;
    case kBF16 * 3 + kBF16: scale_chunk<kBF16, kBF16>(in, out, at, n, make_factor); break;
    case kBF16 * 3 + kF16: scale_chunk<kBF16, kF16>(in, out, at, n, make_factor); break;
    case kF16 * 3 + kF32: scale_chunk<kF16, kF32>(in, out, at, n, make_factor); break;
    case kF16 * 3 + kBF16: scale_chunk<kF16, kBF16>(in, out, at, n, make_factor); break;
    default: scale_chunk<kF16, kF16>(in, out, at, n, make_factor); break;
  }
}

// ---- AdamW -----------------------------------------------------------------------------

struct AdamwArgs {
  const char* grad;
  const double* slots;
  float *param, *m, *v;
  char* half;
  float* norm_out;
  const double* state;     // NULL, or what counts in place of lr and the corrections
  size_t n;
  float lr, beta1, rest1, beta2, rest2, eps, weight_decay, correct1, correct2;   // correct: 1 / (1 - beta^step)
  float scale, max_norm;
};

// The state of a step that counts itself: the steps taken, the learning rate, and the corrections of the step that is being taken.
enum { kSteps, kRate, kCorrect1, kCorrect2, kState };

// Whether there is a step: the norm as it is reported tells the caller.
__device__ __forceinline__ bool step_is_taken(double norm) { return (float)norm < __builtin_inff(); }

// Counts a step that is taken and leaves its corrections for the workgroups of the step itself, which come in a launch of their own: none
// of them may count while others still read.  One workgroup, 2.7 to 3.2 us between two steps in a graph.
__global__ void __launch_bounds__(kThreads) adamw_count_kernel(const double* slots, float scale, double beta1, double beta2, double* state, float* norm_out) {
  __shared__ double buffer[1][kMostWaves];
  bool taken = true;
  if (slots) {
    const double norm = (double)scale * sqrt(slots_total(slots, buffer));
    if (norm_out && threadIdx.x == 0) norm_out[0] = (float)norm;
    taken = step_is_taken(norm);
  }
  if (taken && threadIdx.x == 0) {
    const double step = state[kSteps] + 1.0;
    state[kSteps] = step;
    state[kCorrect1] = 1.0 / (1.0 - pow(beta1, step));
    state[kCorrect2] = 1.0 / (1.0 - pow(beta2, step));
  }
}

// Four values per lane.  (Two and four times as many, with fewer workgroups: 1.5e8 parameters with bf16 gradients 688 us, 757 and 737; 2^21 12.8, 12.1 and
// 11.6; 2^18 3.5 and, with four, 5.0.)
constexpr int kAdamwTile = kThreads * 4;

template <int DG, int DH, bool FULL>
__device__ __forceinline__ void adamw_tile(const AdamwArgs& a, size_t start, int left, double (&buffer)[1][kMostWaves]) {
  constexpr int kN = 4;
  const char* grad = a.grad + start * kBytes<DG>;
  char *param = reinterpret_cast<char*>(a.param + start), *first = reinterpret_cast<char*>(a.m + start), *second = reinterpret_cast<char*>(a.v + start);
  const int at = threadIdx.x * kN;
  Raw<DG, kN> rg;
  Raw<kF32, kN> rp, rm, rv;
  if constexpr (FULL) {
    rg.template load<true>(grad, at * kBytes<DG>);
    rp.template load<true>(param, at * 4);
    rm.template load<true>(first, at * 4);
    rv.template load<true>(second, at * 4);
  } else {
    rg.load(grad, at * kBytes<DG>, left - at);
    rp.load(param, at * 4, left - at);
    rm.load(first, at * 4, left - at);
    rv.load(second, at * 4, left - at);
  }
  float lr = a.lr, correct1 = a.correct1, correct2 = a.correct2;
  if (a.state) {
    lr = (float)a.state[kRate];
    correct1 = (float)a.state[kCorrect1];
    correct2 = (float)a.state[kCorrect2];
  }
  // the factor, while the loads are under way
  float factor = a.scale;
  bool taken = true;
  if (a.slots) {
    const double norm = (double)a.scale * sqrt(slots_total(a.slots, buffer));
    if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) a.norm_out[0] = (float)norm;
    factor = clip_factor(norm, a.scale, a.max_norm);
    taken = step_is_taken(norm);
  }
  float g[kN], p[kN], m[kN], v[kN];
  rg.unpack(g);
  rp.unpack(p);
  rm.unpack(m);
  rv.unpack(v);
  if (taken) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const float gc = g[j] * factor;
      m[j] = fmaf(a.beta1, m[j], a.rest1 * gc);
      v[j] = fmaf(a.beta2, v[j], a.rest2 * (gc * gc));
      const float update = (m[j] * correct1) / (sqrtf(v[j] * correct2) + a.eps);
      p[j] = fmaf(-lr, fmaf(a.weight_decay, p[j], update), p[j]);
    }
    rp.pack(p);
    rm.pack(m);
    rv.pack(v);
    if constexpr (FULL) {
      rp.template store<true>(param, at * 4);
      rm.template store<true>(first, at * 4);
      rv.template store<true>(second, at * 4);
    } else {
      rp.store(param, at * 4, left - at);
      rm.store(first, at * 4, left - at);
      rv.store(second, at * 4, left - at);
    }
  }
  if constexpr (DH != kF32) {
    Raw<DH, kN> rh;
    rh.pack(p);
    if constexpr (FULL) rh.template store<true>(a.half + start * 2, at * 2);
    else rh.store(a.half + start * 2, at * 2, left - at);
  }
}

// One tile for each workgroup.  DG: the gradients' type; DH: that of the copy, kF32 for none.
template <int DG, int DH>
__global__ void __launch_bounds__(kThreads) adamw_kernel(AdamwArgs a) {
  __shared__ double buffer[1][kMostWaves];
  const size_t start = (size_t)blockIdx.x * kAdamwTile, left = a.n - start;
  if (left >= (size_t)kAdamwTile) adamw_tile<DG, DH, true>(a, start, 0, buffer);
  else adamw_tile<DG, DH, false>(a, start, (int)left, buffer);
}

// ---- host ------------------------------------------------------------------------------

// Checks a list of tensors; `out` NULL for the sum of squares.
int check_list(const void* const* d_in, const size_t* n, const int* in_type, void* const* d_out, const int* out_type, int count, bool writes) {
  if (count < 0) return ZC_ERR_K;
  if (count == 0) return ZC_OK;
  if (!d_in || !n || !in_type || (writes && (!d_out || !out_type))) return ZC_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    if (!known_dtype(in_type[i]) || (writes && !known_dtype(out_type[i]))) return ZC_ERR_DTYPE;
    if (n[i] == 0) continue;
    if (n[i] > kMaxValues) return ZC_ERR_SIZE;
    if (!d_in[i] || (writes && !d_out[i])) return ZC_ERR_NULL;
    if (writes && d_in[i] == d_out[i] && in_type[i] != out_type[i]) return ZC_ERR_ARG;
    if (!aligned(d_in[i], dtype_bytes(in_type[i])) || (writes && !aligned(d_out[i], dtype_bytes(out_type[i])))) return ZC_ERR_ALIGN;
  }
  return ZC_OK;
}

// Fills `list` with the tensors from `from` on that one launch takes; returns the first that it does not.
int fill_list(TensorList& list, const void* const* d_in, const size_t* n, const int* in_type, void* const* d_out, const int* out_type, int count, int from) {
  list.count = 0;
  list.first[0] = 0;
  size_t chunks = 0;
  int i = from;
  for (; i < count && list.count < kMostTensors; ++i) {
    if (n[i] == 0) continue;
    const size_t more = (n[i] + kChunk - 1) / kChunk;
    if (chunks + more > kMostChunks && list.count > 0) break;
    const int t = list.count++;
    list.in[t] = static_cast<const char*>(d_in[i]);
    list.out[t] = d_out ? static_cast<char*>(d_out[i]) : nullptr;
    list.n[t] = n[i];
    list.types[t] = (uint32_t)in_type[i] | (out_type ? (uint32_t)out_type[i] : 0u) << 8;
    chunks += more;
    list.first[t + 1] = (uint32_t)chunks;
  }
  return i;
}

bool good_scale(float scale) { return scale > 0.0f && scale < INFINITY; }
bool good_max_norm(float max_norm) { return max_norm > 0.0f; }

}  // namespace

extern "C" {

int zt_sum_squares(const void* const* d_in, const size_t* n, const int* dtype, int count, int accumulate, double* d_slots, void* stream) {
  const int rc = check_list(d_in, n, dtype, nullptr, nullptr, count, false);
  if (rc != ZC_OK) return rc;
  if (!d_slots) return ZC_ERR_NULL;
  if (!aligned(d_slots, 16)) return ZC_ERR_ALIGN;
  TensorList list;
  int next = 0;
  bool launched = false;
  do {
    next = fill_list(list, d_in, n, dtype, nullptr, nullptr, count, next);
    if (list.count == 0 && accumulate) break;      // nothing (more) to add
    hipLaunchKernelGGL(sum_squares_kernel, dim3(ZT_SLOTS), dim3(kSumThreads), 0, static_cast<hipStream_t>(stream), list, accumulate, d_slots);
    accumulate = 1;
    launched = true;
  } while (next < count);
  return launched ? finish_launch() : ZC_OK;
}

int zt_norm(const double* d_slots, float scale, float* d_norm, void* stream) {
  if (!good_scale(scale)) return ZC_ERR_ARG;
  if (!d_slots || !d_norm) return ZC_ERR_NULL;
  if (!aligned(d_slots, 16) || !aligned(d_norm, 4)) return ZC_ERR_ALIGN;
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), d_slots, scale, d_norm);
  return finish_launch();
}

int zt_clip(const void* const* d_in, const size_t* n, const int* dtype_in, void* const* d_out, const int* dtype_out, int count,
            const double* d_slots, float scale, float max_norm, float* d_norm, void* stream) {
  const int rc = check_list(d_in, n, dtype_in, d_out, dtype_out, count, true);
  if (rc != ZC_OK) return rc;
  if (!good_scale(scale) || !good_max_norm(max_norm)) return ZC_ERR_ARG;
  if (!d_slots) return ZC_ERR_NULL;
  if (!aligned(d_slots, 16) || !aligned(d_norm, 4)) return ZC_ERR_ALIGN;
  TensorList list;
  int next = 0;
  bool launched = false;
  do {
    next = fill_list(list, d_in, n, dtype_in, d_out, dtype_out, count, next);
    const size_t chunks = list.first[list.count];
    if (chunks == 0 && !d_norm) break;
    for (size_t from = 0; from < chunks || from == 0; from += kMostGroups) {
      const size_t groups = chunks == 0 ? 1 : chunks - from < kMostGroups ? chunks - from : kMostGroups;
      hipLaunchKernelGGL(clip_kernel, dim3((unsigned)groups), dim3(kThreads), 0, static_cast<hipStream_t>(stream), list, (uint32_t)from, d_slots, scale, max_norm, d_norm);
      d_norm = nullptr;
    }
    launched = true;
  } while (next < count);
  return launched ? finish_launch() : ZC_OK;
}

int zt_adamw(const struct zt_adamw_form* form, const void* d_grad, const double* d_slots, float* d_param, float* d_m, float* d_v, void* d_half,
             float* d_norm, void* stream) {
  if (!form) return ZC_ERR_NULL;
  if (!known_dtype(form->grad_dtype) || (d_half && form->half_dtype != ZC_BF16 && form->half_dtype != ZC_F16)) return ZC_ERR_DTYPE;
  const auto within = [](double v) { return v >= 0.0 && v <= (double)FLT_MAX; };
  double* const state = form->d_state;     // in place of step and lr
  if ((!state && (form->step < 1 || !within(form->lr))) || !within(form->eps) || !within(form->weight_decay) ||
      !(form->beta1 >= 0.0 && form->beta1 < 1.0) || !(form->beta2 >= 0.0 && form->beta2 < 1.0) || !good_scale(form->scale) ||
      (d_slots && !good_max_norm(form->max_norm)))
    return ZC_ERR_ARG;
  if (form->n > kMaxValues) return ZC_ERR_SIZE;
  if (form->n != 0 && (!d_grad || !d_param || !d_m || !d_v)) return ZC_ERR_NULL;
  if (!d_slots && d_norm) return ZC_ERR_NULL;
  if (!aligned(d_slots, 16) || !aligned(state, 16) || !aligned(d_norm, 4) || !aligned(d_grad, dtype_bytes(form->grad_dtype)) || !aligned(d_param, 4) || !aligned(d_m, 4) ||
      !aligned(d_v, 4) || !aligned(d_half, 2))
    return ZC_ERR_ALIGN;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (state) {
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(kThreads), 0, s, d_slots, form->scale, form->beta1, form->beta2, state, d_norm);
    if (form->n == 0) return finish_launch();
  }
  if (form->n == 0) return d_norm ? zt_norm(d_slots, form->scale, d_norm, stream) : ZC_OK;
  AdamwArgs a;
  a.grad = static_cast<const char*>(d_grad);
  a.slots = d_slots;
  a.param = d_param;
  a.m = d_m;
  a.v = d_v;
  a.half = static_cast<char*>(d_half);
  a.norm_out = state ? nullptr : d_norm;
  a.state = state;
  a.lr = state ? 0.0f : (float)form->lr;
  a.beta1 = (float)form->beta1;
  a.rest1 = (float)(1.0 - form->beta1);
  a.beta2 = (float)form->beta2;
  a.rest2 = (float)(1.0 - form->beta2);
  a.eps = (float)form->eps;
  a.weight_decay = (float)form->weight_decay;
  a.correct1 = state ? 0.0f : (float)(1.0 / (1.0 - pow(form->beta1, (double)form->step)));
  a.correct2 = state ? 0.0f : (float)(1.0 / (1.0 - pow(form->beta2, (double)form->step)));
  a.scale = form->scale;
  a.max_norm = form->max_norm;
  const int dh = d_half ? form->half_dtype : ZC_F32;
  for (size_t left = form->n; left != 0; left -= a.n) {
    a.n = left < kMostGroups * kAdamwTile ? left : kMostGroups * kAdamwTile;
    const dim3 grid((unsigned)((a.n + kAdamwTile - 1) / kAdamwTile));
#define LAUNCH(DG)                                                                                         \
  do {                                                                                                     \
    if (dh == ZC_F32) hipLaunchKernelGGL((adamw_kernel<DG, kF32>), grid, dim3(kThreads), 0, s, a);         \
    else if (dh == ZC_BF16) hipLaunchKernelGGL((adamw_kernel<DG, kBF16>), grid, dim3(kThreads), 0, s, a);  \
    else hipLaunchKernelGGL((adamw_kernel<DG, kF16>), grid, dim3(kThreads), 0, s, a);                      \
  } while (0)
    if (form->grad_dtype == ZC_F32) LAUNCH(kF32);
    else if (form->grad_dtype == ZC_BF16) LAUNCH(kBF16);
    else LAUNCH(kF16);
#undef LAUNCH
    a.grad += a.n * dtype_bytes(form->grad_dtype);
    a.param += a.n;
    a.m += a.n;
    a.v += a.n;
    if (a.half) a.half += a.n * 2;
    a.norm_out = nullptr;
  }
  return finish_launch();
}

}  // extern "C"
