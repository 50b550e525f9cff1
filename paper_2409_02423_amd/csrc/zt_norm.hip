// zt_norm.hip -- gfx950 kernel and C ABI of the residual join with the norms around a block, forward (include/zt.h).
//
// A row stays in registers from its loads to its stores, so every value is read and written once: 8 bytes a value in half
// precision for some 15 operations, which memory bounds.  Mean and deviation are taken one after the other over the registers, which keeps them
// exact where a row's mean is far from zero.  One workgroup for each row: what overlaps one row's sums with another's
// loads is the other workgroups of the CU (a loop over rows with 2048 workgroups took 81 us where this takes 73).  8192 x 6144 values in bf16
// with both norms and a gate per channel take 73 us, 5.5 TB/s of what is read and written (a copy of 4 GiB: 4.8); four rows 3.7 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zt_norm.h"

namespace {

struct NormArgs {
  const char *x, *b, *gate, *pre_w, *pre_c, *post_w, *post_c;
  char *y, *h;
  float4* stats;
  size_t sx, sb, sg, sy, sh;     // bytes from row to row
  uint32_t rows;
  int cols;
  float scale, eps, inv_cols;
};

// Takes the mean from a row's values (with LAYER); its 1 / deviation.
template <int DT, bool LAYER, int NV, int MOST>
__device__ __forceinline__ void centre(Values<DT, NV, MOST>& values, const Lanes<DT, NV>& at, Sums<1, NV>& sums, float inv_cols, float eps, float& mean, float& r) {
  constexpr int V = kVec<DT>;
  float s[1] = {0.0f};
  mean = 0.0f;
  if constexpr (LAYER) {
    at.each([&](int i) {
      float v[V];
      values.get(at, i, v);
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] += v[j];
    });
    sums(s);
    mean = s[0] * inv_cols;
    s[0] = 0.0f;
  }
  at.each([&](int i) {
    float v[V];
    values.get(at, i, v);
    if constexpr (LAYER) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] -= mean;
      at.clear_rest(v, i);
      values.set(at, i, v);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[0] = fmaf(v[j], v[j], s[0]);
  });
  sums(s);
  r = 1.0f / sqrtf(fmaf(s[0], inv_cols, eps));
}

// v r w (+ c) of one vector.
template <int DT, bool LAYER, int NV>
__device__ __forceinline__ void weigh(float (&v)[kVec<DT>], float r, const Operand<DT, NV>& w, const Operand<DT, NV>& c, const Lanes<DT, NV>& at, int i) {
  float wv[kVec<DT>], cv[kVec<DT>];
  w.get(at, i, wv);
  if constexpr (LAYER) c.get(at, i, cv);
#pragma unroll
  for (int j = 0; j < kVec<DT>; ++j) v[j] = LAYER ? fmaf(v[j] * r, wv[j], cv[j]) : v[j] * r * wv[j];
}

template <int DT, bool LAYER, bool POST, int NV, int MOST>
__global__ void __launch_bounds__(MOST) norm_kernel(NormArgs a) {
  constexpr int V = kVec<DT>;
  __shared__ float buffers[2][1][kMostWaves];
  Sums<1, NV> sums{buffers};
  const Lanes<DT, NV> at(a.cols);
  const size_t row = at.first;
  if (NV < 0 && row >= a.rows) return;
  Values<DT, NV, MOST> values;
  Operand<DT, NV> pre_w, pre_c, post_w, post_c, gate, x, b;
  x.open(at, a.x + row * a.sx);
  b.open(at, a.b ? a.b + row * a.sb : nullptr);
  gate.open(at, a.gate ? a.gate + row * a.sg : nullptr, 1.0f);
  pre_w.open(at, a.pre_w, 1.0f);
  if constexpr (LAYER) pre_c.open(at, a.pre_c);
  if constexpr (POST) post_w.open(at, a.post_w, 1.0f);
  if constexpr (POST && LAYER) post_c.open(at, a.post_c);
  float4 stats = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (POST) {
    at.each([&](int i) {
      float v[V];
      b.get(at, i, v);
      at.clear_rest(v, i);
      values.set(at, i, v);
    });
    centre<DT, LAYER>(values, at, sums, a.inv_cols, a.eps, stats.x, stats.y);
  }
  at.each([&](int i) {
    float v[V], g[V], xv[V];
    if constexpr (POST) {
      values.get(at, i, v);
      weigh<DT, LAYER>(v, stats.y, post_w, post_c, at, i);
    } else {
      b.get(at, i, v);
    }
    gate.get(at, i, g);
    x.get(at, i, xv);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = fmaf(g[j], v[j], a.scale * xv[j]);
    at.clear_rest(v, i);
    values.set(at, i, v);
    if (a.y) at.store(a.y + row * a.sy, i, v);
  });
  centre<DT, LAYER>(values, at, sums, a.inv_cols, a.eps, stats.z, stats.w);
  at.each([&](int i) {
    float v[V];
    values.get(at, i, v);
    weigh<DT, LAYER>(v, stats.w, pre_w, pre_c, at, i);
    at.store(a.h + row * a.sh, i, v);
  });
  if (a.stats && at.lane == 0) a.stats[row] = stats;
}

// ---- host ------------------------------------------------------------------------------

// As few vectors a lane as leave a row to one wavefront, or to at most four, one for each SIMD of a CU: more vectors a lane take
// registers and with them rows that are under way, more wavefronts wait for one another at each sum.  us forward, with 1, 2, 3, 4 and 5
// vectors a lane: 8192 x 1500 in bf16 18.4, 22.8, 22.0, 29.2 and 33.1 (3, 2, 1, 1 and 1 wavefronts); x 2561 44.4, 36.8, 37.5, 43.7, 58.7 (6, 3, 2, 2, 2);
// x 4099 84.7, 68.7, 61.8, 74.4, 74.0 (9, 5, 3, 3, 2); x 6144 74.1, 72.9, 69.8, 74.6, 93.2 (12, 6, 4, 3, 3); 4000 x 4099 in fp32, a gate for each
// value, 2 to 5 vectors 78.1, 82.9, 90.1, 64.2 (9, 6, 5, 4).
// Rows of more than 2048 vectors have 16 wavefronts and lie in LDS, one workgroup a CU: 4096 x 8193 in fp32 133 us, 4.0 TB/s (x 8192, in registers, 100);
// x 12288 165, 4.9; 2048 x 16391 in bf16 93, 2.9 (x 16384 53); x 20480 84, 4.0; x 32768 119, 4.5.
Layout forward_layout(size_t cols, int dtype) {
  const size_t vectors = row_vectors(cols, dtype);
  if (short_rows(vectors)) return short_layout(vectors);
  const int each = (int)((vectors + 255) / 256);
  if (each <= 5) return {each, lanes_for(vectors, each), 256};
  if (vectors <= 2048) return {vectors <= 1536 ? 3 : 4, lanes_for(vectors, vectors <= 1536 ? 3 : 4), 512};
  return {0, 1024, 1024};
}

template <int DT, bool LAYER, bool POST>
void launch(const NormArgs& a, const Layout& l, hipStream_t s) {
  const dim3 grid((a.rows + l.rows - 1) / l.rows);
#define CALL(NV, MOST) hipLaunchKernelGGL((norm_kernel<DT, LAYER, POST, NV, MOST>), grid, dim3(l.lanes), 0, s, a)
  switch (l.most * 8 + l.vectors) {
    case 256 * 8 + kShort16: CALL(kShort16, 256); break;
    case 256 * 8 + kShort32: CALL(kShort32, 256); break;
    case 256 * 8 + kShort64: CALL(kShort64, 256); break;
    case 256 * 8 + 1: CALL(1, 256); break;
    case 256 * 8 + 2: CALL(2, 256); break;
    case 256 * 8 + 3: CALL(3, 256); break;
    case 256 * 8 + 4: CALL(4, 256); break;
    case 256 * 8 + 5: CALL(5, 256); break;
    case 512 * 8 + 3: CALL(3, 512); break;
    case 512 * 8 + 4: CALL(4, 512); break;
    default: CALL(0, 1024); break;
  }
#undef CALL
}
template <int DT>
void launch(const zt_residual& f, const NormArgs& a, const Layout& l, hipStream_t s) {
  if (f.kind == ZT_LAYER) f.post ? launch<DT, true, true>(a, l, s) : launch<DT, true, false>(a, l, s);
  else f.post ? launch<DT, false, true>(a, l, s) : launch<DT, false, false>(a, l, s);
}

constexpr size_t kMostRows = (size_t)1 << 21;   // of one launch: a grid has fewer than 2^32 lanes

}  // namespace

extern "C" {

int zt_residual_norm(const struct zt_residual* form, const void* d_x, const void* d_b, const void* d_gate, const void* d_pre_weight,
                     const void* d_pre_bias, const void* d_post_weight, const void* d_post_bias, void* d_y, void* d_h, float* d_stats, void* stream) {
  const int rc = check_form(form);
  if (rc != ZC_OK) return rc;
  const zt_residual& f = *form;
  if (f.kind == ZT_RMS && (d_pre_bias || d_post_bias)) return ZC_ERR_ARG;
  if (!good_strides({f.stride_x, f.stride_b, f.stride_gate}, {f.stride_y, f.stride_h}, f.cols)) return ZC_ERR_ARG;
  if (!d_b && (f.post || f.gate != ZT_GATE_NONE)) return ZC_ERR_NULL;
  if (f.rows == 0 || f.cols == 0) return ZC_OK;
  if (!d_x || !d_h || (f.gate != ZT_GATE_NONE && !d_gate)) return ZC_ERR_NULL;
  const size_t e = dtype_bytes(f.dtype);
  if (!all_aligned({d_x, d_b, d_gate, d_pre_weight, d_pre_bias, d_post_weight, d_post_bias, d_y, d_h}, e) || !aligned(d_stats, 16)) return ZC_ERR_ALIGN;
  NormArgs a;
  a.x = bytes_of(d_x);
  a.b = bytes_of(d_b);
  a.gate = f.gate == ZT_GATE_NONE ? nullptr : bytes_of(d_gate);
  a.pre_w = bytes_of(d_pre_weight);
  a.pre_c = bytes_of(d_pre_bias);
  a.post_w = bytes_of(d_post_weight);
  a.post_c = bytes_of(d_post_bias);
  a.y = static_cast<char*>(d_y);
  a.h = static_cast<char*>(d_h);
  a.stats = reinterpret_cast<float4*>(d_stats);
  a.sx = stride_of(f.stride_x, f.cols) * e;
  a.sb = stride_of(f.stride_b, f.cols) * e;
  a.sg = f.gate == ZT_GATE_FULL ? stride_of(f.stride_gate, f.cols) * e : 0;   // a gate per channel is the same for every row
  a.sy = stride_of(f.stride_y, f.cols) * e;
  a.sh = stride_of(f.stride_h, f.cols) * e;
  a.cols = (int)f.cols;
  a.scale = f.residual_scale;
  a.eps = f.eps;
  a.inv_cols = (float)(1.0 / (double)f.cols);
  const Layout l = forward_layout(f.cols, f.dtype);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  for (size_t done = 0; done < f.rows; done += kMostRows) {
    const size_t rows = f.rows - done < kMostRows ? f.rows - done : kMostRows;
    a.rows = (uint32_t)rows;
    if (f.dtype == ZC_F32) launch<kF32>(f, a, l, s);
    else if (f.dtype == ZC_BF16) launch<kBF16>(f, a, l, s);
    else launch<kF16>(f, a, l, s);
    a.x += rows * a.sx;
    if (a.b) a.b += rows * a.sb;
    if (a.gate) a.gate += rows * a.sg;
    if (a.y) a.y += rows * a.sy;
    a.h += rows * a.sh;
    if (a.stats) a.stats += rows;
  }
  return finish_launch();
}

}  // extern "C"
