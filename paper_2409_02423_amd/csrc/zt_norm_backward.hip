// zt_norm_backward.hip -- gfx950 kernels and C ABI of the residual join with the norms around a block, backward (include/zt.h).
//
// The gradient of unit = (v - mean) r is r (t - unit mean(t unit) - mean(t)) for that of the norm's output times its weights, t; through the
// join it is followed from h to y, to x and the block's output, and through the gate and the other norm to b.  As forward, a row
// stays in registers (12 bytes a value in half precision for some 30 operations: memory bounds it).  The sums over the rows, for weights, biases and a gate per
// channel, stay there too: a workgroup takes many rows, adds their terms up lane by lane and leaves one partial sum for each column; a second kernel adds the
// partial sums up in a fixed order, so the result does not depend on which workgroup was first.  8192 x 6144 values in bf16 with both norms and a gate per
// channel: 110 us, 5.5 TB/s, and 5.5 us for 256 partial sums of 18432 columns.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zt_norm.h"

namespace {

struct BackwardArgs {
  const char *dy, *dh, *y, *b, *gate, *pre_w, *post_w, *post_c;
  const float4* stats;
  char *dx, *db, *dgate;
  float* partial;                // [workgroup][sum][columns, padded]
  size_t sdy, sdh, sy, sb, sg, sdx, sdb, sdg;
  uint32_t rows;
  int cols, padded;
  float scale, inv_cols;
};

// The sums over rows, in their order in the workspace.
template <bool LAYER, bool POST, bool CHANNEL>
struct SumIndex {
  static constexpr int pre_w = 0, pre_c = 1, post_w = 1 + LAYER, post_c = 2 + LAYER, gate = 1 + LAYER + (POST ? 1 + LAYER : 0), count = gate + CHANNEL;
};

// A sum is added up where that stands and not at the end of the row, where the compiler would move it: what is added takes more
// registers till then than all the sums.
__device__ __forceinline__ void now(float& sum) { asm volatile("" : "+v"(sum)); }

// A lane's sums over rows: in registers, or for wide rows (NV = 0) in the workspace, of which a workgroup has a part to itself.
template <int COUNT, int DT, int NV>
struct Columns {
  static constexpr int V = kVec<DT>;
  float held[COUNT][kHeld<NV>][V];
  float* partial;
  size_t padded;       // columns
  bool fresh = true;   // nothing in the workspace yet
  __device__ __forceinline__ Columns(float* p, size_t columns) : partial(p), padded(columns) {
    if constexpr (NV != 0) {
#pragma unroll
      for (int k = 0; k < COUNT; ++k)
#pragma unroll
        for (int i = 0; i < kHeld<NV>; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) held[k][i][j] = 0.0f;
    }
  }
  // Sum k of vector i: += a * b
  __device__ __forceinline__ void add(const Lanes<DT, NV>& at, int k, int i, const float (&a)[V], const float (&b)[V]) {
    if constexpr (NV != 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        held[k][i][j] = fmaf(a[j], b[j], held[k][i][j]);
        if constexpr (NV > 1) now(held[k][i][j]);
      }
    } else {
      float* sums = partial + k * padded + at.col(i);
      if (at.whole(i)) {
        Raw<kF32, V> r = {};
        if (!fresh) r.load(reinterpret_cast<char*>(sums - at.col(i)), (uint32_t)at.col(i) * 4);
        float s[V];
        r.unpack(s);
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] = fmaf(a[j], b[j], s[j]);
        r.pack(s);
        r.store(reinterpret_cast<char*>(sums - at.col(i)), (uint32_t)at.col(i) * 4);
      } else if (at.any(i)) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j >= at.from(i) && j < at.to()) sums[j] = fmaf(a[j], b[j], fresh ? 0.0f : sums[j]);
      }
    }
  }
  __device__ __forceinline__ void add(const Lanes<DT, NV>& at, int k, int i, const float (&a)[V]) {
    float ones[V];
#pragma unroll
    for (int j = 0; j < V; ++j) ones[j] = 1.0f;
    add(at, k, i, a, ones);
  }
  __device__ __forceinline__ void leave(const Lanes<DT, NV>& at) {
    if constexpr (NV < 0) {      // of the rows that a workgroup has at a time: over a wavefront's, then over the wavefronts
      constexpr int kLanes = kShortLanes<NV>;
      __shared__ float parts[COUNT][4][kLanes][V];
      const int wave = threadIdx.x / 64;
#pragma unroll
      for (int k = 0; k < COUNT; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float s = held[k][0][j];
          if constexpr (kLanes == 16) s += __shfl_xor(s, 16);
          if constexpr (kLanes < 64) s += __shfl_xor(s, 32);
          if ((threadIdx.x & 63) < kLanes) parts[k][wave][at.lane][j] = s;
        }
      __syncthreads();
      if (threadIdx.x >= kLanes) return;
#pragma unroll
      for (int k = 0; k < COUNT; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) held[k][0][j] = (parts[k][0][at.lane][j] + parts[k][1][at.lane][j]) + (parts[k][2][at.lane][j] + parts[k][3][at.lane][j]);
    }
    if constexpr (NV != 0) {
#pragma unroll
      for (int k = 0; k < COUNT; ++k)
        at.each([&](int i) {
          Raw<kF32, V> r;
          r.pack(held[k][i]);
          char* sums = reinterpret_cast<char*>(partial + k * padded);
          if (at.whole(i)) r.store(sums, (uint32_t)at.col(i) * 4);
          else if (at.any(i)) r.store(sums, (uint32_t)at.col(i) * 4, at.from(i), at.to());
        });
    }
  }
};

// What a row is made of, apart from the weights.
template <int DT, int NV, bool HOLD>
struct BackwardRow {
  Operand<DT, NV, HOLD> dh, y, dy, b, gate;
  float4 stats;
  __device__ __forceinline__ void open(const Lanes<DT, NV>& at, const BackwardArgs& a, uint32_t row) {
    stats = a.stats[row];
    dh.open(at, a.dh + row * a.sdh);
    y.open(at, a.y + row * a.sy);
    dy.open(at, a.dy ? a.dy + row * a.sdy : nullptr);
    b.open(at, a.b ? a.b + row * a.sb : nullptr);
    gate.open(at, a.gate ? a.gate + row * a.sg : nullptr, 1.0f);
  }
};

// What registers hold of a row and the weights besides the sums: all of it, the row, or what is worked on.
enum Hold { kNothing, kRow, kAll };

template <int DT, bool LAYER, bool POST, bool CHANNEL, int NV, int MOST, Hold HOW>
__global__ void __launch_bounds__(MOST) norm_backward_kernel(BackwardArgs a) {
  constexpr bool HOLD = HOW == kAll, ROW = HOW != kNothing;
  constexpr int V = kVec<DT>, K = LAYER ? 2 : 1;
  typedef SumIndex<LAYER, POST, CHANNEL> Index;
  __shared__ float buffers[2][K][kMostWaves];
  Sums<K, NV> sums{buffers};
  const Lanes<DT, NV> at(a.cols);
  Values<DT, NV, MOST, HOLD> values;   // the gradient of y, then of z
  Operand<DT, NV, HOLD> pre_w, post_w, post_c;
  const auto open_weights = [&] {
    pre_w.open(at, a.pre_w, 1.0f);
    if constexpr (POST) post_w.open(at, a.post_w, 1.0f);
    if constexpr (POST && LAYER) post_c.open(at, a.post_c);
  };
  Columns<Index::count, DT, NV> columns(a.partial + (size_t)blockIdx.x * Index::count * a.padded, a.padded);
  // The weights stay, and the next row is under way while this one is worked on, where registers hold all that.
  constexpr bool kAhead = HOLD && (NV < 2 || DT == kF32 || !(LAYER && POST && CHANNEL));
  BackwardRow<DT, NV, ROW> current, next;
  if constexpr (kAhead) {
    open_weights();
    if (at.first < a.rows) next.open(at, a, at.first);
  }
  for (uint32_t row = at.first; row < a.rows; row += at.step) {
    if constexpr (kAhead) {
      current = next;
      if (row + at.step < a.rows) next.open(at, a, row + at.step);
    } else {
      open_weights();
      current.open(at, a, row);
    }
    const float4 stats = current.stats;
    const auto &dh = current.dh, &y = current.y, &dy = current.dy, &b = current.b, &gate = current.gate;
    // a norm's input as it was normed, before weight and bias
    const auto unit = [&](const Operand<DT, NV, ROW>& from, int i, float mean, float r, float (&u)[V]) {
      from.get(at, i, u);
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] = LAYER ? (u[j] - mean) * r : u[j] * r;
    };
    // what a norm's gradient is made of: the sums of t = g w along u, and with LAYER of t
    const auto add_sums = [&](float (&s)[K], const float (&g)[V], const float (&w)[V], const float (&u)[V]) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float t = g[j] * w[j];
        s[0] = fmaf(t, u[j], s[0]);
        if constexpr (LAYER) s[K - 1] += t;
      }
      if constexpr (NV > 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) now(s[k]);
      }
    };
    // through the pre norm
    float s[K] = {};
    at.each([&](int i) {
      if constexpr (NV > 1 && !HOLD) at.forget();
      float g[V], u[V], w[V];
      dh.get(at, i, g);
      at.clear_rest(g, i);
      unit(y, i, stats.z, stats.w, u);
      pre_w.get(at, i, w);
      columns.add(at, Index::pre_w, i, g, u);
      if constexpr (LAYER) columns.add(at, Index::pre_c, i, g);
      add_sums(s, g, w, u);
    });
    sums(s);
    const float along = s[0] * a.inv_cols, mean = s[K - 1] * a.inv_cols;
    float s2[K] = {};
    at.each([&](int i) {
      if constexpr (NV > 1 && !HOLD) at.forget();
      float g[V], u[V], w[V], d[V], v[V];
      dh.get(at, i, g);
      unit(y, i, stats.z, stats.w, u);
      pre_w.get(at, i, w);
      dy.get(at, i, d);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float t = fmaf(-u[j], along, g[j] * w[j]);
        if constexpr (LAYER) t -= mean;
        d[j] = fmaf(stats.w, t, d[j]);
        v[j] = a.scale * d[j];
      }
      if (a.dx) at.store(a.dx + row * a.sdx, i, v);
      // through the gate
      if constexpr (POST) {
        unit(b, i, stats.x, stats.y, u);
        post_w.get(at, i, w);
      } else {
        b.get(at, i, u);
      }
      if (CHANNEL || a.dgate) {
        float z[V], c[V];
        if constexpr (POST && LAYER) post_c.get(at, i, c);
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = !POST ? u[j] : LAYER ? fmaf(u[j], w[j], c[j]) : u[j] * w[j];
        if constexpr (CHANNEL) {
          columns.add(at, Index::gate, i, d, z);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) z[j] *= d[j];
          at.store(a.dgate + row * a.sdg, i, z);
        }
      }
      gate.get(at, i, g);
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] *= g[j];
      if constexpr (POST) {
        at.clear_rest(d, i);
        columns.add(at, Index::post_w, i, d, u);
        if constexpr (LAYER) columns.add(at, Index::post_c, i, d);
        add_sums(s2, d, w, u);
        values.set(at, i, d);
      } else if (a.db) {
        at.store(a.db + row * a.sdb, i, d);
      }
    });
    // through the post norm
    if constexpr (POST) {
      sums(s2);
      const float along2 = s2[0] * a.inv_cols, mean2 = s2[K - 1] * a.inv_cols;
      if (a.db) {
        at.each([&](int i) {
          if constexpr (NV > 1 && !HOLD) at.forget();
          float d[V], u[V], w[V];
          values.get(at, i, d);
          unit(b, i, stats.x, stats.y, u);
          post_w.get(at, i, w);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float t = fmaf(-u[j], along2, d[j] * w[j]);
            if constexpr (LAYER) t -= mean2;
            d[j] = stats.y * t;
          }
          at.store(a.db + row * a.sdb, i, d);
        });
      }
    }
    columns.fresh = false;
  }
  columns.leave(at);
}

// Adds the partial sums up, in a fixed order: a workgroup takes 64 columns of one sum, 16 lanes with four columns each and 64 slices of the
// partial sums.  The slices are added up as a tree: a term goes through six additions there, not through up to 63 (512 rows of 516 fp32 values,
// one of them with gradient 1 and the rest with 2^-28: what is small was lost, 1.9e-6).
struct ColumnArgs {
  const float* partial;
  float* out[5];
  int partials, count, cols, padded;
};
constexpr int kSlices = 64;
template <int N>
__device__ __forceinline__ float tree_sum(const float4 (*slices)[16], int column) {
  if constexpr (N == 1) return reinterpret_cast<const float*>(slices[0])[column];
  else return tree_sum<N / 2>(slices, column) + tree_sum<N / 2>(slices + N / 2, column);
}
__global__ void __launch_bounds__(16 * kSlices) column_sums_kernel(ColumnArgs a) {
  __shared__ float4 slices[kSlices][16];
  const int lane = threadIdx.x & 15, slice = threadIdx.x / 16, k = blockIdx.y;
  const int col = (blockIdx.x * 16 + lane) * 4;
  float4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (col < a.padded) {
    const float* p = a.partial + (size_t)k * a.padded + col;
    const size_t step = (size_t)a.count * a.padded;
#pragma unroll 4
    for (int i = slice; i < a.partials; i += kSlices) {
      const float4 v = *reinterpret_cast<const float4*>(p + i * step);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  }
  slices[slice][lane] = s;
  __syncthreads();
  float* out = a.out[k];
  if (threadIdx.x < 64 && out) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    const float t = tree_sum<kSlices>(slices, threadIdx.x);
    if (c < a.cols) out[c] = t;
  }
}

// ---- host ------------------------------------------------------------------------------

// One vector a lane where a workgroup can have as many lanes: more of them take registers and no more bytes are under way.  us
// with 1, 2, 3 and 4 vectors a lane, each at its best number of workgroups: 8192 x 6144 values in bf16 with both norms and a gate per channel 115.7, 116.2,
// 124.4 and 149.1; x 4096 78.2, 79.1, 104.1 and 88.5; x 2048 45.3, 47.4, 58.9 and 73.0.  Beyond 768 lanes, whose registers still hold two rows, two
// vectors.  Wider ones have fewer registers for a value: rows of more than 1024 vectors keep their sums there and, where
// it fits, the row. us in the form for any width, whose sums are in the workspace, with the sums in registers and with the row as
// well, with both norms and a gate per channel: 4096 x 12288 in bf16 312, 169 and, with at most 768 lanes, which have more registers each, 152; x 8200 225, 150
// and 119; 2048 x 16384 212, 112, and it does not fit; 4096 x 8193 in fp32 302, 257, and it does not fit; x 8192 the latter two 175 and 171. With sums of
// all five kinds in half precision it takes fewer lanes, without the row: 4096 x 12288 448 and 273.
Layout backward_layout(const zt_residual& f) {
  const size_t vectors = row_vectors(f.cols, f.dtype);
  if (short_rows(vectors)) return short_layout(vectors);
  if (vectors <= 256) return {1, lanes_for(vectors, 1), 256};
  if (vectors <= 768) return {1, lanes_for(vectors, 1), 768};
  if (vectors <= 1024) return {2, lanes_for(vectors, 2), 512};
  if (f.dtype == ZC_F32) {
    if (vectors <= 2048) return {2, lanes_for(vectors, 2), 1024};
    if (vectors <= 4096) return {4, lanes_for(vectors, 4), 1024};
  } else if (vectors <= 2048) {
    if (f.kind == ZT_LAYER && f.post && f.gate == ZT_GATE_CHANNEL) return {4, lanes_for(vectors, 4), 512};
    return {2, lanes_for(vectors, 2), vectors <= 1536 ? 768 : 1024};
  }
  return {0, 1024, 1024};
}

// Workgroups, each of which leaves one partial sum for each column: as few as keep memory busy.  us with 1, 2, 3, 4, 6, 8 and 12
// a CU: 256 lanes (8192 x 2048 as above) 49.2, 45.3, 46.8, 52.8, 54.5, 57.0, 63.4; 128 lanes (16384 x 1024) 81.9, 56.1, 45.2, 48.5, 49.9, 57.4, 61.8; 512 and 768 lanes with 1 and 2 78.2 and 83.2, 115.7 and 123.5.
// Short rows with 2, 3, 4 and 6: 262144 x 64 in bf16 57.1, 53.4, 50.4, 54.6; 131072 x 128 45.1, 45.0, 47.3, 50.1; x 200 65.6, 65.2, 70.7, 74.4; 65536 x 512
// 78.3, 81.5, 88.1, 84.8; in fp32, whose vectors have half the sums and leave room for more, 262144 x 64 101, 81.3, 76.3, 93.0; 65536 x 256 113, 88.9, 79.3, 81.7.
size_t backward_groups(const zt_residual& f, const Layout& l) {
  const size_t rows = f.rows;
  const size_t per_cu = l.vectors < 0 ? (f.dtype == ZC_F32 ? 4 : 3) : l.vectors == 0 || l.lanes > 256 ? 1 : l.lanes > 128 ? 2 : 3;
  const size_t groups = (rows + l.rows - 1) / l.rows;
  return groups < kCUs * per_cu ? groups : kCUs * per_cu;
}

int sums_of(const zt_residual& f) {
  const int layer = f.kind == ZT_LAYER;
  return 1 + layer + (f.post ? 1 + layer : 0) + (f.gate == ZT_GATE_CHANNEL);
}
size_t padded_cols(size_t cols) { return (cols + 7) / 8 * 8; }

template <int DT, bool LAYER, bool POST, bool CHANNEL>
void launch(const BackwardArgs& a, const Layout& l, unsigned groups, hipStream_t s) {
#define CALL(NV, MOST, HOW) hipLaunchKernelGGL((norm_backward_kernel<DT, LAYER, POST, CHANNEL, NV, MOST, HOW>), dim3(groups), dim3(l.lanes), 0, s, a)
  if (l.vectors == kShort16) CALL(kShort16, 256, kAll);
  else if (l.vectors == kShort32) CALL(kShort32, 256, kAll);
  else if (l.vectors == kShort64) CALL(kShort64, 256, kAll);
  else if (l.vectors == 1 && l.most == 256) CALL(1, 256, kAll);
  else if (l.vectors == 1) CALL(1, 768, kAll);
  else if (l.vectors == 2 && l.most == 512) CALL(2, 512, kAll);
  else if (l.vectors == 0) CALL(0, 1024, kNothing);
  else if constexpr (DT == kF32) {
    if (l.vectors == 2) CALL(2, 1024, kRow);
    else CALL(4, 1024, kNothing);
  } else if constexpr (LAYER && POST && CHANNEL) {
    CALL(4, 512, kNothing);
  } else {
    if (l.most == 768) CALL(2, 768, kRow);
    else CALL(2, 1024, (CHANNEL || (LAYER && POST)) ? kNothing : kRow);
  }
#undef CALL
}
template <int DT, bool LAYER, bool POST>
void launch(const zt_residual& f, const BackwardArgs& a, const Layout& l, unsigned groups, hipStream_t s) {
  f.gate == ZT_GATE_CHANNEL ? launch<DT, LAYER, POST, true>(a, l, groups, s) : launch<DT, LAYER, POST, false>(a, l, groups, s);
}
template <int DT>
void launch(const zt_residual& f, const BackwardArgs& a, const Layout& l, unsigned groups, hipStream_t s) {
  if (f.kind == ZT_LAYER) f.post ? launch<DT, true, true>(f, a, l, groups, s) : launch<DT, true, false>(f, a, l, groups, s);
  else f.post ? launch<DT, false, true>(f, a, l, groups, s) : launch<DT, false, false>(f, a, l, groups, s);
}

}  // namespace

extern "C" {

size_t zt_residual_work_bytes(const struct zt_residual* form) {
  if (check_form(form) != ZC_OK || form->rows == 0 || form->cols == 0) return 0;
  const Layout l = backward_layout(*form);
  return backward_groups(*form, l) * (size_t)sums_of(*form) * padded_cols(form->cols) * sizeof(float);
}

int zt_residual_norm_backward(const struct zt_residual* form, const void* d_dy, const void* d_dh, const void* d_y, const void* d_b,
                              const void* d_gate, const void* d_pre_weight, const void* d_post_weight, const void* d_post_bias,
                              const float* d_stats, void* d_dx, void* d_db, void* d_dgate, float* d_dpre_weight, float* d_dpre_bias,
                              float* d_dpost_weight, float* d_dpost_bias, void* d_work, size_t work_bytes, void* stream) {
  const int rc = check_form(form);
  if (rc != ZC_OK) return rc;
  const zt_residual& f = *form;
  if (f.kind == ZT_RMS && (d_dpre_bias || d_dpost_bias || d_post_bias)) return ZC_ERR_ARG;
  if ((!f.post && (d_dpost_weight || d_dpost_bias)) || (f.gate == ZT_GATE_NONE && d_dgate)) return ZC_ERR_ARG;
  if (!good_strides({f.stride_dy, f.stride_dh, f.stride_y, f.stride_b, f.stride_gate}, {f.stride_dx, f.stride_db, f.stride_dgate}, f.cols)) return ZC_ERR_ARG;
  if (!d_b && (f.post || f.gate != ZT_GATE_NONE || d_db)) return ZC_ERR_NULL;
  if (f.cols == 0) return ZC_OK;
  const size_t e = dtype_bytes(f.dtype);
  const bool channel = f.gate == ZT_GATE_CHANNEL;
  if (f.rows != 0 && (!d_dh || !d_y || !d_stats || !d_work || (f.gate != ZT_GATE_NONE && !d_gate))) return ZC_ERR_NULL;
  if (!all_aligned({d_dy, d_dh, d_y, d_b, d_gate, d_pre_weight, d_post_weight, d_post_bias, d_dx, d_db}, e) || !aligned(d_dgate, channel ? 4 : e) ||
      !all_aligned({d_dpre_weight, d_dpre_bias, d_dpost_weight, d_dpost_bias}, 4) || !aligned(d_stats, 16) || !aligned(d_work, 16))
    return ZC_ERR_ALIGN;
  if (work_bytes < zt_residual_work_bytes(form)) return ZC_ERR_CAPACITY;
  BackwardArgs a;
  a.dy = bytes_of(d_dy);
  a.dh = bytes_of(d_dh);
  a.y = bytes_of(d_y);
  a.b = bytes_of(d_b);
  a.gate = f.gate == ZT_GATE_NONE ? nullptr : bytes_of(d_gate);
  a.pre_w = bytes_of(d_pre_weight);
  a.post_w = bytes_of(d_post_weight);
  a.post_c = bytes_of(d_post_bias);
  a.stats = reinterpret_cast<const float4*>(d_stats);
  a.dx = static_cast<char*>(d_dx);
  a.db = static_cast<char*>(d_db);
  a.dgate = channel ? nullptr : static_cast<char*>(d_dgate);
  a.partial = static_cast<float*>(d_work);
  a.sdy = stride_of(f.stride_dy, f.cols) * e;
  a.sdh = stride_of(f.stride_dh, f.cols) * e;
  a.sy = stride_of(f.stride_y, f.cols) * e;
  a.sb = stride_of(f.stride_b, f.cols) * e;
  a.sg = f.gate == ZT_GATE_FULL ? stride_of(f.stride_gate, f.cols) * e : 0;   // a gate per channel is the same for every row
  a.sdx = stride_of(f.stride_dx, f.cols) * e;
  a.sdb = stride_of(f.stride_db, f.cols) * e;
  a.sdg = stride_of(f.stride_dgate, f.cols) * e;
  a.rows = (uint32_t)f.rows;
  a.cols = (int)f.cols;
  a.padded = (int)padded_cols(f.cols);
  a.scale = f.residual_scale;
  a.inv_cols = (float)(1.0 / (double)f.cols);
  const Layout l = backward_layout(f);
  const size_t groups = backward_groups(f, l);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (f.rows != 0) {
    if (f.dtype == ZC_F32) launch<kF32>(f, a, l, (unsigned)groups, s);
    else if (f.dtype == ZC_BF16) launch<kBF16>(f, a, l, (unsigned)groups, s);
    else launch<kF16>(f, a, l, (unsigned)groups, s);
  }
  ColumnArgs c;      // with no rows the sums are zero
  int k = 0;
  c.out[k++] = d_dpre_weight;
  if (f.kind == ZT_LAYER) c.out[k++] = d_dpre_bias;
  if (f.post) c.out[k++] = d_dpost_weight;
  if (f.post && f.kind == ZT_LAYER) c.out[k++] = d_dpost_bias;
  if (channel) c.out[k++] = static_cast<float*>(d_dgate);
  bool wanted = false;
  for (int i = 0; i < k; ++i) wanted = wanted || c.out[i];
  if (wanted) {
    c.partial = a.partial;
    c.partials = (int)groups;
    c.count = k;
    c.cols = a.cols;
    c.padded = a.padded;
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((a.padded + 63) / 64), (unsigned)k), dim3(16 * kSlices), 0, s, c);
  }
  return finish_launch();
}

}  // extern "C"
