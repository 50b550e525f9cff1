// ze_common.h -- what the vocabulary's operators share: sums over the lanes up to one, checks of a form, places in a workspace.
#ifndef ZE_COMMON_H
#define ZE_COMMON_H

#include <limits.h>
#include <math.h>

#include "../../include/ze.h"
#include "zt_device.h"

namespace {

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_count(uint32_t v) {
  return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true);
}
// The sum over the lanes up to each one.  All 64 have to be active.
__device__ __forceinline__ uint32_t sum_up_to(uint32_t v) {
  v = dpp_count<0x111, 0xF>(v);   // row_shr 1, 2, 4, 8
  v = dpp_count<0x112, 0xF>(v);
  v = dpp_count<0x114, 0xF>(v);
  v = dpp_count<0x118, 0xF>(v);
  v = dpp_count<0x142, 0xA>(v);   // each row's last lane to the next row, then the second row's to the last two
  return dpp_count<0x143, 0xC>(v);
}

// Which of this rank's rows an id names, of `rows` from `first` on, or -1.  (first is at most 2^63 - 1 - ZE_MAX_ROWS: then the least of ids is no row either.)
__device__ __forceinline__ long long row_of_id(long long id, long long first, long long rows) {
  const unsigned long long at = (unsigned long long)id - (unsigned long long)first;   // (below `first`, and negative: more than any number of rows)
  return at < (unsigned long long)rows ? (long long)at : -1;
}

constexpr size_t kMaxStride = (size_t)1 << 20;   // elements: a tile's rows are told apart by 32 bits

size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }
size_t parts(size_t n, size_t of) { return (n + of - 1) / of; }

int check_form(const struct ze_form* f) {
  if (!f) return ZC_ERR_NULL;
  if (!known_dtype(f->dtype)) return ZC_ERR_DTYPE;
  if ((f->id_dtype != ZE_I32 && f->id_dtype != ZE_I64) || f->first < 0 || f->first > LLONG_MAX - ZE_MAX_ROWS || !isfinite(f->scale)) return ZC_ERR_ARG;
  if (f->tokens > ZE_MAX_TOKENS || f->rows > ZE_MAX_ROWS || f->cols > ZE_MAX_COLS) return ZC_ERR_SIZE;
  if (f->stride_table > kMaxStride || f->stride_tokens > kMaxStride) return ZC_ERR_ARG;
  return ZC_OK;
}
// An output's rows do not overlap.
bool good_output(size_t stride, size_t cols) { return stride == 0 || (stride >= cols && stride <= kMaxStride); }
size_t stride_of(size_t stride, size_t cols) { return stride ? stride : cols; }
bool aligned_ids(const void* p, int id_dtype) { return aligned(p, id_dtype == ZE_I64 ? 8 : 4); }

// Places in a workspace, one behind the other, at multiples of 256 bytes.
struct Places {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t here = at;
    at += up(bytes, 256);
    return here;
  }
};

}  // namespace
#endif  // ZE_COMMON_H
