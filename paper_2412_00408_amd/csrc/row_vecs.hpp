// row_vecs.hpp — a row of any element alignment as aligned 16-byte vectors, for the
// kernels that stream vocabulary rows.
#pragma once

#include "quake_device.hpp"

namespace qk {

// Row r of a matrix as the aligned 16-byte vectors that cover it: vector element
// e is row element e - skip (elements outside the row read as -inf, at most 15
// bytes before and after it, inside vectors that hold some of its bytes).
template <int DT>
struct RowVecs {
  const u32x4* v;
  uint32_t skip, cols, n;
  __device__ __forceinline__ RowVecs(const char* row, uint32_t cols_) : cols(cols_) {
    const uint32_t off = (uint32_t)((uintptr_t)row & 15u);
    v = reinterpret_cast<const u32x4*>(row - off);
    skip = off / kEsz<DT>;
    n = (skip + cols + kV<DT> - 1) / kV<DT>;
  }
  __device__ __forceinline__ void mask(uint32_t i, float* f) const {
    if (i == 0 || i + 1 == n) {
#pragma unroll
      for (int k = 0; k < kV<DT>; ++k) {
        const uint32_t e = i * kV<DT> + k;
        if (e < skip || e >= skip + cols) f[k] = -INFINITY;
      }
    }
  }
};

}  // namespace qk
