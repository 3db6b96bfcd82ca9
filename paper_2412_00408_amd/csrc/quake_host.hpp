// quake_host.hpp — host-side helpers of libquake: the folded constants of
// QuAKE (each evaluated in double from its definition and rounded once to
// binary32), argument validation, and launch bookkeeping.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "quake.h"

namespace qk {

constexpr double kLn2 = 0.693147180559945309417232121458176568;
constexpr double kTwo23 = 8388608.0;      // 2^l_m, l_m = 23 (Sec. II-A)
constexpr double kBias = 127.0;           // B (Sec. II-A)
constexpr double kSchraudolph = 0.0436;   // bias of first-order QuAKE (Sec. III-A)
constexpr double kGeluC = 0.044715;       // Eq. 4
constexpr double kPi = 3.14159265358979323846264338327950288;

// The two constants of one QuAKE call (Eq. 5), or of its EXACT counterpart
// (the same affine map in base 2 without the 2^23 scale and 127 offset).
struct Affine {
  float c0, c1;
};

// e^(a x + b): p = a / ln2, q = b / ln2 in Eq. 5.
inline Affine exp_affine(double a, double b, int mode) {
  if (mode == QUAKE_EXACT) return {(float)(a / kLn2), (float)(b / kLn2)};
  const double beta = (mode == QUAKE_1) ? kSchraudolph : 0.0;
  return {(float)((a / kLn2) * kTwo23), (float)(((kBias - beta) + b / kLn2) * kTwo23)};
}

// Scale of the logistic argument in Eq. 7: 2 * 0.044715 * sqrt(2/pi).
inline double gelu_k() { return 2.0 * kGeluC * std::sqrt(2.0 / kPi); }

// 1/0.044715 + x^2 is one FMA with this addend (Eq. 7).
inline float gelu_a() { return (float)(1.0 / kGeluC); }

// e^(-k w) for w = x (1/0.044715 + x^2): Eq. 5 with p = -k.
inline Affine gelu_affine(int mode) { return exp_affine(-gelu_k(), 0.0, mode); }

// e^(-x) of the logistic function: Eq. 5 with p = -1.
inline Affine sigmoid_affine(int mode) { return exp_affine(-1.0, 0.0, mode); }

// Algorithm 2: c0 = 2^23 t / ln2 (EXACT: t / ln2); c1 is per row on the GPU.
inline float softmax_c0(double t, int mode) {
  if (mode == QUAKE_EXACT) return (float)(t / kLn2);
  return (float)((t / kLn2) * kTwo23);
}

inline bool valid_dtype(int d) { return d == QUAKE_F32 || d == QUAKE_F16 || d == QUAKE_BF16; }
inline bool valid_mode(int m) {
  return m == QUAKE_EXACT || m == QUAKE_1 || m == QUAKE_2 || m == QUAKE_2M;
}
inline int64_t elem_size(int d) { return d == QUAKE_F32 ? 4 : 2; }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Whether bytes [a, a + na) and [b, b + nb) meet (a null pointer has none).
inline bool meet(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a != nullptr && b != nullptr && na > 0 && nb > 0 && x < y + (uint64_t)nb && y < x + (uint64_t)na;
}
// Bytes from the first to behind the last of rows x cols elements, rows ld apart.
inline int64_t rows_bytes(int64_t rows, int64_t cols, int64_t ld, int64_t elem) {
  return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * elem : 0;
}

// Whether no row of a tensor with n <= 4 outer dimensions shares elements with another:
// in ascending order each stride reaches past what the smaller ones span. (Layouts that
// interleave otherwise without meeting are refused as well; no view of a larger tensor by
// slices and permutations is one.)
inline bool rows_apart(const int64_t* stride, const int64_t* count, int n, int64_t row) {
  int order[4] = {0, 1, 2, 3};
  std::sort(order, order + n, [&](int a, int b) { return stride[a] < stride[b]; });
  int64_t span = row;
  for (int k = 0; k < n; ++k) {
    const int i = order[k];
    if (count[i] <= 1) continue;
    if (stride[i] < span) return false;
    span += stride[i] * (count[i] - 1);
  }
  return true;
}
// Bytes from the first to behind the last of count[0] x .. x count[n - 1] rows of `row`
// elements of `elem` bytes.
inline int64_t span_bytes(const int64_t* stride, const int64_t* count, int n, int64_t row, int64_t elem) {
  int64_t last = row;
  for (int i = 0; i < n; ++i) {
    if (count[i] == 0) return 0;
    last += count[i] > 1 ? stride[i] * (count[i] - 1) : 0;
  }
  return last * elem;
}

inline quake_status launch_status() {
  return hipGetLastError() == hipSuccess ? QUAKE_OK : QUAKE_EHIP;
}

}  // namespace qk
