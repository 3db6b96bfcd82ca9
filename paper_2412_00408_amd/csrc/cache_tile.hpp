// cache_tile.hpp — what the attention kernels over a key/value cache share: the
// matrix-core products S^T = K Q^T and O^T = V^T P on blocks of 32 keys x 32 rows,
// their operands in LDS, and a row's accumulators against a whole exponent M.
#pragma once

#include <hip/hip_runtime.h>

#include "quake_device.hpp"

namespace qk {

typedef __bf16 wbf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 wf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLazy = 8.0f;      // how far the running max may rise before M follows
// A largest probability is held at 2^kLift or below when M is set: binary16's steps end
// at 2^-24, and held against 1 keys of 2^-14 of the largest and less would lose digits,
// those below 2^-25 all of them (a sink over thousands of keys). 2^(kLift + kLazy) fits.
template <int DT>
constexpr float kLift = DT == F16 ? 7.0f : 0.0f;
constexpr float kNoMax = -1e30f;   // M of a row that has seen no key

template <int DT>
__device__ __forceinline__ f32x16 wmma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (DT == BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(wbf16x8_t, a),
                                                   __builtin_bit_cast(wbf16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(wf16x8_t, a),
                                                  __builtin_bit_cast(wf16x8_t, b), c, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ uint32_t wpack(float a, float b) {
  return DT == BF16 ? pack_bf16(a, b) : pack_f16(a, b);
}
// The loads of v done here: waited for at their first use, inside the loop, they would
// be waited for there every time, and with them the keys on their way to LDS.
template <int N>
__device__ __forceinline__ void settle(u32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}
// a + the sum of a pair, of its rounded values
template <int DT>
__device__ __forceinline__ float wsum(uint32_t pair, float a) {
  if constexpr (DT == BF16)
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair),
                                           bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, a, false);
  else
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, pair),
                                  f16x2_t{(_Float16)1.0f, (_Float16)1.0f}, a, false);
}
__device__ __forceinline__ float other_half(float v) {   // the value of lane l xor 32
  const auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
  return as_f((threadIdx.x & 32) ? r[0] : r[1]);
}

// Blocks of 32 keys in LDS, rows of D 16-bit elements in 16-byte chunks; chunk c
// of row r sits at chunk c ^ swizzle(r). K's operand reads take one chunk of 32
// consecutive rows, V's transposed reads 64 bytes of 8 consecutive rows: with
// these swizzles neither meets a bank twice beyond what its width costs.
template <int D>
__device__ __forceinline__ int kswizzle(int r) {
  return D == 128 ? (r & 15) : ((r & 7) ^ ((r >> 3) & 1));
}
template <int D>
__device__ __forceinline__ int vswizzle(int r) {
  return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
}

template <int D>
__device__ __forceinline__ u32x4 read_k(const char* blk, int fr, int h, int ks) {
  return *reinterpret_cast<const u32x4*>(blk + fr * (2 * D) + 16 * ((2 * ks + h) ^ kswizzle<D>(fr)));
}
// dims 32 db + lane mod 32, keys 16 ks + 8 u + 4 h + 0 .. 3, u = 0, 1
template <int D>
__device__ __forceinline__ u32x4 read_v(const char* blk, int lane, int ks, int db) {
  typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
  u32x2 p[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = 16 * ks + 8 * u + 4 * (lane >> 5) + ((lane >> 2) & 3);
    const int c = 4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    const char* a = blk + row * (2 * D) + 16 * (c ^ vswizzle<D>(row)) + 8 * (lane & 1);
    p[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)a));
  }
  return u32x4{p[0][0], p[0][1], p[1][0], p[1][1]};
}

// 2^(from - to), from <= to whole numbers, as an exponent
__device__ __forceinline__ int32_t down_shift(float from, float to) {
  return (int32_t)fmaxf(from - to, -1000.0f);
}

// What a row has accumulated: D / 32 blocks of O^T, this lane's part of the sum.
template <int D>
struct RowAcc {
  f32x16 o[D / 32];
  float sum, m;
};

// the larger of the row's scores in a block, in base-2 units
template <int MODE>
__device__ __forceinline__ float block_top(const f32x16& s, float c0) {
  float top = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
  return fmaxf(top, other_half(top)) * (c0 * (MODE == EXACT ? 1.0f : 0x1p-23f));
}
// M brought to kLift below `top` where that is more than kLazy further above it, and what
// is accumulated rescaled; returns the exponent it was rescaled by.
template <int DT, int D>
__device__ __forceinline__ int32_t raise_max(float top, RowAcc<D>& acc) {
  const float m = top > acc.m + (kLift<DT> + kLazy) ? __builtin_ceilf(top) - kLift<DT> : acc.m;
  const int32_t e = down_shift(acc.m, m);
  acc.m = m;
  acc.sum = __builtin_amdgcn_ldexpf(acc.sum, e);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc.o[d][r] = __builtin_amdgcn_ldexpf(acc.o[d][r], e);
  return e;
}
// a 16-bit pair times 2^e
template <int DT>
__device__ __forceinline__ uint32_t scale_pair(uint32_t p, int32_t e) {
  const float a = DT == BF16 ? bf16_lo(p) : f16_lo(p), b = DT == BF16 ? bf16_hi(p) : f16_hi(p);
  return wpack<DT>(__builtin_amdgcn_ldexpf(a, e), __builtin_amdgcn_ldexpf(b, e));
}
template <int MODE>
__device__ __forceinline__ float row_c1(float m) {
  return MODE == EXACT ? -m : (127.0f - m) * 0x1p23f;
}
// Scores r, r + 1 to a pair of probabilities, added to the sum as rounded: numerator
// and denominator then share the rounding.
template <int DT, int MODE>
__device__ __forceinline__ uint32_t prob_pair(const f32x16& s, int r, float c0, float c1, float& sum) {
  const uint32_t p = wpack<DT>(qexp_row<MODE, true>(s[r], c0, c1),
                               qexp_row<MODE, true>(s[r + 1], c0, c1));
  sum = wsum<DT>(p, sum);
  return p;
}

__device__ __forceinline__ int32_t seq_len(const int32_t* lens, int b, int32_t most) {
  return lens == nullptr ? most : min(max(lens[b], 0), most);
}

}  // namespace qk
