// sample.hip — quake_sample: the next token of each row of logits, with
// temperature, top-k, top-p and min-p, from one given random number per row.
//
// Weights are QuAKE's exponentials (arXiv:2412.00408) of (x - m) / temperature
// against the row max m: l = fma(x - m, c0, 127 2^23) (x = m gives exactly 1),
// then Eq. 3 and Eq. 2 / Algorithm 1. Every sum is over W = floor(w 2^40) in
// 64-bit integers (rows of up to 2^22 words stay below 2^62): integer sums are
// exact, so no split, order or atomic changes a token, and the masses of any part
// of a row can be added up by anyone.
//
// Words are ranked by (w descending, index ascending); each filter keeps a prefix
// of that ranking: the first k; those with less than p of the mass before them;
// those with at least min_p of the largest weight. The token is the first kept
// word, in the order of the vocabulary, at which the running mass exceeds u times
// the kept mass. A prefix is given by its last word, (weight, index), found by
// three rounds of a 1024-bin histogram over the weight's bits (counts for k,
// masses for p) and, among equal weights, by a search over the index.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "quake_device.hpp"
#include "quake_host.hpp"

namespace qk {

constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / 64;
constexpr int kBins = 1024;
constexpr uint32_t kOne = 0x3F800000u;   // bits of the weight 1

struct SampleArgs {
  const char* x;
  const float* u;
  const float *temperature, *top_p, *min_p;   // each or null
  const int32_t* top_k;                       // or null
  int32_t* token;
  float* prob;                                // or null
  int64_t ldx;
  uint32_t cols;
};

// A row's parameters, as the header states them for out-of-range values.
struct RowParams {
  float c0, c1;        // c1 = -inf (greedy): every word below the max weighs 0
  uint32_t k;          // words kept by top-k; cols: all
  uint32_t f_top, f_min, f_u;   // 24-bit fractions; f_top = 2^24: no top-p
};
template <int MODE>
__device__ __forceinline__ RowParams row_params(const SampleArgs& g, uint32_t row) {
  RowParams p;
  const float temp = g.temperature ? g.temperature[row] : 1.0f;
  const bool greedy = !(temp > 0.0f);
  const double c = (1.0 / (double)temp) / 0.693147180559945309417232121458176568;
  p.c0 = greedy ? 1.0f : (float)(MODE == EXACT ? c : c * 8388608.0);
  p.c1 = greedy ? -INFINITY : (MODE == EXACT ? 0.0f : kK127);
  const int32_t k = g.top_k ? g.top_k[row] : 0;
  p.k = greedy ? 1u : (k > 0 && (uint32_t)k < g.cols) ? (uint32_t)k : g.cols;
  auto fraction = [](float v) {   // NaN: 0
    return (uint32_t)((double)fminf(fmaxf(v, 0.0f), 1.0f) * 16777216.0);
  };
  const float tp = g.top_p ? g.top_p[row] : 1.0f;
  p.f_top = tp < 1.0f ? fraction(tp) : 1u << 24;
  p.f_min = g.min_p ? fraction(g.min_p[row]) : 0u;
  p.f_u = min(fraction(g.u[row]), (1u << 24) - 1u);
  return p;
}

// NaN counts as -inf: never drawn
__device__ __forceinline__ float no_nan(float v) { return v == v ? v : -INFINITY; }

// bits of the weight of x (canonical) against the row max m
template <int MODE>
__device__ __forceinline__ uint32_t weight_bits(float x, float m, const RowParams& p) {
  const float l = __builtin_fmaf(x - m, p.c0, p.c1);
  const float w = MODE == EXACT ? __builtin_amdgcn_exp2f(l) : quake_of_l_below<MODE>(l);
  return x == m ? kOne : x == -INFINITY ? 0u : as_u(w);
}
// floor(w 2^40) from w's bits (w <= 1; subnormal and smaller than 2^-41: 0)
__device__ __forceinline__ uint64_t mass_of(uint32_t bits) {
  const uint32_t s = 127u - (bits >> 23);
  const uint64_t v = (uint64_t)((bits & kMantMask) | 0x800000u) << 17;
  return s < 64u ? v >> s : 0u;
}
// floor(f 2^-24 mass), f <= 2^24, mass < 2^62
__device__ __forceinline__ uint64_t times(uint32_t f, uint64_t mass) {
  return f * (mass >> 24) + ((f * (mass & 0xFFFFFFu)) >> 24);
}

__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int d) { return __shfl_up(v, d, 64); }
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {   // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = shfl_up64(v, d);
    if ((int)(threadIdx.x & 63u) >= d) v += o;
  }
  return v;
}

struct RowShared {
  uint64_t hist[kBins];
  uint64_t wave[kRowWaves];
  uint64_t pick_before;
  uint32_t pick_bin, found;
  float fwave[kRowWaves];
};

// Inclusive scan over the workgroup; `all` its total.
__device__ __forceinline__ uint64_t block_scan64(uint64_t v, RowShared& sh, uint64_t* all) {
  const int wave = threadIdx.x >> 6;
  v = wave_scan64(v);
  __syncthreads();
  if ((threadIdx.x & 63u) == 63u) sh.wave[wave] = v;
  __syncthreads();
  uint64_t before = 0, total = 0;
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) before += sh.wave[w];
    total += sh.wave[w];
  }
  *all = total;
  return v + before;
}
__device__ __forceinline__ uint64_t block_sum64(uint64_t v, RowShared& sh) {
  uint64_t all;
  block_scan64(v, sh, &all);
  return all;
}

// One row by the whole workgroup, any length, layout and parameters.
template <int DT, int MODE>
struct RowSampler {
  const char* x;
  uint32_t cols;
  float m;
  RowParams p;
  // words kept by the filters so far: weight above w_cut, or w_cut itself up to
  // index i_cut; mass at least m_cut
  uint32_t w_cut = 0, i_cut = 0xFFFFFFFFu;
  uint64_t m_cut = 1;

  __device__ __forceinline__ uint32_t bits(uint32_t i) const {
    return weight_bits<MODE>(no_nan(load1<DT>(x, i)), m, p);
  }
  __device__ __forceinline__ bool kept(uint32_t b, uint32_t i) const {
    return b > w_cut || (b == w_cut && i <= i_cut);
  }

  // First index at which the running sum of f exceeds `target` (f's total is
  // above it): every round cuts the range by the number of waves.
  template <typename F>
  __device__ uint32_t find(F f, uint64_t target, RowShared& sh) const {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t lo = 0, hi = cols;
    while (hi - lo > 64u) {
      const uint32_t seg = ((hi - lo + kRowWaves * 64u - 1u) / (kRowWaves * 64u)) * 64u;
      const uint32_t a = lo + wave * seg, z = min(a + seg, hi);
      uint64_t s = 0;
      for (uint32_t i = a + lane; i < z && i >= a; i += 64u) s += f(i);
      s = wave_scan64(s);
      __syncthreads();
      if (lane == 63u) sh.wave[wave] = s;
      __syncthreads();
      uint64_t before = 0;
      uint32_t w = 0;
      while (w + 1u < kRowWaves && before + sh.wave[w] <= target) before += sh.wave[w++];
      target -= before;
      lo += w * seg;
      hi = min(lo + seg, hi);
    }
    __syncthreads();
    if (wave == 0) {
      const uint32_t i = lo + lane;
      const uint64_t s = wave_scan64(i < hi ? f(i) : 0u);
      const uint64_t past = __ballot(s > target);
      if (lane == 0) sh.found = lo + (past ? (uint32_t)__builtin_ctzll(past) : hi - lo - 1u);
    }
    __syncthreads();
    return sh.found;
  }

  // The word at which the ranking's running sum (of masses, or of ones) reaches
  // `goal` >= 1: the last word of the prefix. Sets w_cut, i_cut.
  template <bool MASS>
  __device__ void cut_at(uint64_t goal, RowShared& sh) {
    uint32_t prefix = 0;
    uint64_t above = 0;
#pragma unroll 1
    for (int shift = 20; shift >= 0; shift -= 10) {
      __syncthreads();
      sh.hist[threadIdx.x] = 0;
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < cols; i += kRowThreads) {
        const uint32_t b = bits(i);
        if (!kept(b, i) || (shift < 20 && (b >> (shift + 10)) != prefix)) continue;
        atomicAdd((unsigned long long*)&sh.hist[(b >> shift) & (kBins - 1u)],
                  MASS ? mass_of(b) : 1ull);
      }
      __syncthreads();
      const uint32_t bin = kBins - 1u - threadIdx.x;   // heaviest first
      const uint64_t here = sh.hist[bin];
      uint64_t all;
      const uint64_t upto = above + block_scan64(here, sh, &all);
      if (upto >= goal && upto - here < goal) {
        sh.pick_bin = bin;
        sh.pick_before = upto - here;
      }
      __syncthreads();
      above = sh.pick_before;
      prefix = (prefix << 10) | sh.pick_bin;
    }
    const uint64_t each = MASS ? mass_of(prefix) : 1u;
    const uint64_t ties = (goal - above + each - 1u) / each;   // how many of weight w_cut
    const uint32_t w0 = w_cut, i0 = i_cut;
    w_cut = prefix;
    i_cut = find([&](uint32_t i) -> uint64_t {
      const uint32_t b = bits(i);
      return b == prefix && (b > w0 || i <= i0) ? 1u : 0u;
    }, ties - 1u, sh);
  }

  __device__ uint64_t kept_mass(RowShared& sh) const {
    uint64_t s = 0;
    for (uint32_t i = threadIdx.x; i < cols; i += kRowThreads) {
      const uint32_t b = bits(i);
      const uint64_t w = mass_of(b);
      if (kept(b, i) && w >= m_cut) s += w;
    }
    return block_sum64(s, sh);
  }
};

template <int DT, int MODE>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs g, uint32_t row0) {
  __shared__ RowShared sh;
  const uint32_t row = row0 + blockIdx.x;
  RowSampler<DT, MODE> r;
  r.x = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  r.cols = g.cols;
  r.p = row_params<MODE>(g, row);
  float m = -INFINITY;
  for (uint32_t i = threadIdx.x; i < g.cols; i += kRowThreads) m = fmaxf(m, no_nan(load1<DT>(r.x, i)));
  m = wave_max(m);
  if ((threadIdx.x & 63u) == 0) sh.fwave[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int w = 0; w < kRowWaves; ++w) m = fmaxf(m, sh.fwave[w]);
  r.m = m;
  if (m == -INFINITY) {   // no word is allowed
    if (threadIdx.x == 0) {
      g.token[row] = -1;
      if (g.prob) g.prob[row] = 0.0f;
    }
    return;
  }
  if (r.p.k < g.cols) r.template cut_at<false>(r.p.k, sh);
  if (r.p.f_top < (1u << 24)) {
    const uint64_t goal = times(r.p.f_top, r.kept_mass(sh));
    r.template cut_at<true>(goal > 0 ? goal : 1, sh);
  }
  const uint64_t least = times(r.p.f_min, 1ull << 40);
  r.m_cut = least > 0 ? least : 1;
  const uint64_t all = r.kept_mass(sh);
  const uint32_t i = r.find([&](uint32_t j) -> uint64_t {
    const uint32_t b = r.bits(j);
    const uint64_t w = mass_of(b);
    return r.kept(b, j) && w >= r.m_cut ? w : 0u;
  }, times(r.p.f_u, all), sh);
  if (threadIdx.x == 0) {
    g.token[row] = (int32_t)i;
    if (g.prob) g.prob[row] = (float)((double)mass_of(r.bits(i)) / (double)all);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kSampleMaxCols = 1 << 22;   // sums below 2^62

template <int DT>
static void launch_sample(int mode, dim3 grid, hipStream_t s, const SampleArgs& g, uint32_t row0) {
  const dim3 b(kRowThreads);
  switch (mode) {
    case QUAKE_EXACT: hipLaunchKernelGGL((sample_row_kernel<DT, EXACT>), grid, b, 0, s, g, row0); break;
    case QUAKE_1: hipLaunchKernelGGL((sample_row_kernel<DT, Q1>), grid, b, 0, s, g, row0); break;
    case QUAKE_2: hipLaunchKernelGGL((sample_row_kernel<DT, Q2>), grid, b, 0, s, g, row0); break;
    default: hipLaunchKernelGGL((sample_row_kernel<DT, Q2M>), grid, b, 0, s, g, row0); break;
  }
}

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_sample_workspace_size(int64_t rows, int64_t cols, int64_t* bytes) {
  if (bytes == nullptr || rows < 0 || cols < 0 || cols > kSampleMaxCols) return QUAKE_EINVAL;
  *bytes = 0;
  return QUAKE_OK;
}

extern "C" quake_status quake_sample(const void* x, const float* u, int32_t* token, float* prob,
                                     int64_t rows, int64_t cols, int64_t ldx,
                                     const float* temperature, const int32_t* top_k,
                                     const float* top_p, const float* min_p, quake_dtype dtype,
                                     quake_mode mode, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  if (!valid_dtype(dtype)) return QUAKE_EDTYPE;
  if (!valid_mode(mode)) return QUAKE_EMODE;
  if (rows < 0 || cols < 0 || cols > kSampleMaxCols || ldx < cols) return QUAKE_EINVAL;
  if (rows > INT32_MAX || ldx > INT64_MAX / 8 / (rows > 0 ? rows : 1)) return QUAKE_EINVAL;
  if (workspace_bytes < 0 || (workspace != nullptr && !aligned16(workspace))) return QUAKE_EINVAL;
  if (rows == 0) return QUAKE_OK;
  if (cols == 0 || x == nullptr || u == nullptr || token == nullptr) return QUAKE_EINVAL;
  const uintptr_t odd = (uintptr_t)u | (uintptr_t)token | (uintptr_t)prob |
                        (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p |
                        (uintptr_t)min_p;
  if ((odd & 3u) != 0 || ((uintptr_t)x & (uintptr_t)(elem_size(dtype) - 1)) != 0)
    return QUAKE_EINVAL;
  const SampleArgs g{static_cast<const char*>(x), u, temperature, top_p, min_p, top_k, token, prob,
                     ldx, (uint32_t)cols};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  constexpr int64_t kMost = 1 << 20;   // rows a launch: below 2^32 threads
  for (int64_t r = 0; r < rows; r += kMost) {
    const dim3 grid((uint32_t)std::min(kMost, rows - r));
    if (dtype == QUAKE_F32) launch_sample<F32>(mode, grid, s, g, (uint32_t)r);
    else if (dtype == QUAKE_F16) launch_sample<F16>(mode, grid, s, g, (uint32_t)r);
    else launch_sample<BF16>(mode, grid, s, g, (uint32_t)r);
    const quake_status st = launch_status();
    if (st != QUAKE_OK) return st;
  }
  return QUAKE_OK;
}
