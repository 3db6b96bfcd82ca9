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
#include "row_vecs.hpp"

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
// (a 64-bit shift by the last register a wave has goes wrong on this GPU: the build
// refuses compiled code that has one)
__device__ __forceinline__ uint64_t mass_of(uint32_t bits) {
  const uint64_t v = (uint64_t)((bits & kMantMask) | 0x800000u) << 17;   // below 2^41
  return v >> min(127u - (bits >> 23), 63u);
}
// the least bits whose mass is at least m (m <= 2^40)
__device__ __forceinline__ uint32_t bits_from(uint64_t m) {
  const double w = (double)m * 0x1p-40;
  const float f = (float)w;
  return as_u(f) + ((double)f < w ? 1u : 0u);
}
// floor(f 2^-24 mass), f <= 2^24, mass < 2^62
__device__ __forceinline__ uint64_t times(uint32_t f, uint64_t mass) {
  return f * (mass >> 24) + ((f * (mass & 0xFFFFFFu)) >> 24);
}

// v of the lane that CTRL names, 0 where there is none
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t v) {
  return ((uint64_t)dpp_u32<CTRL, ROWS>(0u, (uint32_t)(v >> 32)) << 32) |
         dpp_u32<CTRL, ROWS>(0u, (uint32_t)v);
}
// Inclusive scan of a row of 16 lanes (row_shr:1, 2, 4, 8), then of the wave.
__device__ __forceinline__ uint64_t row_scan64(uint64_t v) {
  v += dpp_u64<0x111>(v);
  v += dpp_u64<0x112>(v);
  v += dpp_u64<0x114>(v);
  v += dpp_u64<0x118>(v);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {
  v = row_scan64(v);
  v += dpp_u64<kDppRowBcast15, 0xA>(v);
  v += dpp_u64<kDppRowBcast31, 0xC>(v);
  return v;
}
__device__ __forceinline__ uint64_t readlane64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

constexpr uint32_t kCap = 4096;          // candidates that a row's ranking holds
constexpr uint32_t kMaxSegs = 520;       // segments of a row with masses of their own
template <uint32_t CAP>
struct ListShared {
  uint64_t list[CAP];                    // candidates
  uint32_t count;
};
struct SampleShared : ListShared<kCap> {
  uint64_t hist[kBins];
  uint64_t wave[kRowWaves];
  uint64_t seg[kMaxSegs];
  uint64_t pick_before;
  uint32_t pick_bin, found;
  float fwave[kRowWaves];
  uint32_t cwave[2][kRowWaves];
};

// Inclusive scan over a workgroup of NW waves; `all` its total.
template <int NW>
__device__ __forceinline__ uint64_t block_scan64(uint64_t v, SampleShared& sh, uint64_t* all) {
  static_assert(NW <= 16, "a lane of a row each");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  v = wave_scan64(v);
  __syncthreads();
  if ((threadIdx.x & 63u) == 63u) sh.wave[wave] = v;
  __syncthreads();
  const uint32_t lane = threadIdx.x & 63u;
  const uint64_t sums = row_scan64(lane < NW ? sh.wave[lane] : 0u);
  *all = readlane64(sums, NW - 1);
  return v + (wave > 0 ? readlane64(sums, wave - 1) : 0u);
}
template <int NW>
__device__ __forceinline__ uint64_t block_sum64(uint64_t v, SampleShared& sh) {
  uint64_t all;
  block_scan64<NW>(v, sh, &all);
  return all;
}
template <int NW>
__device__ __forceinline__ float block_max(float v, SampleShared& sh) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) sh.fwave[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) v = fmaxf(v, sh.fwave[w]);
  return v;
}

// The bin, heaviest first, at which `above` plus the running sum of sh.hist
// reaches goal; `above` becomes the sum before it.
template <int NW>
__device__ __forceinline__ uint32_t pick_bin(uint64_t goal, uint64_t& above, SampleShared& sh) {
  constexpr int N = kBins / (64 * NW);
  __syncthreads();
  if (threadIdx.x == 0) {   // should nothing reach it
    sh.pick_bin = 0;
    sh.pick_before = above;
  }
  uint64_t here[N], sum = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) sum += here[j] = sh.hist[kBins - 1u - (threadIdx.x * N + j)];
  uint64_t all;
  uint64_t before = above + block_scan64<NW>(sum, sh, &all) - sum;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (before < goal && before + here[j] >= goal) {
      sh.pick_bin = kBins - 1u - (threadIdx.x * N + j);
      sh.pick_before = before;
    }
    before += here[j];
  }
  __syncthreads();
  above = sh.pick_before;
  return sh.pick_bin;
}
template <int NW>
__device__ __forceinline__ void clear_hist(SampleShared& sh) {
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < kBins; i += 64 * NW) sh.hist[i] = 0;
  __syncthreads();
}

// One row by the whole workgroup, any length, layout and parameters.
template <int DT, int MODE>
struct RowSampler {
  const char* x;
  uint32_t cols;
  float m;
  RowParams p;
  // words kept by the filters so far: weight above w_cut, or w_cut itself before
  // index i_cut; mass at least m_cut
  uint32_t w_cut = 0, i_cut = 0xFFFFFFFFu;
  uint64_t m_cut = 1;

  __device__ __forceinline__ uint32_t bits(uint32_t i) const {
    return weight_bits<MODE>(no_nan(load1<DT>(x, i)), m, p);
  }
  __device__ __forceinline__ bool kept(uint32_t b, uint32_t i) const {
    return b > w_cut || (b == w_cut && i < i_cut);
  }

  // First index of lo .. hi - 1 at which the running sum of f exceeds `target` (its
  // total does). Rounds cut the range by the number of waves until a lane holds
  // what is left, kOwn consecutive words.
  static constexpr uint32_t kOwn = 8;
  template <typename F>
  __device__ uint32_t find(F f, uint32_t lo, uint32_t hi, uint64_t target, SampleShared& sh) const {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    while (hi - lo > kOwn * kRowThreads) {
      const uint32_t seg = ((hi - lo + kRowThreads - 1u) / kRowThreads) * 64u;
      const uint32_t a = lo + wave * seg, z = min(a + seg, hi);
      uint64_t s = 0;
#pragma unroll 4
      for (uint32_t i = a + lane; i < z; i += 64u) s += f(i);
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
    if (threadIdx.x == 0) sh.found = lo;   // should nothing exceed it
    const uint32_t first = lo + threadIdx.x * kOwn;
    uint64_t w[kOwn], sum = 0, all;
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j) w[j] = f(min(first + j, hi - 1u));
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j) {
      if (first + j >= hi) w[j] = 0;
      sum += w[j];
    }
    uint64_t upto = block_scan64<kRowWaves>(sum, sh, &all) - sum;
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j) {
      if (upto <= target && upto + w[j] > target) sh.found = first + j;
      upto += w[j];
    }
    __syncthreads();
    return sh.found;
  }

  // The word at which the ranking's running sum (of masses, or of ones) reaches
  // `goal` >= 1: the last word of the prefix. Sets
  // w_cut, i_cut.
  template <bool MASS>
  __device__ void cut_at(uint64_t goal, SampleShared& sh) {
    uint32_t prefix = 0;
    uint64_t above = 0;
#pragma unroll 1
    for (int shift = 20; shift >= 0; shift -= 10) {
      clear_hist<kRowWaves>(sh);
      for (uint32_t i = threadIdx.x; i < cols; i += kRowThreads) {
        const uint32_t b = bits(i);
        if (!kept(b, i) || (shift < 20 && (b >> (shift + 10)) != prefix)) continue;
        atomicAdd((unsigned long long*)&sh.hist[(b >> shift) & (kBins - 1u)],
                  MASS ? mass_of(b) : 1ull);
      }
      prefix = (prefix << 10) | pick_bin<kRowWaves>(goal, above, sh);
    }
    const uint64_t each = MASS ? mass_of(prefix) : 1u;
    const uint64_t ties = (goal - above + each - 1u) / each;   // how many of weight w_cut
    const uint32_t w0 = w_cut, i0 = i_cut;
    w_cut = prefix;
    i_cut = 1u + find([&](uint32_t i) -> uint64_t {
      const uint32_t b = bits(i);
      return b == prefix && (b > w0 || i < i0) ? 1u : 0u;
    }, 0, cols, ties - 1u, sh);
  }

  __device__ uint64_t kept_mass(SampleShared& sh) const {
    uint64_t s = 0;
    for (uint32_t i = threadIdx.x; i < cols; i += kRowThreads) {
      const uint32_t b = bits(i);
      const uint64_t w = mass_of(b);
      if (kept(b, i) && w >= m_cut) s += w;
    }
    return block_sum64<kRowWaves>(s, sh);
  }
};

// The row by three rounds of histograms per filter, whatever its parameters.
template <int DT, int MODE>
__device__ __forceinline__ void sample_any(const SampleArgs& g, uint32_t row, float m,
                                        const RowParams& p, SampleShared& sh) {
  RowSampler<DT, MODE> r;
  r.x = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  r.cols = g.cols;
  r.p = p;
  r.m = m;
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
  }, 0, g.cols, times(r.p.f_u, all), sh);
  if (threadIdx.x == 0) {
    g.token[row] = (int32_t)i;
    if (g.prob) g.prob[row] = (float)((double)mass_of(r.bits(i)) / (double)all);
  }
}

// ---------------------------------------------------------------------------
// The usual rows, in passes over the logits that keep little of them.
//   top-k   A lower bound of the k-th largest logit is the k-th largest of the lanes'
//           maxima (at least k words are as large); words not below it, nor within
//           the slack below it in which two words may weigh the same, are the
//           candidates, a little more than k. They are ranked in LDS.
//   top-p   Masses by bins of the weight (16 to the octave) give the bin in which the
//           running mass reaches p Z; words above it are kept, and only those in it
//           are ranked. Words lighter than (1 - p) 2^40 / cols weigh together less
//           than (1 - p) of the max alone: they enter Z, but no bin.
//   else    Words of at least min_p are kept, unranked.
// The kept mass of each segment of the row (top-p, else) leads to the segment that
// holds the token, which alone is read again.
// ---------------------------------------------------------------------------
enum RowKind : uint32_t { kNone, kTopK, kTopP, kPlain, kAny };
// known before the max
__device__ __forceinline__ RowKind row_kind(const RowParams& p, uint32_t cols) {
  const bool greedy = p.c1 == -INFINITY;
  if (!(p.c0 < INFINITY) || !(p.c0 >= 0x1p-60f)) return kAny;
  if (p.k < cols) return kTopK;
  if (greedy) return kAny;   // one word
  return p.f_top < (1u << 24) ? kTopP : kPlain;
}
__device__ __forceinline__ RowKind row_kind(const RowParams& p, uint32_t cols, float m) {
  return m == -INFINITY ? kNone : m < INFINITY ? row_kind(p, cols) : kAny;
}

// Vectors [begin(s), begin(s + 1)) of a row are segment s of nseg.
__device__ __forceinline__ uint32_t seg_begin(uint32_t n, uint32_t s, uint32_t nseg) {
  return (uint32_t)((uint64_t)n * s / nseg);
}
// the segment that holds a vector
__device__ __forceinline__ uint32_t seg_of(uint32_t n, uint32_t vec, uint32_t nseg) {
  return (uint32_t)(((uint64_t)(vec + 1u) * nseg - 1u) / n);
}

// f(vector index, elements) for vectors [a, z) by NW waves, each by one lane; elements
// outside the row are -inf (the row's first and last vector are masked, no others).
template <int NW, int U, int DT, typename F>
__device__ __forceinline__ void each_vector(const RowVecs<DT>& r, uint32_t a, uint32_t z, F f) {
  constexpr uint32_t V = kV<DT>, T = 64 * NW;
  const uint32_t t = threadIdx.x & (T - 1u), in = min(z, r.n - 1u);
  uint32_t i = max(a, 1u) + t;
  for (; i + (U - 1) * T < in; i += U * T) {
    u32x4 w[U];
#pragma unroll
    for (uint32_t j = 0; j < U; ++j) w[j] = r.v[i + T * j];
#pragma unroll
    for (uint32_t j = 0; j < U; ++j) {
      float v[V];
      unpack<DT>(w[j], v);
      f(i + T * j, v);
    }
  }
  if (i < in) {
    u32x4 w[U];
#pragma unroll
    for (uint32_t j = 0; j < U; ++j) w[j] = r.v[min(i + T * j, in - 1u)];
#pragma unroll
    for (uint32_t j = 0; j < U; ++j) {
      if (i + T * j < in) {
        float v[V];
        unpack<DT>(w[j], v);
        f(i + T * j, v);
      }
    }
  }
  const bool head = a == 0 && z > 0 && t == 0, tail = a < z && z == r.n && r.n > 1u && t == T - 1u;
  if (head || tail) {
    const uint32_t e = head ? 0u : r.n - 1u;
    float v[V];
    unpack<DT>(r.v[e], v);
    r.mask(e, v);
    f(e, v);
  }
}

// A value that at least k of the workgroup's values reach and few more do: bisection
// between their least and largest, counting by ballots. -inf where fewer are above it.
template <int NW, int N>
__device__ __forceinline__ float kth_bound(const float (&v)[N], uint32_t k, SampleShared& sh) {
  const int wave = threadIdx.x >> 6;
  int parity = 0;
  auto count = [&](float x) {
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) c += (uint32_t)__popcll(__ballot(v[j] >= x));
    if ((threadIdx.x & 63u) == 0) sh.cwave[parity][wave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) c += sh.cwave[parity][w];
    parity ^= 1;
    return c;
  };
  float lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (v[j] > -INFINITY) lo = fminf(lo, v[j]);
    hi = fmaxf(hi, v[j]);
  }
  hi = block_max<NW>(hi, sh);
  lo = -block_max<NW>(-lo, sh);
  if (!(lo <= hi) || count(lo) < k) return -INFINITY;
  for (int i = 0; i < 24; ++i) {
    const float mid = 0.5f * lo + 0.5f * hi;
    const uint32_t c = count(mid);
    if (c >= k) {
      lo = mid;
      if (c <= k + k / 8u + 4u) break;
    } else {
      hi = mid;
    }
  }
  return lo;
}

// How far below a word another may lie and weigh the same (while W > 0, that is
// within 41 base-2 units of the max): one step of l (64 units of 2^23; the exact
// exponential's few last bits), and the rounding of both differences to the max,
// 41 * 2^-23 units each.
template <int MODE>
__device__ __forceinline__ float slack(const RowParams& p) {
  return p.c1 == -INFINITY ? 0.0f : (MODE == EXACT ? 0x1p-16f : 256.0f) / p.c0;
}

// candidates: of top-k the logit's bits, of top-p a key that ranks ascending
__device__ __forceinline__ uint64_t pair64(uint32_t hi, uint32_t lo) {
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t rank_key(uint32_t bits, uint32_t i) { return pair64(~bits, i); }
template <uint32_t CAP>
__device__ __forceinline__ void add_candidate(uint64_t c, ListShared<CAP>& sh) {
  const uint32_t n = atomicAdd(&sh.count, 1u);   // counted past the list's end, too
  if (n < CAP) sh.list[n] = c;
}

// Words of a vector from `above` on.
template <int DT, uint32_t CAP>
__device__ __forceinline__ void add_above(const float* f, uint32_t e, float above,
                                          ListShared<CAP>& sh) {
  float top = f[0];
#pragma unroll
  for (int k = 1; k < kV<DT>; ++k) top = fmaxf(top, f[k]);
  if (!(top >= above) || top == -INFINITY) return;
#pragma unroll
  for (int k = 0; k < kV<DT>; ++k)
    if (f[k] >= above && f[k] > -INFINITY) add_candidate(pair64(as_u(f[k]), e + k), sh);
}

// A logit's weight where the row is neither greedy nor holds +inf (x - m = 0 gives
// l = 127 2^23, weight 1, by itself).
template <int MODE>
__device__ __forceinline__ uint32_t usual_bits(float x, float m, const RowParams& p) {
  const float l = __builtin_fmaf(x - m, p.c0, p.c1);
  return as_u(MODE == EXACT ? __builtin_amdgcn_exp2f(l) : quake_of_l_below<MODE>(l));
}

// Mass of at least `least` in vectors [a, z), this lane's.
template <int DT, int MODE, int NW, int U>
__device__ __forceinline__ uint64_t plain_mass(const RowVecs<DT>& r, uint32_t a, uint32_t z, float m,
                                               const RowParams& p, uint64_t least) {
  const uint32_t from = bits_from(least);
  uint64_t mass = 0;
  each_vector<NW, U>(r, a, z, [&](uint32_t, const float* f) {
#pragma unroll
    for (int k = 0; k < kV<DT>; ++k) {
      const uint32_t b = usual_bits<MODE>(f[k], m, p);
      mass += mass_of(b >= from ? b : 0u);
    }
  });
  return mass;
}
__device__ __forceinline__ uint64_t least_kept(const RowParams& p) {
  return max(times(p.f_min, 1ull << 40), (uint64_t)1);
}

// Bins of the weight: 16 to the octave, heaviest (weight 1) first, down to 2^-40 (W = 1,
// bin 640); sh.hist holds them from its end on, as pick_bin reads it.
constexpr uint32_t kWeightBins = 641;
__device__ __forceinline__ uint32_t weight_bin(uint32_t bits) { return (kOne - bits) >> 19; }
__device__ __forceinline__ uint32_t bin_top(uint32_t bin) { return kOne - (bin << 19); }

// Adds vectors [a, z) to the bins; returns this lane's mass of the words in none.
template <int DT, int MODE, int NW, int U>
__device__ __forceinline__ uint64_t bin_masses(const RowVecs<DT>& r, uint32_t a, uint32_t z, float m,
                                               const RowParams& p, SampleShared& sh) {
  const uint32_t from =
      bits_from(max(((uint64_t)((1u << 24) - p.f_top) << 16) / r.cols, (uint64_t)1));
  uint64_t light = 0;
  each_vector<NW, U>(r, a, z, [&](uint32_t, const float* f) {
#pragma unroll
    for (int k = 0; k < kV<DT>; ++k) {
      const uint32_t b = usual_bits<MODE>(f[k], m, p);
      const uint64_t w = mass_of(b);
      const bool in = b >= from && b <= kOne;   // (NaN: above 1)
      if (in)
        atomicAdd((unsigned long long*)&sh.hist[kBins - 1u - weight_bin(b)], (unsigned long long)w);
      light += in ? 0u : w;
    }
  });
  return light;
}

// Where the ranking is cut: the bin, the mass above it, and the mass to reach.
struct Cut {
  uint32_t bin;
  uint64_t above, goal;
};
// from sh.hist and the mass in no bin
template <int NW>
__device__ __forceinline__ Cut pick_cut(uint64_t light, const RowParams& p, SampleShared& sh) {
  __syncthreads();
  uint64_t z = 0;
  for (uint32_t i = threadIdx.x; i < kBins; i += 64 * NW) z += sh.hist[i];
  z = block_sum64<NW>(z, sh) + light;
  Cut c{0, 0, max(times(p.f_top, z), (uint64_t)1)};
  c.bin = kBins - 1u - pick_bin<NW>(c.goal, c.above, sh);
  return c;
}

// The words above the cut bin, [a, z): this lane's kept mass; those in it: candidates.
template <int DT, int MODE, int NW, int U>
__device__ __forceinline__ uint64_t cut_mass(const RowVecs<DT>& r, uint32_t a, uint32_t z, float m,
                                             const RowParams& p, const Cut& c, SampleShared& sh) {
  const uint32_t top = bin_top(c.bin), next = bin_top(c.bin + 1u);
  const uint32_t from = bits_from(least_kept(p));
  uint64_t mass = 0;
  each_vector<NW, U>(r, a, z, [&](uint32_t i, const float* f) {
#pragma unroll
    for (int k = 0; k < kV<DT>; ++k) {
      const uint32_t b = usual_bits<MODE>(f[k], m, p);
      if (b <= next || b > kOne) continue;   // below the bin (NaN: above 1)
      if (b > top) {
        mass += mass_of(b >= from ? b : 0u);
      } else {
        add_candidate(rank_key(b, i * kV<DT> + k - r.skip), sh);
      }
    }
  });
  return mass;
}

// Ascending sort of the first n entries of sh.list (n <= kCap) by NW waves. Strides up
// to 64 stay inside the 128 entries that a wave's lanes hold, where LDS operations
// complete in order.
template <int NW>
__device__ __forceinline__ void sort_list(uint32_t n, SampleShared& sh) {
  uint32_t size = 2;
  while (size < n) size <<= 1;
  for (uint32_t i = n + threadIdx.x; i < size; i += 64 * NW) sh.list[i] = ~0ull;
  __syncthreads();
  for (uint32_t k = 2; k <= size; k <<= 1) {
    for (uint32_t j = k >> 1; j > 0; j >>= 1) {
      for (uint32_t t = threadIdx.x; t < size / 2; t += 64 * NW) {
        const uint32_t i = 2 * t - (t & (j - 1)), o = i + j;
        const uint64_t a = sh.list[i], b = sh.list[o];
        if ((a > b) == ((i & k) == 0)) {
          sh.list[i] = b;
          sh.list[o] = a;
        }
      }
      if (j > 64 || (j == 1 && k >= 64))
        __syncthreads();   // the next stride, or the next k's first, crosses waves
      else
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
  __syncthreads();
}

// The n candidates of sh.list, in ranking order.
__device__ __forceinline__ void rank_list(uint32_t n, SampleShared& sh) {
  if (n > 128u) {
    sort_list<kRowWaves>(n, sh);
    return;
  }
  // each entry's place by counting, eight lanes an entry
  const uint32_t i = threadIdx.x >> 3;
  __syncthreads();
  const uint64_t mine = i < n ? sh.list[i] : 0u;
  uint32_t rank = 0;
  for (uint32_t j = threadIdx.x & 7u; j < n; j += 8) rank += sh.list[j] < mine ? 1u : 0u;
  rank += dpp_u32<kDppXor1>(0u, rank);
  rank += dpp_u32<kDppXor2>(0u, rank);
  rank += dpp_u32<kDppHalfMirror>(0u, rank);
  __syncthreads();
  if ((threadIdx.x & 7u) == 0 && i < n) sh.list[rank] = mine;
  __syncthreads();
}

constexpr uint32_t kListN = kCap / kRowThreads;   // consecutive entries of a thread

// How many of the n ranked candidates are kept, with `above` ranked before them all;
// *mass: theirs together.
__device__ __forceinline__ uint32_t keep_prefix(uint32_t n, uint64_t above, uint64_t goal,
                                                const RowParams& p, uint64_t* mass,
                                                SampleShared& sh) {
  const uint64_t least = least_kept(p);
  const uint32_t t0 = threadIdx.x * kListN;
  uint64_t w[kListN], sum = 0;
#pragma unroll
  for (uint32_t j = 0; j < kListN; ++j)
    sum += w[j] = t0 + j < n ? mass_of(~(uint32_t)(sh.list[t0 + j] >> 32)) : 0u;
  uint64_t all;
  uint64_t before = above + block_scan64<kRowWaves>(sum, sh, &all) - sum;
  if (goal == 0) goal = max(times(p.f_top, all), (uint64_t)1);   // of these words alone
  uint32_t kept = 0;
  sum = 0;
#pragma unroll
  for (uint32_t j = 0; j < kListN; ++j) {
    if (before < goal && w[j] >= least) {
      ++kept;
      sum += w[j];
    }
    before += w[j];
  }
  *mass = block_sum64<kRowWaves>(sum, sh);
  return (uint32_t)block_sum64<kRowWaves>(kept, sh);
}

__device__ __forceinline__ void write_row(const SampleArgs& g, uint32_t row, uint32_t token,
                                          uint64_t w, uint64_t all) {
  g.token[row] = (int32_t)token;
  if (g.prob) g.prob[row] = (float)((double)w / (double)all);
}

// The token of a row whose top-k candidates, n of them, are in sh.list.
__device__ __forceinline__ void finish_top_k(const SampleArgs& g, uint32_t row, uint32_t n,
                                             const RowParams& p, SampleShared& sh) {
  rank_list(n, sh);
  uint64_t all;
  const uint32_t kept = keep_prefix(min(n, p.k), 0, p.f_top < (1u << 24) ? 0u : ~0ull, p, &all, sh);
  const uint64_t target = times(p.f_u, all);
  const uint32_t t0 = threadIdx.x * kListN;
#pragma unroll
  for (uint32_t j = 0; j < kListN; ++j) {   // by index
    if (t0 + j < kept) {
      const uint64_t e = sh.list[t0 + j];
      sh.list[t0 + j] = pair64((uint32_t)e, ~(uint32_t)(e >> 32));
    }
  }
  __syncthreads();
  rank_list(kept, sh);
  uint64_t w[kListN], sum = 0, unused;
#pragma unroll
  for (uint32_t j = 0; j < kListN; ++j)
    sum += w[j] = t0 + j < kept ? mass_of((uint32_t)sh.list[t0 + j]) : 0u;
  uint64_t upto = block_scan64<kRowWaves>(sum, sh, &unused) - sum;
#pragma unroll
  for (uint32_t j = 0; j < kListN; ++j) {
    if (upto <= target && upto + w[j] > target)
      write_row(g, row, (uint32_t)(sh.list[t0 + j] >> 32), w[j], all);
    upto += w[j];
  }
}

// The token of a row from the kept masses of its nseg segments in sh.seg and r's cuts.
template <int DT, int MODE>
__device__ __forceinline__ void finish_segments(const SampleArgs& g, uint32_t row,
                                                const RowVecs<DT>& v, uint32_t nseg,
                                                const RowSampler<DT, MODE>& r, SampleShared& sh) {
  static_assert(kMaxSegs <= (uint32_t)kRowThreads, "a segment a thread");
  __syncthreads();
  uint64_t all;
  const uint64_t here = threadIdx.x < nseg ? sh.seg[threadIdx.x] : 0u;
  const uint64_t upto = block_scan64<kRowWaves>(here, sh, &all);
  const uint64_t target = times(r.p.f_u, all);
  if (threadIdx.x == 0) {
    sh.pick_bin = 0;
    sh.pick_before = 0;
  }
  __syncthreads();
  if (upto - here <= target && upto > target) {
    sh.pick_bin = threadIdx.x;
    sh.pick_before = upto - here;
  }
  __syncthreads();
  const uint32_t s = sh.pick_bin;
  auto element = [&](uint32_t vec) {
    const uint32_t e = vec * kV<DT>;
    return e < v.skip ? 0u : min(e - v.skip, g.cols);
  };
  const uint32_t i = r.find([&](uint32_t j) -> uint64_t {
    const uint32_t b = r.bits(j);
    const uint64_t w = mass_of(b);
    return r.kept(b, j) && w >= r.m_cut ? w : 0u;
  }, element(seg_begin(v.n, s, nseg)), element(seg_begin(v.n, s + 1, nseg)),
  target - sh.pick_before, sh);
  if (threadIdx.x == 0) write_row(g, row, i, mass_of(r.bits(i)), all);
}

// The same of a top-p row: n candidates of the cut bin in sh.list.
template <int DT, int MODE>
__device__ __forceinline__ void finish_top_p(const SampleArgs& g, uint32_t row,
                                             const RowVecs<DT>& v, uint32_t nseg, uint32_t n,
                                             const Cut& c, RowSampler<DT, MODE>& r,
                                             SampleShared& sh) {
  rank_list(n, sh);
  uint64_t unused;
  const uint32_t kept = keep_prefix(n, c.above, c.goal, r.p, &unused, sh);
  r.m_cut = least_kept(r.p);
  r.w_cut = bin_top(c.bin);
  r.i_cut = 0;
  if (kept > 0) {
    const uint64_t e = sh.list[kept - 1u];
    r.w_cut = ~(uint32_t)(e >> 32);
    r.i_cut = (uint32_t)e + 1u;
  }
  for (uint32_t i = threadIdx.x; i < kept; i += kRowThreads) {
    const uint64_t e = sh.list[i];
    atomicAdd((unsigned long long*)&sh.seg[seg_of(v.n, ((uint32_t)e + v.skip) / kV<DT>, nseg)],
              (unsigned long long)mass_of(~(uint32_t)(e >> 32)));
  }
  finish_segments<DT, MODE>(g, row, v, nseg, r, sh);
}

__device__ __forceinline__ void write_none(const SampleArgs& g, uint32_t row) {
  if (threadIdx.x == 0) {
    g.token[row] = -1;
    if (g.prob) g.prob[row] = 0.0f;
  }
}

// The n top-k candidates in sh.list (logit bits and index) to ranking keys, after a
// bound of the k-th largest among them where they are many; returns how many are left.
template <int MODE, int N>
__device__ __forceinline__ uint32_t weigh_some(uint32_t n, float m, const RowParams& p,
                                               SampleShared& sh) {
  uint64_t e[N];
  float v[N], above = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t i = threadIdx.x + j * kRowThreads;
    e[j] = i < n ? sh.list[i] : 0u;
    v[j] = i < n ? as_f((uint32_t)(e[j] >> 32)) : -INFINITY;
  }
  if (n > 128u) above = kth_bound<kRowWaves>(v, p.k, sh) - slack<MODE>(p);
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (v[j] >= above && v[j] > -INFINITY)
      add_candidate(rank_key(weight_bits<MODE>(v[j], m, p), (uint32_t)e[j]), sh);
  __syncthreads();
  return sh.count;
}
template <int MODE>
__device__ __forceinline__ uint32_t weigh_list(uint32_t n, float m, const RowParams& p,
                                               SampleShared& sh) {
  return n <= (uint32_t)kRowThreads ? weigh_some<MODE, 1>(n, m, p, sh)
                                    : weigh_some<MODE, kCap / kRowThreads>(n, m, p, sh);
}

// One workgroup per row: every pass after the first finds most of the row in L2 (1.05 to
// 1.2 readings past it by the counters). 64 x 128256 binary32 with a top-k 21.6 to 23 us
// (1.4 TB/s), bound by one compute unit's loads; 256 x 50257 bf16 with a top-p 26 us at
// temperature 1 and 0.9, 36 us with both drawn row by row, bound by its VALU (67
// instructions a word in three passes). Rows that overflow the candidates take longer
// (64 x 128256 binary32, top-k 500 49 us, 900 200 us, 1100 and more 290 us; a top-p of 0.9
// over logits of standard deviation 3, 0.5, 0.05 and 0 67, 300, 440 and 660 us; a top-k
// over words masked by the type's lowest value, where fewer lanes than k hold others, 360
// to 510 us, by -inf 20 us).
template <int DT, int MODE>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(4, 4)))
void sample_row_kernel(SampleArgs g, uint32_t row0) {
  __shared__ SampleShared sh;
  constexpr int U = kV<DT> == 4 ? 4 : 2;   // vectors in flight: no more registers than there are
  const uint32_t row = row0 + blockIdx.x;
  const RowVecs<DT> v(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  RowSampler<DT, MODE> r;
  r.x = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  r.cols = g.cols;
  r.p = row_params<MODE>(g, row);
  float top[1] = {-INFINITY};
  each_vector<kRowWaves, 8>(v, 0, v.n, [&](uint32_t, const float* f) {
#pragma unroll
    for (int k = 0; k < kV<DT>; ++k) top[0] = fmaxf(top[0], f[k]);
  });
  const float m = r.m = block_max<kRowWaves>(top[0], sh);
  const RowKind kind = row_kind(r.p, g.cols, m);
  if (kind == kNone) {
    write_none(g, row);
    return;
  }
  if (threadIdx.x == 0) sh.count = 0;
  // the waves' segments
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t a = seg_begin(v.n, wave, kRowWaves), z = seg_begin(v.n, wave + 1, kRowWaves);
  if (kind == kTopK) {
    const float above = kth_bound<kRowWaves>(top, r.p.k, sh) - slack<MODE>(r.p);
    __syncthreads();
    each_vector<kRowWaves, 8>(v, 0, v.n, [&](uint32_t i, const float* f) {
      add_above<DT>(f, i * kV<DT> - v.skip, above, sh);
    });
    __syncthreads();
    const uint32_t n = sh.count;
    if (n <= kCap) {
      finish_top_k(g, row, weigh_list<MODE>(n, m, r.p, sh), r.p, sh);
      return;
    }
  } else if (kind == kTopP) {
    clear_hist<kRowWaves>(sh);
    const uint64_t light = block_sum64<kRowWaves>(
        bin_masses<DT, MODE, kRowWaves, U>(v, 0, v.n, m, r.p, sh), sh);
    const Cut c = pick_cut<kRowWaves>(light, r.p, sh);
    const uint64_t mass = wave_scan64(cut_mass<DT, MODE, 1, U>(v, a, z, m, r.p, c, sh));
    if ((threadIdx.x & 63u) == 63u) sh.seg[wave] = mass;
    __syncthreads();
    const uint32_t n = sh.count;
    if (n <= kCap) {
      finish_top_p<DT, MODE>(g, row, v, kRowWaves, n, c, r, sh);
      return;
    }
  } else if (kind == kPlain) {
    r.m_cut = least_kept(r.p);
    const uint64_t mass = wave_scan64(plain_mass<DT, MODE, 1, U>(v, a, z, m, r.p, r.m_cut));
    if ((threadIdx.x & 63u) == 63u) sh.seg[wave] = mass;
    finish_segments<DT, MODE>(g, row, v, kRowWaves, r, sh);
    return;
  }
  sample_any<DT, MODE>(g, row, m, r.p, sh);
}

// ---------------------------------------------------------------------------
// Few long rows without a top-k: the passes by several workgroups per row (one would
// be bound by one compute unit's loads and arithmetic), a launch each, the rest by one.
//   scan    each part's max; greedy rows: its first word
//   mass    top-p rows: the bins; unranked rows: the parts' kept masses
//   cut     top-p rows: the cut bin's candidates and the parts' kept masses
//   finish  the token
// (With a top-k this form had a launch that did nothing for such rows, and one workgroup
// a row was faster at every size: two passes of a compare a word and one launch, 22
// against 26 us for 64 x 128256 binary32.)
// ---------------------------------------------------------------------------
constexpr int kPartThreads = 256, kPartWaves = 4;
constexpr uint32_t kWsCap = 16384;       // candidates of a row in the workspace

// Workspace of a row: bins, candidates (each part has its share of the places), the
// parts' masses, masses kept, maxima and counts of candidates (greedy rows: the first
// word of the part's max). Every word that a launch reads, an earlier one of the same
// call has written.
struct SampleWs {
  char* base;
  int64_t stride;
  uint32_t parts;
  __device__ __forceinline__ uint64_t* hist(uint32_t row) const {
    return reinterpret_cast<uint64_t*>(base + row * stride);
  }
  __device__ __forceinline__ uint64_t* list(uint32_t row) const { return hist(row) + kWeightBins; }
  __device__ __forceinline__ uint64_t* mass(uint32_t row) const { return list(row) + kWsCap; }
  __device__ __forceinline__ uint64_t* kept(uint32_t row) const { return mass(row) + parts; }
  __device__ __forceinline__ float* maxima(uint32_t row) const {
    return reinterpret_cast<float*>(kept(row) + parts);
  }
  __device__ __forceinline__ uint32_t* count(uint32_t row) const {
    return reinterpret_cast<uint32_t*>(maxima(row) + parts);
  }
  __device__ __forceinline__ uint32_t share() const { return kWsCap / parts; }
};
// a part's candidates from sh.list to its places
template <uint32_t CAP>
__device__ __forceinline__ void flush_list(const SampleWs& ws, uint32_t row, uint32_t part,
                                           ListShared<CAP>& sh) {
  __syncthreads();
  const uint32_t n = sh.count, share = ws.share();
  if (threadIdx.x == 0) ws.count(row)[part] = n > CAP ? share + 1u : n;   // more: not all there
  for (uint32_t i = threadIdx.x; i < min(min(n, CAP), share); i += kPartThreads)
    ws.list(row)[part * share + i] = sh.list[i];
}
// The candidates of a row to sh.list; returns how many there are, above kCap where
// they are not all there.
__device__ __forceinline__ uint32_t fetch_list(const SampleWs& ws, uint32_t row, SampleShared& sh) {
  static_assert(kMaxSegs <= (uint32_t)kRowThreads, "a part a thread");
  const uint32_t share = ws.share();
  const uint32_t c = threadIdx.x < ws.parts ? ws.count(row)[threadIdx.x] : 0u;
  uint64_t all;
  const uint64_t upto = block_scan64<kRowWaves>(c <= share ? c : kCap + 1u, sh, &all);
  if (all > kCap) return kCap + 1u;
  if (threadIdx.x < ws.parts) sh.seg[threadIdx.x] = pair64((uint32_t)upto - c, c);
  __syncthreads();
  for (uint32_t part = threadIdx.x >> 6; part < ws.parts; part += kRowWaves) {
    const uint32_t at = (uint32_t)(sh.seg[part] >> 32), n = (uint32_t)sh.seg[part];
    for (uint32_t i = threadIdx.x & 63u; i < n; i += 64u)
      sh.list[at + i] = ws.list(row)[part * share + i];
  }
  __syncthreads();
  return (uint32_t)all;
}

// a greedy row of a call without a top-k
__device__ __forceinline__ bool is_greedy(const SampleArgs& g, uint32_t row) {
  return g.temperature != nullptr && !(g.temperature[row] > 0.0f);
}

template <int DT>
__global__ __launch_bounds__(kPartThreads) void sample_scan_kernel(SampleArgs g, SampleWs ws) {
  __shared__ float s_top[kPartWaves];
  __shared__ uint32_t s_first;
  constexpr int V = kV<DT>, N = 8192 / (V * kPartThreads);
  const uint32_t row = blockIdx.x / ws.parts, part = blockIdx.x % ws.parts;
  const RowVecs<DT> v(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const uint32_t a = seg_begin(v.n, part, ws.parts), z = seg_begin(v.n, part + 1, ws.parts);
  u32x4 w[N];   // the part, in registers
#pragma unroll
  for (int j = 0; j < N; ++j) w[j] = v.v[min(a + threadIdx.x + j * kPartThreads, z - 1u)];
  if (part == 0)
    for (uint32_t i = threadIdx.x; i < kWeightBins; i += kPartThreads) ws.hist(row)[i] = 0;
  if (threadIdx.x == 0) s_first = 0xFFFFFFFFu;
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float f[V];
    unpack<DT>(w[j], f);
    v.mask(min(a + threadIdx.x + j * kPartThreads, z - 1u), f);
#pragma unroll
    for (int k = 0; k < V; ++k) top = fmaxf(top, f[k]);
  }
  top = wave_max(top);
  if ((threadIdx.x & 63u) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
  if (threadIdx.x == 0) ws.maxima(row)[part] = top;
  if (!is_greedy(g, row)) return;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t i = min(a + threadIdx.x + j * kPartThreads, z - 1u);
    float f[V];
    unpack<DT>(w[j], f);
    v.mask(i, f);
#pragma unroll
    for (int k = V - 1; k >= 0; --k)
      if (f[k] == top && f[k] > -INFINITY) atomicMin(&s_first, i * V + k - v.skip);
  }
  __syncthreads();
  if (threadIdx.x == 0) ws.count(row)[part] = s_first;
}

template <int NW>
__device__ __forceinline__ float row_max(const SampleWs& ws, uint32_t row, SampleShared& sh) {
  float m = -INFINITY;
  for (uint32_t i = threadIdx.x; i < ws.parts; i += 64 * NW) m = fmaxf(m, ws.maxima(row)[i]);
  return block_max<NW>(m, sh);
}

template <int DT, int MODE>
__global__ __launch_bounds__(kPartThreads) void sample_mass_kernel(SampleArgs g, SampleWs ws) {
  __shared__ SampleShared sh;
  const uint32_t row = blockIdx.x / ws.parts, part = blockIdx.x % ws.parts;
  const RowParams p = row_params<MODE>(g, row);
  const float m = row_max<kPartWaves>(ws, row, sh);
  const RowKind kind = row_kind(p, g.cols, m);
  if (is_greedy(g, row) || (kind != kTopP && kind != kPlain)) return;
  const RowVecs<DT> v(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const uint32_t a = seg_begin(v.n, part, ws.parts), z = seg_begin(v.n, part + 1, ws.parts);
  constexpr int U = kV<DT> == 4 ? 4 : 2;
  uint64_t mass;
  if (kind == kPlain) {
    mass = plain_mass<DT, MODE, kPartWaves, U>(v, a, z, m, p, least_kept(p));
  } else {
    clear_hist<kPartWaves>(sh);
    mass = bin_masses<DT, MODE, kPartWaves, U>(v, a, z, m, p, sh);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kWeightBins; i += kPartThreads) {
      const uint64_t w = sh.hist[kBins - 1u - i];
      if (w) atomicAdd((unsigned long long*)&ws.hist(row)[i], (unsigned long long)w);
    }
  }
  mass = block_sum64<kPartWaves>(mass, sh);
  if (threadIdx.x == 0) ws.mass(row)[part] = mass;
}

// The cut of a top-p row from the workspace's bins and light masses.
template <int NW>
__device__ __forceinline__ Cut row_cut(const SampleWs& ws, uint32_t row, const uint64_t* light,
                                       const RowParams& p, SampleShared& sh) {
  for (uint32_t i = threadIdx.x; i < kBins; i += 64 * NW)
    sh.hist[kBins - 1u - i] = i < kWeightBins ? ws.hist(row)[i] : 0u;
  uint64_t s = 0;
  for (uint32_t i = threadIdx.x; i < ws.parts; i += 64 * NW) s += light[i];
  return pick_cut<NW>(block_sum64<NW>(s, sh), p, sh);
}

template <int DT, int MODE>
__global__ __launch_bounds__(kPartThreads) void sample_cut_kernel(SampleArgs g, SampleWs ws) {
  __shared__ SampleShared sh;
  const uint32_t row = blockIdx.x / ws.parts, part = blockIdx.x % ws.parts;
  const RowParams p = row_params<MODE>(g, row);
  const float m = row_max<kPartWaves>(ws, row, sh);
  if (is_greedy(g, row) || row_kind(p, g.cols, m) != kTopP) return;
  if (threadIdx.x == 0) sh.count = 0;
  const Cut c = row_cut<kPartWaves>(ws, row, ws.mass(row), p, sh);
  const RowVecs<DT> v(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const uint32_t a = seg_begin(v.n, part, ws.parts), z = seg_begin(v.n, part + 1, ws.parts);
  const uint64_t mass = block_sum64<kPartWaves>(
      cut_mass<DT, MODE, kPartWaves, kV<DT> == 4 ? 4 : 2>(v, a, z, m, p, c, sh), sh);
  if (threadIdx.x == 0) ws.kept(row)[part] = mass;
  flush_list(ws, row, part, sh);
}

template <int DT, int MODE>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(4, 4)))
void sample_finish_kernel(SampleArgs g, SampleWs ws) {
  __shared__ SampleShared sh;
  const uint32_t row = blockIdx.x;
  const RowVecs<DT> v(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  RowSampler<DT, MODE> r;
  r.x = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  r.cols = g.cols;
  r.p = row_params<MODE>(g, row);
  const float m = r.m = row_max<kRowWaves>(ws, row, sh);
  const RowKind kind = row_kind(r.p, g.cols, m);
  if (kind == kNone) {
    write_none(g, row);
    return;
  }
  if (is_greedy(g, row)) {   // the first word of the row's max
    uint32_t first = 0xFFFFFFFFu;
    if (threadIdx.x < ws.parts && ws.maxima(row)[threadIdx.x] == m) first = ws.count(row)[threadIdx.x];
    if (threadIdx.x == 0) sh.found = 0xFFFFFFFFu;
    __syncthreads();
    if (first != 0xFFFFFFFFu) atomicMin(&sh.found, first);
    __syncthreads();
    if (threadIdx.x == 0) write_row(g, row, sh.found, 1u, 1u);
    return;
  }
  const uint32_t n = kind == kTopP ? fetch_list(ws, row, sh) : 0u;
  if (kind == kTopP && n <= kCap) {
    const Cut c = row_cut<kRowWaves>(ws, row, ws.mass(row), r.p, sh);
    if (threadIdx.x < ws.parts) sh.seg[threadIdx.x] = ws.kept(row)[threadIdx.x];
    __syncthreads();
    finish_top_p<DT, MODE>(g, row, v, ws.parts, n, c, r, sh);
    return;
  } else if (kind == kPlain) {
    r.m_cut = least_kept(r.p);
    if (threadIdx.x < ws.parts) sh.seg[threadIdx.x] = ws.mass(row)[threadIdx.x];
    finish_segments<DT, MODE>(g, row, v, ws.parts, r, sh);
    return;
  }
  sample_any<DT, MODE>(g, row, m, r.p, sh);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kSampleMaxCols = 1 << 22;   // sums below 2^62
// Rows of kSplitCols words or more are split into parts of kPartCols (with the vectors
// at both ends at most 8192 elements, as the scan holds) up to kSplitRows rows, with a
// top-p up to half as many: one workgroup a row against the split, binary32, no filter
// 1 x 50257 14.6 / 15.3 us, 1 x 128256 26.3 / 15.7, 64 x 128256 28.8 / 23.9, 127 x 128256
// 33.2 / 36.6; top-p 1 x 50257 25.2 / 28.9, 32 x 128256 52.8 / 34.6, 64 x 128256 48.2 / 47.8.
constexpr int64_t kPartCols = 8160, kSplitCols = 65536, kSplitRows = 64;

static int64_t sample_parts(int64_t rows, int64_t cols) {
  return rows > 0 && rows <= kSplitRows && cols >= kSplitCols ? (cols + kPartCols - 1) / kPartCols : 1;
}
static_assert((kSampleMaxCols + kPartCols - 1) / kPartCols <= kMaxSegs, "a segment a part");
static int64_t sample_row_ws(int64_t parts) {
  return (kWeightBins + kWsCap + 2 * parts) * 8 + parts * 8;
}
static int64_t sample_ws_bytes(int64_t rows, int64_t parts) {
  return parts == 1 ? 0 : rows * sample_row_ws(parts);
}

template <int DT, int MODE>
static void launch_sample(uint32_t n, hipStream_t s, const SampleArgs& g, uint32_t row0,
                          const SampleWs& ws) {
  if (ws.base == nullptr) {
    hipLaunchKernelGGL((sample_row_kernel<DT, MODE>), dim3(n), dim3(kRowThreads), 0, s, g, row0);
    return;
  }
  const dim3 parts(n * ws.parts), b(kPartThreads);
  hipLaunchKernelGGL((sample_scan_kernel<DT>), parts, b, 0, s, g, ws);
  hipLaunchKernelGGL((sample_mass_kernel<DT, MODE>), parts, b, 0, s, g, ws);
  if (g.top_p != nullptr)
    hipLaunchKernelGGL((sample_cut_kernel<DT, MODE>), parts, b, 0, s, g, ws);
  hipLaunchKernelGGL((sample_finish_kernel<DT, MODE>), dim3(n), dim3(kRowThreads), 0, s, g, ws);
}
template <int DT>
static void launch_sample(int mode, uint32_t n, hipStream_t s, const SampleArgs& g, uint32_t row0,
                          const SampleWs& ws) {
  switch (mode) {
    case QUAKE_EXACT: launch_sample<DT, EXACT>(n, s, g, row0, ws); break;
    case QUAKE_1: launch_sample<DT, Q1>(n, s, g, row0, ws); break;
    case QUAKE_2: launch_sample<DT, Q2>(n, s, g, row0, ws); break;
    default: launch_sample<DT, Q2M>(n, s, g, row0, ws); break;
  }
}

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_sample_workspace_size(int64_t rows, int64_t cols, int64_t* bytes) {
  if (bytes == nullptr || rows < 0 || cols < 0 || cols > kSampleMaxCols) return QUAKE_EINVAL;
  const int64_t parts = sample_parts(rows, cols);
  *bytes = sample_ws_bytes(rows, parts);
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
  const int64_t parts = sample_parts(rows, cols);
  SampleWs ws{nullptr, 0, 1};
  if (workspace != nullptr && workspace_bytes < sample_ws_bytes(rows, parts)) return QUAKE_EINVAL;
  if (workspace != nullptr && parts > 1 && top_k == nullptr &&
      (top_p == nullptr || 2 * rows <= kSplitRows)) {
    const int64_t need = sample_ws_bytes(rows, parts);
    if (meet(workspace, need, x, rows_bytes(rows, cols, ldx, elem_size(dtype)))) return QUAKE_EINVAL;
    for (const void* p : {(const void*)u, (const void*)token, (const void*)prob,
                          (const void*)temperature, (const void*)top_p, (const void*)min_p})
      if (meet(workspace, need, p, 4 * rows)) return QUAKE_EINVAL;
    ws = {static_cast<char*>(workspace), sample_row_ws(parts), (uint32_t)parts};
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  constexpr int64_t kMost = 1 << 20;   // rows a launch: below 2^32 threads
  for (int64_t r = 0; r < rows; r += kMost) {
    const uint32_t n = (uint32_t)std::min(kMost, rows - r);
    if (dtype == QUAKE_F32) launch_sample<F32>(mode, n, s, g, (uint32_t)r, ws);
    else if (dtype == QUAKE_F16) launch_sample<F16>(mode, n, s, g, (uint32_t)r, ws);
    else launch_sample<BF16>(mode, n, s, g, (uint32_t)r, ws);
    const quake_status st = launch_status();
    if (st != QUAKE_OK) return st;
  }
  return QUAKE_OK;
}
