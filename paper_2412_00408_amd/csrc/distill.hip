// distill.hip — quake_distill and quake_distill_grad: the divergence of a
// student's row of logits from a teacher's distribution over its top logits,
//   loss = sum_k p_k (log p_k - log q_{i_k}),   d loss / d x_v = t (q_v - P_v),
// p = softmax(t y) over the row's K entries, q = softmax(t x) over the
// vocabulary, P_v = sum of the p_k whose index is v.
//
// Both softmaxes take QuAKE's exponentials (arXiv:2412.00408) against a whole
// number M of base-2 units: Q(y - M) = 2^-M Q(y) exactly (only the exponent field
// moves), so a thread raises its M as it meets larger logits, partial sums of a
// row join exactly, and a row's statistics take one pass. c1 = (127 - M) 2^23 is
// exact in binary32. Final M: the row max, t/ln2 times, rounded up.
//
// What bounds it is memory: the logits in, twice, their gradient out. One workgroup
// takes a row for statistics, loss and gradient (distill_row_kernel); few rows are cut into chunks over more workgroups, with
// the chunks' (M, sum) in a workspace (part, finish and grad kernels).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "quake_device.hpp"
#include "quake_host.hpp"
#include "row_vecs.hpp"

namespace qk {

constexpr int kDsThreads = 512, kDsWaves = kDsThreads / 64;
constexpr int kDsTopk = 1024;            // most teacher entries per row
constexpr float kDsNoMax = -1e30f;       // M before any logit

struct DistillArgs {
  const char* x;
  const int32_t* idx;
  const char* y;
  const float* weight;   // or null: 1
  float* loss;
  float* stats;          // [rows][2]: M, S
  char* grad;            // or null
  float* part;           // [rows][chunks][2]
  int64_t ldx, ldi, ldy, ldg;
  uint32_t cols, topk, chunks;   // chunks: of a row, 1 where not split
  int32_t ydt;
  float c0, t;           // 2^23 t / ln2 (EXACT: t / ln2)
};

template <int MODE>
__device__ __forceinline__ float c1_of(float M) {
  return MODE == EXACT ? -M : (127.0f - M) * 0x1p23f;
}
template <int MODE>
constexpr float kToUnits = MODE == EXACT ? 1.0f : 0x1p-23f;   // c0 to t / ln2, exactly

__device__ __forceinline__ int32_t ds_shift(float from, float to) {   // from <= to
  return (int32_t)fmaxf(from - to, -2000.0f);
}

// Sum of exponentials relative to 2^M.
struct Sum {
  double s = 0.0;
  float M = kDsNoMax;
  __device__ __forceinline__ void join(double os, float oM) {
    const float top = fmaxf(M, oM);
    s = ldexp(s, ds_shift(M, top)) + ldexp(os, ds_shift(oM, top));
    M = top;
  }
};

template <int MODE, int N>
__device__ __forceinline__ void add_values(const float (&f)[N], float c0, Sum& a) {
  float top = f[0];
#pragma unroll
  for (int k = 1; k < N; ++k) top = fmaxf(top, f[k]);
  top *= c0 * kToUnits<MODE>;
  if (top > a.M) {
    const float M = __builtin_ceilf(top);
    a.s = ldexp(a.s, ds_shift(a.M, M));
    a.M = M;
  }
  const float c1 = c1_of<MODE>(a.M);
  float s[4] = {};
#pragma unroll
  for (int k = 0; k < N; ++k) s[k & 3] += qexp_row<MODE, true>(f[k], c0, c1);
  a.s += (double)((s[0] + s[1]) + (s[2] + s[3]));
}

// Vectors of [a, z) that lie inside the row as a whole; the row's first and last are
// taken by one thread each.
template <int DT>
struct Inner {
  uint32_t a, z;
  bool head, tail;
  __device__ __forceinline__ Inner(const RowVecs<DT>& r, uint32_t a_, uint32_t z_)
      : a(max(a_, 1u)), z(min(z_, r.n - 1u)), head(a_ == 0 && z_ > 0 && threadIdx.x == 0),
        tail(z_ == r.n && r.n > 1u && a_ < z_ && threadIdx.x == 64) {}
};

// Statistics of vectors [a, z) of a row by the workgroup: values four vectors at a
// time (one max, one binary64 addition).
template <int DT, int MODE>
__device__ __forceinline__ Sum row_sum(const RowVecs<DT>& r, uint32_t a, uint32_t z, float c0) {
  constexpr int V = kV<DT>, U = 4;
  const Inner<DT> in(r, a, z);
  Sum acc;
  uint32_t i = in.a + threadIdx.x;
  for (; i + (U - 1) * kDsThreads < in.z; i += U * kDsThreads) {
    u32x4 w[U];
#pragma unroll
    for (int j = 0; j < U; ++j) w[j] = r.v[i + j * kDsThreads];
    float f[U * V];
#pragma unroll
    for (int j = 0; j < U; ++j) unpack<DT>(w[j], f + V * j);
    add_values<MODE>(f, c0, acc);
  }
  for (; i < in.z; i += kDsThreads) {
    float f[V];
    unpack<DT>(r.v[i], f);
    add_values<MODE>(f, c0, acc);
  }
  if (in.head || in.tail) {
    float f[V];
    const uint32_t e = in.head ? 0u : r.n - 1u;
    unpack<DT>(r.v[e], f);
    r.mask(e, f);
    add_values<MODE>(f, c0, acc);
  }
  return acc;
}

struct DistillShared {
  double s[kDsWaves];
  float M[kDsWaves];
  __attribute__((aligned(16))) float p[kDsTopk];     // teacher's exponentials
  __attribute__((aligned(16))) int32_t idx[kDsTopk]; // -1: no entry
};

// The workgroup's sum, on every thread (a fixed order: lanes, then waves).
__device__ __forceinline__ Sum block_join(Sum a, DistillShared& sh) {
  const float M = wave_max(a.M);
  const double s = wave_sum(ldexp(a.s, ds_shift(a.M, M)));
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) {
    sh.s[threadIdx.x >> 6] = s;
    sh.M[threadIdx.x >> 6] = M;
  }
  __syncthreads();
  Sum r;
#pragma unroll
  for (int w = 0; w < kDsWaves; ++w) r.join(sh.s[w], sh.M[w]);
  return r;
}
// the statistics as they are kept: S in binary32 (M = 0 where nothing is finite)
__device__ __forceinline__ float2 kept_stats(const Sum& a) {
  return a.M == kDsNoMax ? float2{0.0f, 0.0f} : float2{a.M, (float)a.s};
}

__device__ __forceinline__ float load_y(const char* p, int32_t dt, int64_t i) {
  return dt == F32 ? load1<F32>(p, i) : dt == F16 ? load1<F16>(p, i) : load1<BF16>(p, i);
}

// The teacher's row: exponentials and indices into LDS, their sum (M of the sum:
// of the largest entry). Entries with an index outside the row are left out.
template <int MODE>
__device__ __forceinline__ Sum teacher(const DistillArgs& g, uint32_t row, DistillShared& sh) {
  const uint32_t padded = (g.topk + 3u) & ~3u;
  const int32_t* idx = g.idx + (int64_t)row * g.ldi;
  const char* y = g.y + (int64_t)row * g.ldy * (g.ydt == F32 ? 4 : 2);
  float top = -INFINITY;
  for (uint32_t k = threadIdx.x; k < padded; k += kDsThreads) {
    const int32_t i = k < g.topk ? idx[k] : -1;
    const bool live = i >= 0 && (uint32_t)i < g.cols;
    const float v = live ? load_y(y, g.ydt, k) : -INFINITY;
    sh.idx[k] = live ? i : -1;
    sh.p[k] = v;
    top = fmaxf(top, v);
  }
  Sum a;
  a.s = 0.0;
  a.M = top == -INFINITY ? kDsNoMax : __builtin_ceilf(top * (g.c0 * kToUnits<MODE>));
  a = block_join(a, sh);
  const float c1 = c1_of<MODE>(a.M);
  Sum b;
  b.M = a.M;
  for (uint32_t k = threadIdx.x; k < padded; k += kDsThreads) {
    const float e = sh.p[k] == -INFINITY ? 0.0f : qexp_row<MODE, true>(sh.p[k], g.c0, c1);
    sh.p[k] = e;
    b.s += (double)e;
  }
  return block_join(b, sh);
}

// loss of the row by the workgroup (valid on thread 0)
template <int DT, int MODE>
__device__ __forceinline__ double row_loss(const DistillArgs& g, uint32_t row, float2 st,
                                           const Sum& ts, DistillShared& sh) {
  const double c = (double)(g.c0 * kToUnits<MODE>);
  const char* x = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  const char* y = g.y + (int64_t)row * g.ldy * (g.ydt == F32 ? 4 : 2);
  const double logs = log2((double)st.y) + (double)st.x, logt = log2(ts.s) + (double)ts.M;
  double l = 0.0;
  for (uint32_t k = threadIdx.x; k < g.topk; k += kDsThreads) {
    if (!(sh.p[k] > 0.0f)) continue;
    const float v = load1<DT>(x, sh.idx[k]);
    const double logq = v == -INFINITY ? -INFINITY : (double)v * c - logs;
    l += ((double)sh.p[k] / ts.s) * (((double)load_y(y, g.ydt, k) * c - logt) - logq);
  }
  l = wave_sum(l);
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) sh.s[threadIdx.x >> 6] = l;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kDsWaves; ++w) all += sh.s[w];
  return all * 0.693147180559945309417232121458176568;
}

// past the caches: they hold the rows that are read again
__device__ __forceinline__ void store_vec(u32x4* p, u32x4 v) { __builtin_nontemporal_store(v, p); }

// Gradient of vectors [a, z) of the row: w t (q - P). The teacher's entries are put
// right after the vectors are written, each index by its first entry, from the
// logit read before (grad may be x).
template <int DT, int MODE>
__device__ __forceinline__ void row_grad(const DistillArgs& g, uint32_t row, uint32_t a, uint32_t z,
                                         float2 st, double ts, const DistillShared& sh) {
  constexpr int V = kV<DT>;
  const char* xrow = g.x + (int64_t)row * g.ldx * kEsz<DT>;
  char* grow = g.grad + (int64_t)row * g.ldg * kEsz<DT>;
  const RowVecs<DT> r(xrow, g.cols);
  const double wt = (double)(g.weight ? g.weight[row] : 1.0f) * (double)g.t;
  const bool live = ts > 0.0 && wt != 0.0;
  const float scale = live && st.y > 0.0f ? (float)(wt / (double)st.y) : 0.0f;
  const float c1 = c1_of<MODE>(st.x);
  const uint32_t e0 = a * V, e1 = z * V;   // vector elements of this part
  // first entries of their index among those of this part, two a thread at most
  constexpr int N = kDsTopk / kDsThreads;
  float fix[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const uint32_t k = threadIdx.x + n * kDsThreads;
    fix[n] = 0.0f;
    if (k >= g.topk || !live) continue;
    const int32_t i = sh.idx[k];
    if (i < 0 || (uint32_t)i + r.skip < e0 || (uint32_t)i + r.skip >= e1) continue;
    fix[n] = load1<DT>(xrow, i);
  }
  const bool same = ((uintptr_t)grow & 15u) == ((uintptr_t)xrow & 15u);
  u32x4* gv = reinterpret_cast<u32x4*>(grow - ((uintptr_t)grow & 15u));
  __syncthreads();   // every entry's logit has been read
  auto values = [&](const u32x4& w, float* f) {
    unpack<DT>(w, f);
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = qexp_row<MODE, true>(f[k], g.c0, c1) * scale;
  };
  auto put = [&](uint32_t i, const float* f) {   // element by element
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const uint32_t e = i * V + k;
      if (e >= r.skip && e < r.skip + r.cols) store1<DT>(grow, e - r.skip, f[k]);
    }
  };
  const Inner<DT> in(r, a, z);
  float f[V] = {};
  if (scale == 0.0f) {
    for (uint32_t i = in.a + threadIdx.x; i < in.z; i += kDsThreads) {
      if (same) gv[i] = u32x4{};
      else put(i, f);
    }
    if (in.head) put(0, f);
    if (in.tail) put(r.n - 1u, f);
  } else {
    // from the row's end on, which a pass before left in the nearest cache
    const uint32_t count = in.z > in.a ? in.z - in.a : 0u;
    uint32_t n = threadIdx.x;   // vectors from the end
    if (same) {
      for (; n + 3 * kDsThreads < count; n += 4 * kDsThreads) {
        const uint32_t i = in.z - 1u - n;
        u32x4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = r.v[i - j * kDsThreads];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          values(w[j], f);
          store_vec(gv + (i - j * kDsThreads), pack<DT>(f));
        }
      }
    }
    for (; n < count; n += kDsThreads) {
      const uint32_t i = in.z - 1u - n;
      values(r.v[i], f);
      if (same) gv[i] = pack<DT>(f);
      else put(i, f);
    }
    if (in.head || in.tail) {
      const uint32_t e = in.head ? 0u : r.n - 1u;
      values(r.v[e], f);
      put(e, f);
    }
  }
  if (!live) return;
  __syncthreads();   // the vectors are written
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const uint32_t k = threadIdx.x + n * kDsThreads;
    if (k >= g.topk) continue;
    const int32_t v = sh.idx[k];
    if (v < 0 || (uint32_t)v + r.skip < e0 || (uint32_t)v + r.skip >= e1) continue;
    double p = 0.0;
    bool first = true;
    for (uint32_t j = 0; j < g.topk; j += 4) {
      const int4 o = *reinterpret_cast<const int4*>(&sh.idx[j]);
      const int32_t ov[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (ov[q] == v) {
          first = first && j + q >= k;
          p += (double)sh.p[j + q];
        }
      }
    }
    if (!first) continue;
    const double q = st.y > 0.0f ? (double)qexp_row<MODE, true>(fix[n], g.c0, c1) / (double)st.y : 0.0;
    store1<DT>(grow, v, (float)(wt * (q - p / ts)));
  }
}

// The whole row by one workgroup. 2048 x 128256 bf16: 285 to 294 us, 3.6 TB/s of the
// logits in and the gradient out (the statistics alone 100 us, 5.2 TB/s). The second
// reading goes past L2 as the first does (1.03 GB read in all by the counters), so it is
// three passes of 525 MB at 5.4 TB/s; 21 VALU instructions an element run beside them.
// Rows of the gradient that do not lie as the logits' do in their 16 bytes (a fresh
// gradient of columns 0 .. 50256 of wider rows) are stored element by element: 2048 rows
// 179 us, 100 with a gradient padded alike.
template <int DT, int MODE>
__global__ __launch_bounds__(kDsThreads) void distill_row_kernel(DistillArgs g, uint32_t row0) {
  __shared__ DistillShared sh;
  const uint32_t row = row0 + blockIdx.x;
  const RowVecs<DT> r(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const float2 st = kept_stats(block_join(row_sum<DT, MODE>(r, 0, r.n, g.c0), sh));
  const Sum ts = teacher<MODE>(g, row, sh);
  const double loss = ts.s > 0.0 ? row_loss<DT, MODE>(g, row, st, ts, sh) : 0.0;
  if (threadIdx.x == 0) {
    g.loss[row] = (float)loss;
    if (g.stats) {
      g.stats[2 * (int64_t)row] = st.x;
      g.stats[2 * (int64_t)row + 1] = st.y;
    }
  }
  if (g.grad) row_grad<DT, MODE>(g, row, 0, r.n, st, ts.s, sh);
}

__device__ __forceinline__ uint32_t chunk_begin(uint32_t n, uint32_t chunk, uint32_t chunks) {
  return (uint32_t)((uint64_t)n * chunk / chunks);
}

// (M, S) of one chunk of a row
template <int DT, int MODE>
__global__ __launch_bounds__(kDsThreads) void distill_part_kernel(DistillArgs g, uint32_t row0) {
  __shared__ DistillShared sh;
  const uint32_t row = row0 + blockIdx.x / g.chunks, c = blockIdx.x % g.chunks;
  const RowVecs<DT> r(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const Sum a = block_join(row_sum<DT, MODE>(r, chunk_begin(r.n, c, g.chunks),
                                             chunk_begin(r.n, c + 1, g.chunks), g.c0), sh);
  if (threadIdx.x == 0) {
    float* p = g.part + 4 * (int64_t)blockIdx.x;
    *reinterpret_cast<double*>(p) = a.s;
    p[2] = a.M;
  }
}

// Joins a row's chunks; loss and statistics.
template <int DT, int MODE>
__global__ __launch_bounds__(kDsThreads) void distill_finish_kernel(DistillArgs g, uint32_t row0) {
  __shared__ DistillShared sh;
  const uint32_t row = row0 + blockIdx.x;
  const float* p = g.part + 4 * (int64_t)blockIdx.x * g.chunks;
  Sum a;
  for (uint32_t c = 0; c < g.chunks; ++c)
    a.join(*reinterpret_cast<const double*>(p + 4 * c), p[4 * c + 2]);
  const float2 st = kept_stats(a);
  const Sum ts = teacher<MODE>(g, row, sh);
  const double loss = ts.s > 0.0 ? row_loss<DT, MODE>(g, row, st, ts, sh) : 0.0;
  if (threadIdx.x == 0) {
    g.loss[row] = (float)loss;
    g.stats[2 * (int64_t)row] = st.x;
    g.stats[2 * (int64_t)row + 1] = st.y;
  }
}

// Gradient of one chunk of a row from its statistics.
template <int DT, int MODE>
__global__ __launch_bounds__(kDsThreads) void distill_grad_kernel(DistillArgs g, uint32_t row0) {
  __shared__ DistillShared sh;
  const uint32_t row = row0 + blockIdx.x / g.chunks, c = blockIdx.x % g.chunks;
  const RowVecs<DT> r(g.x + (int64_t)row * g.ldx * kEsz<DT>, g.cols);
  const float2 st{g.stats[2 * (int64_t)row], g.stats[2 * (int64_t)row + 1]};
  const Sum ts = teacher<MODE>(g, row, sh);
  row_grad<DT, MODE>(g, row, chunk_begin(r.n, c, g.chunks), chunk_begin(r.n, c + 1, g.chunks), st,
                     ts.s, sh);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Rows a launch takes; a workspace holds the chunk sums and statistics of one.
constexpr int64_t kDsRows = 1 << 20;
constexpr int64_t kDsMaxCols = 1 << 30;

// Chunks of a row: below kDsFull rows one workgroup a row leaves compute units
// idle, so rows are cut until the launch has that many, no chunk below 8192 elements.
constexpr int64_t kDsFull = 512;
static int64_t distill_chunks(int64_t rows, int64_t cols) {
  if (rows <= 0 || rows >= kDsFull) return 1;
  return std::max<int64_t>(1, std::min(kDsFull / rows, cols / 8192));
}
// Chunks of a row for the gradient alone: of 16384 elements also where the rows would
// fill the GPU, as then the launch sweeps through memory from front to back (2048 x
// 128256 bf16: 236 us with a workgroup per row, 190 us in chunks).
static int64_t grad_chunks(int64_t rows, int64_t cols) {
  return std::max(distill_chunks(rows, cols), std::max<int64_t>(1, cols / 16384));
}
static int64_t distill_ws_bytes(int64_t rows, int64_t cols) {
  const int64_t c = distill_chunks(rows, cols);
  return c == 1 ? 0 : rows * (16 * c + 8);
}

enum DistillStep { kRow, kPart, kFinish, kGrad };

template <int DT, int MODE>
static void launch_step(DistillStep step, uint32_t n, hipStream_t s, const DistillArgs& g, uint32_t r) {
  const dim3 b(kDsThreads);
  switch (step) {
    case kRow: hipLaunchKernelGGL((distill_row_kernel<DT, MODE>), dim3(n), b, 0, s, g, r); break;
    case kPart: hipLaunchKernelGGL((distill_part_kernel<DT, MODE>), dim3(n * g.chunks), b, 0, s, g, r); break;
    case kFinish: hipLaunchKernelGGL((distill_finish_kernel<DT, MODE>), dim3(n), b, 0, s, g, r); break;
    default: hipLaunchKernelGGL((distill_grad_kernel<DT, MODE>), dim3(n * g.chunks), b, 0, s, g, r); break;
  }
}
template <int DT>
static void launch_mode(DistillStep step, int mode, uint32_t n, hipStream_t s, const DistillArgs& g,
                        uint32_t r) {
  switch (mode) {
    case QUAKE_EXACT: launch_step<DT, EXACT>(step, n, s, g, r); break;
    case QUAKE_1: launch_step<DT, Q1>(step, n, s, g, r); break;
    case QUAKE_2: launch_step<DT, Q2>(step, n, s, g, r); break;
    default: launch_step<DT, Q2M>(step, n, s, g, r); break;
  }
}
static quake_status launch_distill(DistillStep step, quake_dtype dt, int mode, int64_t n,
                                   hipStream_t s, const DistillArgs& g, int64_t r) {
  if (dt == QUAKE_F32) launch_mode<F32>(step, mode, (uint32_t)n, s, g, (uint32_t)r);
  else if (dt == QUAKE_F16) launch_mode<F16>(step, mode, (uint32_t)n, s, g, (uint32_t)r);
  else launch_mode<BF16>(step, mode, (uint32_t)n, s, g, (uint32_t)r);
  return launch_status();
}

// Checks that both entry points share; *c0 on success.
static quake_status distill_check(const void* x, const int32_t* idx, const void* y, int64_t rows,
                                  int64_t cols, int64_t topk, int64_t ldx, int64_t ldi, int64_t ldy,
                                  int64_t ldg, quake_dtype dtype, quake_dtype ydtype,
                                  quake_mode mode, float t, float* c0) {
  if (!valid_dtype(dtype) || !valid_dtype(ydtype)) return QUAKE_EDTYPE;
  if (!valid_mode(mode)) return QUAKE_EMODE;
  if (rows < 0 || rows > INT32_MAX || cols < 0 || cols > kDsMaxCols || topk < 0 || topk > kDsTopk)
    return QUAKE_EINVAL;
  if (ldx < cols || ldi < topk || ldy < topk || ldg < cols) return QUAKE_EINVAL;
  if (std::max(std::max(ldx, ldg), std::max(ldi, ldy)) > INT64_MAX / 8 / (rows > 0 ? rows : 1))
    return QUAKE_EINVAL;
  if (!std::isfinite(t) || !(t > 0.0f)) return QUAKE_EINVAL;
  *c0 = softmax_c0(t, mode);
  if (!std::isfinite(*c0) || *c0 == 0.0f) return QUAKE_EINVAL;
  if (rows == 0) return QUAKE_OK;
  if (cols == 0 || x == nullptr || (topk > 0 && (idx == nullptr || y == nullptr))) return QUAKE_EINVAL;
  if (((uintptr_t)x & (uintptr_t)(elem_size(dtype) - 1)) != 0 || ((uintptr_t)idx & 3u) != 0 ||
      ((uintptr_t)y & (uintptr_t)(elem_size(ydtype) - 1)) != 0)
    return QUAKE_EINVAL;
  return QUAKE_OK;
}

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_distill_workspace_size(int64_t rows, int64_t cols, int64_t* bytes) {
  if (bytes == nullptr || rows < 0 || rows > INT32_MAX || cols < 0 || cols > kDsMaxCols)
    return QUAKE_EINVAL;
  *bytes = distill_ws_bytes(rows, cols);
  return QUAKE_OK;
}

extern "C" quake_status quake_distill(const void* x, const int32_t* idx, const void* y,
                                      const float* weight, float* loss, float* stats, void* grad,
                                      int64_t rows, int64_t cols, int64_t topk, int64_t ldx,
                                      int64_t ldi, int64_t ldy, int64_t ldg, quake_dtype dtype,
                                      quake_dtype ydtype, quake_mode mode, float t,
                                      void* workspace, int64_t workspace_bytes, void* stream) {
  float c0 = 0.0f;
  const quake_status ok = distill_check(x, idx, y, rows, cols, topk, ldx, ldi, ldy,
                                        grad ? ldg : cols, dtype, ydtype, mode, t, &c0);
  if (ok != QUAKE_OK) return ok;
  if (workspace_bytes < 0 || (workspace != nullptr && !aligned16(workspace))) return QUAKE_EINVAL;
  if (rows == 0) return QUAKE_OK;
  if (loss == nullptr || (((uintptr_t)loss | (uintptr_t)stats | (uintptr_t)weight) & 3u) != 0 ||
      ((uintptr_t)grad & (uintptr_t)(elem_size(dtype) - 1)) != 0)
    return QUAKE_EINVAL;
  const int64_t need = distill_ws_bytes(rows, cols);
  if (workspace != nullptr && workspace_bytes < need) return QUAKE_EINVAL;
  DistillArgs g{static_cast<const char*>(x), idx, static_cast<const char*>(y), weight, loss, stats,
                static_cast<char*>(grad), static_cast<float*>(workspace), ldx, ldi, ldy, ldg,
                (uint32_t)cols, (uint32_t)topk, 1u, (int32_t)ydtype, c0, t};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (workspace != nullptr && need > 0) {
    if (meet(workspace, need, x, rows_bytes(rows, cols, ldx, elem_size(dtype))) ||
        meet(workspace, need, grad, rows_bytes(rows, cols, ldg, elem_size(dtype))) ||
        meet(workspace, need, idx, rows_bytes(rows, topk, ldi, 4)) ||
        meet(workspace, need, y, rows_bytes(rows, topk, ldy, elem_size(ydtype))) ||
        meet(workspace, need, weight, 4 * rows) || meet(workspace, need, loss, 4 * rows) ||
        meet(workspace, need, stats, 8 * rows))
      return QUAKE_EINVAL;
    g.chunks = (uint32_t)distill_chunks(rows, cols);
    if (g.stats == nullptr)
      g.stats = reinterpret_cast<float*>(static_cast<char*>(workspace) + rows * 16 * g.chunks);
    quake_status st = launch_distill(kPart, dtype, mode, rows, s, g, 0);
    if (st == QUAKE_OK) st = launch_distill(kFinish, dtype, mode, rows, s, g, 0);
    if (st == QUAKE_OK && grad != nullptr) st = launch_distill(kGrad, dtype, mode, rows, s, g, 0);
    return st;
  }
  for (int64_t r = 0; r < rows; r += kDsRows) {
    const quake_status st = launch_distill(kRow, dtype, mode, std::min(kDsRows, rows - r), s, g, r);
    if (st != QUAKE_OK) return st;
  }
  return QUAKE_OK;
}

extern "C" quake_status quake_distill_grad(const void* x, const int32_t* idx, const void* y,
                                           const float* stats, const float* weight, void* grad,
                                           int64_t rows, int64_t cols, int64_t topk, int64_t ldx,
                                           int64_t ldi, int64_t ldy, int64_t ldg,
                                           quake_dtype dtype, quake_dtype ydtype, quake_mode mode,
                                           float t, void* stream) {
  float c0 = 0.0f;
  const quake_status ok = distill_check(x, idx, y, rows, cols, topk, ldx, ldi, ldy, ldg, dtype,
                                        ydtype, mode, t, &c0);
  if (ok != QUAKE_OK) return ok;
  if (rows == 0) return QUAKE_OK;
  if (stats == nullptr || grad == nullptr || (((uintptr_t)stats | (uintptr_t)weight) & 3u) != 0 ||
      ((uintptr_t)grad & (uintptr_t)(elem_size(dtype) - 1)) != 0)
    return QUAKE_EINVAL;
  DistillArgs g{static_cast<const char*>(x), idx, static_cast<const char*>(y), weight, nullptr,
                const_cast<float*>(stats), static_cast<char*>(grad), nullptr, ldx, ldi, ldy, ldg,
                (uint32_t)cols, (uint32_t)topk, (uint32_t)grad_chunks(rows, cols),
                (int32_t)ydtype, c0, t};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t most = std::max<int64_t>(1, kDsRows / g.chunks);
  for (int64_t r = 0; r < rows; r += most) {
    const quake_status st = launch_distill(kGrad, dtype, mode, std::min(most, rows - r), s, g, r);
    if (st != QUAKE_OK) return st;
  }
  return QUAKE_OK;
}
