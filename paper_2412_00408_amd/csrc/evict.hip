// evict.hip — quake_cache_evict: a key/value cache brought down to `budget` keys a key
// head: the first ones, the newest ones, and of those between the ones that gathered the
// most attention weight. The kept keys stay in order, in slots 0 on.
//
// Which: the weights as order-preserving unsigned keys; the key of the last one that fits
// by counting digits from the top (11, 11 and 10 bits, counts in LDS), then the kept
// slots in order by ballots, of equal ones the first. Whole numbers: the same slots
// every time.
//
// Moving: slot i of the result comes from kept[i] >= i, ascending. Rounds of consecutive
// slots, all read before any is written, are therefore right in place: a round writes
// nothing that a later one reads.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "cache_tile.hpp"
#include "quake_device.hpp"
#include "quake_host.hpp"

namespace qk {

struct EvictArgs {
  const char *k, *v;
  const float* weight;
  const int32_t* lens;                     // or null: skv
  char *ko, *vo;
  float* wo;
  int32_t* lens_out;                       // or null
  int32_t *kept, *evicted;
  quake_evict_strides st;                  // k's and v's in bytes here
  int32_t skv, slots, kv_heads, budget, sinks, recent;
  int32_t row16, slice, slices;            // 16-byte chunks of a row; in place: chunks of a slice of
                                           // it, slices of a row, else rows of a run, runs
};

// Weights in ascending order as unsigned numbers: NaN below all, -0 as 0. What is kept
// whatever its weight is above all, what is no slot below all.
constexpr uint32_t kAlways = 0xFFFFFFFFu, kNever = 0u;
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 1u;
  const uint32_t u = as_u(w == 0.0f ? 0.0f : w);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// A workgroup a sequence and key head; a wave has a run of the slots. The key of the last one
// that fits comes digit by digit from the top (11, 11 and 10 bits), by counting in LDS those
// whose upper digits are the key's. Up to kHeldLong slots a thread stay in registers, longer
// rows are read again for each digit and twice for the result. One compute unit's instructions
// and barriers bound it: rows of 300 slots 7.8 us, 512 rows of 2560 12 us, 8 of 16384 15 us, 32
// of up to 39106 35 us.
constexpr int kBins = 2048, kHeld = 16, kHeldLong = 40, kEach = 8;

template <int THREADS>
struct ChooseShared {
  uint32_t bins[3 * kBins];                          // of a digit each
  uint32_t wave[THREADS / 64], equal[THREADS / 64], found[3];
};

template <int THREADS, int HELD>     // HELD: slots a thread holds, 0: reads them again
__device__ __forceinline__ void choose_slots(const EvictArgs& g, const float* w, int32_t len, int32_t* kept,
                                             ChooseShared<THREADS>& sh) {
  constexpr int E = HELD > 0 ? HELD : kEach, W = THREADS / 64, N = kBins / THREADS;   // bins a thread
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t lo = g.sinks, hi = len - g.recent;
  const int32_t run = (len + THREADS - 1) / THREADS * 64;
  const int32_t from = wave * run, to = min(from + run, len);
  uint32_t u[E];
  const auto fetch = [&](int32_t i0) {
    constexpr int F = E < 16 ? E : 16;               // loads in flight; the last ones may be fewer
#pragma unroll
    for (int e0 = 0; e0 < E; e0 += F) {
      const int end = e0 + F < E ? e0 + F : E;
      float x[F];
#pragma unroll
      for (int e = e0; e < end; ++e) {
        const int32_t i = i0 + 64 * e + lane;
        x[e - e0] = i < to ? w[i] : 0.0f;
      }
#pragma unroll
      for (int e = e0; e < end; ++e) {
        const int32_t i = i0 + 64 * e + lane;
        u[e] = i >= to ? kNever : i < lo || i >= hi ? kAlways : weight_key(x[e - e0]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto each = [&](auto f) {      // f(slot of lane 0, this lane's key), of this wave's run
    for (int32_t i0 = from; i0 < to; i0 += 64 * E) {
      if (HELD == 0) fetch(i0);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i0 + 64 * e < to) f(i0 + 64 * e, u[e]);
    }
  };
  if (HELD > 0) fetch(from);
  for (int i = threadIdx.x; i < 3 * kBins; i += THREADS) sh.bins[i] = 0;
  __syncthreads();
  uint32_t key = 0, left = (uint32_t)g.budget;       // of the slots whose upper digits are key's
  const auto digit = [&](uint32_t* bins, int shift, uint32_t mask, uint32_t upper) {
    each([&](int32_t, uint32_t k) {
      if ((k & upper) == key) atomicAdd(&bins[(k >> shift) & mask], 1u);
    });
    __syncthreads();
    // thread t: N bins from the top
    const int top = kBins - 1 - N * (int)threadIdx.x;
    uint32_t c[N], mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += c[i] = bins[top - i];
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t other = __shfl_up(upto, o, 64);
      upto += lane >= o ? other : 0u;
    }
    if (lane == 63) sh.wave[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) upto += i < wave ? sh.wave[i] : 0u;
    uint32_t above = upto - mine;                    // in the bins above this thread's
    if (above < left && left <= upto) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (above < left && left <= above + c[i]) {
          sh.found[0] = (uint32_t)(top - i);
          sh.found[1] = above;
          sh.found[2] = c[i];
        }
        above += c[i];
      }
    }
    __syncthreads();
    key |= sh.found[0] << shift;
    left -= sh.found[1];
    if (left < sh.found[2] || key == 0) return false;
    --key;                                           // all of these fit: what is above them and they
    left = 0;
    return true;
  };
  if (!digit(sh.bins, 21, 0x7FFu, 0u) && !digit(sh.bins + kBins, 10, 0x7FFu, 0xFFE00000u))
    digit(sh.bins + 2 * kBins, 0, 0x3FFu, 0xFFFFFC00u);
  // kept slots in order: those above the key and, of its equals, the first `left`
  uint32_t n = 0, ne = 0;
  each([&](int32_t, uint32_t k) {
    n += (uint32_t)__popcll(__ballot(k > key));
    ne += (uint32_t)__popcll(__ballot(k == key));
  });
  if (lane == 0) {
    sh.wave[wave] = n;
    sh.equal[wave] = ne;
  }
  __syncthreads();
  n = ne = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    n += i < wave ? sh.wave[i] : 0u;
    ne += i < wave ? sh.equal[i] : 0u;
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  each([&](int32_t i, uint32_t k) {
    const uint64_t more = __ballot(k > key), equal = __ballot(k == key);
    const uint32_t rank = ne + (uint32_t)__popcll(equal & below);   // among the equal ones
    if (k > key || (k == key && rank < left))
      kept[n + (uint32_t)__popcll(more & below) + min(rank, left)] = i + lane;
    n += (uint32_t)__popcll(more);
    ne += (uint32_t)__popcll(equal);
  });
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_choose_kernel(EvictArgs g) {
  __shared__ ChooseShared<THREADS> sh;
  const int b = (int)(blockIdx.x / (uint32_t)g.kv_heads), hk = (int)blockIdx.x - b * g.kv_heads;
  const int32_t len = seq_len(g.lens, b, g.skv);
  int32_t* kept = g.kept + (int64_t)blockIdx.x * g.budget;
  if (hk == 0 && threadIdx.x == 0) g.evicted[b] = max(len - g.budget, 0);
  if (len <= g.budget) {
    for (int32_t i = threadIdx.x; i < g.budget; i += THREADS) kept[i] = i < len ? i : -1;
    return;
  }
  const float* w = g.weight + b * g.st.weight[0] + hk * g.st.weight[1];
  if (THREADS == 256 || len <= kHeld * THREADS) {    // 256 threads are launched for no longer rows
    choose_slots<THREADS, kHeld>(g, w, len, kept, sh);
  } else if constexpr (THREADS > 256) {
    if (len <= kHeldLong * THREADS)
      choose_slots<THREADS, kHeldLong>(g, w, len, kept, sh);
    else
      choose_slots<THREADS, 0>(g, w, len, kept, sh);
  }
}

constexpr int kMvEach = 4, kCopyEach = 8;

// How many of kept[0 .. n) there are (the rest is -1 and behind them), by one wave.
__device__ __forceinline__ int32_t count_kept(const int32_t* kept, int32_t n) {
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, hi = n;                            // kept[lo - 1] is one, kept[hi] is none
  while (lo < hi) {
    const int32_t step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int32_t m = (int32_t)__popcll(__ballot(i < hi && kept[min(i, n - 1)] >= 0));
    // probes 0 .. m - 1 are there, probe m is not
    const int32_t top = lo + m * step;
    lo = m == 0 ? lo : lo + (m - 1) * step + 1;
    hi = m == 0 ? lo : min(hi, top);
  }
  return lo;
}
__device__ __forceinline__ void put_length(const EvictArgs& g, int b, int hk, const int32_t* kept) {
  if (hk > 0 || g.lens_out == nullptr || threadIdx.x >= 64) return;
  const int32_t n = count_kept(kept, g.budget);
  if (threadIdx.x == 0) g.lens_out[b] = n;
}

// Weights [i, end) of a key head's kept slots; IN: in place, as shift_rows.
template <int THREADS, bool IN>
__device__ __forceinline__ void move_weights(const EvictArgs& g, const float* w, float* wo, const int32_t* kept,
                                             int32_t i, int32_t end) {
  for (; i < end; i += THREADS * kMvEach) {
    float x[kMvEach];
    int32_t from[kMvEach];
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      const int32_t k = i + j * THREADS + (int32_t)threadIdx.x;
      from[j] = k < end ? kept[k] : -1;
    }
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) x[j] = from[j] >= 0 ? w[from[j]] : 0.0f;
    if (IN) {
#pragma unroll
      for (int j = 0; j < kMvEach; ++j) asm volatile("" : "+v"(x[j]));
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      const int32_t k = i + j * THREADS + (int32_t)threadIdx.x;
      if (k < end) wo[k] = x[j];
    }
  }
}

// Rows [i, end) of a slice of K or V of one key head: a thread's chunk of a row, kMvEach rows
// at a time.
struct RowsOf {
  uint32_t rows, r, c;      // rows at a time (the last threads may have none), this thread's
  __device__ __forceinline__ RowsOf(uint32_t threads, uint32_t width) {
    rows = threads / width;
    r = threadIdx.x / width;
    c = threadIdx.x - r * width;
  }
};
template <int THREADS>
__device__ __forceinline__ void copy_rows(const char* src, char* dst, int64_t ss, int64_t sd, const int32_t* kept,
                                          int32_t i, int32_t end, uint32_t c0, uint32_t width) {
  const RowsOf t(THREADS, width);
  src += 16 * (int64_t)(c0 + t.c);
  dst += 16 * (int64_t)(c0 + t.c);
  const int32_t any = kept[0];                       // what is read in the place of none
  if (t.r >= t.rows || any < 0) return;              // a cache may have no slot at all
  for (int32_t k0 = i + (int32_t)t.r; k0 < end; k0 += (int32_t)(kCopyEach * t.rows)) {
    int32_t from[kCopyEach];
    u32x4 x[kCopyEach];
#pragma unroll
    for (int j = 0; j < kCopyEach; ++j) from[j] = kept[min(k0 + (int32_t)(j * t.rows), end - 1)];
#pragma unroll
    for (int j = 0; j < kCopyEach; ++j)
      x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (from[j] < 0 ? any : from[j]) * ss));
#pragma unroll
    for (int j = 0; j < kCopyEach; ++j) {
      const int32_t k = k0 + (int32_t)(j * t.rows);
      if (k < end && from[j] >= 0) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4*>(dst + k * sd));
    }
  }
}
// In place: a round's rows are all read before one is written, and the next round's are on
// their way meanwhile.
template <int THREADS>
__device__ __forceinline__ void shift_rows(char* at, int64_t stride, const int32_t* kept, int32_t end, uint32_t c0,
                                           uint32_t width) {
  const RowsOf t(THREADS, width);
  at += 16 * (int64_t)(c0 + t.c);
  int32_t from[kMvEach], next[kMvEach];
  u32x4 x[kMvEach], y[kMvEach];
  const int32_t step = (int32_t)(kMvEach * t.rows);
  const auto read = [&](int32_t k0, int32_t (&f)[kMvEach], u32x4 (&v)[kMvEach]) {
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      const int32_t k = k0 + (int32_t)(j * t.rows + t.r);
      f[j] = t.r < t.rows && k < end ? kept[k] : -1;
      if (f[j] == k) f[j] = -1;                      // stays where it is
    }
#pragma unroll
    for (int j = 0; j < kMvEach; ++j)
      v[j] = f[j] >= 0 ? *reinterpret_cast<const u32x4*>(at + f[j] * stride) : u32x4{0u, 0u, 0u, 0u};
  };
  read(0, from, x);
  for (int32_t k0 = 0; k0 < end; k0 += step) {
    read(k0 + step, next, y);
    // these are in registers, in every wave
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) asm volatile("" : "+v"(x[j]));
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      if (from[j] >= 0)
        *reinterpret_cast<u32x4*>(at + (int64_t)(k0 + (int32_t)(j * t.rows + t.r)) * stride) = x[j];
      from[j] = next[j];
      x[j] = y[j];
    }
  }
}

// In place: slices of rows, and the weights, a workgroup each; rows that stay are not moved.
// 2048 of the 2560 keys of 64 x 8 key heads (dim 128), whose kept keys are spread over the
// cache: 225 us, where copying them takes 203; of 64 sequences of 1536 to 2560 keys, of which
// those up to 2048 stay, 126, and 197; 2048 of the 16384 keys of 8 key heads 12, and 7: there
// few workgroups go through rounds, a barrier and the memory's latency each.
constexpr int kInThreads = 1024;
__global__ __launch_bounds__(kInThreads) void evict_shift_kernel(EvictArgs g) {
  const uint32_t parts = 2u * (uint32_t)g.slices + 1u;
  const uint32_t bh = blockIdx.x / parts, part = blockIdx.x - bh * parts;
  const int b = (int)(bh / (uint32_t)g.kv_heads), hk = (int)bh - b * g.kv_heads;
  const int32_t* kept = g.kept + (int64_t)bh * g.budget;
  if (part == parts - 1u) {
    float* w = g.wo + b * g.st.weight_out[0] + hk * g.st.weight_out[1];
    put_length(g, b, hk, kept);
    move_weights<kInThreads, true>(g, w, w, kept, 0, g.budget);
    for (int32_t i = g.budget + (int32_t)threadIdx.x; i < g.slots; i += kInThreads) w[i] = 0.0f;
    return;
  }
  const bool value = part >= (uint32_t)g.slices;
  const uint32_t c0 = (part - (value ? (uint32_t)g.slices : 0u)) * (uint32_t)g.slice;
  const auto pick = [&](int64_t of_k, int64_t of_v) { return value ? of_v : of_k; };
  char* at = (value ? g.vo : g.ko) + b * pick(g.st.k[0], g.st.v[0]) + hk * pick(g.st.k[2], g.st.v[2]);
  shift_rows<kInThreads>(at, pick(g.st.k[1], g.st.v[1]), kept, g.budget, c0, min((uint32_t)g.slice, (uint32_t)g.row16 - c0));
}

// Into another cache: runs of g.slice rows of K, with their weights, and of V. Memory bounds
// it: 2048 of 2560 keys of 64 x 8 key heads (dim 128, 1.03 GB) 187 to 197 us, 5.2 to 5.5 TB/s.
constexpr int kCopyThreads = 256;
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(EvictArgs g) {
  const uint32_t parts = 2u * (uint32_t)g.slices;
  const uint32_t bh = blockIdx.x / parts, part = blockIdx.x - bh * parts;
  const int b = (int)(bh / (uint32_t)g.kv_heads), hk = (int)bh - b * g.kv_heads;
  const int32_t* kept = g.kept + (int64_t)bh * g.budget;
  const bool value = part >= (uint32_t)g.slices;
  const int32_t i = (int32_t)(part - (value ? (uint32_t)g.slices : 0u)) * g.slice, end = min(i + g.slice, g.budget);
  const auto pick = [&](int64_t of_k, int64_t of_v) { return value ? of_v : of_k; };
  const char* src = (value ? g.v : g.k) + b * pick(g.st.k[0], g.st.v[0]) + hk * pick(g.st.k[2], g.st.v[2]);
  char* dst = (value ? g.vo : g.ko) + b * pick(g.st.k_out[0], g.st.v_out[0]) + hk * pick(g.st.k_out[2], g.st.v_out[2]);
  for (uint32_t c0 = 0; c0 < (uint32_t)g.row16; c0 += kCopyThreads)
    copy_rows<kCopyThreads>(src, dst, pick(g.st.k[1], g.st.v[1]), pick(g.st.k_out[1], g.st.v_out[1]), kept, i, end, c0, min((uint32_t)g.row16 - c0, (uint32_t)kCopyThreads));
  if (!value) {
    const float* w = g.weight + b * g.st.weight[0] + hk * g.st.weight[1];
    float* wo = g.wo + b * g.st.weight_out[0] + hk * g.st.weight_out[1];
    move_weights<kCopyThreads, false>(g, w, wo, kept, i, end);
    if (i == 0) {
      put_length(g, b, hk, kept);
      for (int32_t j = g.budget + (int32_t)threadIdx.x; j < g.slots; j += kCopyThreads) wo[j] = 0.0f;
    }
  }
}

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_cache_evict(const void* k, const void* v, const float* weight,
                                          const int32_t* kv_lens, void* k_out, void* v_out,
                                          float* weight_out, int32_t* lens_out, int32_t* kept,
                                          int32_t* evicted, int64_t batch, int64_t skv, int64_t slots,
                                          int64_t kv_heads, int64_t dim,
                                          const quake_evict_strides* strides, int64_t budget,
                                          int64_t sinks, int64_t recent, quake_dtype dtype,
                                          void* stream) {
  if (!valid_dtype(dtype)) return QUAKE_EDTYPE;
  const int64_t e = elem_size(dtype), chunk = 16 / e;
  if (batch < 0 || skv < 0 || kv_heads < 1 || dim < 1 || dim % chunk != 0 || dim > 4096) return QUAKE_EINVAL;
  if (skv > (1 << 30) || slots > (1 << 30) || batch > (1 << 20) || kv_heads > (1 << 16) ||
      batch * kv_heads > (1 << 20))
    return QUAKE_EINVAL;
  if (budget < 1 || budget > slots || sinks < 0 || recent < 0 || sinks > budget || recent > budget - sinks)
    return QUAKE_EINVAL;
  if (batch == 0) return QUAKE_OK;
  if (strides == nullptr || k_out == nullptr || v_out == nullptr || weight_out == nullptr ||
      kept == nullptr || evicted == nullptr)
    return QUAKE_EINVAL;
  if (skv > 0 && (k == nullptr || v == nullptr || weight == nullptr)) return QUAKE_EINVAL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_out) || !aligned16(v_out) ||
      (((uintptr_t)weight | (uintptr_t)weight_out | (uintptr_t)kv_lens | (uintptr_t)lens_out |
        (uintptr_t)kept | (uintptr_t)evicted) & 3u) != 0)
    return QUAKE_EINVAL;
  const quake_evict_strides& st = *strides;
  const int64_t ni[3] = {batch, skv, kv_heads}, no[3] = {batch, slots, kv_heads}, nw[2] = {batch, kv_heads};
  for (const int64_t* x : {st.k, st.v, st.k_out, st.v_out}) {
    const int64_t* n = x == st.k || x == st.v ? ni : no;
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && (x[i] < 0 || x[i] % chunk != 0 || x[i] > INT64_MAX / 32 / n[i])) return QUAKE_EINVAL;
  }
  for (const int64_t* x : {st.weight, st.weight_out})
    for (int i = 0; i < 2; ++i)
      if (nw[i] > 1 && (x[i] < 0 || x[i] > INT64_MAX / 32 / nw[i])) return QUAKE_EINVAL;
  // rows that are written: apart, also K's from V's where the two interleave
  if (!rows_apart(st.k_out, no, 3, dim) || !rows_apart(st.v_out, no, 3, dim) ||
      !rows_apart(st.weight_out, nw, 2, slots))
    return QUAKE_EINVAL;
  const auto same = [](const int64_t* a, const int64_t* b, const int64_t* n, int count) {
    for (int i = 0; i < count; ++i)
      if (n[i] > 1 && a[i] != b[i]) return false;
    return true;
  };
  const int64_t ki = span_bytes(st.k, ni, 3, dim, e), vi = span_bytes(st.v, ni, 3, dim, e);
  const int64_t ko = span_bytes(st.k_out, no, 3, dim, e), vo = span_bytes(st.v_out, no, 3, dim, e);
  const int64_t wi = span_bytes(st.weight, nw, 2, skv, 4), wo = span_bytes(st.weight_out, nw, 2, slots, 4);
  if (meet(k_out, ko, v_out, vo)) {
    const char *a = std::min((const char*)k_out, (const char*)v_out), *z = std::max((const char*)k_out, (const char*)v_out);
    const int64_t s4[4] = {st.k_out[0], st.k_out[1], st.k_out[2], (z - a) / e}, n4[4] = {no[0], no[1], no[2], 2};
    if (!same(st.k_out, st.v_out, no, 3) || !rows_apart(s4, n4, 4, dim)) return QUAKE_EINVAL;
  }
  // in place as a whole, or into a cache of its own
  if (k_out == k || v_out == v || weight_out == weight) {
    if (k_out != k || v_out != v || weight_out != weight || slots != skv || !same(st.k, st.k_out, ni, 3) ||
        !same(st.v, st.v_out, ni, 3) || !same(st.weight, st.weight_out, nw, 2))
      return QUAKE_EINVAL;
    if (meet(weight_out, wo, k, ki) || meet(weight_out, wo, v, vi)) return QUAKE_EINVAL;
  } else {
    const std::pair<const void*, int64_t> ins[] = {{k, ki}, {v, vi}, {weight, wi}};
    for (const auto& [p, n] : ins)
      if (meet(k_out, ko, p, n) || meet(v_out, vo, p, n) || meet(weight_out, wo, p, n)) return QUAKE_EINVAL;
    if (meet(weight_out, wo, k_out, ko) || meet(weight_out, wo, v_out, vo)) return QUAKE_EINVAL;
  }
  const int64_t nkept = 4 * batch * kv_heads * budget;
  const std::pair<const void*, int64_t> outs[] = {{kept, nkept}, {evicted, 4 * batch}, {lens_out, 4 * batch}};
  for (const auto& [p, n] : outs) {
    if (meet(p, n, k, ki) || meet(p, n, v, vi) || meet(p, n, weight, wi) || meet(p, n, k_out, ko) ||
        meet(p, n, v_out, vo) || meet(p, n, weight_out, wo))
      return QUAKE_EINVAL;
  }
  if (meet(kept, nkept, evicted, 4 * batch)) return QUAKE_EINVAL;
  for (const int32_t* p : {(const int32_t*)kv_lens, (const int32_t*)lens_out})
    if (meet(kept, nkept, p, 4 * batch) || meet(evicted, 4 * batch, p, 4 * batch)) return QUAKE_EINVAL;
  if (lens_out != kv_lens && meet(lens_out, 4 * batch, kv_lens, 4 * batch)) return QUAKE_EINVAL;
  if (kv_lens != nullptr && (meet(kv_lens, 4 * batch, k_out, ko) || meet(kv_lens, 4 * batch, v_out, vo) ||
                             meet(kv_lens, 4 * batch, weight_out, wo)))
    return QUAKE_EINVAL;
  EvictArgs g{};
  g.k = static_cast<const char*>(k);
  g.v = static_cast<const char*>(v);
  g.weight = weight;
  g.lens = kv_lens;
  g.ko = static_cast<char*>(k_out);
  g.vo = static_cast<char*>(v_out);
  g.wo = weight_out;
  g.lens_out = lens_out;
  g.kept = kept;
  g.evicted = evicted;
  g.st = st;
  for (int64_t* x : {g.st.k, g.st.v, g.st.k_out, g.st.v_out})
    for (int i = 0; i < 3; ++i) x[i] *= e;
  g.skv = (int32_t)skv;
  g.slots = (int32_t)slots;
  g.kv_heads = (int32_t)kv_heads;
  g.budget = (int32_t)budget;
  g.sinks = (int32_t)sinks;
  g.recent = (int32_t)recent;
  g.row16 = (int32_t)(dim * e / 16);
  const int64_t heads = batch * kv_heads;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  // four waves a row where its slots fit their registers, which leaves room for more rows
  if (skv <= kHeld * 256)
    hipLaunchKernelGGL(evict_choose_kernel<256>, dim3((uint32_t)heads), dim3(256), 0, s, g);
  else
    hipLaunchKernelGGL(evict_choose_kernel<1024>, dim3((uint32_t)heads), dim3(1024), 0, s, g);
  if (k_out == k) {
    // a row whole where there are heads enough, else in up to as many slices as fill the GPU
    g.slice = (int32_t)std::max<int64_t>(g.row16 * 2 * heads / 512, std::min(g.row16, 4));
    g.slice = std::min(g.slice, g.row16);
    g.slices = (g.row16 + g.slice - 1) / g.slice;
    hipLaunchKernelGGL(evict_shift_kernel, dim3((uint32_t)(heads * (2 * g.slices + 1))), dim3(kInThreads), 0, s, g);
  } else {
    // runs of about 64 KiB, of fewer where that leaves the GPU idle
    int64_t rows = std::max<int64_t>(1, (1 << 16) / (dim * e));
    rows = std::max<int64_t>(std::min(rows, budget * heads * 2 / 1024), std::max<int64_t>(1, 4096 / (dim * e)));
    rows = std::max(rows, budget * heads / (1 << 22) + 1);       // a launch takes fewer than 2^32 threads
    g.slice = (int32_t)std::min(rows, budget);
    g.slices = (int32_t)((budget + g.slice - 1) / g.slice);
    hipLaunchKernelGGL(evict_copy_kernel, dim3((uint32_t)(heads * 2 * g.slices)), dim3(kCopyThreads), 0, s, g);
  }
  return launch_status();
}
