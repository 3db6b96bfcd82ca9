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
  int32_t row16, slice, slices;            // 16-byte chunks of a row, of a slice; slices of a row
};

constexpr int kEvThreads = 1024, kEvWaves = kEvThreads / 64, kEvBins = 2048;

// weights in ascending order as unsigned: NaN below all, -0 as 0
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = as_u(w == 0.0f ? 0.0f : w);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// One workgroup a sequence and key head.
__global__ __launch_bounds__(kEvThreads) void evict_choose_kernel(EvictArgs g) {
  __shared__ uint32_t s_bin[kEvBins];
  __shared__ uint32_t s_wave[kEvWaves], s_eq[kEvWaves], s_found[2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hk = blockIdx.x % (uint32_t)g.kv_heads, b = blockIdx.x / (uint32_t)g.kv_heads;
  const int32_t len = seq_len(g.lens, b, g.skv);
  int32_t* kept = g.kept + (int64_t)blockIdx.x * g.budget;
  if (hk == 0 && threadIdx.x == 0) g.evicted[b] = max(len - g.budget, 0);
  if (len <= g.budget) {
    for (int32_t i = threadIdx.x; i < g.budget; i += kEvThreads) kept[i] = i < len ? i : -1;
    return;
  }
  const float* w = g.weight + b * g.st.weight[0] + hk * g.st.weight[1];
  const int32_t lo = g.sinks, hi = len - g.recent;
  // the key of the last one that fits, and how many of its equals do
  uint32_t key = 0xFFFFFFFFu, left = (uint32_t)(g.budget - g.sinks - g.recent);
  if (left > 0) {
    uint32_t mask = 0;
    key = 0;
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {
      const uint32_t digit = shift == 0 ? 0x3FFu : 0x7FFu;
      for (int i = threadIdx.x; i < kEvBins; i += kEvThreads) s_bin[i] = 0;
      __syncthreads();
      for (int32_t i = lo + (int32_t)threadIdx.x; i < hi; i += kEvThreads) {
        const uint32_t u = weight_key(w[i]);
        if ((u & mask) == key) atomicAdd(&s_bin[(u >> shift) & digit], 1u);
      }
      __syncthreads();
      // thread t: bins 2047 - 2 t and the one below, from the top
      const int top = kEvBins - 1 - 2 * (int)threadIdx.x;
      const uint32_t a = s_bin[top], z = s_bin[top - 1];
      uint32_t upto = a + z;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t other = __shfl_up(upto, o, 64);
        upto += lane >= o ? other : 0u;
      }
      if (lane == 63) s_wave[wave] = upto;
      __syncthreads();
      for (int i = 0; i < wave; ++i) upto += s_wave[i];
      const uint32_t above = upto - a - z;          // in the bins above both
      if (above < left && left <= upto) {
        const bool first = left <= above + a;
        s_found[0] = (uint32_t)(first ? top : top - 1);
        s_found[1] = first ? above : above + a;
      }
      __syncthreads();
      key |= s_found[0] << shift;
      mask |= digit << shift;
      left -= s_found[1];
    }
  }
  // kept slots in order; a wave takes a run of them
  const int32_t run = (len + kEvThreads - 1) / kEvThreads * 64;
  const int32_t from = wave * run, to = min(from + run, len);
  auto look = [&](int32_t i, uint64_t& more, uint64_t& equal) {
    const bool in = i < to, mid = in && i >= lo && i < hi;
    const uint32_t u = mid ? weight_key(w[i]) : 0u;
    more = __ballot(in && (!mid || u > key));
    equal = __ballot(mid && u == key && left > 0);
  };
  uint32_t n = 0, ne = 0;
  for (int32_t i = from; i < to; i += 64) {
    uint64_t more, equal;
    look(i + lane, more, equal);
    n += (uint32_t)__popcll(more);
    ne += (uint32_t)__popcll(equal);
  }
  __syncthreads();
  if (lane == 0) {
    s_wave[wave] = n;
    s_eq[wave] = ne;
  }
  __syncthreads();
  n = ne = 0;
  for (int i = 0; i < wave; ++i) {
    n += s_wave[i];
    ne += s_eq[i];
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int32_t i = from; i < to; i += 64) {
    uint64_t more, equal;
    look(i + lane, more, equal);
    const uint32_t rank = ne + (uint32_t)__popcll(equal & below);   // among the equal ones
    const bool mine = ((more >> lane) & 1) != 0 || (((equal >> lane) & 1) != 0 && rank < left);
    const uint32_t at = n + (uint32_t)__popcll(more & below) + min(rank, left);
    if (mine) kept[at] = i + lane;
    n += (uint32_t)__popcll(more);
    ne += (uint32_t)__popcll(equal);
  }
}

constexpr int kMvThreads = 256, kMvEach = 4;

// A slice of the rows of K or V of one key head, or its weights, by one workgroup.
__global__ __launch_bounds__(kMvThreads) void evict_move_kernel(EvictArgs g) {
  const uint32_t parts = 2u * (uint32_t)g.slices + 1u;
  const uint32_t part = blockIdx.x % parts, bh = blockIdx.x / parts;
  const int hk = bh % (uint32_t)g.kv_heads, b = bh / (uint32_t)g.kv_heads;
  const int32_t* kept = g.kept + (int64_t)bh * g.budget;
  if (part == parts - 1u) {
    const float* w = g.weight + b * g.st.weight[0] + hk * g.st.weight[1];
    float* wo = g.wo + b * g.st.weight_out[0] + hk * g.st.weight_out[1];
    int32_t n = 0;                                   // kept
    for (int32_t i0 = 0; i0 < g.budget; i0 += kMvThreads * kMvEach) {
      float x[kMvEach];
      int32_t live = 0;
#pragma unroll
      for (int j = 0; j < kMvEach; ++j) {
        const int32_t i = i0 + j * kMvThreads + (int32_t)threadIdx.x;
        const int32_t from = i < g.budget ? kept[i] : -1;
        x[j] = from >= 0 ? w[from] : 0.0f;
        live += from >= 0;
      }
      n += live;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMvEach; ++j) {
        const int32_t i = i0 + j * kMvThreads + (int32_t)threadIdx.x;
        if (i < g.budget) wo[i] = x[j];
      }
    }
    for (int32_t i = g.budget + (int32_t)threadIdx.x; i < g.slots; i += kMvThreads) wo[i] = 0.0f;
    if (hk == 0 && g.lens_out != nullptr) {
      __shared__ int32_t s_n[kMvThreads / 64];
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o, 64);
      if ((threadIdx.x & 63) == 0) s_n[threadIdx.x >> 6] = n;
      __syncthreads();
      if (threadIdx.x == 0) {
        for (int i = 1; i < kMvThreads / 64; ++i) n += s_n[i];
        g.lens_out[b] = n;
      }
    }
    return;
  }
  const bool value = part >= (uint32_t)g.slices;
  const uint32_t c0 = (part - (value ? (uint32_t)g.slices : 0u)) * (uint32_t)g.slice;
  const int64_t* si = value ? g.st.v : g.st.k;
  const int64_t* so = value ? g.st.v_out : g.st.k_out;
  const char* src = (value ? g.v : g.k) + b * si[0] + hk * si[2];
  char* dst = (value ? g.vo : g.ko) + b * so[0] + hk * so[2];
  const bool same = src == dst;
  const int64_t ss = si[1], sd = so[1];
  const uint32_t width = min((uint32_t)g.slice, (uint32_t)g.row16 - c0);
  const uint64_t all = (uint64_t)g.budget * width;
  for (uint64_t e0 = 0; e0 < all; e0 += kMvThreads * kMvEach) {
    u32x4 x[kMvEach];
    int32_t from[kMvEach];
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      const uint64_t e = e0 + (uint32_t)(j * kMvThreads) + threadIdx.x;
      const int32_t i = (int32_t)(e / width);
      const uint32_t c = (uint32_t)(e % width);
      from[j] = e < all ? kept[i] : -1;
      if (same && from[j] == i) from[j] = -1;        // stays where it is
      if (from[j] >= 0) x[j] = *reinterpret_cast<const u32x4*>(src + from[j] * ss + 16 * (int64_t)(c0 + c));
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMvEach; ++j) {
      const uint64_t e = e0 + (uint32_t)(j * kMvThreads) + threadIdx.x;
      const int32_t i = (int32_t)(e / width);
      const uint32_t c = (uint32_t)(e % width);
      if (from[j] >= 0) *reinterpret_cast<u32x4*>(dst + i * sd + 16 * (int64_t)(c0 + c)) = x[j];
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
  const uint32_t heads = (uint32_t)(batch * kv_heads);
  g.slice = heads >= 256 ? g.row16 : std::min(g.row16, 4);
  g.slices = (g.row16 + g.slice - 1) / g.slice;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(evict_choose_kernel, dim3(heads), dim3(kEvThreads), 0, s, g);
  hipLaunchKernelGGL(evict_move_kernel, dim3(heads * (2u * (uint32_t)g.slices + 1u)), dim3(kMvThreads), 0, s, g);
  return launch_status();
}
