// shared.hip — quake_attention_shared: attention of a batch whose sequences share a
// prefix, o_i = sum_j p_ij v_j / sum_j p_ij over the prefix's keys, all of which every
// query sees, and the sequence's own keys j <= pos_i; and the weight that each own key
// gathers, weight_j += sum_i p_ij / sum_j p_ij over the rows of a key head.
//
// The exponentials are QuAKE's (arXiv:2412.00408) against a whole number M of base-2
// units, Q(y - M) = 2^-M Q(y) exactly, as in quake_attention_window: results over
// different keys are brought to one M by exact powers of two.
//
// Rows: the queries of all heads that share a key head, row r = query r / group, head
// r mod group of the group. Keys: blocks of 32, the prefix's first, then the
// sequence's own. Products as cache_tile.hpp describes them: a lane holds row
// l mod 32 of a tile and keys 8 g + 4 (l / 32) + i of a block, i, g < 4.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cache_tile.hpp"
#include "quake_device.hpp"
#include "quake_host.hpp"

namespace qk {

constexpr int kShWaves = 4;

struct SharedArgs {
  const uint16_t *q, *pk, *pv, *k, *v;
  uint16_t* o;
  float* weight;                                // or null
  const int32_t *prefix_lens, *q_lens, *kv_lens;   // or null: sp, sq, skv
  float2* stats;                                // of a row: M, 1 / sum of p; weight only
  quake_shared_strides st;
  int32_t sq, sp, skv, group, kv_heads, members, tiles;
  float c0;                                     // 2^23 t / ln2 (EXACT: t / ln2)
};

// Loads ROWS keys from n0 on into LDS rows, as a cache's keys lie one after the other
// (1024 bytes a load: 64 lanes x 16; ROWS a multiple of 16, the period of the
// swizzles). The last of the n keys stands for those behind it, whose probabilities
// are 0.
template <int D, bool IS_V, int ROWS>
__device__ __forceinline__ void stage_run(uint32_t lds, const uint16_t* base, int64_t stride,
                                          int32_t n0, int32_t n, int lane) {
  constexpr int CH = D / 8, RPL = 64 / CH, N = ROWS / RPL;   // chunks a row, rows a load, loads
  const int r = lane / CH, pc = lane % CH;
  asm volatile("" : "+s"(lds));   // else its sums are kept in vector registers, which M0 cannot take
  if (n0 + ROWS <= n) {
    const char* b = scalar_base(base + (int64_t)n0 * stride);
    const uint32_t row = (uint32_t)r * (uint32_t)stride * 2u;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int sw = IS_V ? vswizzle<D>(RPL * j + r) : kswizzle<D>(RPL * j + r);
      lds_load16(lds + 1024 * j, row + 16u * (uint32_t)(pc ^ sw), b + (int64_t)2 * RPL * j * stride);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int sw = IS_V ? vswizzle<D>(RPL * j + r) : kswizzle<D>(RPL * j + r);
      lds_load16(lds + 1024 * j, base + (int64_t)min(n0 + RPL * j + r, n - 1) * stride + 8 * (pc ^ sw));
    }
  }
}

// -inf for the keys of the block from n0 on that lie behind key `lim`
__device__ __forceinline__ void hide_behind(f32x16& s, int32_t n0, int32_t lim, int h) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = n0 + 8 * (r >> 2) + 4 * h + (r & 3) <= lim ? s[r] : -INFINITY;
}

// sum of 16 values in pairs of pairs
__device__ __forceinline__ float sum16(const float (&e)[16]) {
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = e[2 * i] + e[2 * i + 1];
#pragma unroll
  for (int n = 4; n > 0; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) s[i] += s[i + n];
  return s[0];
}

// A tile of 32 rows of one sequence in one workgroup; the waves take every fourth block
// of its keys and join at the end. K's next block is on its way while V of this one is
// used, and the other way round.
template <int DT, int MODE, int D, bool WEIGH>
__global__ __launch_bounds__(64 * kShWaves, 2) void shared_few_kernel(SharedArgs g) {
  constexpr int kBlk = 64 * D;                      // bytes of a block of 32 rows
  constexpr int kWave = 2 * kBlk;                   // K and V
  __shared__ __attribute__((aligned(16))) char s_buf[kShWaves * kWave];
  __shared__ float s_m[kShWaves][32], s_sum[kShWaves][32], s_all[kShWaves][32];

  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.x % (uint32_t)g.tiles;
  const uint32_t bh = blockIdx.x / (uint32_t)g.tiles;
  const int hk = bh % (uint32_t)g.kv_heads, b = bh / (uint32_t)g.kv_heads;
  const int grp = b / g.members;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t plen = g.sp == 0 ? 0 : seq_len(g.prefix_lens, grp, g.sp);
  const int32_t rows = qlen * g.group, r0 = 32 * tile;
  if (r0 >= rows) return;
  const int32_t row = min(r0 + fr, rows - 1);
  const int32_t off = kvlen - qlen;                 // position of query 0
  const int32_t query = row / g.group, head = hk * g.group + row % g.group;
  const int32_t pos = off + query;
  const int32_t first = off + r0 / g.group, last = off + min(r0 + 31, rows - 1) / g.group;
  const int32_t pblocks = (plen + 31) >> 5, own = last < 0 ? 0 : last + 1;
  const int32_t blocks = pblocks + ((own + 31) >> 5);

  u32x4 qf[D / 16];
  {
    const uint16_t* qr = g.q + b * g.st.q[0] + query * g.st.q[1] + head * g.st.q[2] + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const u32x4*>(qr + 16 * ks);
  }
  settle(qf);
  const uint16_t* PK = g.pk + grp * g.st.prefix_k[0] + hk * g.st.prefix_k[2];
  const uint16_t* PV = g.pv + grp * g.st.prefix_v[0] + hk * g.st.prefix_v[2];
  const uint16_t* K = g.k + b * g.st.k[0] + hk * g.st.k[2];
  const uint16_t* V = g.v + b * g.st.v[0] + hk * g.st.v[2];
  char* buf = s_buf + wave * kWave;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf + wave * kWave);
  auto load_k = [&](int32_t n) {
    const bool p = n < pblocks;
    stage_run<D, false, 32>(lds, p ? PK : K, p ? g.st.prefix_k[1] : g.st.k[1], 32 * (p ? n : n - pblocks),
                            p ? plen : own, lane);
  };
  auto load_v = [&](int32_t n) {
    const bool p = n < pblocks;
    stage_run<D, true, 32>(lds + kBlk, p ? PV : V, p ? g.st.prefix_v[1] : g.st.v[1], 32 * (p ? n : n - pblocks),
                           p ? plen : own, lane);
  };

  RowAcc<D> acc;
  acc.sum = 0.0f;
  acc.m = kNoMax;
  float all = 0.0f;                                 // of p as it is, not rounded to 16 bits
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc.o[d] = f32x16{};
  constexpr int kLoads = D / 16;                    // of a block's K or V
  if (wave < blocks) {
    load_k(wave);
    load_v(wave);
  }
  for (int32_t n = wave; n < blocks; n += kShWaves) {
    const bool more = n + kShWaves < blocks;
    wait_loads<kLoads>();                           // K is here, V may be on its way
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = wmma<DT>(read_k<D>(buf, fr, h, ks), qf[ks], s);
    wait_lds();                                     // K's reads, before it is loaded again
    if (more) load_k(n + kShWaves);
    const bool p = n < pblocks;
    const int32_t n0 = 32 * (p ? n : n - pblocks);
    if (n0 + 31 > (p ? plen - 1 : first)) hide_behind(s, n0, p ? plen - 1 : pos, h);
    const float top = block_top<MODE>(s, g.c0);
    if (__any(top > acc.m + (kLift<DT> + kLazy))) {
      const int32_t e = raise_max<DT>(top, acc);
      if constexpr (WEIGH) all = __builtin_amdgcn_ldexpf(all, e);
    }
    const float c1 = row_c1<MODE>(acc.m);
    u32x4 pr[2];
    if constexpr (WEIGH) {
      float e[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) e[r] = qexp_row<MODE, true>(s[r], g.c0, c1);
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const uint32_t w = wpack<DT>(e[r], e[r + 1]);
        acc.sum = wsum<DT>(w, acc.sum);
        pr[r >> 3][(r >> 1) & 3] = w;
      }
      all += sum16(e);
    } else {
#pragma unroll
      for (int r = 0; r < 16; r += 2)
        pr[r >> 3][(r >> 1) & 3] = prob_pair<DT, MODE>(s, r, g.c0, c1, acc.sum);
    }
    if (more)
      wait_loads<kLoads>();                         // V is here, the next K may be on its way
    else
      wait_loads<0>();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        acc.o[d] = wmma<DT>(read_v<D>(buf + kBlk, lane, ks, d), pr[ks], acc.o[d]);
    wait_lds();
    if (more) load_v(n + kShWaves);
  }

  // join the waves: their M, then sums and O^T brought to the largest M
  acc.sum += other_half(acc.sum);
  if constexpr (WEIGH) all += other_half(all);
  __syncthreads();
  if (lane < 32) {
    s_m[wave][fr] = acc.m;
    s_sum[wave][fr] = acc.sum;
    if constexpr (WEIGH) s_all[wave][fr] = all;
  }
  float* part = reinterpret_cast<float*>(s_buf + wave * kWave);   // [D][32] floats
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      part[(32 * d + 8 * (r >> 2) + 4 * h + (r & 3)) * 32 + fr] = acc.o[d][r];
  __syncthreads();
  float m = s_m[0][fr];
#pragma unroll
  for (int w = 1; w < kShWaves; ++w) m = fmaxf(m, s_m[w][fr]);
  float sum = 0.0f, every = 0.0f;
  int32_t e[kShWaves];
#pragma unroll
  for (int w = 0; w < kShWaves; ++w) {
    e[w] = down_shift(s_m[w][fr], m);
    sum += __builtin_amdgcn_ldexpf(s_sum[w][fr], e[w]);
    if constexpr (WEIGH) every += __builtin_amdgcn_ldexpf(s_all[w][fr], e[w]);
  }
  // this wave's dims: D / 4, each half of its lanes D / 8 of them
  constexpr int N = D / 8;
  const int d0 = wave * (D / 4) + h * N;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kShWaves; ++w)
      v[i] += __builtin_amdgcn_ldexpf(
          reinterpret_cast<const float*>(s_buf + w * kWave)[(d0 + i) * 32 + fr], e[w]);
  }
  if (r0 + fr >= rows) return;
  if constexpr (WEIGH) {
    if (wave == 0 && h == 0)
      g.stats[(int64_t)bh * g.sq * g.group + r0 + fr] =
          every > 0.0f ? float2{m, 1.0f / every} : float2{0.0f, 0.0f};
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* orow = g.o + b * g.st.o[0] + query * g.st.o[1] + head * g.st.o[2] + d0;
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = wpack<DT>(v[i + 2 * j] * inv, v[i + 2 * j + 1] * inv);
    *reinterpret_cast<u32x4*>(orow + i) = w;
  }
}

// The weight that 128 slots gather, 32 a wave, which holds their K and goes over the rows
// that see them: the scores again, the exponentials against the row's final M, times
// 1 / sum. Each slot has one wave and a fixed order of rows.
constexpr int kWeighSlots = 32 * kShWaves;

template <int DT, int MODE, int D>
__global__ __launch_bounds__(64 * kShWaves, 2) void weigh_rows_kernel(SharedArgs g, uint32_t slot_tiles) {
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t bh = blockIdx.x / slot_tiles;
  const int hk = bh % (uint32_t)g.kv_heads, b = bh / (uint32_t)g.kv_heads;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t j0 = (int32_t)(blockIdx.x % slot_tiles) * kWeighSlots + 32 * wave;
  if (j0 >= kvlen) return;
  u32x4 kf[D / 16];
  {
    const uint16_t* kr = g.k + b * g.st.k[0] + min(j0 + fr, kvlen - 1) * g.st.k[1] + hk * g.st.k[2] + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[ks] = *reinterpret_cast<const u32x4*>(kr + 16 * ks);
  }
  const int32_t off = kvlen - qlen, rows = qlen * g.group;
  const int32_t from = max(0, j0 - off);             // the first query that sees slot j0
  const float2* stats = g.stats + (int64_t)bh * g.sq * g.group;
  float acc[16] = {};
  for (int32_t r0 = from >= qlen ? rows : from * g.group & ~31; r0 < rows; r0 += 32) {
    const int32_t row = min(r0 + fr, rows - 1);
    const int32_t query = row / g.group, head = hk * g.group + row % g.group;
    const uint16_t* qr = g.q + b * g.st.q[0] + query * g.st.q[1] + head * g.st.q[2] + 8 * h;
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      s = wmma<DT>(kf[ks], *reinterpret_cast<const u32x4*>(qr + 16 * ks), s);
    if (off + r0 / g.group < j0 + 31) hide_behind(s, j0, off + query, h);
    const float2 ms = stats[row];
    const float c1 = row_c1<MODE>(ms.x), inv = r0 + fr < rows ? ms.y : 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      acc[r] = __builtin_fmaf(qexp_row<MODE, true>(s[r], g.c0, c1), inv, acc[r]);
  }
  float mine = 0.0f;                                 // lane r < 16 of a half: slot r's sum
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float v = acc[r];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) v += __shfl_xor(v, o, 64);
    mine = fr == r ? v : mine;
  }
  const int32_t j = j0 + 8 * (fr >> 2) + 4 * h + (fr & 3);
  if (fr < 16 && j < kvlen) g.weight[b * g.st.weight[0] + hk * g.st.weight[1] + j] += mine;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct SharedShape {
  int64_t batch, groups, sq, sp, skv, heads, kv_heads, dim;
  int64_t group() const { return heads / kv_heads; }
  int64_t tiles() const { return (sq * group() + 31) / 32; }
};

static bool shared_shape_ok(const SharedShape& s) {
  if (s.batch < 0 || s.groups < 1 || s.batch % s.groups != 0 || s.sq < 0 || s.sp < 0 || s.skv < 0)
    return false;
  if (s.heads < 1 || s.kv_heads < 1 || s.heads % s.kv_heads != 0 || (s.dim != 64 && s.dim != 128))
    return false;
  if (s.batch > (1 << 24) || s.sq > (1 << 24) || s.heads > (1 << 16)) return false;
  if (s.sp > (1 << 30) || s.skv > (1 << 30) || s.sp + s.skv > (1 << 30)) return false;
  if (s.sq * s.group() > (1 << 30) || s.batch / s.groups * s.sq > (1 << 30) / s.group()) return false;
  // workgroups of 256 threads: a launch takes fewer than 2^32 threads
  return s.batch * s.kv_heads < (1 << 24) && s.batch * s.kv_heads * s.tiles() < (1 << 24);
}
static int64_t slot_tiles(const SharedShape& s) { return (s.skv + kWeighSlots - 1) / kWeighSlots; }
static bool weigh_shape_ok(const SharedShape& s) {
  return s.batch * s.kv_heads * slot_tiles(s) < (1 << 24);
}
static int64_t stats_bytes(const SharedShape& s) {
  return (s.batch * s.heads * s.sq * 8 + 15) / 16 * 16;
}

template <int DT, int MODE, int D>
static void launch_shared(const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  const int64_t heads = s.batch * s.kv_heads;
  const dim3 grid((uint32_t)(heads * s.tiles())), block(64 * kShWaves);
  if (g.weight == nullptr) {
    hipLaunchKernelGGL((shared_few_kernel<DT, MODE, D, false>), grid, block, 0, stream, g);
    return;
  }
  hipLaunchKernelGGL((shared_few_kernel<DT, MODE, D, true>), grid, block, 0, stream, g);
  const uint32_t n = (uint32_t)slot_tiles(s);
  if (n > 0)
    hipLaunchKernelGGL((weigh_rows_kernel<DT, MODE, D>), dim3((uint32_t)heads * n), block, 0, stream, g, n);
}
template <int DT, int D>
static void launch_shared(int mode, const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  switch (mode) {
    case QUAKE_EXACT: launch_shared<DT, EXACT, D>(s, stream, g); break;
    case QUAKE_1: launch_shared<DT, Q1, D>(s, stream, g); break;
    case QUAKE_2: launch_shared<DT, Q2, D>(s, stream, g); break;
    default: launch_shared<DT, Q2M, D>(s, stream, g); break;
  }
}

static int64_t shared_ws_bytes(const SharedShape& s, bool weigh) { return weigh ? stats_bytes(s) : 0; }

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_attention_shared_workspace_size(int64_t batch, int64_t groups, int64_t sq,
                                                              int64_t sp, int64_t skv, int64_t heads,
                                                              int64_t kv_heads, int64_t dim, int weigh,
                                                              int64_t* bytes) {
  const SharedShape s{batch, groups, sq, sp, skv, heads, kv_heads, dim};
  if (bytes == nullptr || !shared_shape_ok(s) || (weigh && !weigh_shape_ok(s))) return QUAKE_EINVAL;
  *bytes = shared_ws_bytes(s, weigh != 0);
  return QUAKE_OK;
}

extern "C" quake_status quake_attention_shared(
    const void* q, const void* prefix_k, const void* prefix_v, const void* k, const void* v, void* o,
    float* weight, const int32_t* prefix_lens, const int32_t* q_lens, const int32_t* kv_lens,
    int64_t batch, int64_t groups, int64_t sq, int64_t sp, int64_t skv, int64_t heads, int64_t kv_heads,
    int64_t dim, const quake_shared_strides* strides, quake_dtype dtype, quake_mode mode, float t,
    void* workspace, int64_t workspace_bytes, void* stream) {
  if (dtype != QUAKE_BF16 && dtype != QUAKE_F16) return QUAKE_EDTYPE;
  if (!valid_mode(mode)) return QUAKE_EMODE;
  const SharedShape s{batch, groups, sq, sp, skv, heads, kv_heads, dim};
  if (!shared_shape_ok(s)) return QUAKE_EINVAL;
  if (!std::isfinite(t) || !(t > 0.0f)) return QUAKE_EINVAL;
  const float c0 = softmax_c0(t, mode);
  if (!std::isfinite(c0) || c0 == 0.0f) return QUAKE_EINVAL;
  if (workspace_bytes < 0 || (workspace != nullptr && !aligned16(workspace))) return QUAKE_EINVAL;
  if (batch == 0 || sq == 0) return QUAKE_OK;
  if (strides == nullptr || q == nullptr || o == nullptr) return QUAKE_EINVAL;
  if (skv > 0 && (k == nullptr || v == nullptr)) return QUAKE_EINVAL;
  if (sp > 0 && (prefix_k == nullptr || prefix_v == nullptr)) return QUAKE_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(prefix_k) || !aligned16(prefix_v) ||
      !aligned16(o) ||
      (((uintptr_t)weight | (uintptr_t)prefix_lens | (uintptr_t)q_lens | (uintptr_t)kv_lens) & 3u) != 0)
    return QUAKE_EINVAL;
  const quake_shared_strides& st = *strides;
  const int64_t nq[3] = {batch, sq, heads}, nk[3] = {batch, skv, kv_heads}, np[3] = {groups, sp, kv_heads};
  for (const int64_t* x : {st.q, st.o, st.k, st.v, st.prefix_k, st.prefix_v}) {
    const bool pre = x == st.prefix_k || x == st.prefix_v, kv = pre || x == st.k || x == st.v;
    const int64_t(&count)[3] = pre ? np : kv ? nk : nq;
    for (int i = 0; i < 3; ++i) {
      if (count[i] <= 1) continue;   // never multiplied by anything but 0
      if (x[i] < 0 || x[i] % 8 != 0 || x[i] > INT64_MAX / 8 / count[i]) return QUAKE_EINVAL;
      if (i == 1 && kv && x[i] > (1 << 24)) return QUAKE_EINVAL;   // 32-row offsets in 32 bits
    }
  }
  if (!rows_apart(st.o, nq, 3, dim)) return QUAKE_EINVAL;
  const bool weigh = weight != nullptr;
  const int64_t nw[2] = {batch, kv_heads};
  const int64_t* sw = st.weight;
  if (weigh) {
    if (!weigh_shape_ok(s)) return QUAKE_EINVAL;
    for (int i = 0; i < 2; ++i)
      if (nw[i] > 1 && (sw[i] < 0 || sw[i] > INT64_MAX / 8 / nw[i])) return QUAKE_EINVAL;
    if (!rows_apart(sw, nw, 2, skv)) return QUAKE_EINVAL;
    if (workspace == nullptr) return QUAKE_EINVAL;
  }
  const int64_t need = shared_ws_bytes(s, weigh);
  if (workspace != nullptr && need > 0) {
    if (workspace_bytes < need) return QUAKE_EINVAL;
    if (meet(workspace, need, q, span_bytes(st.q, nq, 3, dim, 2)) ||
        meet(workspace, need, o, span_bytes(st.o, nq, 3, dim, 2)) ||
        meet(workspace, need, k, span_bytes(st.k, nk, 3, dim, 2)) ||
        meet(workspace, need, v, span_bytes(st.v, nk, 3, dim, 2)) ||
        meet(workspace, need, prefix_k, span_bytes(st.prefix_k, np, 3, dim, 2)) ||
        meet(workspace, need, prefix_v, span_bytes(st.prefix_v, np, 3, dim, 2)) ||
        meet(workspace, need, weight, span_bytes(sw, nw, 2, skv, 4)) ||
        meet(workspace, need, prefix_lens, 4 * groups) || meet(workspace, need, q_lens, 4 * batch) ||
        meet(workspace, need, kv_lens, 4 * batch))
      return QUAKE_EINVAL;
  }
  SharedArgs g{};
  g.q = static_cast<const uint16_t*>(q);
  g.pk = static_cast<const uint16_t*>(prefix_k);
  g.pv = static_cast<const uint16_t*>(prefix_v);
  g.k = static_cast<const uint16_t*>(k);
  g.v = static_cast<const uint16_t*>(v);
  g.o = static_cast<uint16_t*>(o);
  g.weight = weight;
  g.prefix_lens = prefix_lens;
  g.q_lens = q_lens;
  g.kv_lens = kv_lens;
  g.stats = static_cast<float2*>(workspace);
  g.st = st;
  g.sq = (int32_t)sq;
  g.sp = (int32_t)sp;
  g.skv = (int32_t)skv;
  g.group = (int32_t)s.group();
  g.kv_heads = (int32_t)kv_heads;
  g.members = (int32_t)(batch / groups);
  g.tiles = (int32_t)s.tiles();
  g.c0 = c0;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  if (dtype == QUAKE_BF16) {
    if (dim == 64) launch_shared<BF16, 64>(mode, s, on, g);
    else launch_shared<BF16, 128>(mode, s, on, g);
  } else {
    if (dim == 64) launch_shared<F16, 64>(mode, s, on, g);
    else launch_shared<F16, 128>(mode, s, on, g);
  }
  return launch_status();
}
