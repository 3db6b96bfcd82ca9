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
#include <type_traits>

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
  float* part;                                  // partial results, the groups' then the sequences'
  quake_shared_strides st;
  int32_t groups, sq, sp, skv, group, kv_heads, members;
  int32_t gtiles, gsplit, gmany;                // of a group's rows (gsplit 0: none) ..
  int32_t tiles, nsplit, many;                  // .. and a sequence's: tiles of 32 rows, splits,
                                                // whether 128 rows share a workgroup
  uint32_t gwork;                               // workgroups of the groups' rows
  float c0;                                     // 2^23 t / ln2 (EXACT: t / ln2)
};

// Partial results of a tile of 32 rows: M, sum, sum of p as it is, O.
template <int D>
constexpr int64_t kPart = 96 + 32 * D;

__device__ __forceinline__ int64_t group_part(const SharedArgs& g, int64_t bh, int32_t tile) {
  return (bh * g.gtiles + tile) * g.gsplit;     // first split's
}
__device__ __forceinline__ int64_t own_part(const SharedArgs& g, int64_t bh, int32_t tile, int64_t groups) {
  return groups * g.kv_heads * g.gtiles * g.gsplit + (bh * g.tiles + tile) * g.nsplit;
}

// What a workgroup does: rows r0 on of a list, against a split of its keys.
struct Work {
  bool whole;               // the rows of a whole group, against its prefix alone
  int32_t b, hk;            // sequence (of a group: its first), key head
  int32_t r0, rows;         // first row, rows of the list
  int32_t qlen, off;        // of the sequence; position of its query 0
  int32_t plen, own;        // keys of the list: the prefix's, then the sequence's
  int32_t split, nsplit;
  int64_t part;             // of the workgroup's first 32 rows, split 0; -1: straight to o
};
struct RowOf {
  int32_t b, query, head, pos;
  bool live;
};

__device__ __forceinline__ RowOf row_of(const SharedArgs& g, const Work& w, int32_t r) {
  RowOf x;
  x.live = r < w.rows;
  r = min(r, w.rows - 1);
  x.b = w.b;
  x.query = r / g.group;
  x.head = w.hk * g.group + r % g.group;
  x.pos = w.off + x.query;
  if (w.whole) {
    const int32_t m = x.query / g.sq;
    x.b += m;
    x.query -= m * g.sq;
    x.pos = -1;
    x.live = x.live && x.query < seq_len(g.q_lens, x.b, g.sq);
  }
  return x;
}
template <int D>
__device__ __forceinline__ void load_q(const SharedArgs& g, const RowOf& x, int h, u32x4 (&qf)[D / 16]) {
  const uint16_t* qr = g.q + x.b * g.st.q[0] + x.query * g.st.q[1] + x.head * g.st.q[2] + 8 * h;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    qf[ks] = x.live ? *reinterpret_cast<const u32x4*>(qr + 16 * ks) : u32x4{0u, 0u, 0u, 0u};
  settle(qf);
}

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

// The bases of a list's keys and values.
struct Lists {
  const uint16_t *pk, *pv, *k, *v;
  __device__ __forceinline__ Lists(const SharedArgs& g, const Work& w) {
    const int32_t grp = w.b / g.members;
    pk = g.pk + grp * g.st.prefix_k[0] + w.hk * g.st.prefix_k[2];
    pv = g.pv + grp * g.st.prefix_v[0] + w.hk * g.st.prefix_v[2];
    k = g.k + w.b * g.st.k[0] + w.hk * g.st.k[2];
    v = g.v + w.b * g.st.v[0] + w.hk * g.st.v[2];
  }
};
template <int D, bool IS_V, int ROWS>
__device__ __forceinline__ void stage_list(uint32_t lds, const SharedArgs& g, const Work& w, const Lists& l,
                                           bool prefix, int32_t n0, int lane) {
  if (IS_V)
    stage_run<D, true, ROWS>(lds, prefix ? l.pv : l.v, prefix ? g.st.prefix_v[1] : g.st.v[1], n0,
                             prefix ? w.plen : w.own, lane);
  else
    stage_run<D, false, ROWS>(lds, prefix ? l.pk : l.k, prefix ? g.st.prefix_k[1] : g.st.k[1], n0,
                              prefix ? w.plen : w.own, lane);
}

// 32 rows in one workgroup; the waves take every fourth block of the keys and join at the
// end. K's next block is on its way while V of this one is used, and the other way round.
template <int DT, int MODE, int D, bool WEIGH>
__device__ __forceinline__ void few_rows(const SharedArgs& g, const Work& w, char* s_buf, float* s_row) {
  constexpr int kBlk = 64 * D;                      // bytes of a block of 32 rows
  constexpr int kWave = 2 * kBlk;                   // K and V
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RowOf x = row_of(g, w, w.r0 + fr);
  if (!__any(x.live)) return;
  u32x4 qf[D / 16];
  load_q<D>(g, x, h, qf);
  const Lists lists(g, w);
  const int32_t first = w.off + w.r0 / g.group;     // position of the first row
  const int32_t pblocks = (w.plen + 31) >> 5, blocks = pblocks + ((w.own + 31) >> 5);
  const int32_t n_lo = (int32_t)((int64_t)blocks * w.split / w.nsplit);
  const int32_t n_hi = (int32_t)((int64_t)blocks * (w.split + 1) / w.nsplit);
  char* buf = s_buf + wave * kWave;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf + wave * kWave);
  auto load_k = [&](int32_t n) {
    stage_list<D, false, 32>(lds, g, w, lists, n < pblocks, 32 * (n < pblocks ? n : n - pblocks), lane);
  };
  auto load_v = [&](int32_t n) {
    stage_list<D, true, 32>(lds + kBlk, g, w, lists, n < pblocks, 32 * (n < pblocks ? n : n - pblocks), lane);
  };

  RowAcc<D> acc;
  acc.sum = 0.0f;
  acc.m = kNoMax;
  float all = 0.0f;                                 // of p as it is, not rounded to 16 bits
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc.o[d] = f32x16{};
  constexpr int kLoads = D / 16;                    // of a block's K or V
  if (n_lo + wave < n_hi) {
    load_k(n_lo + wave);
    load_v(n_lo + wave);
  }
  for (int32_t n = n_lo + wave; n < n_hi; n += kShWaves) {
    const bool more = n + kShWaves < n_hi;
    wait_loads<kLoads>();                           // K is here, V may be on its way
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = wmma<DT>(read_k<D>(buf, fr, h, ks), qf[ks], s);
    wait_lds();                                     // K's reads, before it is loaded again
    if (more) load_k(n + kShWaves);
    const bool p = n < pblocks;
    const int32_t n0 = 32 * (p ? n : n - pblocks);
    if (n0 + 31 > (p ? w.plen - 1 : first)) hide_behind(s, n0, p ? w.plen - 1 : x.pos, h);
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
        const uint32_t pair = wpack<DT>(e[r], e[r + 1]);
        acc.sum = wsum<DT>(pair, acc.sum);
        pr[r >> 3][(r >> 1) & 3] = pair;
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
  float (*s_m)[32] = reinterpret_cast<float (*)[32]>(s_row);
  float (*s_sum)[32] = s_m + kShWaves, (*s_all)[32] = s_sum + kShWaves;
  acc.sum += other_half(acc.sum);
  if constexpr (WEIGH) all += other_half(all);
  __syncthreads();
  if (lane < 32) {
    s_m[wave][fr] = acc.m;
    s_sum[wave][fr] = acc.sum;
    if constexpr (WEIGH) s_all[wave][fr] = all;
  }
  float* mine = reinterpret_cast<float*>(s_buf + wave * kWave);   // [D][32] floats
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      mine[(32 * d + 8 * (r >> 2) + 4 * h + (r & 3)) * 32 + fr] = acc.o[d][r];
  __syncthreads();
  float m = s_m[0][fr];
#pragma unroll
  for (int i = 1; i < kShWaves; ++i) m = fmaxf(m, s_m[i][fr]);
  float sum = 0.0f, every = 0.0f;
  int32_t e[kShWaves];
#pragma unroll
  for (int i = 0; i < kShWaves; ++i) {
    e[i] = down_shift(s_m[i][fr], m);
    sum += __builtin_amdgcn_ldexpf(s_sum[i][fr], e[i]);
    if constexpr (WEIGH) every += __builtin_amdgcn_ldexpf(s_all[i][fr], e[i]);
  }
  // this wave's dims: D / 4, each half of its lanes D / 8 of them
  constexpr int N = D / 8;
  const int d0 = wave * (D / 4) + h * N;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < kShWaves; ++j)
      v[i] += __builtin_amdgcn_ldexpf(
          reinterpret_cast<const float*>(s_buf + j * kWave)[(d0 + i) * 32 + fr], e[j]);
  }
  if (!x.live) return;
  if (w.part >= 0) {
    float* to = g.part + (w.part + w.split) * kPart<D>;
    if (wave == 0 && h == 0) {
      to[fr] = m;
      to[32 + fr] = sum;
      if constexpr (WEIGH) to[64 + fr] = every;
    }
    float4* wo = reinterpret_cast<float4*>(to + 96 + fr * D + d0);
#pragma unroll
    for (int i = 0; i < N; i += 4) wo[i / 4] = float4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    return;
  }
  if constexpr (WEIGH) {
    if (wave == 0 && h == 0)
      g.stats[((int64_t)w.b * g.kv_heads + w.hk) * g.sq * g.group + w.r0 + fr] =
          every > 0.0f ? float2{m, 1.0f / every} : float2{0.0f, 0.0f};
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* orow = g.o + x.b * g.st.o[0] + x.query * g.st.o[1] + x.head * g.st.o[2] + d0;
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    u32x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = wpack<DT>(v[i + 2 * j] * inv, v[i + 2 * j + 1] * inv);
    *reinterpret_cast<u32x4*>(orow + i) = y;
  }
}

// 128 rows in one workgroup, 32 a wave, which share tiles of 64 keys in LDS (two blocks of
// 32; two tiles each of K and V), in the software pipeline of window_many_kernel: while
// block n's scores become probabilities, the scores of block n + 1 and the second product
// of block n - 1 are computed; one barrier a tile, between its blocks.
constexpr int kShKeys = 64;

template <int DT, int MODE, int D, bool WEIGH>
__device__ __forceinline__ void many_rows(const SharedArgs& g, const Work& w, char* s_buf) {
  constexpr int kTile = 2 * kShKeys * D;            // bytes of K or V of a tile
  constexpr int kRows = kShKeys / kShWaves;         // a wave loads
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t w0 = w.r0 + 32 * wave;
  const RowOf x = row_of(g, w, w0 + fr);
  const int32_t first = w.off + min(w0, w.rows - 1) / g.group;
  const int32_t last = w.off + min(w0 + 31, w.rows - 1) / g.group;
  const int32_t ptiles = (w.plen + kShKeys - 1) / kShKeys;
  const int32_t steps = ptiles + (w.own + kShKeys - 1) / kShKeys;
  const int32_t n_lo = (int32_t)((int64_t)steps * w.split / w.nsplit);
  const int32_t n_hi = (int32_t)((int64_t)steps * (w.split + 1) / w.nsplit);
  // tiles of which this wave's rows may see something
  const int32_t seen = w.whole || last < 0 ? 0 : last / kShKeys + 1;
  const int32_t t_hi = __any(x.live) ? min(n_hi, ptiles + seen) : n_lo;

  u32x4 qf[D / 16];
  load_q<D>(g, x, h, qf);
  const Lists lists(g, w);
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf + wave * kRows * 2 * D);
  auto load_k = [&](int32_t t, uint32_t at) {
    stage_list<D, false, kRows>(lds + kTile * at, g, w, lists, t < ptiles,
                                kShKeys * (t < ptiles ? t : t - ptiles) + kRows * wave, lane);
  };
  auto load_v = [&](int32_t t) {
    stage_list<D, true, kRows>(lds + kTile * (2 + ((t - n_lo) & 1)), g, w, lists, t < ptiles,
                               kShKeys * (t < ptiles ? t : t - ptiles) + kRows * wave, lane);
  };

  RowAcc<D> acc;
  acc.sum = 0.0f;
  acc.m = kNoMax;
  float all = 0.0f;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc.o[d] = f32x16{};

  constexpr int NU = D / 16, NE = 16 / NU;   // products of a kind a block; values for each
  constexpr int ND = D / 32;
  // Where this lane reads its operands in block 0: K's chunk of step ks, V's of dims
  // 32 d on; other blocks and keys at constant distances.
  typedef __attribute__((address_space(3))) const char* lds_ptr;
  lds_ptr kat[NU], vat[ND];
  {
    const lds_ptr base = (lds_ptr)s_buf;
#pragma unroll
    for (int ks = 0; ks < NU; ++ks)
      kat[ks] = base + fr * (2 * D) + 16 * ((2 * ks + h) ^ kswizzle<D>(fr));
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const int r = 4 * h + ((lane >> 2) & 3);
      const int c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
      vat[d] = base + 2 * kTile + r * (2 * D) + 16 * (c ^ vswizzle<D>(r)) + 8 * (lane & 1);
    }
  }
  auto get_k = [&](int blk, int ks) {
    return *(__attribute__((address_space(3))) const u32x4*)(kat[ks] + 64 * D * blk);
  };
  auto get_v = [&](int blk, int u) {   // of product u: keys 16 (u / ND) on, dims 32 (u mod ND) on
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const lds_ptr a = vat[u % ND] + 64 * D * blk + 32 * D * (u / ND);
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)a));
    const u32x2 hi = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(a + 16 * D)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };
  const float units = g.c0 * (MODE == EXACT ? 1.0f : 0x1p-23f);
  float limit = -INFINITY;   // scores up to here leave M as it is
  // Block n (scores s, in LDS block KN - 1) while the scores of block n + 1 (KN) go to
  // sn; pp: the probabilities of block n - 1, whose values lie in block VP; pn: block
  // n's.
  auto step = [&](int32_t n, auto kn, auto vp, f32x16& s, f32x16& sn, u32x4 (&pp)[2], u32x4 (&pn)[2]) {
    constexpr int KN = decltype(kn)::value, VP = decltype(vp)::value;
    u32x4 ka[NU], va[NU];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ka[u] = get_k(KN, u);
      va[u] = get_v(VP, u);
    }
    const bool p = n < 2 * ptiles;
    const int32_t n0 = 32 * (p ? n : n - 2 * ptiles);
    if (n0 + 31 > (p ? w.plen - 1 : first)) hide_behind(s, n0, p ? w.plen - 1 : x.pos, h);
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    if (__any(top > limit)) {
      const int32_t e = raise_max<DT>(fmaxf(top, other_half(top)) * units, acc);
      if constexpr (WEIGH) all = __builtin_amdgcn_ldexpf(all, e);
#pragma unroll
      for (int i = 0; i < 8; ++i) pp[i >> 2][i & 3] = scale_pair<DT>(pp[i >> 2][i & 3], e);
      limit = (acc.m + (kLift<DT> + kLazy)) / units;
    }
    const float c1 = row_c1<MODE>(acc.m);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if (u + 2 < NU) {
        ka[u + 2] = get_k(KN, u + 2);
        va[u + 2] = get_v(VP, u + 2);
      }
      const f32x16 zero = {};
      sn = wmma<DT>(ka[u], qf[u], u == 0 ? zero : sn);
      acc.o[u % ND] = wmma<DT>(va[u], pp[u / ND], acc.o[u % ND]);
#pragma unroll
      for (int r = NE * u; r < NE * u + NE; r += 2) {
        const float a = qexp_row<MODE, true>(s[r], g.c0, c1), z = qexp_row<MODE, true>(s[r + 1], g.c0, c1);
        const uint32_t pair = wpack<DT>(a, z);
        acc.sum = wsum<DT>(pair, acc.sum);
        if constexpr (WEIGH) all += a + z;
        pn[r >> 3][(r >> 1) & 3] = pair;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  u32x4 pa[2], pb[2];
  f32x16 sa, sb;
  auto two_blocks = [&](int32_t t, auto parity) {
    constexpr int B = 2 * decltype(parity)::value;   // the tile's first block in LDS
    const bool mine = t < t_hi;
    if (mine && t == n_lo) {
      sa = f32x16{};
#pragma unroll
      for (int u = 0; u < NU; ++u) sa = wmma<DT>(get_k(B, u), qf[u], sa);
      pb[0] = pb[1] = u32x4{0u, 0u, 0u, 0u};   // no block before
    }
    if (mine)
      step(2 * t, std::integral_constant<int, B + 1>{}, std::integral_constant<int, 3 - B>{}, sa, sb, pb, pa);
    wait_lds();
    wait_loads<0>();
    __syncthreads();
    if (t + 2 < n_hi) load_k(t + 2, (t - n_lo) & 1);
    if (t + 1 < n_hi) load_v(t + 1);
    if (!mine) return;
    step(2 * t + 1, std::integral_constant<int, 2 - B>{}, std::integral_constant<int, B>{}, sb, sa, pa, pb);
    if (t + 1 == t_hi) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
        acc.o[u % ND] = wmma<DT>(get_v(B + 1, u), pb[u / ND], acc.o[u % ND]);
    }
  };
  if (n_lo < n_hi) {
    load_k(n_lo, 3);   // V of the tile before the first is read (times 0): K's rows, finite where K is
    load_k(n_lo, 0);
    load_v(n_lo);
    if (n_lo + 1 < n_hi) load_k(n_lo + 1, 1);
    wait_loads<0>();
    __syncthreads();
  }
  for (int32_t t = n_lo; t < n_hi; t += 2) {
    two_blocks(t, std::integral_constant<int, 0>{});
    if (t + 1 < n_hi) two_blocks(t + 1, std::integral_constant<int, 1>{});
  }

  const float sum = acc.sum + other_half(acc.sum);
  if constexpr (WEIGH) all += other_half(all);
  if (w.part >= 0) {
    if (!x.live) return;
    float* to = g.part + (w.part + (int64_t)wave * w.nsplit + w.split) * kPart<D>;
    if (h == 0) {
      to[fr] = acc.m;
      to[32 + fr] = sum;
      if constexpr (WEIGH) to[64 + fr] = all;
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(to + 96 + fr * D + 32 * d + 8 * i + 4 * h) =
            float4{acc.o[d][4 * i], acc.o[d][4 * i + 1], acc.o[d][4 * i + 2], acc.o[d][4 * i + 3]};
    return;
  }
  if constexpr (WEIGH) {
    if (h == 0 && x.live)
      g.stats[((int64_t)w.b * g.kv_heads + w.hk) * g.sq * g.group + w0 + fr] =
          all > 0.0f ? float2{acc.m, 1.0f / all} : float2{0.0f, 0.0f};
  }
  // Rows of the output through LDS (the wave's own rows, chunks swizzled as K's), so
  // that whole rows are stored 16 bytes a lane.
  __syncthreads();
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  char* ow = s_buf + wave * 64 * D;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x2 y = {wpack<DT>(acc.o[d][4 * i] * inv, acc.o[d][4 * i + 1] * inv),
                       wpack<DT>(acc.o[d][4 * i + 2] * inv, acc.o[d][4 * i + 3] * inv)};
      *reinterpret_cast<u32x2*>(ow + fr * 2 * D + 16 * ((4 * d + i) ^ kswizzle<D>(fr)) + 8 * h) = y;
    }
  __builtin_amdgcn_wave_barrier();
  wait_lds();
  constexpr int CH = D / 8, RPL = 64 / CH;
#pragma unroll
  for (int j = 0; j < 32 / RPL; ++j) {
    const int r = RPL * j + lane / CH, c = lane % CH;
    if (w0 + r >= w.rows) continue;
    const int32_t qi = (w0 + r) / g.group, hd = w.hk * g.group + (w0 + r) % g.group;
    *reinterpret_cast<u32x4*>(g.o + w.b * g.st.o[0] + qi * g.st.o[1] + hd * g.st.o[2] + 8 * c) =
        *reinterpret_cast<const u32x4*>(ow + r * 2 * D + 16 * (c ^ kswizzle<D>(r)));
  }
}

// The groups' rows against the prefixes, then each sequence's against its own keys (where no
// rows of groups are formed: against the prefix, too). Workgroups go round the 8 XCDs: each
// gets consecutive ones of either kind, which share most of their keys, for its own L2.
template <int DT, int MODE, int D, bool WEIGH>
__global__ __launch_bounds__(64 * kShWaves, 2) void shared_kernel(SharedArgs g) {
  __shared__ __attribute__((aligned(16))) char s_buf[4 * 2 * kShKeys * D];
  __shared__ float s_row[3 * kShWaves * 32];
  const bool whole = blockIdx.x < g.gwork;
  const uint32_t at = whole ? blockIdx.x : blockIdx.x - g.gwork, work = whole ? g.gwork : gridDim.x - g.gwork;
  const uint32_t c = at & 7u, per = work >> 3, rest = work & 7u;
  uint32_t id = c * per + min(c, rest) + (at >> 3);
  Work w;
  w.whole = whole;
  const bool many = (whole ? g.gmany : g.many) != 0;
  const uint32_t tiles = ((uint32_t)(whole ? g.gtiles : g.tiles) + (many ? kShWaves - 1 : 0)) / (many ? kShWaves : 1);
  w.nsplit = whole ? g.gsplit : g.nsplit;
  const uint32_t tile = id % tiles;
  id /= tiles;
  w.split = (int32_t)(id % (uint32_t)w.nsplit);
  const uint32_t bh = id / (uint32_t)w.nsplit;
  w.hk = (int32_t)(bh % (uint32_t)g.kv_heads);
  w.b = (int32_t)(bh / (uint32_t)g.kv_heads) * (whole ? g.members : 1);
  const int32_t t32 = (int32_t)tile * (many ? kShWaves : 1);
  w.r0 = 32 * t32;
  const int32_t grp = w.b / g.members;
  const int32_t plen = g.sp == 0 ? 0 : seq_len(g.prefix_lens, grp, g.sp);
  if (whole) {
    w.qlen = w.off = w.own = 0;
    w.rows = g.members * g.sq * g.group;
    w.plen = plen;
    w.part = group_part(g, bh, t32);
  } else {
    w.qlen = seq_len(g.q_lens, w.b, g.sq);
    w.off = seq_len(g.kv_lens, w.b, g.skv) - w.qlen;
    w.rows = w.qlen * g.group;
    const int32_t last = w.off + min(w.r0 + (many ? 32 * kShWaves : 32) - 1, w.rows - 1) / g.group;
    w.own = max(last + 1, 0);
    w.plen = g.gsplit > 0 ? 0 : plen;
    w.part = g.gsplit == 0 && g.nsplit == 1 ? -1 : own_part(g, bh, t32, g.groups);
  }
  if (w.r0 >= w.rows) return;
  if (many)
    many_rows<DT, MODE, D, WEIGH>(g, w, s_buf);
  else
    few_rows<DT, MODE, D, WEIGH>(g, w, s_buf, s_row);
}

// Joins a row's partial results, the group's and the sequence's, a lane for every four dims:
// D / 4 lanes, which take the results one after the other, or (WIDE) the whole workgroup,
// whose 1024 / D such teams take every so many-th. Several loads are in flight; the order
// is fixed.
template <int DT, int D, bool WEIGH, bool WIDE>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs g) {
  constexpr int C = D / 4, SL = WIDE ? 256 / C : 1, U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t id = WIDE ? blockIdx.x : blockIdx.x * (256u / C) + threadIdx.x / C;   // of all rows
  const uint32_t item = id >> 5, bh = item / (uint32_t)g.tiles;
  const int32_t row = 32 * (int32_t)(item % (uint32_t)g.tiles) + (int32_t)(id & 31u);
  const int hk = bh % (uint32_t)g.kv_heads, b = bh / (uint32_t)g.kv_heads;
  if (b >= g.members * g.groups || row >= seq_len(g.q_lens, b, g.sq) * g.group) return;
  const int grp = b / g.members;
  const int32_t of_group = (b - grp * g.members) * g.sq * g.group + row;   // among the group's rows
  const float* pg = g.part + group_part(g, (int64_t)grp * g.kv_heads + hk, of_group >> 5) * kPart<D>;
  const float* po = g.part + own_part(g, bh, row >> 5, g.groups) * kPart<D>;
  const int c = lane % C, total = g.gsplit + g.nsplit;
  float m = kNoMax, sum = 0.0f, every = 0.0f;
  float4 v{0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](float om, float os, float oe, float4 ov) {
    const float top = fmaxf(m, om);
    const int32_t e = down_shift(m, top), oe2 = down_shift(om, top);
    auto two = [&](float a, float o) {
      return __builtin_amdgcn_ldexpf(a, e) + __builtin_amdgcn_ldexpf(o, oe2);
    };
    sum = two(sum, os);
    if constexpr (WEIGH) every = two(every, oe);
    v = float4{two(v.x, ov.x), two(v.y, ov.y), two(v.z, ov.z), two(v.w, ov.w)};
    m = top;
  };
  for (int s0 = WIDE ? threadIdx.x / C : 0; s0 < total; s0 += U * SL) {
    float om[U], os[U], oe[U];
    float4 ov[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {   // past the last one: that one again, not added
      const int i = min(s0 + j * SL, total - 1);
      const bool own = i >= g.gsplit;
      const float* p = own ? po + (i - g.gsplit) * kPart<D> : pg + i * kPart<D>;
      const int fr = (own ? row : of_group) & 31;
      om[j] = p[fr];
      os[j] = p[32 + fr];
      oe[j] = WEIGH ? p[64 + fr] : 0.0f;
      ov[j] = *reinterpret_cast<const float4*>(p + 96 + fr * D + 4 * c);
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (s0 + j * SL < total) add(om[j], os[j], oe[j], ov[j]);
  }
  if constexpr (WIDE) {
    constexpr int W = 4;
#pragma unroll
    for (int o = C; o < 64; o <<= 1)
      add(__shfl_xor(m, o, 64), __shfl_xor(sum, o, 64), __shfl_xor(every, o, 64),
          float4{__shfl_xor(v.x, o, 64), __shfl_xor(v.y, o, 64), __shfl_xor(v.z, o, 64),
                 __shfl_xor(v.w, o, 64)});
    __shared__ float s_m[W], s_sum[W], s_all[W];
    __shared__ float4 s_v[W][C];
    if (lane < C) s_v[wave][c] = v;
    if (lane == 0) {
      s_m[wave] = m;
      s_sum[wave] = sum;
      s_all[wave] = every;
    }
    __syncthreads();
    if (wave > 0 || lane >= C) return;
#pragma unroll
    for (int o = 1; o < W; ++o) add(s_m[o], s_sum[o], s_all[o], s_v[o][c]);
  }
  if constexpr (WEIGH) {
    if (c == 0)
      g.stats[(int64_t)bh * g.sq * g.group + row] = every > 0.0f ? float2{m, 1.0f / every} : float2{0.0f, 0.0f};
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* orow = g.o + b * g.st.o[0] + (row / g.group) * g.st.o[1] + (hk * g.group + row % g.group) * g.st.o[2];
  *reinterpret_cast<u32x2*>(orow + 4 * c) =
      u32x2{wpack<DT>(v.x * inv, v.y * inv), wpack<DT>(v.z * inv, v.w * inv)};
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

// How a call is cut up. Rows of a whole group against the prefix where a sequence alone has
// few: the prefix is then read once for all, and its scores are full tiles.
struct SharedPlan {
  int64_t gtiles = 0, gsplit = 0, tiles = 0, nsplit = 1;
  bool gmany = false, many = false;
  bool join() const { return gsplit > 0 || nsplit > 1; }
};
constexpr int64_t kShTarget = 512, kShSplitKeys = 128, kShSplitFrom = 512;
constexpr int64_t kShJoinFew = 8;

static SharedPlan shared_plan(const SharedShape& s) {
  SharedPlan p;
  const int64_t rows = s.sq * s.group(), all = rows * (s.batch / s.groups);
  const auto wide = [](int64_t n, bool many) { return many ? (n + 127) / 128 : (n + 31) / 32; };
  const auto splits = [&](int64_t items, int64_t keys) {
    return items == 0 || keys < kShSplitFrom ? 1
                                             : std::max<int64_t>(1, std::min(keys / kShSplitKeys, kShTarget / items));
  };
  p.tiles = (rows + 31) / 32;
  p.many = rows >= 96;
  int64_t own = s.skv;
  if (s.sp > 0 && rows < 96 && all > rows) {
    p.gtiles = (all + 31) / 32;
    p.gmany = all > 32;
    p.gsplit = splits(s.groups * s.kv_heads * wide(all, p.gmany), s.sp);
  } else {
    own += s.sp;
  }
  p.nsplit = splits(s.batch * s.kv_heads * wide(rows, p.many), own);
  return p;
}
static int64_t part_bytes(const SharedShape& s, const SharedPlan& p) {
  if (!p.join()) return 0;
  const int64_t n = s.groups * s.kv_heads * p.gtiles * p.gsplit + s.batch * s.kv_heads * p.tiles * p.nsplit;
  return n * (96 + 32 * s.dim) * 4;
}
static int64_t shared_ws_bytes(const SharedShape& s, bool weigh) {
  return part_bytes(s, shared_plan(s)) + (weigh ? stats_bytes(s) : 0);
}

template <int DT, int MODE, int D, bool WEIGH>
static void launch_shared(const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  const int64_t heads = s.batch * s.kv_heads;
  const dim3 block(64 * kShWaves);
  const int64_t own = heads * (g.many ? (g.tiles + kShWaves - 1) / kShWaves : g.tiles) * g.nsplit;
  hipLaunchKernelGGL((shared_kernel<DT, MODE, D, WEIGH>), dim3((uint32_t)(g.gwork + own)), block, 0, stream, g);
  if (g.gsplit > 0 || g.nsplit > 1) {
    if (g.gsplit + g.nsplit > kShJoinFew)
      hipLaunchKernelGGL((shared_join_kernel<DT, D, WEIGH, true>), dim3((uint32_t)(heads * g.tiles * 32)),
                         dim3(256), 0, stream, g);
    else
      hipLaunchKernelGGL((shared_join_kernel<DT, D, WEIGH, false>), dim3((uint32_t)(heads * g.tiles * D / 32)),
                         dim3(256), 0, stream, g);
  }
  const uint32_t n = (uint32_t)slot_tiles(s);
  if constexpr (WEIGH)
    if (n > 0)
      hipLaunchKernelGGL((weigh_rows_kernel<DT, MODE, D>), dim3((uint32_t)heads * n), block, 0, stream, g, n);
}
template <int DT, int D, bool WEIGH>
static void launch_shared(int mode, const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  switch (mode) {
    case QUAKE_EXACT: launch_shared<DT, EXACT, D, WEIGH>(s, stream, g); break;
    case QUAKE_1: launch_shared<DT, Q1, D, WEIGH>(s, stream, g); break;
    case QUAKE_2: launch_shared<DT, Q2, D, WEIGH>(s, stream, g); break;
    default: launch_shared<DT, Q2M, D, WEIGH>(s, stream, g); break;
  }
}
template <int DT, int D>
static void launch_shared(int mode, const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  if (g.weight == nullptr)
    launch_shared<DT, D, false>(mode, s, stream, g);
  else
    launch_shared<DT, D, true>(mode, s, stream, g);
}

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
  SharedPlan p;
  p.tiles = s.tiles();
  if (workspace != nullptr) p = shared_plan(s);
  else p.many = s.sq * s.group() >= 96;
  g.part = static_cast<float*>(workspace);
  g.stats = reinterpret_cast<float2*>(static_cast<char*>(workspace) + part_bytes(s, p));
  g.st = st;
  g.sq = (int32_t)sq;
  g.sp = (int32_t)sp;
  g.skv = (int32_t)skv;
  g.group = (int32_t)s.group();
  g.kv_heads = (int32_t)kv_heads;
  g.members = (int32_t)(batch / groups);
  g.groups = (int32_t)groups;
  g.gtiles = (int32_t)p.gtiles;
  g.gsplit = (int32_t)p.gsplit;
  g.gmany = p.gmany;
  g.tiles = (int32_t)p.tiles;
  g.nsplit = (int32_t)p.nsplit;
  g.many = p.many;
  g.gwork = (uint32_t)(groups * kv_heads * (p.gmany ? (p.gtiles + kShWaves - 1) / kShWaves : p.gtiles) * p.gsplit);
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
