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
//
// Bits: scores, M, row sums, O and weights are binary32. The probabilities of the second
// product alone are rounded to the operands' 16 bits, as the matrix cores take no wider ones
// beside 16-bit values at this rate (twice the products would carry their lower halves); the
// output's denominator is the sum of the rounded ones. In the norm an output is then 2.3e-3
// (bf16) or 2.9e-4 (f16) off the 64-bit one, 1.4 times the 1.7e-3 or 2.1e-4 of its own
// rounding. Weights are taken from the probabilities as they are: 1e-6.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache_tile.hpp"
#include "quake_device.hpp"
#include "quake_host.hpp"

namespace qk {

constexpr int kShWaves = 4;

// Division by a number the host knows: n / d = floor(n m / 2^(32 + s)) for n < 2^31 with
// 2^s < d <= 2^(s + 1), m = ceil(2^(32 + s) / d) < 2^32: n m / 2^(32 + s) exceeds n / d by less
// than n / 2^(32 + s) <= 2^-(s + 1) <= 1 / d.
struct Div {
  uint32_t d = 1, m = 0, s = 0;
  Div() = default;
  explicit Div(int64_t by) : d((uint32_t)std::max<int64_t>(by, 1)) {
    if (d == 1) return;
    while (((uint64_t)2 << s) < d) ++s;
    m = (uint32_t)((((uint64_t)1 << (32 + s)) + d - 1) / d);
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> s; }
  __device__ __forceinline__ int32_t of(int32_t n) const { return (int32_t)of((uint32_t)n); }   // n >= 0
};

// A token's stride is below 2^24 + 1, so the strides that loops use are 32-bit ones.
struct SharedArgs {
  const uint16_t *q, *pk, *pv, *k, *v;
  uint16_t* o;
  float* weight;                                // or null
  const int32_t *prefix_lens, *q_lens, *kv_lens;   // or null: sp, sq, skv
  float2* stats;                                // of a row: M, 1 / sum of p (weights by rows)
  float* part;                                  // partial results, the groups' then the sequences'
  float* scores;                                // or null; [row of a key head][slot] (weights by slots)
  float* sums;                                  // parts of weights, by chunks of rows
  quake_shared_strides st;
  int32_t pkt, pvt, kt, vt;                     // token strides
  int32_t groups, sq, sp, skv, group, kv_heads, members;
  int32_t gtiles, gmany, gsplit;                // of a group's rows (gsplit 0: none) ..
  int32_t tiles, many, cut, nsplit;             // .. and a sequence's: tiles of 32 rows, whether 128 rows
                                                // share a workgroup, whether tiles are cut into parts, the most of one
  uint32_t heads, gwork, items;                 // key heads of all sequences; workgroups of groups' rows; the
                                                // sequences' tiles in units of one workgroup's
  Div by_group, by_sq, by_members, by_heads;    // heads: key heads
  Div by_gtiles, by_gsplit, by_tiles, by_items;    // tiles: in units of one workgroup's
  Div by_gper, by_per, by_rows;                 // blocks of a part; rows of a key head or, many, 128
  float c0;                                     // 2^23 t / ln2 (EXACT: t / ln2)
};

// Partial results of a tile of 32 rows: M, sum, sum of p as it is, O.
template <int D>
constexpr int64_t kPart = 96 + 32 * D;
constexpr int kShKeys = 64;                     // keys of a step

// What a workgroup does: rows r0 on of a list, against a part of its keys.
struct Work {
  bool whole;               // the rows of a whole group, against its prefix alone
  int32_t b, hk;            // sequence (of a group: its first), key head
  int32_t r0, rows;         // first row, rows of the list
  int32_t off;              // position of the sequence's query 0
  int32_t plen, own;        // keys of the list: the prefix's, then the sequence's
  int32_t n_lo, n_hi;       // blocks of 32 (128 rows: steps of 64) keys of the list
  int64_t part;             // of the workgroup's first 32 rows; -1: straight to o
  int32_t apart;            // parts from one tile's to the next one's
};
__device__ __forceinline__ int32_t list_blocks(int32_t plen, int32_t own, bool many) {
  return many ? (plen + 63) / 64 + (own + 63) / 64 : (plen + 31) / 32 + (own + 31) / 32;
}
// parts that a list is cut into
__device__ __forceinline__ int32_t list_parts(int32_t plen, int32_t own, bool many, const Div& per) {
  return per.of(list_blocks(plen, own, many) + (int32_t)per.d - 1);
}
// own keys that the rows of the tile at r0 see
__device__ __forceinline__ int32_t tile_keys(const SharedArgs& g, int32_t off, int32_t r0, int32_t rows) {
  return rows == 0 ? 0 : max(off + g.by_group.of(min(r0 + (g.many ? 32 * kShWaves : 32), rows) - 1) + 1, 0);
}
__device__ __forceinline__ int32_t prefix_len(const SharedArgs& g, int32_t group) {
  return g.sp == 0 ? 0 : seq_len(g.prefix_lens, group, g.sp);
}
// The first part of a tile: a group's; a sequence's, the tiles numbered as they are launched.
__device__ __forceinline__ int64_t group_part(const SharedArgs& g, int64_t bh, int32_t tile) {
  return (bh * g.gtiles + tile) * g.gsplit;
}
__device__ __forceinline__ int64_t own_part(const SharedArgs& g, int64_t tile) {
  return (int64_t)g.groups * g.kv_heads * g.gtiles * g.gsplit + tile * g.nsplit;
}
// Workgroups go round the 8 XCDs: number `at` of n as each XCD takes consecutive ones, which
// share most of their keys, for its own L2.
__device__ __forceinline__ uint32_t by_xcd(uint32_t at, uint32_t n) {
  const uint32_t x = at & 7u, per = n >> 3, rest = n & 7u;
  return x * per + min(x, rest) + (at >> 3);
}
// Number `at` of the sequences' tiles (in units of one workgroup's), in the order of their
// launch: key head of a sequence, tile, those that see most first. The tiles of a key head
// share an XCD, and key heads go round the XCDs one by one where they come out even: runs of
// them would give one XCD the long sequences.
struct TileOf {
  uint32_t bh;
  int32_t tile;
};
__device__ __forceinline__ TileOf tile_of(const SharedArgs& g, uint32_t at) {
  const uint32_t tiles = g.by_tiles.d;
  uint32_t id = at;
  if (tiles > 1 && (g.heads & 7u) == 0) {
    const uint32_t k = at >> 3, round = g.by_tiles.of(k);
    return {8 * round + (at & 7u), (int32_t)(tiles - 1u - (k - round * tiles))};
  }
  if (tiles > 1) id = by_xcd(at, g.heads * tiles);
  const uint32_t bh = g.by_tiles.of(id);
  return {bh, (int32_t)(tiles - 1u - (id - bh * tiles))};
}
// The number of a key head's tile.
__device__ __forceinline__ uint32_t number_of(const SharedArgs& g, uint32_t bh, int32_t tile) {
  const uint32_t tiles = g.by_tiles.d, back = tiles - 1u - (uint32_t)tile;
  if (tiles > 1 && (g.heads & 7u) == 0) return 8 * ((bh >> 3) * tiles + back) + (bh & 7u);
  const uint32_t id = bh * tiles + back;
  if (tiles == 1) return id;
  // by_xcd's inverse
  const uint32_t n = g.heads * tiles, per = n >> 3, rest = n & 7u, first = rest * (per + 1u);
  const uint32_t x = id < first ? id / (per + 1u) : rest + (id - first) / per;
  return 8 * (id - (x * per + min(x, rest))) + x;
}
struct RowOf {
  int32_t b, query, head, pos;
  bool live;
};

__device__ __forceinline__ RowOf row_of(const SharedArgs& g, const Work& w, int32_t r) {
  RowOf x;
  x.live = r < w.rows;
  r = min(r, w.rows - 1);
  x.b = w.b;
  x.query = g.by_group.of(r);
  x.head = w.hk * g.group + r - x.query * g.group;
  x.pos = w.off + x.query;
  if (w.whole) {
    const int32_t m = g.by_sq.of(x.query);
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
__device__ __forceinline__ void stage_run(uint32_t lds, const uint16_t* base, int32_t stride,
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
      lds_load16(lds + 1024 * j, row + 16u * (uint32_t)(pc ^ sw), b + (int64_t)(2 * RPL * j) * stride);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int sw = IS_V ? vswizzle<D>(RPL * j + r) : kswizzle<D>(RPL * j + r);
      lds_load16(lds + 1024 * j, base + (int64_t)min(n0 + RPL * j + r, n - 1) * stride + 8 * (pc ^ sw));
    }
  }
}

// slots of a row of scores
__host__ __device__ constexpr int64_t score_row(int64_t skv) { return (skv + 31) / 32 * 32; }

// -inf for the keys of the block from n0 on that lie behind key `lim`
__device__ __forceinline__ void hide_behind(f32x16& s, int32_t n0, int32_t lim, int h) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = n0 + 8 * (r >> 2) + 4 * h + (r & 3) <= lim ? s[r] : -INFINITY;
}

// The exponential of `mode` times a constant that all of a row share, so that it cancels.
// QuAKE2's is (a_m^2 + 2) / 3 with the exponent of z, which has the value 2^i a_m itself: 3/2
// times it is one multiply-add, z (a_m / 2) + 2^i. An instruction less than with the mantissa
// joined to the exponent, and two roundings.
template <int MODE>
__device__ __forceinline__ float q2_of_z(uint32_t z) {
  return __builtin_fmaf(as_f(z), as_f((z & kMantMask) | 0x3F000000u), as_f(z & kSignExpMask));
}
// Two at a time: a wait state follows each piece of inline assembly.
template <int MODE>
__device__ __forceinline__ void row_exp(float x, float y, float c0, float c1, float& ex, float& ey) {
  if constexpr (MODE == Q2) {
    uint32_t zx, zy;
    asm("v_cvt_u32_f32 %0, %2\n\tv_cvt_u32_f32 %1, %3"
        : "=&v"(zx), "=v"(zy)
        : "v"(__builtin_fmaf(x, c0, c1)), "v"(__builtin_fmaf(y, c0, c1)));
    ex = q2_of_z<MODE>(zx);
    ey = q2_of_z<MODE>(zy);
  } else {
    ex = qexp_row<MODE, true>(x, c0, c1);
    ey = qexp_row<MODE, true>(y, c0, c1);
  }
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
    const int32_t grp = g.by_members.of(w.b);
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
    stage_run<D, true, ROWS>(lds, prefix ? l.pv : l.v, prefix ? g.pvt : g.vt, n0,
                             prefix ? w.plen : w.own, lane);
  else
    stage_run<D, false, ROWS>(lds, prefix ? l.pk : l.k, prefix ? g.pkt : g.kt, n0,
                              prefix ? w.plen : w.own, lane);
}

// 32 rows in one workgroup; the waves take every fourth block of the keys and join at the
// end. K's next block is on its way while V of this one is used, and the other way round: one
// buffer of each a wave, so that two workgroups fit a compute unit. What bounds it is reading
// the keys: one token for each of 32 caches of 4096 (32 heads over 8, head dim 128, bf16) 100
// us, 5.3 TB/s; of 256 caches of 512 93 us, 5.8 TB/s; a single one of 8192 keys is bound by
// the latency of its blocks, about 2 us each, and so are the last workgroups of a batch of
// different lengths (32 x 4096, 267 MB: 65 us, 4.1 TB/s).
// The scores kept for the weights cost 8 us of 126 where each of 32 caches has 4096 keys.
template <int DT, int MODE, int D, bool WEIGH>
__device__ __forceinline__ void few_rows(const SharedArgs& g, const Work& w, char* s_buf, float* s_row) {
  constexpr int kBlk = 64 * D;                      // bytes of a block of 32 rows
  constexpr int kWave = 2 * kBlk;                   // K and V
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RowOf x = row_of(g, w, w.r0 + fr);
  if (!__any(x.live)) return;
  const Lists lists(g, w);
  const int32_t first = w.off + g.by_group.of(w.r0);     // position of the first row
  const int32_t pblocks = (w.plen + 31) >> 5;
  const int32_t n_lo = w.n_lo, n_hi = w.n_hi;
  float* scores = nullptr;                          // of this lane's row, for the weights
  if (WEIGH && g.scores != nullptr && !w.whole)
    scores = g.scores + (((int64_t)w.b * g.kv_heads + w.hk) * (g.sq * g.group) + w.r0 + fr) * score_row(g.skv) + 4 * h;
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
  u32x4 qf[D / 16];
  load_q<D>(g, x, h, qf);
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
    float e[16];
#pragma unroll
    for (int r = 0; r < 16; r += 2) row_exp<MODE>(s[r], s[r + 1], g.c0, c1, e[r], e[r + 1]);
#pragma unroll
    for (int r = 0; r < 16; r += 2) {                // summed as rounded: numerator and denominator
      const uint32_t pair = wpack<DT>(e[r], e[r + 1]);   // share the rounding
      acc.sum = wsum<DT>(pair, acc.sum);
      pr[r >> 3][(r >> 1) & 3] = pair;
    }
    if constexpr (WEIGH) all += sum16(e);
    if (more)
      wait_loads<kLoads>();                         // V is here, the next K may be on its way
    else
      wait_loads<0>();
    if constexpr (WEIGH) {
      // between the loads of K and V, whose number the waits go by
      if (scores != nullptr && !p && x.live) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(scores + n0 + 8 * i) = float4{s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]};
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        acc.o[d] = wmma<DT>(read_v<D>(buf + kBlk, lane, ks, d), pr[ks], acc.o[d]);
    wait_lds();
    if (more) load_v(n + kShWaves);
  }

  // join the waves: their M, then sums and O^T brought to the largest M; the rows of the
  // tile alone, four dims a lane
  float (*s_m)[32] = reinterpret_cast<float (*)[32]>(s_row);
  float (*s_sum)[32] = s_m + kShWaves, (*s_all)[32] = s_sum + kShWaves;
  acc.sum += other_half(acc.sum);
  if constexpr (WEIGH) all += other_half(all);
  const int32_t rows = min(32, w.rows - w.r0);
  constexpr int C = D / 4;                          // chunks of a row, swizzled
  if (fr < rows) {
    if (h == 0) {
      s_m[wave][fr] = acc.m;
      s_sum[wave][fr] = acc.sum;
      if constexpr (WEIGH) s_all[wave][fr] = all;
    }
    float4* mine = reinterpret_cast<float4*>(buf) + fr * C;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        mine[(8 * d + 2 * i + h) ^ (fr & 7)] =
            float4{acc.o[d][4 * i], acc.o[d][4 * i + 1], acc.o[d][4 * i + 2], acc.o[d][4 * i + 3]};
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * C; i += 64 * kShWaves) {
    const int r = i / C, c = i % C;
    float m = s_m[0][r];
#pragma unroll
    for (int j = 1; j < kShWaves; ++j) m = fmaxf(m, s_m[j][r]);
    float sum = 0.0f, every = 0.0f;
    float4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kShWaves; ++j) {
      const int32_t e = down_shift(s_m[j][r], m);
      const float4 o = reinterpret_cast<const float4*>(s_buf + j * kWave)[r * C + (c ^ (r & 7))];
      sum += __builtin_amdgcn_ldexpf(s_sum[j][r], e);
      if constexpr (WEIGH) every += __builtin_amdgcn_ldexpf(s_all[j][r], e);
      v.x += __builtin_amdgcn_ldexpf(o.x, e);
      v.y += __builtin_amdgcn_ldexpf(o.y, e);
      v.z += __builtin_amdgcn_ldexpf(o.z, e);
      v.w += __builtin_amdgcn_ldexpf(o.w, e);
    }
    if (w.part >= 0) {
      float* to = g.part + w.part * kPart<D>;
      if (c == 0) {
        to[r] = m;
        to[32 + r] = sum;
        if constexpr (WEIGH) to[64 + r] = every;
      }
      *reinterpret_cast<float4*>(to + 96 + r * D + 4 * c) = v;
      continue;
    }
    if constexpr (WEIGH) {
      if (c == 0)
        g.stats[((int64_t)w.b * g.kv_heads + w.hk) * 32 * g.tiles + w.r0 + r] =
            every > 0.0f ? float2{m, 1.0f / every} : float2{0.0f, 0.0f};
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    const int32_t query = g.by_group.of(w.r0 + r);
    *reinterpret_cast<u32x2*>(g.o + w.b * g.st.o[0] + query * g.st.o[1] +
                              (w.hk * g.group + w.r0 + r - query * g.group) * g.st.o[2] + 4 * c) =
        u32x2{wpack<DT>(v.x * inv, v.y * inv), wpack<DT>(v.z * inv, v.w * inv)};
  }
}

// 128 rows in one workgroup, 32 a wave, which share tiles of 64 keys in LDS (two blocks of
// 32; two tiles each of K and V), in the software pipeline of window_many_kernel: while
// block n's scores become probabilities, the scores of block n + 1 and the second product
// of block n - 1 are computed; one barrier a tile, between its blocks. 256 sequences
// of 32 heads over 8 x 32768 shared keys (head dim 128, bf16): 147 us without the join, 0.93
// PFLOP/s; 120 us, 1.15, where all operands are 0: power and its clock. By the counters
// products take 42 % of the cycles; a wave waits 26 % of its time for memory or a barrier and
// 32 % to issue; of about 220 instructions a wave and block 123 are VALU ones, 16 products, 42
// scalar.
template <int DT, int MODE, int D, bool WEIGH>
__device__ __forceinline__ void many_rows(const SharedArgs& g, const Work& w, char* s_buf) {
  constexpr int kTile = 2 * kShKeys * D;            // bytes of K or V of a tile
  constexpr int kRows = kShKeys / kShWaves;         // a wave loads
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t w0 = w.r0 + 32 * wave;
  const RowOf x = row_of(g, w, w0 + fr);
  const int32_t first = w.off + g.by_group.of(min(w0, w.rows - 1));
  const int32_t last = w.off + g.by_group.of(min(w0 + 31, w.rows - 1));
  const int32_t ptiles = (w.plen + kShKeys - 1) / kShKeys;
  const int32_t n_lo = w.n_lo, n_hi = w.n_hi;
  // blocks of 32 of the prefix, and of the own keys, that all rows of this wave see
  const int32_t pseen = w.plen >> 5, oseen = 2 * ptiles + (first < 0 ? 0 : (first + 1) >> 5);
  // tiles of which this wave's rows may see something
  const int32_t seen = w.whole || last < 0 ? 0 : last / kShKeys + 1;
  const int32_t t_hi = __any(x.live) ? min(n_hi, ptiles + seen) : n_lo;

  u32x4 qf[D / 16];
  load_q<D>(g, x, h, qf);
  const Lists lists(g, w);
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf + wave * kRows * 2 * D);
  // Whole tiles of the longer list go from a running base and this lane's own offsets, which
  // leaves two scalar instructions a load; the others as any run of keys.
  const bool main_p = w.plen >= w.own;
  const int32_t whole_lo = main_p ? 0 : ptiles, whole_hi = whole_lo + (main_p ? w.plen : w.own) / kShKeys;
  constexpr int RPL = 512 / D, NL = kRows / RPL;   // rows a load, loads of K or V of a tile
  uint32_t koff[NL], voff[NL];
  const uint32_t ktok = 2u * (uint32_t)(main_p ? g.pkt : g.kt), vtok = 2u * (uint32_t)(main_p ? g.pvt : g.vt);
  {
    constexpr int CH = D / 8;
    const int r = lane / CH, pc = lane % CH;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const uint32_t in = kRows * wave + RPL * j + r;
      koff[j] = in * ktok + 16u * (uint32_t)(pc ^ kswizzle<D>(RPL * j + r));
      voff[j] = in * vtok + 16u * (uint32_t)(pc ^ vswizzle<D>(RPL * j + r));
    }
  }
  const int64_t kstep = (int64_t)kShKeys * ktok, vstep = (int64_t)kShKeys * vtok;
  const char* kcur = scalar_base((const char*)(main_p ? lists.pk : lists.k) + (n_lo - whole_lo) * kstep);
  const char* vcur = scalar_base((const char*)(main_p ? lists.pv : lists.v) + (n_lo - whole_lo) * vstep);
  auto any_k = [&](int32_t t, uint32_t at) {
    stage_list<D, false, kRows>(lds + kTile * at, g, w, lists, t < ptiles,
                                kShKeys * (t < ptiles ? t : t - ptiles) + kRows * wave, lane);
  };
  // tiles one after the other from n_lo on
  auto load_k = [&](int32_t t) {
    const uint32_t at = (uint32_t)(t - n_lo) & 1u;
    if (t >= whole_lo && t < whole_hi) {
      uint32_t to = lds + kTile * at;
      asm volatile("" : "+s"(to));
#pragma unroll
      for (int j = 0; j < NL; ++j) lds_load16(to + 1024 * j, koff[j], kcur);
    } else {
      any_k(t, at);
    }
    kcur += kstep;
  };
  auto load_v = [&](int32_t t) {
    const uint32_t at = 2u + ((uint32_t)(t - n_lo) & 1u);
    if (t >= whole_lo && t < whole_hi) {
      uint32_t to = lds + kTile * at;
      asm volatile("" : "+s"(to));
#pragma unroll
      for (int j = 0; j < NL; ++j) lds_load16(to + 1024 * j, voff[j], vcur);
    } else {
      stage_list<D, true, kRows>(lds + kTile * at, g, w, lists, t < ptiles,
                                 kShKeys * (t < ptiles ? t : t - ptiles) + kRows * wave, lane);
    }
    vcur += vstep;
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
    if (n >= (n < 2 * ptiles ? pseen : oseen)) {     // not all keys are seen by all rows
      const bool p = n < 2 * ptiles;
      hide_behind(s, 32 * (p ? n : n - 2 * ptiles), p ? w.plen - 1 : x.pos, h);
    }
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
      // the operand that was read last first: one wait for both
      const f32x16 zero = {};
      acc.o[u % ND] = wmma<DT>(va[u], pp[u / ND], acc.o[u % ND]);
      sn = wmma<DT>(ka[u], qf[u], u == 0 ? zero : sn);
#pragma unroll
      for (int r = NE * u; r < NE * u + NE; r += 2) {
        float a, z;
        row_exp<MODE>(s[r], s[r + 1], g.c0, c1, a, z);
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
    if (t + 2 < n_hi) load_k(t + 2);
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
    any_k(n_lo, 3);    // V of the tile before the first is read (times 0): K's rows, finite where K is
    load_k(n_lo);
    load_v(n_lo);
    if (n_lo + 1 < n_hi) load_k(n_lo + 1);
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
    float* to = g.part + (w.part + (int64_t)wave * w.apart) * kPart<D>;
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
      g.stats[((int64_t)w.b * g.kv_heads + w.hk) * 32 * g.tiles + w0 + fr] =
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
  constexpr int CH = D / 8;
#pragma unroll
  for (int j = 0; j < 32 / RPL; ++j) {
    const int r = RPL * j + lane / CH, c = lane % CH;
    if (w0 + r >= w.rows) continue;
    const int32_t qi = g.by_group.of(w0 + r), hd = w.hk * g.group + w0 + r - qi * g.group;
    *reinterpret_cast<u32x4*>(g.o + w.b * g.st.o[0] + qi * g.st.o[1] + hd * g.st.o[2] + 8 * c) =
        *reinterpret_cast<const u32x4*>(ow + r * 2 * D + 16 * (c ^ kswizzle<D>(r)));
  }
}

// The groups' rows against the prefixes, then each sequence's against its own keys (where no
// rows of groups are formed: against the prefix first), whole or cut into parts.
template <int DT, int MODE, int D, bool WEIGH>
__global__ __launch_bounds__(64 * kShWaves, 2) void shared_kernel(SharedArgs g) {
  __shared__ __attribute__((aligned(16))) char s_buf[4 * 2 * kShKeys * D];
  __shared__ float s_row[3 * kShWaves * 32];
  Work w;
  bool many;
  int32_t split = 0;
  if (blockIdx.x < g.gwork) {
    w.whole = true;
    many = g.gmany != 0;
    const uint32_t id = by_xcd(blockIdx.x, g.gwork), rest = g.by_gtiles.of(id);
    const int32_t t32 = (int32_t)(id - rest * g.by_gtiles.d) * (many ? kShWaves : 1);
    const uint32_t bh = g.by_gsplit.of(rest), grp = g.by_heads.of(bh);
    split = (int32_t)(rest - bh * g.by_gsplit.d);
    w.hk = (int32_t)(bh - grp * g.by_heads.d);
    w.b = (int32_t)grp * g.members;
    w.r0 = 32 * t32;
    w.rows = g.members * g.sq * g.group;
    w.off = w.own = 0;
    w.plen = prefix_len(g, (int32_t)grp);
    w.apart = g.gsplit;
    w.part = group_part(g, bh, t32) + split;
  } else {
    w.whole = false;
    many = g.many != 0;
    const uint32_t at = blockIdx.x - g.gwork;
    uint32_t id = at;
    w.part = -1;
    w.apart = g.nsplit;
    if (g.cut) {
      // the first parts of all tiles, then the second ones: as sequences differ in length, the
      // last parts are the ones that have nothing to do
      split = (int32_t)g.by_items.of(at);
      id = at - (uint32_t)split * g.items;
      w.part = own_part(g, (int64_t)id * (many ? kShWaves : 1)) + split;
    }
    const TileOf t = tile_of(g, id);
    w.b = (int32_t)g.by_heads.of(t.bh);
    w.hk = (int32_t)t.bh - w.b * g.kv_heads;
    w.r0 = t.tile * (many ? 32 * kShWaves : 32);
    const int32_t qlen = seq_len(g.q_lens, w.b, g.sq);
    w.off = seq_len(g.kv_lens, w.b, g.skv) - qlen;
    w.rows = qlen * g.group;
    w.own = tile_keys(g, w.off, w.r0, w.rows);
    w.plen = g.gsplit > 0 ? 0 : prefix_len(g, g.by_members.of(w.b));
  }
  if (w.r0 >= w.rows) return;
  w.n_lo = 0;
  w.n_hi = list_blocks(w.plen, w.own, many);
  if (w.part >= 0) {
    const int32_t per = (int32_t)(w.whole ? g.by_gper.d : g.by_per.d);
    w.n_lo = split * per;
    w.n_hi = min(w.n_hi, w.n_lo + per);
    if (w.n_lo >= w.n_hi) return;
  }
  if (many)
    many_rows<DT, MODE, D, WEIGH>(g, w, s_buf);
  else
    few_rows<DT, MODE, D, WEIGH>(g, w, s_buf, s_row);
}

// The parts of a row: first those of the group's tile, then those of the sequence's.
struct Parts {
  const float *pg, *po;      // first parts
  int32_t ng, n;             // the group's, all
  int32_t fg, fo;            // the row in either tile
};
template <int D>
__device__ __forceinline__ Parts parts_of(const SharedArgs& g, uint32_t id, uint32_t bh, int b, int32_t row,
                                          int32_t rows, int32_t off) {
  Parts p;
  const int hk = (int)bh - b * g.kv_heads, grp = g.by_members.of(b);
  const int32_t plen = prefix_len(g, grp);
  const int32_t of_group = (b - grp * g.members) * g.sq * g.group + row;
  const int32_t t32 = row >> 5, in = g.many ? t32 & (kShWaves - 1) : 0;   // in: of the workgroup's tile
  p.ng = g.gsplit > 0 ? list_parts(plen, 0, g.gmany != 0, g.by_gper) : 0;
  p.pg = g.part + group_part(g, (int64_t)grp * g.kv_heads + hk, of_group >> 5) * kPart<D>;
  p.po = g.part + own_part(g, (int64_t)id * (g.many ? kShWaves : 1) + in) * kPart<D>;
  p.n = p.ng + list_parts(g.gsplit > 0 ? 0 : plen, tile_keys(g, off, 32 * (t32 - in), rows), g.many != 0, g.by_per);
  p.fg = of_group & 31;
  p.fo = row & 31;
  return p;
}
template <int D>
__device__ __forceinline__ const float* part_at(const Parts& p, int32_t i, int32_t& fr) {
  fr = i < p.ng ? p.fg : p.fo;
  return i < p.ng ? p.pg + (int64_t)i * kPart<D> : p.po + (int64_t)(i - p.ng) * kPart<D>;
}

// Joins the parts of a row (2048 rows of 10 parts 6 us, 8192 of 9 11 us: the latency of the
// lengths, then the parts): T teams of D / 4 lanes, a lane for every four dims, which take
// every T-th part with several loads in flight; then the teams' results in LDS. The order
// is fixed.
template <int DT, int D, bool WEIGH, int T>
__device__ __forceinline__ void join_rows(const SharedArgs& g, uint32_t block, float* s_row, float4 (*s_v)[D / 4]) {
  constexpr int C = D / 4, TEAMS = 256 / C, R = TEAMS / T, U = 4;
  const int team = threadIdx.x / C, c = threadIdx.x % C, k = team % T;   // team k of its row
  const uint32_t n = block * R + team / T;                               // row of all that are joined
  // all tiles of 128 rows; else all rows of all key heads
  const uint32_t per = g.by_rows.d, item = g.by_rows.of(n);
  int32_t row = (int32_t)(n - item * per);
  uint32_t id = item, bh = item;
  bool in;
  if (g.many) {
    const TileOf t = tile_of(g, id);
    bh = t.bh;
    row += t.tile * (int32_t)per;
    in = item < g.items;
  } else {
    id = number_of(g, bh, row >> 5);
    in = item < g.heads;
  }
  const int b = (int)g.by_heads.of(bh), hk = (int)bh - b * g.kv_heads;
  const int32_t qlen = in ? seq_len(g.q_lens, b, g.sq) : 0, rows = qlen * g.group;
  const bool live = row < rows;
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
  if (live) {
    const Parts p = parts_of<D>(g, id, bh, b, row, rows, seq_len(g.kv_lens, b, g.skv) - qlen);
    for (int32_t s0 = k; s0 < p.n; s0 += U * T) {
      float om[U], os[U], oe[U];
      float4 ov[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {   // past the last one: that one again, not added
        int32_t fr;
        const float* x = part_at<D>(p, min(s0 + j * T, p.n - 1), fr);
        om[j] = x[fr];
        os[j] = x[32 + fr];
        oe[j] = WEIGH ? x[64 + fr] : 0.0f;
        ov[j] = *reinterpret_cast<const float4*>(x + 96 + fr * D + 4 * c);
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (s0 + j * T < p.n) add(om[j], os[j], oe[j], ov[j]);
    }
  }
  if constexpr (T > 1) {
    s_v[team][c] = v;
    if (c == 0) {
      s_row[team] = m;
      s_row[TEAMS + team] = sum;
      s_row[2 * TEAMS + team] = every;
    }
    __syncthreads();
    if (k > 0) return;
#pragma unroll
    for (int o = 1; o < T; ++o)
      add(s_row[team + o], s_row[TEAMS + team + o], s_row[2 * TEAMS + team + o], s_v[team + o][c]);
  }
  if (!live) return;
  if constexpr (WEIGH) {
    if (c == 0 && g.scores == nullptr)
      g.stats[(int64_t)bh * 32 * g.tiles + row] = every > 0.0f ? float2{m, 1.0f / every} : float2{0.0f, 0.0f};
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  const int32_t query = g.by_group.of(row);
  uint16_t* orow = g.o + b * g.st.o[0] + query * g.st.o[1] + (hk * g.group + row - query * g.group) * g.st.o[2];
  *reinterpret_cast<u32x2*>(orow + 4 * c) =
      u32x2{wpack<DT>(v.x * inv, v.y * inv), wpack<DT>(v.z * inv, v.w * inv)};
}

// The weight of kScoreSlots slots of a key head whose rows are one tile of 32: the scores
// that the tiles left, against the rows' final M, which is joined here from the parts. Reading
// 4 bytes a row and key again costs less than the key once more: 32 caches of 4096 keys, head
// dim 128, groups of 4, against weigh_rows_kernel: 1 token 127 / 199 us, 4 tokens 156 / 208, 8
// (32 rows) 195 / 216; 16 x 4096 at head dim 64 with 1 row 69 / 124, 32 rows 134 / 134. Where
// 64 workgroups at most go over at most 1024 keys the second launch is dearer (26 / 23 us for
// 2 caches of 1000 keys and 32 rows), and the rows do it there.
constexpr int kScoreSlots = 1024;

template <int MODE, int D>
__device__ __forceinline__ void weigh_slots(const SharedArgs& g, uint32_t bh, int32_t j0, float* s_row) {
  const int b = (int)g.by_heads.of(bh), hk = (int)bh - b * g.kv_heads;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t rows = qlen * g.group, off = kvlen - qlen;
  if (j0 >= kvlen || rows == 0) return;
  {
    // 8 lanes a row
    const int32_t row = threadIdx.x >> 3, k = threadIdx.x & 7;
    float m = kNoMax, all = 0.0f;
    if (row < rows) {
      const Parts p = parts_of<D>(g, bh, bh, b, row, rows, off);
      for (int32_t i = k; i < p.n; i += 8) {
        int32_t fr;
        const float* x = part_at<D>(p, i, fr);
        const float top = fmaxf(m, x[fr]);
        all = __builtin_amdgcn_ldexpf(all, down_shift(m, top)) +
              __builtin_amdgcn_ldexpf(x[64 + fr], down_shift(x[fr], top));
        m = top;
      }
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      const float om = __shfl_xor(m, o, 64), oa = __shfl_xor(all, o, 64), top = fmaxf(m, om);
      all = __builtin_amdgcn_ldexpf(all, down_shift(m, top)) + __builtin_amdgcn_ldexpf(oa, down_shift(om, top));
      m = top;
    }
    if (k == 0) {
      s_row[row] = all > 0.0f ? row_c1<MODE>(m) : 0.0f;
      s_row[32 + row] = all > 0.0f ? 1.0f / all : 0.0f;
    }
  }
  __syncthreads();
  const int32_t j = j0 + 4 * (int32_t)threadIdx.x;
  if (j >= kvlen) return;
  const int64_t ld = score_row(g.skv);
  const float* x = g.scores + (int64_t)bh * (g.sq * g.group) * ld + j;
  float a[4] = {};
  for (int32_t r = 0; r < rows; ++r) {
    if (off + g.by_group.of(r) < j) continue;            // no part of this row's tile need be there
    const float4 s = *reinterpret_cast<const float4*>(x + r * ld);
    const float c1 = s_row[r], inv = s_row[32 + r];
    float e[4];
    row_exp<MODE>(s.x, s.y, g.c0, c1, e[0], e[1]);
    row_exp<MODE>(s.z, s.w, g.c0, c1, e[2], e[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __builtin_fmaf(e[i], inv, a[i]);
  }
  float* to = g.weight + b * g.st.weight[0] + hk * g.st.weight[1] + j;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (j + i < kvlen) to[i] += a[i];
}

// Joins the parts of the rows and, in workgroups of their own, weighs the slots.
template <int DT, int MODE, int D, bool WEIGH, int T>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs g, uint32_t joins, uint32_t slot_blocks) {
  __shared__ float s_row[3 * 32];
  __shared__ float4 s_v[1024 / D][D / 4];
  if constexpr (WEIGH) {
    if (blockIdx.x >= joins) {
      const uint32_t i = blockIdx.x - joins;
      weigh_slots<MODE, D>(g, i / slot_blocks, (int32_t)(i % slot_blocks) * kScoreSlots, s_row);
      return;
    }
  }
  join_rows<DT, D, WEIGH, T>(g, blockIdx.x, s_row, s_v);
}

// The weight that 256 slots gather from a chunk of the rows. A wave holds the K of 64 slots;
// the rows' queries go through LDS, 64 at a time for all waves, two buffers: the scores
// again, the exponentials against the rows' final M, times 1 / sum. A slot's rows are added
// in a fixed order, chunks by weigh_add_kernel. VALU issue bounds it: a prompt of 4096 tokens
// (32 heads over 8, head dim 128, bf16) 121 us beside the 159 of its attention.
constexpr int kWeighSlots = 64 * kShWaves, kWeighStep = 64, kWeighRows = 1024;

template <int DT, int MODE, int D>
__global__ __launch_bounds__(64 * kShWaves, 2) void weigh_rows_kernel(SharedArgs g, uint32_t slot_tiles,
                                                                      uint32_t chunks) {
  constexpr int kBuf = 2 * kWeighStep * D + 1024;    // bytes: queries, then M and 1 / sum of 128 rows
  constexpr int CH = D / 8, RPL = 64 / CH, kRows = kWeighStep / kShWaves, N = kRows / RPL;
  __shared__ __attribute__((aligned(16))) char s_buf[2 * kBuf];
  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // late slots see few rows: the early ones first
  const uint32_t heads = g.heads, t_chunk = blockIdx.x / heads, bh = blockIdx.x - t_chunk * heads;
  const uint32_t chunk = chunks - 1u - t_chunk % chunks, tile = t_chunk / chunks;
  const int b = (int)g.by_heads.of(bh), hk = (int)bh - b * g.kv_heads;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t first_slot = (int32_t)tile * kWeighSlots, j0 = first_slot + 64 * wave;
  if (first_slot >= kvlen) return;
  const int32_t off = kvlen - qlen, rows = qlen * g.group;
  // rows of this chunk that may see the first slot
  const int32_t from = max(0, first_slot - off);
  const int32_t lo = max(from >= qlen ? rows : (from * g.group) & ~(kWeighStep - 1), (int32_t)chunk * kWeighRows);
  const int32_t hi = min(rows, ((int32_t)chunk + 1) * kWeighRows);

  u32x4 kf[2][D / 16];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint16_t* kr = g.k + b * g.st.k[0] + (int64_t)min(j0 + 32 * u + fr, kvlen - 1) * g.kt + hk * g.st.k[2] + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[u][ks] = *reinterpret_cast<const u32x4*>(kr + 16 * ks);
  }
  settle(kf[0]);
  settle(kf[1]);
  const uint16_t* Q = g.q + b * g.st.q[0] + hk * g.group * g.st.q[2];
  const float2* stats = g.stats + (int64_t)bh * 32 * g.tiles;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf);
  // Queries r0 on to buffer `at`: this wave's kRows of them, chunks swizzled as K's. Where
  // whole queries make up a step and lie close, from a running base and this lane's own
  // offsets.
  const bool near = kWeighStep % g.group == 0 && (g.sq == 1 || g.st.q[1] <= (1 << 23)) &&
                    (g.group == 1 || g.st.q[2] <= (1 << 23));
  const int lr = lane / CH, pc = lane % CH;
  uint32_t qoff[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int32_t in = kRows * wave + RPL * j + lr, query = g.by_group.of(in);
    qoff[j] = 2u * ((uint32_t)query * (uint32_t)g.st.q[1] + (uint32_t)(in - query * g.group) * (uint32_t)g.st.q[2]) +
              16u * (uint32_t)(pc ^ kswizzle<D>(RPL * j + lr));
  }
  auto load = [&](int32_t r0, int at) {
    uint32_t lds = lds0 + kBuf * at;
    asm volatile("" : "+s"(lds));
    if (near && r0 + kWeighStep <= rows) {
      const char* base = scalar_base(Q + (int64_t)g.by_group.of(r0) * g.st.q[1]);
#pragma unroll
      for (int j = 0; j < N; ++j) lds_load16(lds + kRows * 2 * D * wave + 1024 * j, qoff[j], base);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int32_t row = min(r0 + kRows * wave + RPL * j + lr, rows - 1), query = g.by_group.of(row);
        const uint16_t* p = Q + query * g.st.q[1] + (row - query * g.group) * g.st.q[2];
        lds_load16(lds + kRows * 2 * D * wave + 1024 * j, p + 8 * (pc ^ kswizzle<D>(RPL * j + lr)));
      }
    }
    if (wave == 0) lds_load16(lds + 2 * kWeighStep * D, reinterpret_cast<const char*>(stats + r0) + 16 * lane);
  };
  float acc[2][16] = {};
  if (lo < hi) load(lo, 0);
  int at = 0;
  for (int32_t r0 = lo; r0 < hi; r0 += kWeighStep, at ^= 1) {
    wait_loads<0>();
    __syncthreads();                                 // this buffer is here, the other one done with
    if (r0 + kWeighStep < hi) load(r0 + kWeighStep, at ^ 1);
    const char* buf = s_buf + kBuf * at;
#pragma unroll
    for (int t = 0; t < kWeighStep / 32; ++t) {
      const int32_t row = r0 + 32 * t + fr;
      f32x16 s[2] = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const u32x4 qf = read_k<D>(buf + 64 * D * t, fr, h, ks);
        s[0] = wmma<DT>(kf[0][ks], qf, s[0]);
        s[1] = wmma<DT>(kf[1][ks], qf, s[1]);
      }
      const float2 ms = *reinterpret_cast<const float2*>(buf + 2 * kWeighStep * D + 8 * (32 * t + fr));
      const bool in = row < hi;
      const float c1 = in ? row_c1<MODE>(ms.x) : -INFINITY, inv = in ? ms.y : 0.0f;   // e = 0 behind the rows
      const int32_t first = off + g.by_group.of(r0 + 32 * t);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (first < j0 + 32 * u + 31) hide_behind(s[u], j0 + 32 * u, off + g.by_group.of(row), h);
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          float a, z;
          row_exp<MODE>(s[u][r], s[u][r + 1], g.c0, c1, a, z);
          acc[u][r] = __builtin_fmaf(a, inv, acc[u][r]);
          acc[u][r + 1] = __builtin_fmaf(z, inv, acc[u][r + 1]);
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float mine = 0.0f;                               // lane r < 16 of a half: slot r's sum
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float v = acc[u][r];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) v += __shfl_xor(v, o, 64);
      mine = fr == r ? v : mine;
    }
    const int32_t j = j0 + 32 * u + 8 * (fr >> 2) + 4 * h + (fr & 3);
    if (fr >= 16 || j >= kvlen) continue;
    if (chunks == 1)
      g.weight[b * g.st.weight[0] + hk * g.st.weight[1] + j] += mine;
    else
      g.sums[((int64_t)bh * chunks + chunk) * g.skv + j] = mine;
  }
}

__global__ __launch_bounds__(256) void weigh_add_kernel(SharedArgs g, uint32_t blocks, uint32_t chunks) {
  const uint32_t bh = blockIdx.x / blocks;
  const int b = (int)g.by_heads.of(bh), hk = (int)bh - b * g.kv_heads;
  const int32_t kvlen = seq_len(g.kv_lens, b, g.skv), qlen = seq_len(g.q_lens, b, g.sq);
  const int32_t j = (int32_t)(blockIdx.x % blocks) * 256 + (int32_t)threadIdx.x;
  if (j >= kvlen) return;
  const float* x = g.sums + (int64_t)bh * chunks * g.skv + j;
  const uint32_t n = ((uint32_t)(qlen * g.group) + kWeighRows - 1) / kWeighRows;
  float v = 0.0f;
  for (uint32_t i = 0; i < n; ++i) v += x[(int64_t)i * g.skv];
  g.weight[b * g.st.weight[0] + hk * g.st.weight[1] + j] += v;
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
// How a call is cut up. Rows of a whole group against the prefix where a sequence alone has
// few: the prefix is then read once for all, and its scores are full tiles.
struct SharedPlan {
  int64_t gtiles = 0, gchunk = 1, gsplit = 0, gitems = 0;   // items: tiles of a workgroup
  int64_t tiles = 0, chunk = 1, nsplit = 1, items = 0;
  bool gmany = false, many = false, cut = false, stored = false;
};
constexpr int64_t kShSlots = 512;       // workgroups that run at once
// From kManyRows rows on, 128 rows share a workgroup. Up to kBriefSteps steps a compute unit,
// a workgroup a tile goes over all keys and nothing is joined: 4 to 16 sequences, 8 key heads, a
// prefix of 1000 keys 13 to 14 us against 15 with rows of groups and a join, of 2000 21 to 22
// against 16; 64 sequences: 500 keys 14 / 17, 1000 20 / 18.
constexpr int64_t kManyRows = 96, kBriefSteps = 16;

// Steps of 64 keys a workgroup of 32 rows takes of `all`: four rounds of workgroups where
// there is enough, as sequences differ in length; at least 512 keys, unless compute units
// would be left without work. (32 caches of up to 4096: 256 keys each 78 us, 512 70, 1024 70,
// 4096 69; with weights 85, 80, 83, 88. 64 over 8192 shared and up to 1024 own keys: 128 own
// keys a workgroup 65 us, 256 57, 512 55, 1024 55.)
static int64_t few_chunk(int64_t all) {
  const auto per = [&](int64_t n) { return (all + n - 1) / n; };
  return std::max({per(4 * kShSlots), std::min<int64_t>(8, per(kShSlots / 2)), (int64_t)2});
}

// The same for 128 rows: one round; at least 1024 keys, unless most compute units would be
// left without work (they have the sequences' own keys to read meanwhile). 64 over 8192 shared
// keys: 256 keys a workgroup 74 us, 512 62, 1024 55, 1536 58; 16 x 5 tokens over 10007: 512
// keys 48 us, 1024 43, 1280 39, 2048 48.
static int64_t many_chunk(int64_t all) {
  const auto per = [&](int64_t n) { return (all + n - 1) / n; };
  return std::max({per(kShSlots), std::min<int64_t>(16, per(kShSlots / 4)), (int64_t)4});
}

static int64_t wide_tiles(int64_t rows, bool many) { return many ? (rows + 127) / 128 : (rows + 31) / 32; }

static SharedPlan shared_plan(const SharedShape& s, bool weigh, bool workspace) {
  SharedPlan p;
  const int64_t rows = s.sq * s.group(), all = rows * (s.batch / s.groups);
  p.tiles = (rows + 31) / 32;
  p.many = rows >= kManyRows;
  const int64_t items = p.items = s.batch * s.kv_heads * wide_tiles(rows, p.many);
  if (!workspace || items == 0 || items >= (1 << 18)) return p;   // 32 rows a tile are joined in one launch
  const int64_t psteps = (s.sp + 63) / 64;
  int64_t steps = (s.skv + 63) / 64;
  // few keys, which a workgroup a tile goes over in the time that a second launch takes
  const bool brief = !p.many && (psteps + steps) * ((items + 255) / 256) <= kBriefSteps;
  p.stored = weigh && rows <= 32 && !(brief && items <= 64);
  if (s.sp > 0 && rows < kManyRows && all > rows && !brief) {
    p.gtiles = (all + 31) / 32;
    p.gmany = all > 32;
    p.gitems = s.groups * s.kv_heads * wide_tiles(all, p.gmany);
    p.gchunk = std::min(p.gmany ? many_chunk(psteps * p.gitems) : few_chunk(psteps * p.gitems), psteps);
    p.gsplit = (psteps + p.gchunk - 1) / p.gchunk;
  } else {
    steps += psteps;
  }
  if (p.many) {
    // Tiles that leave workgroups idle are cut up: a prompt of 600 tokens behind 4096 shared keys
    // (152 tiles) 64 us, uncut 87; two of 900 behind 2000 (464 tiles) 93 either way, as are 8 of
    // 600 (1216 tiles, 355 us) with the last round's tiles cut or not.
    p.cut = items <= kShSlots * 3 / 4;
    p.chunk = !p.cut ? 1 : std::max<int64_t>(8, (steps * items + kShSlots - 1) / kShSlots);
  } else {
    p.cut = true;
    p.chunk = brief ? steps : few_chunk(steps * items);
  }
  p.chunk = std::max<int64_t>(1, std::min(p.chunk, steps));   // the kernels divide by 31-bit numbers
  p.nsplit = std::max<int64_t>(1, (steps + p.chunk - 1) / p.chunk);
  if (p.nsplit == 1 && p.gsplit == 0 && !p.stored) p.cut = false;   // nothing to join
  if (!p.cut) p.nsplit = 1;
  return p;
}

static int64_t slot_tiles(const SharedShape& s) { return (s.skv + kWeighSlots - 1) / kWeighSlots; }
static int64_t weigh_chunks(const SharedShape& s) { return (s.sq * s.group() + kWeighRows - 1) / kWeighRows; }
static bool weigh_shape_ok(const SharedShape& s) {
  return s.batch * s.kv_heads * slot_tiles(s) < (1 << 24) &&
         s.batch * s.kv_heads * slot_tiles(s) * weigh_chunks(s) < (1 << 24);
}

// The workspace: parts, then what the weights need.
struct SharedSpace {
  int64_t part, stats, scores, sums;
  int64_t total() const { return part + stats + scores + sums; }
};
static SharedSpace shared_space(const SharedShape& s, const SharedPlan& p, bool weigh) {
  SharedSpace x{};
  const int64_t heads = s.batch * s.kv_heads;
  const int64_t n = s.groups * s.kv_heads * p.gtiles * p.gsplit + p.items * (p.many ? kShWaves : 1) * p.nsplit;
  if (p.cut) x.part = n * (96 + 32 * s.dim) * 4;
  if (!weigh || heads * s.sq == 0) return x;
  if (p.stored) {
    x.scores = heads * s.sq * s.group() * score_row(s.skv) * 4;
  } else {
    x.stats = heads * 32 * p.tiles * 8 + 1024;       // whole blocks of 128 rows are read
    if (weigh_chunks(s) > 1) x.sums = (heads * weigh_chunks(s) * s.skv * 4 + 15) / 16 * 16;
  }
  return x;
}

template <int DT, int MODE, int D, bool WEIGH>
static void launch_shared(const SharedShape& s, hipStream_t stream, const SharedArgs& g) {
  const int64_t heads = s.batch * s.kv_heads;
  const dim3 block(64 * kShWaves);
  const uint32_t work = g.gwork + g.items * (uint32_t)g.nsplit;
  hipLaunchKernelGGL((shared_kernel<DT, MODE, D, WEIGH>), dim3(work), block, 0, stream, g);
  const bool stored = WEIGH && g.scores != nullptr;
  if (g.cut) {
    const uint32_t slots = stored ? (uint32_t)((s.skv + kScoreSlots - 1) / kScoreSlots) : 0u;
    const int64_t rows = g.many ? (int64_t)g.items * 32 * kShWaves : heads * s.sq * s.group();
    const auto launch = [&](auto teams) {
      constexpr int T = decltype(teams)::value, R = 1024 / D / T;
      const uint32_t joins = (uint32_t)((rows + R - 1) / R);
      hipLaunchKernelGGL((shared_join_kernel<DT, MODE, D, WEIGH, T>), dim3(joins + (uint32_t)heads * slots), dim3(256), 0,
                         stream, g, joins, slots);
    };
    const int32_t parts = g.gsplit + g.nsplit;
    if (parts <= 16) launch(std::integral_constant<int, 1>{});
    else launch(std::integral_constant<int, 8>{});
  }
  if constexpr (WEIGH) {
    const uint32_t n = (uint32_t)slot_tiles(s), chunks = (uint32_t)weigh_chunks(s);
    if (stored || n == 0) return;
    hipLaunchKernelGGL((weigh_rows_kernel<DT, MODE, D>), dim3((uint32_t)heads * n * chunks), block, 0, stream, g, n, chunks);
    if (chunks > 1) {
      const uint32_t blocks = (uint32_t)((s.skv + 255) / 256);
      hipLaunchKernelGGL(weigh_add_kernel, dim3((uint32_t)heads * blocks), dim3(256), 0, stream, g, blocks, chunks);
    }
  }
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
  const bool weighs = weigh != 0 && skv > 0;
  if (bytes == nullptr || !shared_shape_ok(s) || (weighs && !weigh_shape_ok(s))) return QUAKE_EINVAL;
  *bytes = shared_space(s, shared_plan(s, weighs, true), weighs).total();
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
  const bool weigh = weight != nullptr && skv > 0;
  const int64_t nw[2] = {batch, kv_heads};
  const int64_t* sw = st.weight;
  if (weigh) {
    if (!weigh_shape_ok(s)) return QUAKE_EINVAL;
    for (int i = 0; i < 2; ++i)
      if (nw[i] > 1 && (sw[i] < 0 || sw[i] > INT64_MAX / 8 / nw[i])) return QUAKE_EINVAL;
    if (!rows_apart(sw, nw, 2, skv)) return QUAKE_EINVAL;
    if (workspace == nullptr) return QUAKE_EINVAL;
  }
  const SharedPlan p = shared_plan(s, weigh, workspace != nullptr);
  const SharedSpace space = shared_space(s, p, weigh);
  const int64_t need = space.total();
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
  g.weight = weigh ? weight : nullptr;
  g.prefix_lens = prefix_lens;
  g.q_lens = q_lens;
  g.kv_lens = kv_lens;
  char* ws = static_cast<char*>(workspace);
  g.part = reinterpret_cast<float*>(ws);
  if (space.stats > 0) g.stats = reinterpret_cast<float2*>(ws + space.part);
  if (space.scores > 0) g.scores = reinterpret_cast<float*>(ws + space.part + space.stats);
  if (space.sums > 0) g.sums = reinterpret_cast<float*>(ws + space.part + space.stats + space.scores);
  g.st = st;
  g.sq = (int32_t)sq;
  g.sp = (int32_t)sp;
  g.skv = (int32_t)skv;
  g.group = (int32_t)s.group();
  g.kv_heads = (int32_t)kv_heads;
  g.members = (int32_t)(batch / groups);
  g.pkt = (int32_t)st.prefix_k[1];
  g.pvt = (int32_t)st.prefix_v[1];
  g.kt = (int32_t)st.k[1];
  g.vt = (int32_t)st.v[1];
  g.groups = (int32_t)groups;
  g.gtiles = (int32_t)p.gtiles;
  g.gmany = p.gmany;
  g.gsplit = (int32_t)p.gsplit;
  g.gwork = (uint32_t)(p.gitems * p.gsplit);
  g.tiles = (int32_t)p.tiles;
  g.many = p.many;
  g.cut = p.cut;
  g.nsplit = (int32_t)p.nsplit;
  g.by_group = Div(s.group());
  g.by_sq = Div(sq);
  g.by_members = Div(batch / groups);
  g.by_heads = Div(kv_heads);
  g.by_gtiles = Div(p.gmany ? (p.gtiles + kShWaves - 1) / kShWaves : p.gtiles);
  g.by_gsplit = Div(p.gsplit);
  g.by_tiles = Div(p.many ? (p.tiles + kShWaves - 1) / kShWaves : p.tiles);
  g.by_items = Div(p.items);
  g.by_gper = Div(p.gchunk * (p.gmany ? 1 : 2));
  g.by_per = Div(p.chunk * (p.many ? 1 : 2));
  g.by_rows = Div(p.many ? 32 * kShWaves : sq * s.group());
  g.heads = (uint32_t)(batch * kv_heads);
  g.items = (uint32_t)p.items;
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
