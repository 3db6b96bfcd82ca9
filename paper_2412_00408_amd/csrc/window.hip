// window.hip — quake_attention_window: attention over a key/value cache with a
// sliding window and sink tokens, o_i = sum_j p_ij v_j / sum_j p_ij over the keys
// query i sees (j <= pos_i and (j > pos_i - window or j < sinks)).
//
// The exponentials are QuAKE's (arXiv:2412.00408), taken against a whole number M
// of base-2 units instead of the row max itself: Q(y - M) = 2^-M Q(y) exactly for
// the bit constructions too, as M only moves the exponent field (l of Eq. 5 moves
// by M 2^23, its mantissa bits stay). So here, unlike in Algorithm 2 with its
// real-valued max, a running M can be raised later by an exact power of two: the
// keys are read once, and partial results of different keys are brought to one M
// without an error, whatever their number. (Roundings stay: l's at the M of its time,
// the 16-bit ones, and those of binary32 sums in their order.) c1 = (127 - M) 2^23 is
// exact in binary32 for |M| < 2^23, which |t q.k| < 1e6 keeps far from, so
// l = fma(s, c0, c1) has one rounding; M is then off by less than 1/8 unit of the row's
// max, which binary16's largest probability, 2^15, has room for. M follows the
// running max lazily, only when it falls more than kLazy below (probabilities then
// reach 2^kLazy, binary16's 2^(kLift + kLazy), which binary32 sums and both 16-bit
// formats hold with the same relative rounding).
//
// Rows. The queries of all heads that share a key head are one list of rows,
// row r = query r / group, head r mod group of the group, so a single token's
// group fills one tile and a tile of a prompt covers few positions, whose windows
// nearly coincide. Keys. A tile's keys are the list "sinks below the window, then
// the window" (Span), cut into blocks of 32 from its first key on, not at
// multiples of 32; keys that no row of the tile sees are never read.
//
// Products (matrix cores, v_mfma_f32_32x32x16): S^T = K Q^T with K staged in LDS,
// lane l then holding row l mod 32 and keys 8 g + 4 (l / 32) + i of the block,
// i, g < 4; O^T = V^T P with the same lane's exponentials as the B operand as they
// lie: the 16 keys of a step are numbered 8 (e / 4) + 4 (l / 32) + e mod 4, e < 8,
// on both sides, so nothing is exchanged between lanes. The A operand, V^T, comes
// from V's rows in LDS by ds_read_b64_tr_b16 (16 lanes read 4 keys x 16 dims and
// each receives its dim's 4 keys), so V needs no transposed copy.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "quake_device.hpp"
#include "quake_host.hpp"

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
constexpr int kWinWaves = 4;

struct WindowArgs {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  const int32_t *q_lens, *kv_lens;   // or null: sq, skv
  float* ws;                         // partial results, nsplit > 1
  int64_t qb, qs, qh, kb, ks, kh, vb, vs, vh, ob, os, oh;   // strides in elements
  int32_t sq, skv, group, kv_heads, tiles, nsplit;
  uint32_t window, sinks;
  float c0;                          // 2^23 t / ln2 (EXACT: t / ln2)
};

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

// The keys of a tile of rows at positions first .. last: number n of the list is
// key n below `sinks` (of them those below the window), else key n + shift.
struct Span {
  int32_t sinks, shift, total;
  __device__ __forceinline__ Span(int32_t first, int32_t last, const WindowArgs& g) {
    int32_t low = 0;
    if (first >= 0 && (uint32_t)first >= g.window) low = first - (int32_t)g.window + 1;
    sinks = 0;
    if (g.sinks < (uint32_t)low)
      sinks = (int32_t)g.sinks;
    else
      low = 0;
    shift = low - sinks;
    total = last < 0 ? 0 : last + 1 - shift;
  }
  __device__ __forceinline__ int32_t key(int32_t n) const { return n < sinks ? n : n + shift; }
};

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

// Loads ROWS keys of the list from n0 on into LDS rows (1024 bytes a load: 64 lanes x
// 16; ROWS a multiple of 16, the period of the swizzles). Whole runs of the window go
// from a uniform base; those that hold sinks or end behind the list from each lane's
// own row, the list's last key standing for those behind it (their probabilities are
// 0).
template <int D, bool IS_V, int ROWS>
__device__ __forceinline__ void stage_rows(uint32_t lds, const uint16_t* base, int64_t stride,
                                           const Span& sp, int32_t n0, int lane) {
  constexpr int CH = D / 8, RPL = 64 / CH, N = ROWS / RPL;   // chunks a row, rows a load, loads
  const int r = lane / CH, pc = lane % CH;
  if (n0 >= sp.sinks && n0 + ROWS <= sp.total) {
    const char* b = scalar_base(base + (int64_t)(n0 + sp.shift) * stride);
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
      const int32_t key = sp.key(min(n0 + RPL * j + r, sp.total - 1));
      lds_load16(lds + 1024 * j, base + (int64_t)key * stride + 8 * (pc ^ sw));
    }
  }
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

// whether rows at positions first .. last see all of 32 keys of the list
__device__ __forceinline__ bool all_seen(const Span& sp, int32_t n0, int32_t first, int32_t last,
                                         const WindowArgs& g) {
  const int32_t a = sp.key(n0), z = sp.key(n0 + 31);
  return z <= first && z - a == 31 && ((uint32_t)z < g.sinks || (uint32_t)(last - a) < g.window);
}

// -inf for the keys of block n0 that the row at `pos` does not see
__device__ __forceinline__ void mask_block(f32x16& s, const Span& sp, int32_t n0, int32_t pos,
                                           int h, const WindowArgs& g) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int32_t key = sp.key(n0 + 8 * (r >> 2) + 4 * h + (r & 3));
    const uint32_t limit = (uint32_t)key < g.sinks ? 0x80000000u : g.window;
    s[r] = (uint32_t)(pos - key) < limit ? s[r] : -INFINITY;
  }
}

__device__ __forceinline__ int32_t seq_len(const int32_t* lens, int b, int32_t most) {
  return lens == nullptr ? most : min(max(lens[b], 0), most);
}

// A tile of 32 rows in one workgroup; the waves take every fourth block of its
// keys and join at the end. What bounds it is reading the keys (single tokens),
// so each wave keeps the next block's K and V in flight. One token for each of 64
// caches of up to 8192 (window 4096, 32 heads over 8, head dim 128, bf16): 164 us,
// 5.5 TB/s; for one cache of 8192 tokens (32 splits) 10.8 us, 3.1 TB/s, and 3.8 us to
// join them.
template <int DT, int MODE, int D>
__global__ __launch_bounds__(64 * kWinWaves) void window_few_kernel(WindowArgs g) {
  constexpr int kBlk = 64 * D;                      // bytes of a block of 32 rows
  constexpr int kWave = 4 * kBlk;                   // K and V, two buffers
  __shared__ __attribute__((aligned(16))) char s_buf[kWinWaves * kWave];
  __shared__ float s_m[kWinWaves][32], s_sum[kWinWaves][32];

  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % (uint32_t)g.nsplit;
  const uint32_t item = blockIdx.x / (uint32_t)g.nsplit;
  const int tile = item % (uint32_t)g.tiles;
  const int hk = (item / (uint32_t)g.tiles) % (uint32_t)g.kv_heads;
  const int b = item / (uint32_t)g.tiles / (uint32_t)g.kv_heads;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t rows = qlen * g.group, r0 = 32 * tile;
  if (r0 >= rows) return;
  const int32_t row = min(r0 + fr, rows - 1);
  const int32_t first = kvlen - qlen + r0 / g.group;
  const int32_t last = kvlen - qlen + min(r0 + 31, rows - 1) / g.group;
  const int32_t query = row / g.group, head = hk * g.group + row % g.group;
  const int32_t pos = kvlen - qlen + query;
  const Span sp(first, last, g);
  const int32_t blocks = (sp.total + 31) >> 5;
  const int32_t n_lo = (int32_t)((int64_t)blocks * split / g.nsplit);
  const int32_t n_hi = (int32_t)((int64_t)blocks * (split + 1) / g.nsplit);

  u32x4 qf[D / 16];
  {
    const uint16_t* qr = g.q + b * g.qb + query * g.qs + head * g.qh + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const u32x4*>(qr + 16 * ks);
  }
  settle(qf);
  const uint16_t* K = g.k + b * g.kb + hk * g.kh;
  const uint16_t* V = g.v + b * g.vb + hk * g.vh;
  char* buf = s_buf + wave * kWave;
  const uint32_t lds =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf + wave * kWave;
  auto load = [&](int32_t n, int slot) {
    stage_rows<D, false, 32>(lds + 2 * kBlk * slot, K, g.ks, sp, 32 * n, lane);
    stage_rows<D, true, 32>(lds + 2 * kBlk * slot + kBlk, V, g.vs, sp, 32 * n, lane);
  };

  RowAcc<D> acc;
  acc.sum = 0.0f;
  acc.m = kNoMax;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc.o[d] = f32x16{};
  if (n_lo + wave < n_hi) load(n_lo + wave, 0);
  int slot = 0;
  for (int32_t n = n_lo + wave; n < n_hi; n += kWinWaves, slot ^= 1) {
    if (n + kWinWaves < n_hi) {
      load(n + kWinWaves, slot ^ 1);
      wait_loads<D / 8>();   // of the next block: D / 16 loads each for K and V
    } else {
      wait_loads<0>();
    }
    const char* kblk = buf + 2 * kBlk * slot;
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = wmma<DT>(read_k<D>(kblk, fr, h, ks), qf[ks], s);
    if (!all_seen(sp, 32 * n, first, last, g)) mask_block(s, sp, 32 * n, pos, h, g);
    const float top = block_top<MODE>(s, g.c0);
    if (__any(top > acc.m + (kLift<DT> + kLazy))) raise_max<DT>(top, acc);
    const float c1 = row_c1<MODE>(acc.m);
    u32x4 p[2];
#pragma unroll
    for (int r = 0; r < 16; r += 2)
      p[r >> 3][(r >> 1) & 3] = prob_pair<DT, MODE>(s, r, g.c0, c1, acc.sum);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        acc.o[d] = wmma<DT>(read_v<D>(kblk + kBlk, lane, ks, d), p[ks], acc.o[d]);
    wait_lds();   // this buffer's reads, before it is loaded again
  }

  // join the waves: their M, then sums and O^T brought to the largest M
  acc.sum += other_half(acc.sum);
  __syncthreads();   // every wave is done with its buffers
  if (lane < 32) {
    s_m[wave][fr] = acc.m;
    s_sum[wave][fr] = acc.sum;
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
  for (int w = 1; w < kWinWaves; ++w) m = fmaxf(m, s_m[w][fr]);
  float sum = 0.0f;
  int32_t e[kWinWaves];
#pragma unroll
  for (int w = 0; w < kWinWaves; ++w) {
    e[w] = down_shift(s_m[w][fr], m);
    sum += __builtin_amdgcn_ldexpf(s_sum[w][fr], e[w]);
  }
  // this wave's dims: D / 4, each half of its lanes D / 8 of them
  constexpr int N = D / 8;
  const int d0 = wave * (D / 4) + h * N;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWinWaves; ++w)
      v[i] += __builtin_amdgcn_ldexpf(
          reinterpret_cast<const float*>(s_buf + w * kWave)[(d0 + i) * 32 + fr], e[w]);
  }
  if (g.nsplit > 1) {
    if (r0 + fr >= rows) return;
    float* w = g.ws + (int64_t)blockIdx.x * (64 + 32 * D);
    if (wave == 0 && h == 0) {
      w[fr] = m;
      w[32 + fr] = sum;
    }
    float4* wo = reinterpret_cast<float4*>(w + 64 + fr * D + d0);
#pragma unroll
    for (int i = 0; i < N; i += 4) wo[i / 4] = float4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    return;
  }
  if (r0 + fr >= rows) return;
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* orow = g.o + b * g.ob + query * g.os + head * g.oh + d0;
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = wpack<DT>(v[i + 2 * j] * inv, v[i + 2 * j + 1] * inv);
    *reinterpret_cast<u32x4*>(orow + i) = w;
  }
}

// 128 rows in one workgroup, 32 a wave, which share tiles of 64 keys in LDS (two
// blocks of 32; two tiles each of K and V). A wave's products run under its own VALU
// work: while block n's scores become probabilities, the scores of block n + 1 and the
// second product of block n - 1 are computed, one product of each with every 512 / D
// of the block's 16 values a lane. One barrier a tile, between its blocks: by then K
// of the next tile and V of this one have landed, and K of this one and V of the last
// are done with, so the loads of two tiles on start there.
// What bounds it is VALU issue, so whether M has to rise is asked of each lane's own
// scores; only if so are the two halves of a row brought together. A prompt of 16384
// tokens (window 4096, 32 heads over 8, head dim 128, bf16): 1.00 to 1.04 ms, 0.93 to
// 0.96 PFLOP/s; products take 49 % of the cycles and VALU instructions 53 %, and they
// hardly overlap. The operand reads from LDS, by count 16 cycles a wave for two products,
// take nearly as many as both.
constexpr int kManyKeys = 64;

template <int DT, int MODE, int D>
__global__ __launch_bounds__(64 * kWinWaves, 2) void window_many_kernel(WindowArgs g) {
  constexpr int kTile = 2 * kManyKeys * D;          // bytes of K or V of a tile
  constexpr int kRows = kManyKeys / kWinWaves;      // a wave loads
  __shared__ __attribute__((aligned(16))) char s_buf[4 * kTile];   // K and V, two buffers

  const int lane = threadIdx.x & 63, fr = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups go round the 8 XCDs: each XCD gets consecutive tiles, which share
  // most of their keys, for its own L2.
  const uint32_t x = blockIdx.x & 7u, per = gridDim.x >> 3, rest = gridDim.x & 7u;
  const uint32_t id = x * per + min(x, rest) + (blockIdx.x >> 3);
  const int split = id % (uint32_t)g.nsplit;
  const uint32_t item = id / (uint32_t)g.nsplit;
  const uint32_t tiles = ((uint32_t)g.tiles + kWinWaves - 1) / kWinWaves;
  const int tile = item % tiles;
  const uint32_t bh = item / tiles;
  const int hk = bh % (uint32_t)g.kv_heads, b = bh / (uint32_t)g.kv_heads;
  const int32_t qlen = seq_len(g.q_lens, b, g.sq), kvlen = seq_len(g.kv_lens, b, g.skv);
  const int32_t rows = qlen * g.group, r0 = 32 * kWinWaves * tile;
  if (r0 >= rows) return;
  const int32_t off = kvlen - qlen;
  const Span sp(off + r0 / g.group, off + min(r0 + 32 * kWinWaves - 1, rows - 1) / g.group, g);
  const int32_t steps = (sp.total + kManyKeys - 1) / kManyKeys;
  const int32_t n_lo = (int32_t)((int64_t)steps * split / g.nsplit);
  const int32_t n_hi = (int32_t)((int64_t)steps * (split + 1) / g.nsplit);
  // this wave's rows (past the last row: that row again, not stored)
  const int32_t w0 = r0 + 32 * wave;
  const int32_t row = min(w0 + fr, rows - 1);
  const int32_t query = row / g.group, head = hk * g.group + row % g.group;
  const int32_t pos = off + query;
  const int32_t first = off + min(w0, rows - 1) / g.group;
  const int32_t last = off + min(w0 + 31, rows - 1) / g.group;

  u32x4 qf[D / 16];
  {
    const uint16_t* qr = g.q + b * g.qb + query * g.qs + head * g.qh + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const u32x4*>(qr + 16 * ks);
  }
  settle(qf);
  const uint16_t* K = g.k + b * g.kb + hk * g.kh;
  const uint16_t* V = g.v + b * g.vb + hk * g.vh;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_buf +
                       wave * kRows * 2 * D;
  auto load_k = [&](int32_t t) {
    stage_rows<D, false, kRows>(lds + kTile * ((t - n_lo) & 1), K, g.ks, sp, kManyKeys * t + kRows * wave, lane);
  };
  auto load_v = [&](int32_t t) {
    stage_rows<D, true, kRows>(lds + kTile * (2 + ((t - n_lo) & 1)), V, g.vs, sp, kManyKeys * t + kRows * wave,
                               lane);
  };

  RowAcc<D> acc;
  acc.sum = 0.0f;
  acc.m = kNoMax;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc.o[d] = f32x16{};
  // tiles of which this wave's rows may see something, and of which they see all
  const int32_t seen = last < 0 ? 0 : last + 1 - (last < sp.sinks ? 0 : sp.shift);
  const int32_t t_hi = min(n_hi, (seen + kManyKeys - 1) / kManyKeys);
  int32_t t_lo = n_lo;
  const int32_t low = (uint32_t)last >= g.window ? last - (int32_t)g.window + 1 : 0;   // seen by all
  const int32_t all_lo = (max(low - sp.shift, sp.sinks) + kManyKeys - 1) / kManyKeys;
  const int32_t all_hi = first < 0 ? 0 : max(first + 1 - sp.shift, 0) / kManyKeys;
  if (g.sinks == 0 && first >= 0 && (uint32_t)first >= g.window)
    t_lo = max(t_lo, (first - (int32_t)g.window + 1 - sp.shift) / kManyKeys);

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
  auto step = [&](int32_t n, bool plain, auto kn, auto vp, f32x16& s, f32x16& sn, u32x4 (&pp)[2],
                  u32x4 (&pn)[2]) {
    constexpr int KN = decltype(kn)::value, VP = decltype(vp)::value;
    u32x4 ka[NU], va[NU];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ka[u] = get_k(KN, u);
      va[u] = get_v(VP, u);
    }
    if (!plain) mask_block(s, sp, 32 * n, pos, h, g);
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    if (__any(top > limit)) {
      const int32_t e = raise_max<DT>(fmaxf(top, other_half(top)) * units, acc);
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
      for (int r = NE * u; r < NE * u + NE; r += 2)
        pn[r >> 3][(r >> 1) & 3] = prob_pair<DT, MODE>(s, r, g.c0, c1, acc.sum);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  u32x4 pa[2], pb[2];
  f32x16 sa, sb;
  auto two_blocks = [&](int32_t t, auto parity) {
    constexpr int B = 2 * decltype(parity)::value;   // the tile's first block in LDS
    const bool mine = t >= t_lo && t < t_hi, plain = t >= all_lo && t < all_hi;
    if (mine && t == t_lo) {
      sa = f32x16{};
#pragma unroll
      for (int u = 0; u < NU; ++u) sa = wmma<DT>(get_k(B, u), qf[u], sa);
      pb[0] = pb[1] = u32x4{0u, 0u, 0u, 0u};   // no block before
    }
    if (mine)
      step(2 * t, plain, std::integral_constant<int, B + 1>{}, std::integral_constant<int, 3 - B>{},
           sa, sb, pb, pa);
    wait_lds();
    wait_loads<0>();
    __syncthreads();
    if (t + 2 < n_hi) load_k(t + 2);
    if (t + 1 < n_hi) load_v(t + 1);
    if (!mine) return;
    step(2 * t + 1, plain, std::integral_constant<int, 2 - B>{}, std::integral_constant<int, B>{}, sb,
         sa, pa, pb);
    if (t + 1 == t_hi) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
        acc.o[u % ND] = wmma<DT>(get_v(B + 1, u), pb[u / ND], acc.o[u % ND]);
    }
  };
  if (n_lo < n_hi) {
    // V of the tile before the first is read (times 0): K's rows, which are finite
    // where K is
    stage_rows<D, false, kRows>(lds + kTile * 3, K, g.ks, sp, kManyKeys * n_lo + kRows * wave, lane);
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
  if (g.nsplit > 1) {
    if (w0 >= rows) return;
    const int64_t slot32 = ((int64_t)bh * g.tiles + kWinWaves * tile + wave) * g.nsplit + split;
    if (w0 + fr >= rows) return;
    float* w = g.ws + slot32 * (64 + 32 * D);
    if (h == 0) {
      w[fr] = acc.m;
      w[32 + fr] = sum;
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(w + 64 + fr * D + 32 * d + 8 * i + 4 * h) =
            float4{acc.o[d][4 * i], acc.o[d][4 * i + 1], acc.o[d][4 * i + 2], acc.o[d][4 * i + 3]};
    return;
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
      const u32x2 w = {wpack<DT>(acc.o[d][4 * i] * inv, acc.o[d][4 * i + 1] * inv),
                       wpack<DT>(acc.o[d][4 * i + 2] * inv, acc.o[d][4 * i + 3] * inv)};
      *reinterpret_cast<u32x2*>(ow + fr * 2 * D + 16 * ((4 * d + i) ^ kswizzle<D>(fr)) + 8 * h) = w;
    }
  __builtin_amdgcn_wave_barrier();
  wait_lds();
  constexpr int CH = D / 8, RPL = 64 / CH;
#pragma unroll
  for (int j = 0; j < 32 / RPL; ++j) {
    const int r = RPL * j + lane / CH, c = lane % CH;
    if (w0 + r >= rows) continue;
    const int32_t qi = (w0 + r) / g.group, hd = hk * g.group + (w0 + r) % g.group;
    *reinterpret_cast<u32x4*>(g.o + b * g.ob + qi * g.os + hd * g.oh + 8 * c) =
        *reinterpret_cast<const u32x4*>(ow + r * 2 * D + 16 * (c ^ kswizzle<D>(r)));
  }
}

// Joins a row's splits, a lane for every four dims: D / 4 lanes, which take the splits
// one after the other, or (WIDE) the whole workgroup, whose 1024 / D such teams take
// every so many-th. Several loads are in flight; the order is fixed.
template <int DT, int D, bool WIDE>
__global__ __launch_bounds__(256) void window_join_kernel(WindowArgs g) {
  constexpr int C = D / 4, SL = WIDE ? 256 / C : 1, U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t id = WIDE ? blockIdx.x : blockIdx.x * (256u / C) + threadIdx.x / C;   // of all rows
  const uint32_t item = id >> 5;
  const int fr = id & 31u, tile = item % (uint32_t)g.tiles;
  const int hk = (item / (uint32_t)g.tiles) % (uint32_t)g.kv_heads;
  const int b = item / (uint32_t)g.tiles / (uint32_t)g.kv_heads;
  const int32_t row = 32 * tile + fr;
  if (row >= seq_len(g.q_lens, b, g.sq) * g.group) return;
  constexpr int64_t slot = 64 + 32 * D;
  const float* w = g.ws + (int64_t)item * g.nsplit * slot;
  const int c = lane % C;
  float m = kNoMax, sum = 0.0f;
  float4 v{0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](float om, float os, float4 ov) {
    const float top = fmaxf(m, om);
    const int32_t e = down_shift(m, top), oe = down_shift(om, top);
    auto two = [&](float a, float o) {
      return __builtin_amdgcn_ldexpf(a, e) + __builtin_amdgcn_ldexpf(o, oe);
    };
    sum = two(sum, os);
    v = float4{two(v.x, ov.x), two(v.y, ov.y), two(v.z, ov.z), two(v.w, ov.w)};
    m = top;
  };
  for (int s0 = WIDE ? threadIdx.x / C : 0; s0 < g.nsplit; s0 += U * SL) {
    float om[U], os[U];
    float4 ov[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {   // past the last split: that one again, not added
      const float* p = w + (int64_t)min(s0 + j * SL, g.nsplit - 1) * slot;
      om[j] = p[fr];
      os[j] = p[32 + fr];
      ov[j] = *reinterpret_cast<const float4*>(p + 64 + fr * D + 4 * c);
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (s0 + j * SL < g.nsplit) add(om[j], os[j], ov[j]);
  }
  if constexpr (WIDE) {
    constexpr int W = 4;
#pragma unroll
    for (int o = C; o < 64; o <<= 1)
      add(__shfl_xor(m, o, 64), __shfl_xor(sum, o, 64),
          float4{__shfl_xor(v.x, o, 64), __shfl_xor(v.y, o, 64), __shfl_xor(v.z, o, 64),
                 __shfl_xor(v.w, o, 64)});
    __shared__ float s_m[W], s_sum[W];
    __shared__ float4 s_v[W][C];
    if (lane < C) s_v[wave][c] = v;
    if (lane == 0) {
      s_m[wave] = m;
      s_sum[wave] = sum;
    }
    __syncthreads();
    if (wave > 0 || lane >= C) return;
#pragma unroll
    for (int o = 1; o < W; ++o) add(s_m[o], s_sum[o], s_v[o][c]);
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  uint16_t* orow = g.o + b * g.ob + (row / g.group) * g.os + (hk * g.group + row % g.group) * g.oh;
  *reinterpret_cast<u32x2*>(orow + 4 * c) =
      u32x2{wpack<DT>(v.x * inv, v.y * inv), wpack<DT>(v.z * inv, v.w * inv)};
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct WindowPlan {
  int64_t tiles;    // tiles of 32 rows of a key head
  int64_t nsplit;   // workgroups that share a tile's keys
  bool many;        // 128 rows a workgroup
};

// Splits: few tiles leave compute units idle while each walks a long window, so a
// tile's keys go to as many workgroups as bring the launch to kWinTarget (one per
// compute unit), with at least kSplitKeys keys for each. Below kSplitFrom keys the
// second launch costs more than it saves.
constexpr int64_t kWinTarget = 256, kSplitKeys = 128, kSplitFrom = 512;
constexpr int64_t kJoinFew = 8;     // splits up to which D / 4 lanes join a row

// From kManyRows rows on, 128 rows share a workgroup, unless workgroups of 32 rows fit
// one to a compute unit and each walks at most kFewWalk keys: what sharing saves is
// then no compute unit's time, while a short walk's start and end are longer for it.
// 32 rows against 128 (us; heads dim 128 unless said): 300 to 380 rows x 8 key heads,
// 2000 keys, 13.9 to 19.4 / 21.8 to 24.4; 256 rows x 8, 4096 keys (walk 1024) 18.5 /
// 24.0; 128 x 16 x 100 keys at dim 64 5.3 / 7.6; 128 x 64, 512 keys 16.0 / 21.2, 1024
// keys 25.0 / 21.4 (the one found that loses within the limit); a walk of 2040 keys
// 43 / 26, of 4096 83 / 37. Several workgroups of 32 rows a compute unit lose where
// there are many (384: 61 / 34, 768: 233 / 125), though not always (512 over 512 causal
// keys: 18.3 / 24.3). The walk is that of the split call also where a call has no
// workspace: its few workgroups then walk all keys, which 32 rows, whose four waves share
// them, do best (64 queries of 8 heads over 4, 9000 keys, dim 64, 54.5 / 149; 16 of 64
// over 8, 4096 keys, 34.6 / 87.5).
constexpr int64_t kManyRows = 96, kFewWalk = 1024;

static WindowPlan window_plan(int64_t batch, int64_t sq, int64_t skv, int64_t group,
                              int64_t kv_heads, int64_t window, int64_t sinks) {
  WindowPlan p;
  const int64_t rows = sq * group;
  p.tiles = (rows + 31) / 32;
  int64_t walk = 0;   // keys of one workgroup
  const auto split = [&](int64_t wide) {
    const int64_t items = batch * kv_heads * ((rows + wide - 1) / wide);
    const int64_t queries = (wide - 1 + group) / group;   // most positions a tile covers, less one
    const int64_t keys = std::min(skv, std::min(window, skv) + std::min(sinks, skv) + queries);
    const int64_t most = keys < kSplitFrom ? 1 : keys / kSplitKeys;
    p.nsplit = items == 0 ? 1 : std::max<int64_t>(1, std::min(most, kWinTarget / items));
    walk = keys / p.nsplit;
    return items;
  };
  p.many = false;
  if (split(32) > kWinTarget || walk > kFewWalk) p.many = rows >= kManyRows;
  if (p.many) split(128);
  return p;
}

static int64_t window_ws_bytes(const WindowPlan& p, int64_t batch, int64_t kv_heads, int64_t dim) {
  if (p.nsplit == 1) return 0;
  return batch * kv_heads * p.tiles * p.nsplit * (64 + 32 * dim) * 4;
}

static bool window_shape_ok(int64_t batch, int64_t sq, int64_t skv, int64_t heads,
                            int64_t kv_heads, int64_t dim, int64_t window, int64_t sinks) {
  if (batch < 0 || sq < 0 || skv < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0)
    return false;
  if ((dim != 64 && dim != 128) || window < 1 || sinks < 0) return false;
  if (window > INT32_MAX || sinks > INT32_MAX || skv > (1 << 30) || sq > (1 << 24)) return false;
  if (heads > (1 << 16) || batch > (1 << 24)) return false;
  if (sq * (heads / kv_heads) > (1 << 30)) return false;
  // a workgroup of 256 threads a tile: a launch takes fewer than 2^32 threads
  return batch * kv_heads * ((sq * (heads / kv_heads) + 31) / 32) < (1 << 24);
}

// Whether no row of o shares elements with another: in ascending order each stride
// reaches past what the smaller ones span. (Layouts that interleave otherwise without
// meeting are refused as well; no view of a larger tensor by slices and permutations
// is one.)
static bool rows_apart(const int64_t (&stride)[3], const int64_t (&count)[3], int64_t dim) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  int64_t span = dim;
  for (const int i : order) {
    if (count[i] <= 1) continue;
    if (stride[i] < span) return false;
    span += stride[i] * (count[i] - 1);
  }
  return true;
}

template <int DT, int MODE, int D>
static void launch_window(bool many, int64_t heads, hipStream_t s, const WindowArgs& g) {
  const int64_t wide = many ? kWinWaves : 1;   // tiles of 32 rows a workgroup
  const dim3 grid((uint32_t)(heads * ((g.tiles + wide - 1) / wide) * g.nsplit));
  if (many)
    hipLaunchKernelGGL((window_many_kernel<DT, MODE, D>), grid, dim3(64 * kWinWaves), 0, s, g);
  else
    hipLaunchKernelGGL((window_few_kernel<DT, MODE, D>), grid, dim3(64 * kWinWaves), 0, s, g);
  if (g.nsplit > kJoinFew)
    hipLaunchKernelGGL((window_join_kernel<DT, D, true>), dim3((uint32_t)(heads * g.tiles * 32)),
                       dim3(256), 0, s, g);
  else if (g.nsplit > 1)
    hipLaunchKernelGGL((window_join_kernel<DT, D, false>), dim3((uint32_t)(heads * g.tiles * D / 32)),
                       dim3(256), 0, s, g);
}
template <int DT, int D>
static void launch_window(int mode, bool many, int64_t heads, hipStream_t s, const WindowArgs& g) {
  switch (mode) {
    case QUAKE_EXACT: launch_window<DT, EXACT, D>(many, heads, s, g); break;
    case QUAKE_1: launch_window<DT, Q1, D>(many, heads, s, g); break;
    case QUAKE_2: launch_window<DT, Q2, D>(many, heads, s, g); break;
    default: launch_window<DT, Q2M, D>(many, heads, s, g); break;
  }
}

}  // namespace qk

using namespace qk;

extern "C" quake_status quake_attention_window_workspace_size(int64_t batch, int64_t sq,
                                                              int64_t skv, int64_t heads,
                                                              int64_t kv_heads, int64_t dim,
                                                              int64_t window, int64_t sinks,
                                                              int64_t* bytes) {
  if (bytes == nullptr) return QUAKE_EINVAL;
  if (!window_shape_ok(batch, sq, skv, heads, kv_heads, dim, window, sinks)) return QUAKE_EINVAL;
  const WindowPlan p = window_plan(batch, sq, skv, heads / kv_heads, kv_heads, window, sinks);
  *bytes = window_ws_bytes(p, batch, kv_heads, dim);
  return QUAKE_OK;
}

extern "C" quake_status quake_attention_window(
    const void* q, const void* k, const void* v, void* o, const int32_t* q_lens,
    const int32_t* kv_lens, int64_t batch, int64_t sq, int64_t skv, int64_t heads,
    int64_t kv_heads, int64_t dim, const quake_window_strides* strides, int64_t window,
    int64_t sinks, quake_dtype dtype, quake_mode mode, float t, void* workspace,
    int64_t workspace_bytes, void* stream) {
  if (dtype != QUAKE_BF16 && dtype != QUAKE_F16) return QUAKE_EDTYPE;
  if (!valid_mode(mode)) return QUAKE_EMODE;
  if (!window_shape_ok(batch, sq, skv, heads, kv_heads, dim, window, sinks)) return QUAKE_EINVAL;
  if (!std::isfinite(t) || !(t > 0.0f)) return QUAKE_EINVAL;
  const float c0 = softmax_c0(t, mode);
  if (!std::isfinite(c0) || c0 == 0.0f) return QUAKE_EINVAL;
  if (workspace_bytes < 0 || (workspace != nullptr && !aligned16(workspace))) return QUAKE_EINVAL;
  if (batch == 0 || sq == 0) return QUAKE_OK;
  if (strides == nullptr || q == nullptr || o == nullptr) return QUAKE_EINVAL;
  if (skv > 0 && (k == nullptr || v == nullptr)) return QUAKE_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) ||
      ((uintptr_t)q_lens & 3u) != 0 || ((uintptr_t)kv_lens & 3u) != 0)
    return QUAKE_EINVAL;
  const quake_window_strides& st = *strides;
  for (const int64_t* s : {st.q, st.k, st.v, st.o}) {
    const bool kv = s == st.k || s == st.v;
    const int64_t count[3] = {batch, kv ? skv : sq, kv ? kv_heads : heads};
    for (int i = 0; i < 3; ++i) {
      if (count[i] <= 1) continue;   // never multiplied by anything but 0
      if (s[i] < 0 || s[i] % 8 != 0 || s[i] > INT64_MAX / 8 / count[i]) return QUAKE_EINVAL;
      if (i == 1 && kv && s[i] > (1 << 24)) return QUAKE_EINVAL;   // 32-row offsets in 32 bits
    }
    if (s == st.o && !rows_apart(st.o, count, dim)) return QUAKE_EINVAL;
  }
  const WindowPlan p = window_plan(batch, sq, skv, heads / kv_heads, kv_heads, window, sinks);
  const int64_t need = window_ws_bytes(p, batch, kv_heads, dim);
  const bool split = workspace != nullptr && need > 0;
  if (split) {
    if (workspace_bytes < need) return QUAKE_EINVAL;
    const auto bytes = [&](const int64_t (&s)[3], int64_t tokens, int64_t n) {
      const int64_t count[3] = {batch, tokens, n};
      int64_t last = dim;
      for (int i = 0; i < 3; ++i) last += count[i] > 1 ? s[i] * (count[i] - 1) : 0;
      return tokens > 0 ? 2 * last : 0;
    };
    if (meet(workspace, need, q, bytes(st.q, sq, heads)) ||
        meet(workspace, need, k, bytes(st.k, skv, kv_heads)) ||
        meet(workspace, need, v, bytes(st.v, skv, kv_heads)) ||
        meet(workspace, need, o, bytes(st.o, sq, heads)) ||
        meet(workspace, need, q_lens, 4 * batch) || meet(workspace, need, kv_lens, 4 * batch))
      return QUAKE_EINVAL;
  }
  WindowArgs g{};
  g.q = static_cast<const uint16_t*>(q);
  g.k = static_cast<const uint16_t*>(k);
  g.v = static_cast<const uint16_t*>(v);
  g.o = static_cast<uint16_t*>(o);
  g.q_lens = q_lens;
  g.kv_lens = kv_lens;
  g.ws = static_cast<float*>(workspace);
  g.qb = st.q[0], g.qs = st.q[1], g.qh = st.q[2];
  g.kb = st.k[0], g.ks = st.k[1], g.kh = st.k[2];
  g.vb = st.v[0], g.vs = st.v[1], g.vh = st.v[2];
  g.ob = st.o[0], g.os = st.o[1], g.oh = st.o[2];
  g.sq = (int32_t)sq;
  g.skv = (int32_t)skv;
  g.group = (int32_t)(heads / kv_heads);
  g.kv_heads = (int32_t)kv_heads;
  g.tiles = (int32_t)p.tiles;
  g.nsplit = split ? (int32_t)p.nsplit : 1;
  g.window = (uint32_t)window;
  g.sinks = (uint32_t)sinks;
  g.c0 = c0;
  const int64_t kvh = batch * kv_heads;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == QUAKE_BF16) {
    if (dim == 64) launch_window<BF16, 64>(mode, p.many, kvh, s, g);
    else launch_window<BF16, 128>(mode, p.many, kvh, s, g);
  } else {
    if (dim == 64) launch_window<F16, 64>(mode, p.many, kvh, s, g);
    else launch_window<F16, 128>(mode, p.many, kvh, s, g);
  }
  return launch_status();
}
