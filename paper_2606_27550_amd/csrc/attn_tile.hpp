// Pieces of the tree attention that its kernels share: tile sizes, the split
// targets of a batch, the rotation to positions, and the LDS reads of the
// matrix products' operands.  The method is described in tree_attn.hip.
#pragma once

#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "stream_pipe.hpp"

namespace entmtp {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int HD = ENTMTP_HEAD_DIM;  // 128
constexpr int kAttnThreads = 256;
constexpr int KB = 32;               // keys per block
constexpr int kQTile = 32;           // query rows per tile
constexpr float kLazyLog2 = 8.f;     // the running max is raised only past this many doublings
constexpr int kMinBlocksPerSplit = 4;
// Sequences of up to this many key blocks are not split: a merge (launch,
// partials, its gap) costs as much as the blocks it saves.  Captured calls back
// to back, split / unsplit, 32 KV heads: 9 blocks 12.5 / 12.2 us (27 nodes), 10
// 14.1 / 14.4 (64), 11 12.3 / 12.9 (7) and 12.5 / 13.0 (27), where calls from
// Python still gain unsplit (13.9 / 13.1); 12 13.6 / 15.3 (64), 13 12.3 / 14.3,
// 20 13.7 / 18.9 (27).  4 and 8 KV heads alike.
constexpr int kLoneBlocks = 11;
constexpr int kTilesPerWg = 4;       // query tiles per workgroup, one per wave
constexpr int kWgPerCu = 2;          // attend workgroups resident per CU (registers, LDS)

__host__ __device__ inline int rows_padded(int G, int T) {
  return (G * T + kQTile - 1) / kQTile * kQTile;
}

// Workgroups along the query rows: groups of four 32-row tiles.
__host__ __device__ inline int query_groups(int nqt) { return (nqt + kTilesPerWg - 1) / kTilesPerWg; }

// Where split k of ns begins: even shares of nblocks + tree_extra blocks, the
// last split, which holds the tree's keys, shorter by tree_extra.  A block of
// tree keys is rotated and staged through registers (about two prefix blocks'
// time) after a table of fp64 angles (two more): given an even share that
// workgroup ended 8 us after the others at 128 nodes and prefix 8192 (43.8
// against a median of 35), 4 us at 27 nodes and prefix 2048.
constexpr int kTreeSetup = 2;
__host__ __device__ inline int tree_extra(int nblocks, int L, int ns) {
  const int extra = kTreeSetup + nblocks - L / KB, share = nblocks / ns;
  return extra < share ? extra : share;   // (the last split keeps a block)
}
__device__ __forceinline__ int split_begin(int k, int ns, int nblocks, int extra) {
  return k < ns ? static_cast<int>(static_cast<unsigned>(k) * static_cast<unsigned>(nblocks + extra) / ns)
                : nblocks;
}

// A batch of several sequences shares one blocks-per-split target t: sequence
// b, with H_b streams (KV heads x query groups) of nb_b blocks, takes
// ns_b(t) = ceil(nb_b / t) splits (clipped to [1, split_bound]).  Every
// workgroup costs its blocks and a fixed part, and the chip runs `slots` of
// them at a time, so the target minimises
//   rounds(sum H_b ns_b(t)) * (kWgFixed + t)  (+ kMergeCost when any is split)
// over kTargets candidates: the last one splits nothing (t = the longest),
// the others are multiples of the even share work / slots, from half of it
// (two rounds) up.  A fixed number of workgroups per CU instead (three, at two
// resident) left the second round half empty: eight GQA sequences 103 us
// against 88, at prefixes up to 4096 62 us a call against 48.
constexpr int kTargets = 16;
constexpr int kWgFixed = 6;      // a workgroup's fixed part, in blocks (8 us at 1.3-1.7 us a block)
constexpr int kMergeCost = 4;    // the merge kernel, in blocks
__host__ __device__ inline int target_sixteenths(int k) {   // of the even share
  constexpr unsigned long long lo = 0x1413121110'0a0908ull;   // 8 9 10 16 17 18 19 20
  constexpr unsigned long long hi = 0x60402820'1e1c1816ull;   // 22 24 28 30 32 40 64 96
  return static_cast<int>((k < 8 ? lo >> (8 * k) : hi >> (8 * (k - 8))) & 0xff);
}
__host__ __device__ inline int batch_target(int k, long long work, int nb_max, int slots) {
  if (k == kTargets - 1) return nb_max > 1 ? nb_max : 1;
  const long long t = (work * target_sixteenths(k) + 16LL * slots - 1) / (16LL * slots);
  return static_cast<int>(t > kMinBlocksPerSplit ? (t < nb_max ? t : nb_max) : kMinBlocksPerSplit);
}
// One key per candidate: the smallest wins (the lowest candidate among equals).
__host__ __device__ inline unsigned long long batch_cost(int k, int t, long long items, bool split,
                                                         int slots) {
  const long long rounds = (items + slots - 1) / slots;
  return (static_cast<unsigned long long>(rounds * (kWgFixed + t) + (split ? kMergeCost : 0)) << 8) | k;
}
// Most workgroups a planned batch can have (padding aside) when its streams
// number at most `streams`: the two-round candidates are allowed only where
// the streams alone nearly fill the chip, and a split count is below
// nb / t + 1, so the items stay below work / t + streams.
__host__ __device__ inline bool two_rounds(long long streams_bound, int slots) {
  return 4 * streams_bound > 3LL * slots;
}

__device__ __forceinline__ long long uniform(long long x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return static_cast<long long>((static_cast<unsigned long long>(hi) << 32) | lo);
}

// ------------------------------------------------------------------ RoPE --

// Angles of a tree's positions: the turn of pair (c, c + 64) at position
// L + d, d = 0..D, in fp64 (pos * freq[c], freq[c] = theta^(-2c/d) from the
// host), tabulated as (cos, sin) by the workgroup's threads (a multiple of
// 64: each keeps one pair's frequency).
constexpr int kRopePairs = HD / 2;
inline void rope_freqs(float rope_theta, double (&out)[kRopePairs]) {
  const double theta = static_cast<double>(rope_theta);
  // (a model has one base: its 64 powers are kept, per thread, for the next call)
  thread_local double last_theta = -1.0, freq[kRopePairs];
  if (theta != last_theta) {
    for (int c = 0; c < kRopePairs; ++c) freq[c] = theta > 0.0 ? std::pow(theta, -2.0 * c / HD) : 0.0;
    last_theta = theta;
  }
  std::copy(freq, freq + kRopePairs, out);
}

// sin and cos of x in fp64, 0 <= x < 2^31 (positions times frequencies up to
// one radian, those of a base of one or more): x less the nearest multiple n of pi/2 (pi/2 as a sum of two
// doubles, each product exact in its fused multiply-add: the remainder is
// off by a rounding of its own size), then the Taylor series on [-pi/4,
// pi/4], cut where the next term is below 1e-17 of the value.  About 40 fp64
// instructions; the library's sincos, made for all arguments, took most of
// the attention kernels' prologue.  It stays for bases below one, whose
// frequencies grow to 1 / base: the angle of an ordinary position then leaves
// this range (base 1e-6: from position 4200 on), so those calls have an
// instance of the kernel of their own (wide_angles) and the others keep theirs
// as it is.
__device__ __forceinline__ double2 cos_sin(double x) {
  const double n = rint(x * 0.63661977236758134308);   // 2 / pi
  const double r = fma(-n, 6.123233995736766035869e-17, fma(-n, 1.57079632679489655800, x));
  const double z = r * r;
  double s = 1.0 / 355687428096000.0;                  // 1 / 17!
  s = fma(s, z, -1.0 / 1307674368000.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;                   // 1 / 16!
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int q = static_cast<int>(n) & 3;   // quarter turns
  const double a = q & 1 ? s : c, b = q & 1 ? c : s;
  return make_double2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

inline bool wide_angles(double theta) { return theta > 0.0 && theta < 1.0; }

// Calls put(d, c, (cos, sin)) for the angles of positions L + d, d = 0..D,
// over the workgroup.  f: thread tid's pair frequency, freq[tid % 64], loaded by the caller ahead of its bulk loads (a load issued behind
// them would wait for them).
template <bool WIDE, typename F>
__device__ __forceinline__ void rope_table(int tid, int D, int L, double f, F put) {
  const int c = tid % kRopePairs;
  for (int d = tid / kRopePairs; d <= D; d += kAttnThreads / kRopePairs) {
    const double x = (static_cast<double>(L) + static_cast<double>(d)) * f;
    if constexpr (WIDE) {
      double sn, cs;
      sincos(x, &sn, &cs);
      put(d, c, make_double2(cs, sn));
    } else {
      put(d, c, cos_sin(x));
    }
  }
}

// Turns the 8 pairs (c0 + e, c0 + e + 64), e < 8, whose halves lo / hi hold
// (bf16), by the angles at t[0 .. 7] (t = the position's table row at c0, its
// eight entries at index ^ swz, so that the lanes of a row read other banks):
// lo cos - hi sin and hi cos + lo sin in fp64 (each product rounded, then
// the sum: no fused multiply-add), each rounded to bf16 once.
__device__ __forceinline__ void rope_pairs(u32x4& lo, u32x4& hi, const double2* t, int swz) {
#pragma clang fp contract(off)
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t nl = 0u, nh = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const double2 a = t[(2 * w + h) ^ swz];
      const double x = bf16_to_f64(static_cast<uint16_t>(lo[w] >> (16 * h)));
      const double y = bf16_to_f64(static_cast<uint16_t>(hi[w] >> (16 * h)));
      nl |= f64_to_bf16_rne(x * a.x - y * a.y) << (16 * h);
      nh |= f64_to_bf16_rne(y * a.x + x * a.y) << (16 * h);
    }
    lo[w] = nl;
    hi[w] = nh;
  }
}

// The same turn of pairs c0 .. c0 + 7 in fp32 with fp32 angles (pair c at
// t[c ^ swz]: lanes at other depths read other banks), rounded to bf16 by the hardware
// (for the queries, which only enter bf16 products: the cache keeps the
// fp64 form's keys).  Which product is fused is spelled out, so that every
// instance of the kernel rounds alike.
__device__ __forceinline__ void rope_pairs_f32(u32x4& lo, u32x4& hi, const float2* t, int c0, int swz) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float4 a = *reinterpret_cast<const float4*>(t + ((c0 + 2 * w) ^ swz));   // (swz is even)
    const float2 a0 = make_float2(a.x, a.y), a1 = make_float2(a.z, a.w);
    const float x0 = bf16_lo(lo[w]), x1 = bf16_hi(lo[w]);
    const float y0 = bf16_lo(hi[w]), y1 = bf16_hi(hi[w]);
    lo[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                             (f32x2{fmaf(x0, a0.x, -(y0 * a0.y)), fmaf(x1, a1.x, -(y1 * a1.y))}), bf16x2));
    hi[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                             (f32x2{fmaf(x0, a0.y, y0 * a0.x), fmaf(x1, a1.y, y1 * a1.x)}), bf16x2));
  }
}

// ------------------------------------------------------------ ring tiles --

constexpr int kRing = 4;
constexpr int kRingK = KB * HD * 2;          // bytes of a slot's K rows (V follows)
constexpr int kRingSlot = 2 * kRingK;        // 16 KB
constexpr int kRingLoads = kRingSlot / 16 / kAttnThreads;   // copies per thread and block

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Four 16-bit elements of one column of a 4 x 16 block, the 16 lanes of a
// group holding the block's columns: lane j of the group passes the address
// of elements 4 (j % 4) .. + 3 of row j / 4 and receives column j.  (In a
// device-only function, as lds_dma16.)
__device__ __forceinline__ uint2 lds_read_tr(const uint8_t* p) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}

// The larger of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float max_halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Chunk c (16 bytes) of row r of a slot lies at chunk position c ^ k_swz(r)
// (K) or c ^ v_swz(r) (V): a K fragment read takes one chunk of 16 rows, a
// transposing read 32 lanes' 64 bytes of four rows; both then cover all banks.
__device__ __forceinline__ int k_swz(int r) { return r & 15; }
__device__ __forceinline__ int v_swz(int r) { return 4 * (r & 3); }

}  // namespace entmtp
