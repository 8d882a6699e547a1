// LM-head logits from 4-bit weights: z = X W^T, W in codes and group scales.
//
// The weights stream past the hidden states, which stay in registers.  A
// workgroup of eight wavefronts takes up to 32 rows of X (64 short ones); wavefront w keeps
// an eighth of their length, in 128-wide steps, and takes the same steps of each
// 16-row tile of W: a lane's 16 bytes are 32 codes of one group, which become bf16
// numbers, exactly, on the way into the matrix instruction (16 x 16 x 32), so
// that the products are exact and the sums those of the bf16 LM head.  The eight
// partial sums of a tile meet in the LDS.  (The matrix instruction that takes
// codes as they are, with X as two 8-bit numbers, sums its 128 products to
// 4.6e-6 of the logits' norm; this one to 1e-7.)
//
// Up to 32 rows the weights' bytes bound it: one row of 32000 logits of 4096 values
// takes 14 us (5 TB/s), 8 of 128256 50.5 (5.6), 27 of 128256 60 (4.9), where the bf16
// LM head reads 3.8 times the bytes.  Beyond, the weights come once more for every
// 32 rows (64 of up to 2048 values), from the L2 but at about the same 6 TB/s a chip
// can take, and are turned into bf16 once more: 128 rows of 32000 (5120 values) 57 us
// where the products at bf16's rate would take 31, 64 of 128256 87, 256 of 32000 79.
// A tile kernel for many rows (64 x 128 and 128 x 128 logits a workgroup, W and X
// through the LDS) came to 50-55 us for the first and 100-113 for the second: its
// copies of W are 64 bytes a row and a dword of scales.  (Hidden sizes that are no
// multiple of 128 and scales at odd addresses take lm_fp4_kernel, 10-30 % slower.)
#include <algorithm>

#include "fp4.hpp"
#include "paged.hpp"
#include "stream_pipe.hpp"

namespace entmtp {
namespace {

constexpr int kLmWaves = 8, kLmThreads = 64 * kLmWaves;
constexpr int kLmStep = 128;    // values a matrix instruction takes
constexpr int kLmTile = 16;     // rows of W
constexpr int kLmGroup = 2;     // tiles between reductions
constexpr int kLmRound = 4;     // tiles of the unrolled loop
constexpr int kLmHeld = 64;     // 16 x 16 logits that a workgroup holds before it stores them

struct LmFp4Args {
  const uint16_t* x;       // [T][hid]
  const uint8_t* codes;    // [V][hid / 2]
  const uint8_t* scales;   // [V][hid / 32]
  float* out;              // [T][V]
  int T, hid, V;
  int tiles, slices;       // tiles of W, workgroups that share them
  int chunks;              // of X's rows
  int k0;                  // first step of this pass over hid
  int add;                 // a later pass adds to the earlier ones
};

// KS: steps a wavefront; NT: 16-row tiles of X; NBUF: tiles of W in flight and
// in use.
template <int KS, int NT, int NBUF>
__global__ __launch_bounds__(kLmThreads, 2) void lm_fp4_kernel(LmFp4Args p) {
  __shared__ __attribute__((aligned(16))) f32x4 s_part[2][kLmWaves][kLmGroup][NT][64];
  constexpr int kHold = kLmHeld / NT;   // tiles of W
  __shared__ __attribute__((aligned(16))) f32x4 s_out[kHold][NT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, blk = lane >> 4;
  // the chunks of X that share a range of W follow each other on one XCD
  const int grp = static_cast<int>(blockIdx.x) >> 3;
  const int chunk = grp % p.chunks, slice = (grp / p.chunks) * 8 + (static_cast<int>(blockIdx.x) & 7);
  // its tiles are slice, slice + slices, ..: the workgroups then read one stretch
  // of W between them at any time (stretches of their own, a power of two apart,
  // meet in the same memory channels)
  if (slice >= p.slices) return;
  const int n_tiles = (p.tiles - slice + p.slices - 1) / p.slices;
  auto row_of = [&](int i) { return (slice + min(i, n_tiles - 1) * p.slices) * kLmTile; };
  const int row0 = chunk * 16 * NT;
  const int k0 = (p.k0 + wave * KS) * kLmStep + 32 * blk;   // of this lane's first 32 values

  // Step s of a row of W: the lane's 16 bytes of codes and their scale byte.  Past
  // the row the first step's stand in, and X is zero.
  bool there[KS];
  int coff[KS], soff[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int k = k0 + s * kLmStep;
    there[s] = k < p.hid;
    coff[s] = there[s] ? k / 2 : 0;
    soff[s] = there[s] ? k / 32 : 0;
  }
  u32x4 wb[NBUF][KS];
  uint32_t sb[NBUF][KS];
  const int crow = p.hid / 2, srow = p.hid / 32;
  auto load = [&](int buf, int i) {
    const int v = min(row_of(i) + li, p.V - 1);
    const uint8_t* const c = p.codes + static_cast<size_t>(v) * crow;
    const uint8_t* const s8 = p.scales + static_cast<size_t>(v) * srow;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      wb[buf][s] = *reinterpret_cast<const u32x4*>(c + coff[s]);
      sb[buf][s] = s8[soff[s]];
    }
  };
  // this lane's part of X: row li of each tile, the same 32 values of a step
  u32x4 xb[NT][KS][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + 16 * n + li;
    const uint16_t* const xr = p.x + static_cast<size_t>(min(row, p.T - 1)) * p.hid;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        xb[n][s][j] = *reinterpret_cast<const u32x4*>(xr + 2 * coff[s] + 8 * j);
        if (!there[s]) xb[n][s][j] = u32x4{0u, 0u, 0u, 0u};
      }
  }

  // (the loads keep their order: a wait for a tile then leaves the later ones in flight)
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < NBUF - 1; ++k) {
    load(k, k);
    __builtin_amdgcn_sched_barrier(0);
  }

  const bool wide = (p.V & 3) == 0;
  auto compute = [&](int buf, int k, int par) {
    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      // (past the row X is zero and W's first values stand in, as numbers)
      const float step = fp4_step(there[s] ? sb[buf][s] : 127u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 a = as_bf16x8(fp4_values(wb[buf][s][j], step));
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(xb[n][s][j]), acc[n], 0, 0, 0);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) s_part[par][wave][k][n][lane] = acc[n];
  };
  // the sums of tiles first .. first + 1, kept
  auto reduce = [&](int first, int par) {
    for (int i = tid; i < kLmGroup * NT * 64; i += kLmThreads) {
      const int l = i & 63, n = (i >> 6) % NT, k = i / (64 * NT);
      f32x4 z = s_part[par][0][k][n][l];
#pragma unroll
      for (int w = 1; w < kLmWaves; ++w) z += s_part[par][w][k][n][l];
      s_out[(first + k) % kHold][n][l] = z;
    }
  };
  // Stores of tiles first .. end - 1.  (A store is waited for like the loads
  // issued before and after it, so they go out together: two tiles at a time
  // they cost 10 us of 64 at 27 rows of 128256.)
  auto flush = [&](int first, int end) {
    for (int i = tid; i < (end - first) * NT * 64; i += kLmThreads) {
      const int l = i & 63, n = (i >> 6) % NT, k = first + i / (64 * NT);
      const f32x4 z = s_out[k % kHold][n][l];
      const int row = row0 + 16 * n + (l & 15), v = row_of(k) + 4 * (l >> 4);
      if (row >= p.T || v >= p.V) continue;
      float* const o = p.out + static_cast<size_t>(row) * p.V + v;
      if (wide) {
        f32x4* const o4 = reinterpret_cast<f32x4*>(o);
        *o4 = p.add ? *o4 + z : z;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < p.V) o[e] = p.add ? o[e] + z[e] : z[e];
      }
    }
  };
  int par = 0, kept = 0;
  static_assert(kLmRound % NBUF == 0 && kLmRound % kLmGroup == 0, "a tile's buffer is known");
  static_assert(kHold % kLmRound == 0, "a round is kept whole");
  for (int t = 0; t < n_tiles; t += kLmRound) {
#pragma unroll
    for (int k = 0; k < kLmRound; ++k) {
      load((k + NBUF - 1) % NBUF, t + k + NBUF - 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(k % NBUF, k % kLmGroup, par);
      if (k % kLmGroup == kLmGroup - 1) {
        // (the other half is written while this one is read: one barrier a group)
        wait_lds();
        stage_barrier();
        reduce(t + k + 1 - kLmGroup, par);
        par ^= 1;
      }
    }
    if (t + kLmRound - kept == kHold || t + kLmRound >= n_tiles) {
      wait_lds();
      stage_barrier();
      flush(kept, min(t + kLmRound, n_tiles));
      kept = t + kLmRound;
      if (kept < n_tiles) {
        wait_lds();
        stage_barrier();
      }
    }
  }
}

// ---------------------------------------------------------- whole lines --

// The same for rows of whole steps: a wavefront's part of a tile, 16 rows of 64 KS
// bytes, is copied to the LDS by whole lines, two tiles ahead.  ALL: every wavefront
// has KS steps of this pass; otherwise the last ones have fewer or none, and copy
// the row's first step instead.  Against
// a lane's own 16 bytes to registers: one row of 32000 logits 16.6 -> 13.7 us, 27
// rows 21.9 -> 19.0, 128 rows (5120 values) 63 -> 56; 27 rows of 128256 are level
// (58-60, the plain read's rate is 46), 8 rows 49 -> 50.5.  Three tiles ahead are no
// faster, nor one barrier for two tiles.
// Chunk c (16 bytes) of row r of a tile lies at c ^ lm_swz(r), which spreads the 16
// rows that a read takes over all banks.
template <int KS>
__device__ __forceinline__ int lm_swz(int r) {
  return KS % 4 == 0 ? r & 15 : (KS % 2 == 0 ? r >> 1 & 7 : r >> 2 & 3);
}

// A wavefront's part of a tile: codes, and a dword of scale bytes a row and step.
template <int KS>
struct LmPart {
  uint8_t codes[KS * 1024];
  uint32_t scales[(KS + 3) / 4 * 64];
};

template <int KS, int NT, bool ALL>
__global__ __launch_bounds__(kLmThreads, 2) void lm_fp4_stream_kernel(LmFp4Args p) {
  constexpr int kScaleCopies = (KS + 3) / 4, kCopies = KS + kScaleCopies;
  // the LDS: two tiles of W, partial sums of two, logits of kHold
  constexpr int kFree = 160 * 1024 - 2 * static_cast<int>(sizeof(LmPart<KS>)) * kLmWaves - 2 * kLmWaves * NT * 1024;
  constexpr int kHold = std::min(kFree / (NT * 1024), 48 / NT) / 2 * 2;
  static_assert(kHold >= 2, "a round's logits are kept");
  __shared__ __attribute__((aligned(16))) LmPart<KS> ring0[kLmWaves];
  __shared__ __attribute__((aligned(16))) LmPart<KS> ring1[kLmWaves];
  __shared__ __attribute__((aligned(16))) f32x4 s_part[2][kLmWaves][NT][64];
  __shared__ __attribute__((aligned(16))) f32x4 s_out[kHold][NT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, blk = lane >> 4;
  const int grp = static_cast<int>(blockIdx.x) >> 3;
  const int chunk = grp % p.chunks, slice = (grp / p.chunks) * 8 + (static_cast<int>(blockIdx.x) & 7);
  if (slice >= p.slices) return;
  const int n_tiles = (p.tiles - slice + p.slices - 1) / p.slices;
  auto row_of = [&](int i) { return (slice + min(i, n_tiles - 1) * p.slices) * kLmTile; };
  const int row0 = chunk * 16 * NT;
  const int crow = p.hid / 2, srow = p.hid / 32;
  const int left = p.hid / kLmStep - (p.k0 + wave * KS), n_live = ALL ? KS : max(0, min(left, KS));   // steps
  const int k0 = n_live > 0 ? (p.k0 + wave * KS) * kLmStep : 0;   // of this wavefront's values

  // this lane's part of X: row li of each tile, 32 values of every step
  u32x4 xb[NT][KS][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const uint16_t* const xr = p.x + static_cast<size_t>(min(row0 + 16 * n + li, p.T - 1)) * p.hid + k0 + 32 * blk;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) xb[n][s][j] = *reinterpret_cast<const u32x4*>(xr + (s < n_live ? s : 0) * kLmStep + 8 * j);
  }

  // copies of a tile: place q of the part is chunk q % (4 KS) of row q / (4 KS)
  uint32_t coff[KS], soff[kScaleCopies];
  int crw[KS], srw[kScaleCopies];
#pragma unroll
  for (int j = 0; j < KS; ++j) {
    const int q = 64 * j + lane;
    crw[j] = q / (4 * KS);
    coff[j] = 16 * (q % (4 * KS) ^ lm_swz<KS>(crw[j]));
    if (!ALL && coff[j] >= 64u * n_live) coff[j] = 0;
  }
#pragma unroll
  for (int j = 0; j < kScaleCopies; ++j) {
    const int q = 64 * j + lane;
    srw[j] = min(q / KS, 15);
    soff[j] = 4 * (ALL || q % KS < n_live ? q % KS : 0);
  }
  auto copy = [&](LmPart<KS>& to, int i) {
    // (rows past the last are the last again, as are tiles)
    const int v = row_of(i), last = p.V - 1 - v;
    const __amdgpu_buffer_rsrc_t cbuf = dma_buffer(p.codes + static_cast<size_t>(v) * crow + k0 / 2, 0x7fffffff);
    const __amdgpu_buffer_rsrc_t sbuf = dma_buffer(p.scales + static_cast<size_t>(v) * srow + k0 / 32, 0x7fffffff);
#pragma unroll
    for (int j = 0; j < KS; ++j) buf_dma16(cbuf, static_cast<uint32_t>(min(crw[j], last)) * crow + coff[j], to.codes + 1024 * j);
#pragma unroll
    for (int j = 0; j < kScaleCopies; ++j)
      buf_dma4(sbuf, static_cast<uint32_t>(min(srw[j], last)) * srow + soff[j], to.scales + 64 * j);
  };
  u32x4 w[KS];
  uint32_t sc[KS];
  auto read = [&](const LmPart<KS>& from) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      w[s] = *reinterpret_cast<const u32x4*>(from.codes + 16 * (4 * KS * li + (4 * s + blk ^ lm_swz<KS>(li))));
      sc[s] = from.scales[KS * li + s];
    }
  };
  auto compute = [&](int par) {
    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if (!ALL && s >= n_live) break;   // (uniform)
      const float step = fp4_step(sc[s] >> (8 * blk) & 0xffu);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 a = as_bf16x8(fp4_values(w[s][j], step));
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(xb[n][s][j]), acc[n], 0, 0, 0);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) s_part[par][wave][n][lane] = acc[n];
  };
  // (a number a thread: by fours it would be two wavefronts' work, for which the
  // others wait at the next barrier)
  auto reduce = [&](int i, int par) {
#pragma unroll
    for (int at = tid; at < NT * 256; at += kLmThreads) {
      const float* const from = reinterpret_cast<const float*>(s_part[par]) + at;
      float z = from[0];
#pragma unroll
      for (int v = 1; v < kLmWaves; ++v) z += from[v * NT * 256];
      reinterpret_cast<float*>(s_out[i % kHold])[at] = z;
    }
  };
  const bool wide = (p.V & 3) == 0;
  auto flush = [&](int first, int end) {
    for (int i = tid; i < (end - first) * NT * 64; i += kLmThreads) {
      const int l = i & 63, n = (i >> 6) % NT, k = first + i / (64 * NT);
      const f32x4 z = s_out[k % kHold][n][l];
      const int row = row0 + 16 * n + (l & 15), v = row_of(k) + 4 * (l >> 4);
      if (row >= p.T || v >= p.V) continue;
      float* const o = p.out + static_cast<size_t>(row) * p.V + v;
      if (wide) {
        f32x4* const o4 = reinterpret_cast<f32x4*>(o);
        *o4 = p.add ? *o4 + z : z;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < p.V) o[e] = p.add ? o[e] + z[e] : z[e];
      }
    }
  };
  // (X is waited for here, so that the counts are the copies' alone)
  wait_vmcnt<0>();
  copy(ring0[wave], 0);
  copy(ring1[wave], 1);
  int kept = 0;
  for (int t = 0; t < n_tiles; t += 2) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      LmPart<KS>& mine = k ? ring1[wave] : ring0[wave];
      wait_vmcnt<kCopies>();
      read(mine);
      wait_lds();
      asm volatile("" ::: "memory");
      copy(mine, t + k + 2);
      compute(k);
      // (the other half is written while this one is read: one barrier a tile)
      wait_lds();
      stage_barrier();
      reduce(t + k, k);
    }
    if (t + 2 - kept == kHold || t + 2 >= n_tiles) {
      wait_lds();
      stage_barrier();
      flush(kept, min(t + 2, n_tiles));
      kept = t + 2;
      if (kept < n_tiles) {
        wait_lds();
        stage_barrier();
      }
    }
  }
  wait_vmcnt<0>();   // (copies past the last tile)
}

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" int32_t entmtp_verify_logits_fp4(const entmtp_bf16* hidden, const uint8_t* codes, const uint8_t* scales,
                                            int32_t T, int32_t hid, int32_t V, float* logits, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(hidden && codes && scales && logits, ENTMTP_EINVAL, "hidden, codes, scales and logits must be non-NULL");
  ENTMTP_CHECK_ARG(T >= 1 && T <= 4096, ENTMTP_EINVAL, "T = %d outside [1, 4096]", T);
  ENTMTP_CHECK_ARG(hid >= kFp4Group && hid % kFp4Group == 0 && hid <= 65536, ENTMTP_EINVAL,
                   "hid = %d must be a multiple of %d up to 65536", hid, kFp4Group);
  ENTMTP_CHECK_ARG(V >= 1 && V <= INT32_MAX - 4096, ENTMTP_EINVAL, "V = %d out of range", V);
  ENTMTP_CHECK_ARG(aligned16(hidden) && aligned16(codes) && aligned16(logits), ENTMTP_EINVAL,
                   "hidden, codes and logits must be 16-byte aligned");
  LmFp4Args a{};
  a.x = hidden;
  a.codes = codes;
  a.scales = scales;
  a.out = logits;
  a.T = T;
  a.hid = hid;
  a.V = V;
  a.tiles = (V + kLmTile - 1) / kLmTile;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int steps = (hid + kLmStep - 1) / kLmStep;
  // a pass over hid holds at most 8 steps a wavefront (5 where it has two tiles of X,
  // 2 where it has four, which halves the copies of W: of 128256 logits 128 rows of
  // 1024 values 78 -> 61 us, 100 of 1536 94 -> 78; of 32000 33 of 2048 18.1 -> 16.7;
  // 64 rows of 50257 of 2048 lose by it, 30.9 -> 32.0)
  const bool lines = hid % kLmStep == 0 && (reinterpret_cast<uintptr_t>(scales) & 3u) == 0;   // (a step's scale bytes are a dword)
  const int nt = T > 32 && lines && steps <= 2 * kLmWaves ? 4 : (T > 16 ? 2 : 1), most = nt == 4 ? 2 : (nt == 2 ? 5 : 8);
  const int passes = (steps + most * kLmWaves - 1) / (most * kLmWaves);
  const int ks = ((steps + passes - 1) / passes + kLmWaves - 1) / kLmWaves;
  a.chunks = (T + 16 * nt - 1) / (16 * nt);
  a.slices = std::min(std::max(1, device_cus() / a.chunks / 8) * 8, a.tiles);
  const dim3 grid(static_cast<uint32_t>((a.slices + 7) / 8 * 8 * a.chunks));
  for (int pass = 0; pass < passes; ++pass) {
    a.k0 = pass * ks * kLmWaves;
    a.add = pass > 0;
    const bool all = a.k0 + ks * kLmWaves <= steps;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kLmThreads), 0, s, a); };
#define LM_FP4_LINES(KS, NT) go(all ? lm_fp4_stream_kernel<KS, NT, true> : lm_fp4_stream_kernel<KS, NT, false>)
#define LM_FP4(KS, NT)             \
  if (lines)                       \
    LM_FP4_LINES(KS, NT);          \
  else                             \
    go(lm_fp4_kernel<KS, NT, 2>)
    if (nt == 4) {
      if (ks == 1)
        LM_FP4_LINES(1, 4);
      else
        LM_FP4_LINES(2, 4);
    } else if (nt == 1) {
      switch (ks) {
        case 1: LM_FP4(1, 1); break;
        case 2: LM_FP4(2, 1); break;
        case 3: LM_FP4(3, 1); break;
        case 4: LM_FP4(4, 1); break;
        case 5: LM_FP4(5, 1); break;
        case 6: LM_FP4(6, 1); break;
        case 7: LM_FP4(7, 1); break;
        default: LM_FP4(8, 1);
      }
    } else {
      switch (ks) {
        case 1: LM_FP4(1, 2); break;
        case 2: LM_FP4(2, 2); break;
        case 3: LM_FP4(3, 2); break;
        case 4: LM_FP4(4, 2); break;
        default: LM_FP4(5, 2);
      }
    }
#undef LM_FP4
#undef LM_FP4_LINES
    if (int32_t rc = launch_status("verify_logits_fp4 launch")) return rc;
  }
  return ENTMTP_OK;
}
