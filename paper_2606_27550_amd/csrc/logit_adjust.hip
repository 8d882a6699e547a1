// Penalties, biases and grammar masks on the verification logits, with the
// statistics of the result, and the token history the penalties read.
//
// Row i of a batch is a tree node; its logits z are the target's for the token
// after it.  With c(v) = how often v was said so far -- the sequence's history
// plus the drafted tokens on the node's path below the root (the root's token
// is the last one emitted, so the history holds it) -- and seen(v) = c(v) > 0
// or v in the prompt:
//   z(v) <- z(v) > 0 ? z(v) / rep : z(v) rep       where seen(v)
//   z(v) <- (z(v) - freq c(v)) - pres              where c(v) > 0
//   z(v) <- z(v) + bias(v)                         where the sequence has a bias row
//   z(v) <- -inf                                   where the row's mask forbids v
// in fp32, each step rounded (no fused multiply-add, so the result is the
// formula's whatever the compiler does), and of the result, at the sequence's
// own inverse temperature, entropy, top-1 probability and lowest argmax.
//
// One pass over the logits.  A workgroup takes a slice of 4096 entries and up
// to kRows rows after each other: the next row's logits are in flight while
// this one is worked on, and the slice's history and biases stay in registers
// while the rows belong to one sequence (they cost as much as a row's logits
// otherwise).  The drafted tokens of the rows' paths lie in LDS as a byte per
// entry of the slice, so an entry's count is one addition.  Every wavefront
// writes its own statistics partial (no barrier in the row loop) and a second
// kernel merges a row's partials, a wavefront per row.
// HBM bound, 8 bytes an entry and row, once the arithmetic fits beside it: 1024
// rows of 128256 with everything asked for take 209 us, 5.1 TB/s (a large copy
// reaches 5.2; 255 with divisions, reductions by LDS permutes, the argmax's
// index kept entry by entry and stores through the caches).  26 rows of 32000
// take 9.9 us, both kernels' latency.
#include <cfloat>
#include <climits>
#include <type_traits>

#include "paged.hpp"
#include "stats.hpp"

namespace entmtp {
namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjWaves = kAdjThreads / 64;
constexpr int kEntries = 16;                           // entries per thread and row
constexpr int kSlice = kEntries * kAdjThreads;         // 4096
constexpr int kRows = 4;                               // rows a workgroup takes at most
constexpr int kUnits = kEntries / 4;                   // a thread's units of four entries

typedef float f32x4v __attribute__((ext_vector_type(4)));

struct AdjustArgs {
  TreeTable trees;
  const int* topo;
  const int* row_off;
  const int* tok;        // [rows]
  const float* z;        // [rows][V]
  const float4* params;  // [B]: rep, freq, pres, inv_temp
  const int* history;    // [B][V] or NULL
  const float* bias;     // [n_bias][V] or NULL
  const int* bias_idx;   // [B]
  const uint32_t* mask;  // [n_masks][words] or NULL
  const int* mask_idx;   // [rows]
  float* out;            // [rows][V] or NULL
  StatPart* part;        // [rows][slices * kAdjWaves]
  float* entropy;
  float* top1p;
  int* argmax;
  int B, rows, V, n_bias, n_masks, words, slices, group;   // group: rows per workgroup
};

// A row's place: sequence (B: none) and node.
struct RowOf {
  int b, node, row0, tree;
};

__device__ __forceinline__ RowOf row_of(const AdjustArgs& p, int r) {
  RowOf q{p.B, 0, 0, 0};
  const int b = seq_of_row(p.row_off, p.B, r);
  if (b >= p.B || r >= p.rows) return q;
  const int row0 = p.row_off[b], tr = p.topo[b];
  if (row0 < 0 || r < row0 || tr < 0 || tr >= p.trees.n || r - row0 >= p.trees.t[tr].T) return q;
  q.b = b;
  q.node = r - row0;
  q.row0 = row0;
  q.tree = tr;
  return q;
}

// f over the wavefront's 64 lanes, in every lane: within rows of 16 by DPP, then
// the rows and the halves (through LDS permutes a row's reductions are a chain
// of 24 round trips).
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F f) {
  auto dpp = [&](auto ctrl) {
    return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  v = f(v, dpp(std::integral_constant<int, 0xB1>{}));    // lane ^ 1
  v = f(v, dpp(std::integral_constant<int, 0x4E>{}));    // lane ^ 2
  v = f(v, dpp(std::integral_constant<int, 0x141>{}));   // mirrored halves of a row
  v = f(v, dpp(std::integral_constant<int, 0x140>{}));   // mirrored rows
  uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = f(__builtin_bit_cast(T, static_cast<uint32_t>(a[0])), __builtin_bit_cast(T, static_cast<uint32_t>(a[1])));
  u = __builtin_bit_cast(uint32_t, v);
  const auto c = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return f(__builtin_bit_cast(T, static_cast<uint32_t>(c[0])), __builtin_bit_cast(T, static_cast<uint32_t>(c[1])));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int wave_min(int v) {
  return wave_all(v, [](int a, int b) { return a < b ? a : b; });
}

// A thread's units of four entries are 16-byte aligned in the logits.  WHOLE: V
// is a multiple of four, so units start at multiples of four in every row.
// Else row r starts (r V) % 4 entries past a 16-byte boundary: a workgroup then
// takes every fourth row, which start alike, and its slices start that many
// entries early.  (Rows as they come, by 16-byte accesses at any address, took
// 305 us for 1024 rows of 128255 where rows of 128256 took 214.)
template <bool WHOLE>
__global__ __launch_bounds__(kAdjThreads) void logit_adjust_kernel(AdjustArgs p) {
  __shared__ uint32_t s_said[kRows][kSlice / 4];   // a byte per entry: drafted tokens on the row's path
  __shared__ int s_row[kRows][4];                  // RowOf
  constexpr int kStep = WHOLE ? 1 : 4;             // from row to row
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int V = p.V;
  const int part = static_cast<int>(blockIdx.x / p.slices), slice = blockIdx.x % p.slices;
  const int r0 = part / kStep * (kStep * p.group) + part % kStep;
  const int n = min(p.group, (p.rows - r0 + kStep - 1) / kStep);
  if (n <= 0) return;
  const int v0 = slice * kSlice - (WHOLE ? 0 : static_cast<int>(static_cast<unsigned>(r0) * static_cast<unsigned>(V) & 3u));
  auto row_at = [&](int i) { return r0 + kStep * i; };
  auto entry = [&](int u) { return v0 + (u * kAdjThreads + tid) * 4; };
  auto in_row = [&](int v) { return v < V && (WHOLE || v >= 0); };
  // the thread's entries of a row, zeros outside it
  auto load = [&](auto& x, const auto* row, auto aligned) {
    typedef std::remove_reference_t<decltype(x[0])> T;
    typedef T T4 __attribute__((ext_vector_type(4), aligned(decltype(aligned)::value)));
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int v = entry(u);
      T4 t = {0, 0, 0, 0};
      if (v <= V - 4 && (WHOLE || v >= 0)) {
        t = *reinterpret_cast<const T4*>(row + v);
      } else if constexpr (!WHOLE) {   // the row's first or last unit
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (in_row(v + e)) t[e] = row[v + e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * u + e] = t[e];
    }
  };
  constexpr std::integral_constant<int, 16> kAligned{};
  constexpr std::integral_constant<int, WHOLE ? 16 : 4> kAny{};   // history and bias rows start elsewhere
  auto row_ptr = [&](const float* m, int r) { return m + static_cast<size_t>(r) * V; };

  float x[kEntries], nx[kEntries];
  load(x, row_ptr(p.z, r0), kAligned);
  for (int i = tid; i < n * (kSlice / 4); i += kAdjThreads) s_said[0][i] = 0u;
  for (int i = wave; i < n; i += kAdjWaves) {   // a wavefront finds a row's sequence
    const RowOf q = row_of(p, row_at(i));
    if (lane == 0) {
      s_row[i][0] = q.b;
      s_row[i][1] = q.node;
      s_row[i][2] = q.row0;
      s_row[i][3] = q.tree;
    }
  }
  __syncthreads();
  if (tid < 32 * n) {   // 32 threads per row: the path's nodes below the root
    const int i = tid >> 5, j = (tid & 31) + 1;
    const int b = s_row[i][0];
    if (b < p.B) {
      const PagedTree& t = p.trees.t[s_row[i][3]];
      if (j <= t.D) {
        const int node = reinterpret_cast<const int*>(p.trees.arena + t.off_path)[s_row[i][1] * (t.D + 1) + j];
        if (node >= 0 && s_row[i][2] + node < p.rows) {   // (-1 past the node's depth)
          const int tok = p.tok[s_row[i][2] + node], rel = tok - v0;
          if (tok >= 0 && rel >= 0 && rel < kSlice) atomicAdd(&s_said[i][rel >> 2], 1u << (8 * (rel & 3)));
        }
      }
    }
  }
  static_assert(32 * kRows <= kAdjThreads && ENTMTP_D_MAX < 32, "32 threads per row hold a path");
  __syncthreads();

  int hist[kEntries];
  float bias[kEntries];
  int b_held = -1;
  float4 par = make_float4(1.f, 0.f, 0.f, 1.f);
  double rrep = 1.0, rrep_lo = 0.0;   // 1 / rep: rounded, and what that left
  bool biased = false, counts = false;
  auto work = [&](float (&x)[kEntries], int i) {
    const int r = row_at(i);
    const int b = __builtin_amdgcn_readfirstlane(s_row[i][0]);
    if (b >= p.B) return;
    if (b != b_held) {
      b_held = b;
      par = p.params[b];
      rrep = 1.0 / static_cast<double>(par.x);
      rrep_lo = fma(-rrep, static_cast<double>(par.x), 1.0) * rrep;
      rrep_lo = rrep_lo == rrep_lo ? rrep_lo : 0.0;   // (a factor of infinity or zero)
      counts = par.x != 1.f || par.y != 0.f || par.z != 0.f;
      const int bi = p.bias ? p.bias_idx[b] : -1;
      biased = bi >= 0 && bi < p.n_bias;
      const int* h = p.history + static_cast<size_t>(b) * V;
      const float* bs = p.bias + static_cast<size_t>(biased ? bi : 0) * V;
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        hist[e] = 0;
        bias[e] = 0.f;
      }
      if (counts && p.history) load(hist, h, kAny);
      if (biased) load(bias, bs, kAny);
    }
    const int mi = p.mask ? p.mask_idx[r] : -1;
    const bool masked = mi >= 0 && mi < p.n_masks;
    uint32_t allow[kUnits];   // the unit's bits, lowest first
    if (masked) {
      const uint32_t* mw = p.mask + static_cast<size_t>(mi) * p.words;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int v = entry(u), last = (V - 1) >> 5;
        if constexpr (WHOLE) {
          allow[u] = mw[min(v >> 5, last)] >> (v & 31);
        } else {   // (a unit can straddle two words)
          const uint64_t lo = mw[max(0, min(v >> 5, last))], hi = mw[max(0, min((v >> 5) + 1, last))];
          allow[u] = static_cast<uint32_t>((hi << 32 | lo) >> (v & 31));
        }
      }
    }
    {
#pragma clang fp contract(off)
      if (counts) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const uint32_t said = s_said[i][u * kAdjThreads + tid];
          uint32_t any = said;
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= static_cast<uint32_t>(hist[4 * u + e]);
          if (any == 0u) continue;   // (most tokens never were)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int h = hist[4 * u + e], more = (said >> (8 * e)) & 0xff;
            float z = x[4 * u + e];
            // z / rep as fp32 rounds it, by way of 64 bits: with the reciprocal's
            // two words the product is the quotient to 2^-104 before its rounding
            // to 53 bits.  Those hold a quotient that lies right where fp32's
            // rounding turns (only one below the normal numbers can), and any other
            // is 2^-49 of itself or more away from there.  (Infinity, by either.)
            const double zd = static_cast<double>(z);
            const float q = static_cast<float>(fma(zd, rrep, zd * rrep_lo));
            z = z > 0.f && z < INFINITY ? q : z * par.x;
            const int c = (h & INT_MAX) + more;
            if (c > 0) z = (z - par.y * static_cast<float>(c)) - par.z;
            if ((h | more) != 0) x[4 * u + e] = z;
          }
        }
      }
      if (biased) {
#pragma unroll
        for (int e = 0; e < kEntries; ++e) x[e] = x[e] + bias[e];
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < kEntries; ++e)
          if (!((allow[e / 4] >> (e % 4)) & 1u)) x[e] = -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < kEntries; ++e)
        if (!in_row(entry(e / 4) + (WHOLE ? 0 : e % 4))) x[e] = -INFINITY;
    }
    if (p.out) {
      float* o = p.out + static_cast<size_t>(r) * V;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int v = entry(u);
        if (v <= V - 4 && (WHOLE || v >= 0)) {
          // (written past the caches: nothing of this kernel reads it again)
          __builtin_nontemporal_store(f32x4v{x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]},
                                      reinterpret_cast<f32x4v*>(o + v));
        } else if constexpr (!WHOLE) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (in_row(v + e)) o[v + e] = x[4 * u + e];
        }
      }
    }
    if (p.part) {
      float mine = x[0];
#pragma unroll
      for (int e = 1; e < kEntries; ++e) mine = fmaxf(mine, x[e]);   // (a NaN is no maximum, but shows in Z)
      const float best = wave_max(mine);
      int idx = INT_MAX;
      if (mine == best && best > -INFINITY) {
#pragma unroll
        for (int e = kEntries - 1; e >= 0; --e)   // (a thread's entries rise with e)
          if (x[e] == best) idx = entry(e / 4) + e % 4;
      }
      idx = wave_min(idx);
      // (the difference of the raw logits first: exact or nearly, 0 for the
      // largest; base 2 from there on)
      const float m = best > -INFINITY ? best : 0.f, it2 = par.w * 1.44269504088896341f;
      float Z = 0.f, S = 0.f;
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        const float t = (x[e] - m) * it2;
        const float f = __builtin_amdgcn_exp2f(t);
        Z += f;
        S = fmaf(fmaxf(t, -256.f), f, S);   // (2^-256 is 0: keeps (-inf) * 0 out of the sum)
      }
      Z = wave_sum(Z);
      S = wave_sum(S) * 0.693147180559945309f;
      if (lane == 0)
        p.part[(static_cast<size_t>(r) * p.slices + slice) * kAdjWaves + wave] = StatPart{best, Z, S, idx};
    }
  };
  for (int i = 0; i < n; i += 2) {   // (two rows a round: their registers take turns)
    if (i + 1 < n) load(nx, row_ptr(p.z, row_at(i + 1)), kAligned);
    work(x, i);
    if (i + 2 < n) load(x, row_ptr(p.z, row_at(i + 2)), kAligned);
    if (i + 1 < n) work(nx, i + 1);
  }
}

// Merges a row's partials, a wavefront per row; rows of no sequence are left
// alone.  A row with nothing left (every entry -inf) has argmax -1, top-1
// probability 0 and entropy 0; one with a NaN has NaN statistics.
__global__ __launch_bounds__(kAdjThreads) void adjust_stats_kernel(AdjustArgs p) {
  const int lane = threadIdx.x & 63;
  const int r = static_cast<int>(blockIdx.x) * kAdjWaves + (threadIdx.x >> 6);
  if (r >= p.rows) return;
  const RowOf q = row_of(p, r);
  if (q.b >= p.B) return;
  const float it = p.params[q.b].w;
  const int G = p.slices * kAdjWaves;
  const StatPart* src = p.part + static_cast<size_t>(r) * G;
  float best = -INFINITY, bad = 0.f;   // bad: NaN once a partial holds one
  int idx = INT_MAX;
  for (int g = lane; g < G; g += 64) {
    const StatPart a = src[g];
    take_max(best, idx, a.zmax, a.idx);
    bad += a.Z * 0.f;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    take_max(best, idx, __shfl_xor(best, off, 64), __shfl_xor(idx, off, 64));
    bad += __shfl_xor(bad, off, 64);
  }
  float Z = 0.f, S = 0.f;
  for (int g = lane; g < G; g += 64) {
    const StatPart a = src[g];
    if (a.zmax == -INFINITY) continue;
    const float d = (a.zmax - best) * it, f = __expf(d);
    Z += a.Z * f;
    S += f > 0.f ? f * (a.S + d * a.Z) : 0.f;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    Z += __shfl_xor(Z, off, 64);
    S += __shfl_xor(S, off, 64);
  }
  if (lane != 0) return;
  const bool some = best > -INFINITY;
  if (p.entropy) p.entropy[r] = (some ? logf(Z) - S / Z : 0.f) + bad;
  if (p.top1p) p.top1p[r] = (some ? 1.f / Z : 0.f) + bad;
  if (p.argmax) p.argmax[r] = some ? idx : -1;
}

// --------------------------------------------------------------- history --

// An entry of the history counts the tokens said in its lower 31 bits; the
// top bit says that the prompt holds the token.  The threads of a prompt that
// meet at an entry all read the same count and store the same word, so no
// atomic is needed.  Bound by the lines its scattered words lie in, so an
// XCD takes a stretch of the tokens and finds a sequence's lines in its L2: 64
// prompts of 100 to 32768 tokens, vocabulary 128256, take 9.0 us (13.4 with the
// workgroups in order, every XCD fetching every line).
__global__ __launch_bounds__(256) void history_prompt_kernel(const int* __restrict__ tok, int n,
                                                             const int* __restrict__ off, int B, int V,
                                                             uint32_t* history) {
  __shared__ int s_off[kPagedSeqs + 1];
  // (workgroups go to the eight XCDs in turn)
  const int block = static_cast<int>((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3));
  const int i = block * 256 + threadIdx.x;
  const int t = i < n ? tok[i] : -1;   // (in flight with the offsets)
  for (int k = threadIdx.x; k <= B; k += 256) s_off[k] = off[k];
  __syncthreads();
  if (t < 0 || t >= V || i < s_off[0] || i >= s_off[B]) return;
  int b = 0;   // the last sequence that starts at or before i
#pragma unroll
  for (int step = kPagedSeqs / 2; step >= 1; step >>= 1)
    if (b + step < B && s_off[min(b + step, B)] <= i) b += step;
  uint32_t* const h = history + static_cast<size_t>(b) * V + t;
  const uint32_t v = *h;
  if (!(v & 0x80000000u)) *h = v | 0x80000000u;
}

// A wavefront per sequence: the tokens of its accepted path below the root,
// and the bonus token, counted by integer atomics (a token may come twice; their
// order changes nothing).  Three round trips: 2.2 us.
__global__ __launch_bounds__(64) void history_accept_kernel(const int* __restrict__ row_off,
                                                            const int* __restrict__ tok, int rows,
                                                            const int* __restrict__ path, int path_cap,
                                                            const int* __restrict__ accept_len,
                                                            const int* __restrict__ bonus, int V,
                                                            int* __restrict__ history) {
  const int b = blockIdx.x, lane = threadIdx.x;
  const int a = accept_len[b];
  if (a < 0) return;   // not verified
  const int last = min(a, min(path_cap, ENTMTP_D_MAX + 1) - 1);
  int t = -1;
  if (lane >= 1 && lane <= last) {
    const int r0 = row_off[b], node = path[static_cast<size_t>(b) * path_cap + lane];
    const long long r = static_cast<long long>(r0) + node;
    if (r0 >= 0 && node >= 0 && r < row_off[b + 1] && r < rows) t = tok[r];
  } else if (lane == 63) {
    t = bonus[b];
  }
  static_assert(ENTMTP_D_MAX < 63, "a lane per path node, the last one for the bonus token");
  if (t >= 0 && t < V) atomicAdd(history + static_cast<size_t>(b) * V + t, 1);
}

// (a row may start up to three entries into its first slice)
int adjust_slices(int V) { return (V + ((V & 3) ? 3 : 0) + kSlice - 1) / kSlice; }

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" size_t entmtp_logit_adjust_workspace(int32_t rows, int32_t V) {
  if (rows < 1 || V < 1) return 0;
  return static_cast<size_t>(rows) * adjust_slices(V) * kAdjWaves * sizeof(StatPart);
}

extern "C" int32_t entmtp_logit_adjust(const entmtp_bank* bank, int32_t B, const int32_t* topo,
                                       const int32_t* row_off, int32_t rows, const int32_t* draft_tokens,
                                       const float* logits, int32_t V, const float* params,
                                       const int32_t* history, const float* bias, int32_t n_bias,
                                       const int32_t* bias_idx, const uint32_t* mask, int32_t n_masks,
                                       int32_t mask_words, const int32_t* mask_idx, float* out,
                                       float* entropy, float* top1p, int32_t* argmax, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(topo && row_off && draft_tokens && logits && params, ENTMTP_EINVAL,
                   "topo, row_off, draft_tokens, logits and params must be non-NULL device arrays");
  ENTMTP_CHECK_ARG(rows >= 1 && V >= 1, ENTMTP_EINVAL, "rows = %d, V = %d must be >= 1", rows, V);
  ENTMTP_CHECK_ARG(V <= INT32_MAX - 2 * kSlice, ENTMTP_ERANGE, "V = %d too large", V);
  ENTMTP_CHECK_ARG((bias == nullptr) == (bias_idx == nullptr) && (!bias || n_bias >= 1), ENTMTP_EINVAL,
                   "bias (n_bias = %d rows) and bias_idx go together", n_bias);
  ENTMTP_CHECK_ARG((mask == nullptr) == (mask_idx == nullptr) && (!mask || n_masks >= 1), ENTMTP_EINVAL,
                   "mask (n_masks = %d rows) and mask_idx go together", n_masks);
  ENTMTP_CHECK_ARG(!mask || mask_words >= (V + 31) / 32, ENTMTP_EINVAL,
                   "mask rows of %d words are shorter than V = %d bits", mask_words, V);
  ENTMTP_CHECK_ARG(aligned16(logits) && aligned16(out) && aligned16(history) && aligned16(bias) &&
                       aligned16(params) && aligned16(workspace),
                   ENTMTP_EINVAL, "logits, out, history, bias, params and workspace must be 16-byte aligned");
  const bool stats = entropy || top1p || argmax;
  const size_t need = stats ? entmtp_logit_adjust_workspace(rows, V) : 0;
  ENTMTP_CHECK_ARG(!stats || workspace, ENTMTP_EINVAL, "the statistics need a workspace");
  ENTMTP_CHECK_ARG(workspace_bytes >= need, ENTMTP_ENOSPC, "workspace has %zu bytes, needs %zu",
                   workspace_bytes, need);
  AdjustArgs a{};
  if (int32_t rc = tree_table(bank, &a.trees)) return rc;
  if (!stats && !out) return ENTMTP_OK;
  a.topo = topo;
  a.row_off = row_off;
  a.tok = draft_tokens;
  a.z = logits;
  a.params = reinterpret_cast<const float4*>(params);
  a.history = history;
  a.bias = bias;
  a.bias_idx = bias_idx;
  a.mask = mask;
  a.mask_idx = mask_idx;
  a.out = out;
  a.part = stats ? static_cast<StatPart*>(workspace) : nullptr;
  a.entropy = entropy;
  a.top1p = top1p;
  a.argmax = argmax;
  a.B = B;
  a.rows = rows;
  a.V = V;
  a.n_bias = n_bias;
  a.n_masks = n_masks;
  a.words = mask_words;
  a.slices = adjust_slices(V);
  // Rows a workgroup takes: as many as leave two rounds of four workgroups a CU
  // (what registers let reside where V is a multiple of four; three elsewhere),
  // so that few rows fill the chip and many share their start.  128 rows of
  // 128256: one row each 38.6 us, two 35.0; 1024 rows: four 209, eight 215; 26
  // rows of 128256: one 14.7.
  const long long fill = static_cast<long long>(rows) * a.slices / (8 * device_cus());
  a.group = static_cast<int>(fill < 1 ? 1 : (fill > kRows ? kRows : fill));
  const int step = (V & 3) ? 4 : 1;   // rows a workgroup's rows lie apart
  const long long blocks = static_cast<long long>((rows + step * a.group - 1) / (step * a.group)) * step * a.slices;
  ENTMTP_CHECK_ARG(blocks <= INT32_MAX, ENTMTP_ERANGE, "%d rows of %d entries: too many", rows, V);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kAdjThreads), 0, s, a);
  };
  (V & 3) == 0 ? go(logit_adjust_kernel<true>) : go(logit_adjust_kernel<false>);
  if (int32_t rc = launch_status("logit_adjust launch")) return rc;
  if (!stats) return ENTMTP_OK;
  hipLaunchKernelGGL(adjust_stats_kernel, dim3((rows + kAdjWaves - 1) / kAdjWaves), dim3(kAdjThreads), 0, s, a);
  return launch_status("logit_adjust statistics launch");
}

extern "C" int32_t entmtp_token_history_prompt(const int32_t* tokens, int32_t n_tokens, const int32_t* tok_off,
                                               int32_t B, int32_t V, int32_t* history, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(tok_off && history, ENTMTP_EINVAL, "tok_off and history must be non-NULL device arrays");
  ENTMTP_CHECK_ARG(n_tokens >= 0 && n_tokens <= INT32_MAX - (1 << 24) && (tokens || n_tokens == 0), ENTMTP_EINVAL,
                   "tokens is NULL or n_tokens = %d out of range", n_tokens);
  ENTMTP_CHECK_ARG(V >= 1, ENTMTP_EINVAL, "V = %d must be >= 1", V);
  if (n_tokens == 0) return ENTMTP_OK;
  const int blocks = ((n_tokens - 1) / 256 / 8 + 1) * 8;
  hipLaunchKernelGGL(history_prompt_kernel, dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream), tokens,
                     n_tokens, tok_off, B, V, reinterpret_cast<uint32_t*>(history));
  return launch_status("token_history_prompt launch");
}

extern "C" int32_t entmtp_token_history_accept(int32_t B, const int32_t* row_off, const int32_t* draft_tokens,
                                               int32_t rows, const int32_t* path, int32_t path_capacity,
                                               const int32_t* accept_len, const int32_t* bonus, int32_t V,
                                               int32_t* history, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(row_off && draft_tokens && path && accept_len && bonus && history, ENTMTP_EINVAL,
                   "row_off, draft_tokens, path, accept_len, bonus and history must be non-NULL device arrays");
  ENTMTP_CHECK_ARG(rows >= 1 && V >= 1, ENTMTP_EINVAL, "rows = %d, V = %d must be >= 1", rows, V);
  ENTMTP_CHECK_ARG(path_capacity >= 1, ENTMTP_EINVAL, "path_capacity = %d < 1", path_capacity);
  hipLaunchKernelGGL(history_accept_kernel, dim3(B), dim3(64), 0, static_cast<hipStream_t>(stream), row_off,
                     draft_tokens, rows, path, path_capacity, accept_len, bonus, V, history);
  return launch_status("token_history_accept launch");
}
