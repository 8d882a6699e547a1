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
// HBM bound: 8 bytes an entry and row.
#include <cfloat>
#include <climits>

#include "paged.hpp"
#include "stats.hpp"

namespace entmtp {
namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjWaves = kAdjThreads / 64;
constexpr int kEntries = 16;                           // entries per thread and row
constexpr int kSlice = kEntries * kAdjThreads;         // 4096
constexpr int kRows = 4;                               // rows a workgroup takes at most

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

// VEC: V is a multiple of four (16-byte units); entry e of a thread is then
// e % 4 of unit e / 4, else a unit of its own.
template <bool VEC>
__global__ __launch_bounds__(kAdjThreads) void logit_adjust_kernel(AdjustArgs p) {
  constexpr int E = VEC ? 4 : 1, U = kEntries / E;
  __shared__ uint32_t s_said[kRows][kSlice / 4];   // a byte per entry: drafted tokens on the row's path
  __shared__ int s_row[kRows][4];                  // RowOf
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int V = p.V;
  const int r0 = static_cast<int>(blockIdx.x / p.slices) * p.group;
  const int slice = blockIdx.x % p.slices;
  const int v0 = slice * kSlice;
  const int n = min(p.group, p.rows - r0);
  auto entry = [&](int u) { return v0 + (u * kAdjThreads + tid) * E; };
  auto load = [&](float (&x)[kEntries], const float* row) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = entry(u);
      if constexpr (VEC) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if (v < V) t = *reinterpret_cast<const float4*>(row + v);
        x[4 * u] = t.x;
        x[4 * u + 1] = t.y;
        x[4 * u + 2] = t.z;
        x[4 * u + 3] = t.w;
      } else {
        x[u] = v < V ? row[v] : 0.f;
      }
    }
  };
  auto row_ptr = [&](const float* m, int r) { return m + static_cast<size_t>(r) * V; };

  float x[kEntries], nx[kEntries];
  load(x, row_ptr(p.z, r0));
  for (int i = tid; i < n * (kSlice / 4); i += kAdjThreads) s_said[0][i] = 0u;
  if (wave < n) {   // a wavefront per row finds its sequence
    const RowOf q = row_of(p, r0 + wave);
    if (lane == 0) {
      s_row[wave][0] = q.b;
      s_row[wave][1] = q.node;
      s_row[wave][2] = q.row0;
      s_row[wave][3] = q.tree;
    }
  }
  static_assert(kAdjWaves >= kRows, "a wavefront per row");
  __syncthreads();
  if (tid < 32 * n) {   // 32 threads per row: the path's nodes below the root
    const int i = tid >> 5, j = (tid & 31) + 1;
    const int b = s_row[i][0];
    if (b < p.B) {
      const PagedTree& t = p.trees.t[s_row[i][3]];
      if (j <= t.D) {
        const int node = reinterpret_cast<const int*>(p.trees.arena + t.off_path)[s_row[i][1] * (t.D + 1) + j];
        if (node >= 0 && s_row[i][2] + node < p.rows) {   // (-1 past the node's depth)
          const int rel = p.tok[s_row[i][2] + node] - v0;
          if (rel >= 0 && rel < kSlice) atomicAdd(&s_said[i][rel >> 2], 1u << (8 * (rel & 3)));
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
  bool biased = false, counts = false;
  for (int i = 0; i < n; ++i) {
    const int r = r0 + i;
    if (i + 1 < n) load(nx, row_ptr(p.z, r + 1));
    const int b = __builtin_amdgcn_readfirstlane(s_row[i][0]);
    if (b < p.B) {
      if (b != b_held) {
        b_held = b;
        par = p.params[b];
        counts = par.x != 1.f || par.y != 0.f || par.z != 0.f;
        const int bi = p.bias ? p.bias_idx[b] : -1;
        biased = bi >= 0 && bi < p.n_bias;
        const int* h = p.history + static_cast<size_t>(b) * V;
        const float* bs = p.bias + static_cast<size_t>(biased ? bi : 0) * V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int v = entry(u);
          if constexpr (VEC) {
            int4 t = make_int4(0, 0, 0, 0);
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (counts && p.history && v < V) t = *reinterpret_cast<const int4*>(h + v);
            if (biased && v < V) f = *reinterpret_cast<const float4*>(bs + v);
            hist[4 * u] = t.x;
            hist[4 * u + 1] = t.y;
            hist[4 * u + 2] = t.z;
            hist[4 * u + 3] = t.w;
            bias[4 * u] = f.x;
            bias[4 * u + 1] = f.y;
            bias[4 * u + 2] = f.z;
            bias[4 * u + 3] = f.w;
          } else {
            hist[u] = counts && p.history && v < V ? h[v] : 0;
            bias[u] = biased && v < V ? bs[v] : 0.f;
          }
        }
      }
      const int mi = p.mask ? p.mask_idx[r] : -1;
      const bool masked = mi >= 0 && mi < p.n_masks;
      const uint32_t* mw = p.mask + static_cast<size_t>(masked ? mi : 0) * p.words;
      uint32_t allow[U];   // the unit's bits, lowest first
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = entry(u);
        allow[u] = ~0u;
        if (masked && v < V) allow[u] = mw[v >> 5] >> (v & 31);
      }
      {
#pragma clang fp contract(off)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = (u * kAdjThreads + tid) * E;
          uint32_t said = s_said[i][at >> 2];
          if constexpr (!VEC) said = (said >> (8 * (at & 3))) & 0xffu;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float& z = x[E * u + e];
            const int h = hist[E * u + e];
            const int more = VEC ? (said >> (8 * e)) & 0xff : said;
            if (counts && (h | more) != 0) {
              z = z > 0.f ? z / par.x : z * par.x;
              const int c = (h & INT_MAX) + more;
              if (c > 0) z = (z - par.y * static_cast<float>(c)) - par.z;
            }
            if (biased) z = z + bias[E * u + e];
            if (!((allow[u] >> e) & 1u) || entry(u) >= V) z = -INFINITY;
          }
        }
      }
      if (p.out) {
        float* o = p.out + static_cast<size_t>(r) * V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int v = entry(u);
          if (v < V) {
            if constexpr (VEC)
              *reinterpret_cast<float4*>(o + v) = make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
            else
              o[v] = x[u];
          }
        }
      }
      if (p.part) {
        float best = -INFINITY;
        int idx = INT_MAX;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < E; ++e)   // (in index order within a thread)
            if (x[E * u + e] > best) {
              best = x[E * u + e];
              idx = entry(u) + e;
            }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1)
          take_max(best, idx, __shfl_xor(best, off, 64), __shfl_xor(idx, off, 64));
        // (a NaN is no maximum, but shows in Z)
        const float m = best == -INFINITY ? 0.f : best;
        float Z = 0.f, S = 0.f;
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
          const float t = (x[e] - m) * par.w;
          const float f = __expf(t);
          Z += f;
          if (f > 0.f) S = fmaf(t, f, S);   // keeps (-inf) * 0 out of the sum
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
          Z += __shfl_xor(Z, off, 64);
          S += __shfl_xor(S, off, 64);
        }
        if (lane == 0)
          p.part[(static_cast<size_t>(r) * p.slices + slice) * kAdjWaves + wave] = StatPart{best, Z, S, idx};
      }
    }
#pragma unroll
    for (int e = 0; e < kEntries; ++e) x[e] = nx[e];
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
// top bit says that the prompt holds the token.  Integer atomics: the order
// they land in changes nothing.  A token whose bit is set already needs none
// (a text's frequent tokens would queue up on one address).
__global__ __launch_bounds__(256) void history_prompt_kernel(const int* __restrict__ tok, int n,
                                                             const int* __restrict__ off, int B, int V,
                                                             uint32_t* history) {
  __shared__ int s_off[kPagedSeqs + 1];
  for (int i = threadIdx.x; i <= B; i += 256) s_off[i] = off[i];
  __syncthreads();
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    if (i < s_off[0] || i >= s_off[B]) continue;
    int lo = 0, hi = B;   // the last b with s_off[b] <= i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_off[mid] <= i) lo = mid; else hi = mid;
    }
    const int t = tok[i];
    if (t < 0 || t >= V) continue;
    uint32_t* h = history + static_cast<size_t>(lo) * V + t;
    if (!(__hip_atomic_load(h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 0x80000000u)) atomicOr(h, 0x80000000u);
  }
}

// A wavefront per sequence: the tokens of its accepted path below the root,
// and the bonus token.
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

int adjust_slices(int V) { return (V + kSlice - 1) / kSlice; }

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
  ENTMTP_CHECK_ARG(V <= INT32_MAX - kSlice, ENTMTP_ERANGE, "V = %d too large", V);
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
  a.group = static_cast<long long>(rows) * a.slices >= 8192 ? kRows : 1;
  const long long blocks = static_cast<long long>((rows + a.group - 1) / a.group) * a.slices;
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
  const int blocks = n_tokens / 256 + 1 < 4096 ? n_tokens / 256 + 1 : 4096;
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
