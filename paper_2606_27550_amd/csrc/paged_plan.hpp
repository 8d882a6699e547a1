// What the attentions over a page pool share: the plan (the work list that one
// kernel makes for all layers of a step), the merge of split partials, and the
// sizes of both.  The method is described in paged_attn.hip; the pools hold
// bf16 rows there, 4-bit ones in paged_attn_fp4.hip.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attn_tile.hpp"
#include "paged.hpp"

namespace entmtp {

constexpr int kPagedSplits = 128;
constexpr int kMaxKvHeads = 256;   // (work lists are counted in 32 bits)
constexpr float kMaxCap = 1024.f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPlanMagic = 0x50a6ed01;      // of a plan for bf16 pools
constexpr int kPlanMagicFp4 = 0x50a6ed04;   // of one for 4-bit pools

// First 64 bytes of a plan: what it was made for (the attention does nothing
// with a plan of something else) and the length of its work list.
struct PlanHeader {
  int magic, B, Hq, Hkv, shift, n_pages, max_pages, rows_cap, window, items;
  uint32_t bank_lo, bank_hi;
  int pad[4];
};
static_assert(sizeof(PlanHeader) == 64, "plan layout");

// A sequence as the merge finds it.
struct PlanSeq {
  int row0, T, nsplit, rows_pad;
  long long part_off;   // row offset of its split partials
  int pad[2];
};
static_assert(sizeof(PlanSeq) == 32, "plan layout");

// One workgroup's work.
struct PlanItem {
  int T, L, row0, D;         // T = 0: nothing to do
  int off_mask, off_depth;   // the tree, bytes into the bank's arena
  int b, g, qg, split, nsplit, blk_lo, blk_hi, rows_pad;
  uint32_t part_lo, part_hi;
};
static_assert(sizeof(PlanItem) == 64, "plan layout");

// A plan: header, sequences, the tree of every sequence that has work (-1: none),
// the sequence of every tree row (a byte each; only rows that hold one are
// written, the reader checks it against the sequence's record), work items.
inline size_t plan_topo_at(int B) { return sizeof(PlanHeader) + sizeof(PlanSeq) * B; }
inline size_t plan_rows_at(int B) { return plan_topo_at(B) + sizeof(int) * B; }
inline size_t plan_items_at(int B, int rows_cap) { return (plan_rows_at(B) + rows_cap + 63) / 64 * 64; }
static_assert(kPagedSeqs <= 256, "a sequence is a byte");

__host__ __device__ inline int paged_splits(int nb, int t) {
  if (nb <= kLoneBlocks) return 1;
  int bound = nb / kMinBlocksPerSplit;
  bound = bound > kPagedSplits ? kPagedSplits : bound;
  const int ns = (nb + t - 1) / t;
  return ns < 1 ? 1 : (ns > bound ? bound : ns);
}

// First key block a tree at prefix length L reads: the root's window starts at
// position L + 1 - window.
__host__ __device__ inline int first_pos(int L, int window) {
  return window > 0 && L >= window ? L + 1 - window : 0;
}

// What an attention call and its merge know of the plan and the outputs.
struct PagedCall {
  const uint8_t* plan;
  // [part rows][HD]: the split's output, normalised by its sum so that it stays
  // within its values' range.  Of bf16 pools in bf16: in fp32 the whole output's
  // error against 64 bits is 3.4-3.5e-3 instead of 3.7-3.9e-3 (the weights' and the
  // query's roundings stay), and the bytes cost 3-6 % of long prefixes and windows,
  // 15 % of 26 nodes at 8192 (21.5 -> 24.7 us).  Of 4-bit pools in fp16, the
  // row's largest scaled to [2^14, 2^15): the output of split calls is then off by
  // 2.2-2.3e-3 instead of 2.7-2.9e-3 with bf16 (1.7e-3 of it its own rounding, the
  // rest the weights'), at the same bytes.
  void* part_o;
  float* part_ml;        // [part rows][2]: max, sum; of 4-bit pools [4]: what undoes the scaling, too
  uint16_t* out;         // [rows_cap][Hq][HD]
  long long rows_at, items_at;
  uint64_t bank;         // the bank's number
  int B, G, Hq, Hkv, shift, n_pages, max_pages, rows_cap, window, magic;
};

// Memory that earlier kernels wrote and this one only reads, by scalar loads.
template <typename T>
using Const = const __attribute__((address_space(4))) T*;
template <typename T>
__device__ __forceinline__ Const<T> as_const(const void* p) {
  return (Const<T>)reinterpret_cast<uintptr_t>(p);
}

// A 64-byte record in one scalar load (field by field behind branches, a
// header took a dozen round trips).
typedef int i32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ i32x16 record(const uint8_t* p) { return *as_const<i32x16>(p); }

// Whether a plan's header h says that it was made for this call.
__device__ __forceinline__ bool plan_is_ours(const PagedCall& p, const PlanHeader& h) {
  return ((h.magic ^ p.magic) | (h.B ^ p.B) | (h.Hq ^ p.Hq) | (h.Hkv ^ p.Hkv) | (h.shift ^ p.shift) |
          (h.n_pages ^ p.n_pages) | (h.max_pages ^ p.max_pages) | (h.rows_cap ^ p.rows_cap) | (h.window ^ p.window) |
          static_cast<int>(h.bank_lo ^ static_cast<uint32_t>(p.bank)) |
          static_cast<int>(h.bank_hi ^ static_cast<uint32_t>(p.bank >> 32))) == 0;
}

// ----------------------------------------------------------------- merge --

// LANES threads (half a wavefront or a whole one) take a query head of a tree
// row: lane c reads the (max, sum) of splits c, c + LANES, .., and each 32 lanes
// hold the head's dims, four a lane, of kMergeAhead splits at a time -- a whole
// wavefront's halves of 16 splits each, summed up at the end.  The first partial
// outputs are requested with the (max, sum) pairs.  The row's sequence is found
// by scalar loads: its number, then its record.
// Round trips and little data: 512 rows of 32 heads in four splits take 8 us with
// the launch.
constexpr int kMergeThreads = 256;
constexpr int kMergeAhead = 16;

// HALF: partials in scaled fp16.
template <int LANES, bool HALF>
static __global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedCall p) {
  constexpr int kHeads = kMergeThreads / LANES;
  constexpr int kPairs = kPagedSplits / LANES;   // (max, sum) pairs a lane
  constexpr int kRound = LANES / 32 * kMergeAhead;
  static_assert(LANES % kRound == 0, "a round's weights lie in one register");
  const int groups = (p.Hq + kHeads - 1) / kHeads;
  const int r = static_cast<int>(blockIdx.x) / groups;   // (below rows_cap, by the grid)
  const int h = static_cast<int>(blockIdx.x) % groups * kHeads + threadIdx.x / LANES;
  const i32x16 head = record(p.plan);
  const size_t byte = static_cast<size_t>(p.rows_at) + r;
  const uint32_t word = *as_const<uint32_t>(p.plan + (byte & ~size_t(3)));
  const int b = min(static_cast<int>(word >> (8 * (byte & 3)) & 0xffu), p.B - 1);
  typedef int i32x8 __attribute__((ext_vector_type(8)));
  const PlanSeq sq =
      __builtin_bit_cast(PlanSeq, *as_const<i32x8>(p.plan + sizeof(PlanHeader) + static_cast<size_t>(b) * sizeof(PlanSeq)));
  if (!plan_is_ours(p, __builtin_bit_cast(PlanHeader, head)) | (r < sq.row0) | (r >= sq.row0 + sq.T) | (sq.nsplit == 1))
    return;   // (a row of no sequence, or written by the attention)
  if (h >= p.Hq) return;
  const int nsplit = sq.nsplit, lane = threadIdx.x % LANES;
  const int first = lane / 32 * kMergeAhead;   // this half's splits of a round
  const int row = (h % p.G) * sq.T + (r - sq.row0);
  const size_t base = sq.part_off + static_cast<size_t>(h / p.G) * sq.rows_pad + row;
  const size_t stride = static_cast<size_t>(p.Hkv) * sq.rows_pad;   // from split to split
  const uint16_t* const po = static_cast<const uint16_t*>(p.part_o) + base * HD + 4 * (lane & 31);
  float m[kPairs], l[kPairs], scale[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) {
    m[k] = -INFINITY;
    l[k] = 0.f;
    scale[k] = 1.f;
    if (lane + LANES * k < nsplit) {
      const size_t at = base + (lane + LANES * k) * stride;
      if constexpr (HALF) {
        const float4 ml = *reinterpret_cast<const float4*>(p.part_ml + at * 4);
        m[k] = ml.x;
        l[k] = ml.y;
        scale[k] = ml.z;
      } else {
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
        m[k] = ml.x;
        l[k] = ml.y;
      }
    }
  }
  // (kBatch at a time without a branch between them: a split past the last is
  // that one again, at no weight)
  constexpr int kBatch = LANES == 64 ? kMergeAhead : 4;
  uint2 ob[kMergeAhead];
  auto request = [&](int c) {
#pragma unroll
    for (int k = 0; k < kMergeAhead; ++k)
      if (k / kBatch == 0 || c + k / kBatch * kBatch < nsplit)
        ob[k] = *reinterpret_cast<const uint2*>(po + min(c + first + k, nsplit - 1) * stride * HD);
  };
  request(0);
  float M = m[0];
#pragma unroll
  for (int k = 1; k < kPairs; ++k) M = fmaxf(M, m[k]);
#pragma unroll
  for (int off = LANES / 2; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, LANES));
  // (a split that sees no key of the row has max -inf and counts for nothing;
  // where M is -inf too the row has a NaN score, kept in a sum)
  float lsum = 0.f;
#pragma unroll
  for (int k = 0; k < kPairs; ++k) {
    l[k] = m[k] == -INFINITY ? l[k] : l[k] * __builtin_amdgcn_exp2f(m[k] - M);
    lsum += l[k];
    if constexpr (HALF) l[k] *= scale[k];   // (from here on the partial's weight)
  }
#pragma unroll
  for (int off = LANES / 2; off >= 1; off >>= 1) lsum += __shfl_xor(lsum, off, LANES);
  const float inv = 1.f / lsum;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c = 0; c < nsplit; c += kRound) {
    if (c > 0) request(c);
    float w = l[0];   // the splits' weights, lane s % LANES holding split s's
#pragma unroll
    for (int k = 1; k < kPairs; ++k) w = c >= LANES * k ? l[k] : w;   // (0 past the last split)
#pragma unroll
    for (int k = 0; k < kMergeAhead; ++k) {
      const float wc = __shfl(w, (c + first + k) % LANES, LANES);
      if (k / kBatch == 0 || c + k / kBatch * kBatch < nsplit) {
        const bool in = c + first + k < nsplit;   // (the last one again may hold infinities)
        float4 v;
        if constexpr (HALF) {
          typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
          const f16x2 a = __builtin_bit_cast(f16x2, static_cast<uint32_t>(ob[k].x)), b = __builtin_bit_cast(f16x2, static_cast<uint32_t>(ob[k].y));
          v = make_float4(static_cast<float>(a[0]), static_cast<float>(a[1]), static_cast<float>(b[0]), static_cast<float>(b[1]));
        }
        else
          v = make_float4(__uint_as_float(ob[k].x << 16), __uint_as_float(ob[k].x & 0xffff0000u),
                          __uint_as_float(ob[k].y << 16), __uint_as_float(ob[k].y & 0xffff0000u));
        acc.x = fmaf(wc, in ? v.x : 0.f, acc.x);
        acc.y = fmaf(wc, in ? v.y : 0.f, acc.y);
        acc.z = fmaf(wc, in ? v.z : 0.f, acc.z);
        acc.w = fmaf(wc, in ? v.w : 0.f, acc.w);
      }
    }
  }
  if constexpr (LANES == 64) {
    acc.x += __shfl_xor(acc.x, 32, 64);
    acc.y += __shfl_xor(acc.y, 32, 64);
    acc.z += __shfl_xor(acc.z, 32, 64);
    acc.w += __shfl_xor(acc.w, 32, 64);
    if (lane >= 32) return;
  }
  const uint2 pk = {__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.x * inv, acc.y * inv}), bf16x2)),
                    __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc.z * inv, acc.w * inv}), bf16x2))};
  *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(r) * p.Hq + h) * HD + 4 * lane) = pk;
}

// ------------------------------------------------------------------ host --

inline size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// What a batch of these sizes can need at most, wherever its rows lie apart
// from each other.  A sequence has ceil(G T / 128) query groups, so the groups
// number at most rows G / 128 + B, the streams (KV heads x groups) Hkv times
// that; a split target t gives ceil(nb / t) <= nb / t + 1 splits, so the items
// stay below work / t + streams, and t is at least the even share (half of it
// where two rounds are allowed).  A (KV head, split) range is padded to eight.
struct PagedShape {
  int items = 0;
  bool two = false, splits = false;
  long long part_rows = 0;
  size_t plan_bytes = 0, workspace = 0;   // (the workspace: of bf16 pools)
};

inline PagedShape paged_shape(const entmtp_bank* bank, int B, int rows_cap, int Hq, int Hkv, long long cap) {
  PagedShape sh;
  const int G = Hq / Hkv, slots = device_cus() * kWgPerCu;
  int T_max = 0;
  for (const TopoDesc& td : bank->desc) T_max = std::max(T_max, td.T);
  const long long rows = std::min<long long>(rows_cap, static_cast<long long>(B) * T_max);
  const long long groups = rows * G / (kTilesPerWg * kQTile) + B, streams = Hkv * groups;
  sh.two = two_rounds(streams, slots);
  const int bound = paged_splits(static_cast<int>((cap + KB - 1) / KB), 1);
  sh.splits = bound > 1;
  const int nqg = query_groups(rows_padded(G, T_max) / kQTile);
  const long long all = static_cast<long long>(B) * ((static_cast<long long>(Hkv) * bound + 7) / 8 * 8) * nqg;
  const long long most = (sh.two ? 2LL : 1LL) * slots + streams + (Hkv % 8 ? 7 * groups : 0);
  sh.items = static_cast<int>(std::min(std::min(most, all), static_cast<long long>(INT32_MAX)));
  if (sh.splits)
    sh.part_rows = static_cast<long long>(sh.items) * std::min(kTilesPerWg * kQTile, rows_padded(G, T_max));
  sh.plan_bytes = plan_items_at(B, rows_cap) + sizeof(PlanItem) * static_cast<size_t>(sh.items);
  sh.workspace = up256(static_cast<size_t>(sh.part_rows) * HD * sizeof(uint16_t)) +
                 up256(static_cast<size_t>(sh.part_rows) * 2 * sizeof(float));
  return sh;
}

inline bool shape_ok(const entmtp_bank* bank, int B, int rows_cap, int Hq, int Hkv, int max_pages, int page_size) {
  return bank && !bank->desc.empty() && paged_batch(B) && rows_cap >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 &&
         Hq / Hkv <= 32 && Hkv <= kMaxKvHeads && page_shift(page_size) >= 0 && max_pages >= 1 &&
         static_cast<int64_t>(max_pages) * page_size <= INT32_MAX - 1024;
}

inline int32_t check_batch(int32_t B, int32_t rows_cap, int32_t Hq, int32_t Hkv, int32_t max_pages, int32_t page_size,
                    int32_t n_pages, int32_t window) {
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(rows_cap >= 1, ENTMTP_EINVAL, "rows_cap = %d < 1", rows_cap);
  ENTMTP_CHECK_ARG(Hq >= 1 && Hkv >= 1, ENTMTP_EINVAL, "Hq = %d, Hkv = %d must be >= 1", Hq, Hkv);
  ENTMTP_CHECK_ARG(Hq % Hkv == 0, ENTMTP_ERANGE, "Hq = %d is not a multiple of Hkv = %d", Hq, Hkv);
  ENTMTP_CHECK_ARG(Hq / Hkv <= 32, ENTMTP_ERANGE, "query group %d too large", Hq / Hkv);
  ENTMTP_CHECK_ARG(Hkv <= kMaxKvHeads, ENTMTP_ERANGE, "Hkv = %d too large", Hkv);
  if (int32_t rc = check_pool(n_pages, page_size)) return rc;
  if (int32_t rc = check_pages(max_pages, page_size)) return rc;
  ENTMTP_CHECK_ARG(window >= 0, ENTMTP_EINVAL, "window = %d < 0", window);
  return ENTMTP_OK;
}

// The plan of either kind of pool (entmtp_tree_attn_paged_plan; in paged_attn.hip).
int32_t launch_paged_plan(bool fp4, const entmtp_bank* bank, int32_t B, const int32_t* topo, const int32_t* prefix_len,
                          const int32_t* row_off, const int32_t* status, const int32_t* block_table,
                          int32_t max_pages, int32_t page_size, int32_t n_pages, int32_t rows_cap, int32_t Hq,
                          int32_t Hkv, int32_t window, int32_t* bad, void* plan, size_t plan_bytes, void* stream);

// Bytes of a call's workspace over 4-bit pools.
inline size_t fp4_workspace(const PagedShape& sh) {
  return up256(static_cast<size_t>(sh.part_rows) * HD * sizeof(uint16_t)) +
         up256(static_cast<size_t>(sh.part_rows) * 4 * sizeof(float));
}

// Fills what PagedCall holds; the workspace has been checked against sh.
inline void fill_call(PagedCall& a, const TreeTable& trees, const PagedShape& sh, const void* plan, int32_t B,
                      int32_t n_pages, int32_t page_size, int32_t max_pages, int32_t rows_cap, int32_t Hq,
                      int32_t Hkv, int32_t window, entmtp_bf16* out, void* workspace, int magic) {
  a.plan = static_cast<const uint8_t*>(plan);
  a.bank = trees.bank;
  a.part_o = workspace;
  a.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) +
                                       up256(static_cast<size_t>(sh.part_rows) * HD * sizeof(uint16_t)));
  a.out = out;
  a.rows_at = static_cast<long long>(plan_rows_at(B));
  a.items_at = static_cast<long long>(plan_items_at(B, rows_cap));
  a.B = B;
  a.G = Hq / Hkv;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.shift = page_shift(page_size);
  a.n_pages = n_pages;
  a.max_pages = max_pages;
  a.rows_cap = rows_cap;
  a.window = window;
  a.magic = magic;
}

// The merge's grid: a wavefront a head where they are few, so that long
// prefixes' many splits take half the round trips: 26 rows of 32 heads at 8192
// 21.4 us (attention and merge) against 23.9 by half wavefronts, 8 rows of 8
// heads at 32000 18.3 against 26.4; 4096 heads are level, 32768 take 10 us more
// by whole ones.
inline bool merge_few(int32_t rows_cap, int32_t Hq) {
  return static_cast<long long>(rows_cap) * Hq <= 4LL * device_cus();
}
inline long long merge_blocks(int32_t rows_cap, int32_t Hq) {
  const int heads = kMergeThreads / (merge_few(rows_cap, Hq) ? 64 : 32);
  return static_cast<long long>(rows_cap) * ((Hq + heads - 1) / heads);
}
template <bool HALF>
inline int32_t launch_merge(const PagedCall& a, hipStream_t s) {
  const dim3 blocks(static_cast<uint32_t>(merge_blocks(a.rows_cap, a.Hq)));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, blocks, dim3(kMergeThreads), 0, s, a); };
  if (merge_few(a.rows_cap, a.Hq))
    go(paged_merge_kernel<64, HALF>);
  else
    go(paged_merge_kernel<32, HALF>);
  return launch_status("tree_attn_paged merge launch");
}

}  // namespace entmtp
