// Tree attention over a page pool, for batches of up to 256 sequences whose
// trees, prefix lengths and pages the host never reads.
//
// Node i of sequence b (position pos_i = L + depth(i)) and query head h attend
// to the prefix and to i's root-to-node path:
//   s = scale q . k;  s = cap tanh(s / cap) (a score cap);  s = s - slope_h
//   (pos_i - pos_k) (a distance bias);  visible where pos_i - pos_k < window
//   out = softmax(s) V
// with the tree's queries and keys rotated as they are loaded, and its keys
// and values written to their slots of the pool, as tree_attn.hip does it (the
// tile: 32-key blocks through an LDS ring, a 32-row query tile per wave, fp32
// online softmax, bf16 products).  What differs:
//  - A plan kernel makes the work list once for all layers: a workgroup per
//    sequence weighs the batch's split targets, checks the pages its sequence
//    will read and writes its 64-byte work items (tree, rows, head, key
//    blocks), so the attention's workgroups start from one scalar load instead
//    of a scan over the batch.
//  - A wave copies eight rows of a block at a time and a page has at least 16
//    slots, so each wave has one page per block whatever the page size; its
//    number comes by a scalar load one block ahead and costs no wait.  Pages
//    outside the pool read as zeros (an empty buffer), never out of bounds.
//  - Long prefixes split up to 128 ways (few heads and one sequence still fill
//    the chip); half a wavefront merges a row's partials, a whole one where the
//    rows are few.
//  - Rotated queries carry the scale (it shares their one rounding to bf16), and
//    a block's products start from minus the row's reference, so they leave the
//    matrix pipe as exponents of two.  Queries that are not rotated are exact in
//    bf16 and stay as they are; their scores are scaled in fp32.
//  - The score cap, distance bias and window live in an instance of their own;
//    a window also cuts the key blocks that the plan hands out.
// Few rows are HBM bound: 32 single tokens at 8192 (32:8 heads) take 189-196 us,
// 5.5 TB/s (a plain read reaches 6.4; nothing is fetched twice); 26 nodes at
// 131000 110-116 us, 4.8.  Large trees are bound by the issue of both pipes:
// counted per wave and block, 16 products keep the matrix pipe for 512 cycles,
// 64 vector instructions and 16 exponentials the vector pipe for 450, and two
// waves a SIMD (512 registers between them, most of them the outputs and
// queries) overlap 170 of them, 960 cycles in all: eight 128-node trees at 8192
// take 160-171 us, 0.84 PFLOP/s (a large product reaches 1.34).  A score cap's
// tanh adds two transcendentals a score (950 vector cycles): 206-215 us; a
// distance bias takes 211-220, no rotation 165-169.  What is smaller is a chain
// of round trips: one token at 63 takes 7.6 us, 9.0 behind a table of more than
// 22 pages of 16, whose prefixes could be split (a workgroup for every item
// there could be, and the merge, which find nothing to do).
#include <algorithm>
#include <type_traits>

#include "attn_tile.hpp"
#include "paged.hpp"

namespace entmtp {
namespace {

constexpr int kPagedSplits = 128;
constexpr int kMaxKvHeads = 256;   // (work lists are counted in 32 bits)
constexpr float kMaxCap = 1024.f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPlanThreads = kPagedSeqs;   // a thread per sequence
constexpr int kPlanMagic = 0x50a6ed01;

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
size_t plan_topo_at(int B) { return sizeof(PlanHeader) + sizeof(PlanSeq) * B; }
size_t plan_rows_at(int B) { return plan_topo_at(B) + sizeof(int) * B; }
size_t plan_items_at(int B, int rows_cap) { return (plan_rows_at(B) + rows_cap + 63) / 64 * 64; }
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

// What the last split's part of the tree costs beyond its blocks, in prefix
// blocks: a table of fp64 angles and, for each of the ntree blocks with tree
// keys, their rotation and staging through registers (2.7 us against 0.9 at 128
// nodes).  One 128-node tree at 8192: 34.7 us, 39.7 with one block more per tree
// block, 39.2 with two fewer; four mixed trees up to 16384 79.3, 84 with two fewer.
__host__ __device__ inline int paged_tree_extra(int nb, int ntree, int ns) {
  const int extra = 2 + 3 * ntree, share = nb / ns;
  return extra < share ? extra : share;   // (the last split keeps a block)
}

// ------------------------------------------------------------------ plan --

struct PlanArgs {
  TreeTable trees;
  const int* topo;
  const int* len;
  const int* row_off;
  const int* status;
  const int* table;
  int* bad;
  uint8_t* plan;
  long long topo_at, rows_at, items_at, part_cap;
  int B, G, Hq, Hkv, shift, n_pages, max_pages, rows_cap, window, slots, items_cap, two;
};

// ceil(nb / t) as paged_splits clips it: the quotient by t's reciprocal is off
// by less than one up to 200, and past the clip beyond.
__device__ __forceinline__ int paged_splits_by(int nb, int t, float rt) {
  if (nb <= kLoneBlocks) return 1;
  const int bound = min(nb / kMinBlocksPerSplit, kPagedSplits), n = nb + t - 1;
  int q = static_cast<int>(static_cast<float>(n) * rt);
  const int r = n - q * t;
  q += r < 0 ? -1 : (r >= t ? 1 : 0);
  return q < 1 ? 1 : min(q, bound);
}

// Bound by its chain of loads, scans and barriers: one sequence takes 5.2 us, 256
// take 9.2 (each workgroup weighs the whole batch, which is cheaper than a second
// launch or a wait between workgroups).
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PlanArgs p) {
  static_assert(kPlanThreads == 256 && kTargets == 16, "four wavefronts; 16 threads to a candidate");
  __shared__ int2 s_size[kPagedSeqs];   // blocks, streams
  __shared__ long long part_work[4];
  __shared__ int part_max[4], part_items[4], part_rows[4];
  __shared__ int s_items[4][kTargets], s_split[4][kTargets];
  __shared__ PlanSeq s_seq;
  __shared__ int s_tree, s_L, s_len, s_item0, s_nb0, s_end[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int P = 1 << p.shift;
  // every sequence's size, a thread each
  int tr = -1, L = -1, r0 = -1, r1 = -1, st = -1;
  if (tid < p.B) {
    tr = p.topo[tid];
    L = p.len[tid];
    r0 = p.row_off[tid];
    r1 = p.row_off[tid + 1];
    st = p.status[tid];
  }
  const bool named = tr >= 0 && tr < p.trees.n;
  int T = named ? p.trees.t[named ? tr : 0].T : 0;
  const long long end = static_cast<long long>(r0) + T;
  if (st != ENTMTP_PAGE_OK || L < 0 || static_cast<long long>(L) + T > static_cast<long long>(p.max_pages) * P ||
      r0 < 0 || end > r1 || end > p.rows_cap)
    T = 0;
  const int first = T ? first_pos(L, p.window) / KB : 0;
  const int nb = T ? (L + T + KB - 1) / KB - first : 0;
  const int rows_pad = rows_padded(p.G, T);
  const int nqg = query_groups(rows_pad / kQTile);
  const int H = p.Hkv * nqg;
  s_size[tid] = make_int2(nb, H);
  // the split target: thread (sequence group, candidate) weighs its share
  const long long mine = static_cast<long long>(H) * nb;   // (below 2^40: summed up in two pieces of 20 bits)
  const int lo = last_lane(scan_wave(static_cast<int>(mine & 0xfffff), add));
  const int hi = last_lane(scan_wave(static_cast<int>(mine >> 20), add));
  int nb_max = last_lane(scan_wave(nb, larger));
  if (lane == 0) {
    part_work[wave] = (static_cast<long long>(hi) << 20) + lo;
    part_max[wave] = nb_max;
  }
  __syncthreads();
  const long long work = part_work[0] + part_work[1] + part_work[2] + part_work[3];
  nb_max = max(max(part_max[0], part_max[1]), max(part_max[2], part_max[3]));
  const int k = lane & 15;
  const int t = batch_target(k, work, nb_max, p.slots);
  const float rt = 1.f / static_cast<float>(t);
  int items = 0, split = 0;
#pragma unroll 4   // (their LDS reads overlap)
  for (int u = tid >> 4; u < p.B; u += 16) {
    const int2 q = s_size[u];
    const int n = paged_splits_by(q.x, t, rt);
    items += q.y * n;
    split |= q.y > 0 && n > 1;
  }
#pragma unroll
  for (int off = 16; off <= 32; off <<= 1) {
    items += __shfl_xor(items, off, 64);
    split |= __shfl_xor(split, off, 64);
  }
  if (lane < kTargets) {
    s_items[wave][lane] = items;
    s_split[wave][lane] = split;
  }
  __syncthreads();
  items = s_items[0][k] + s_items[1][k] + s_items[2][k] + s_items[3][k];
  split = s_split[0][k] | s_split[1][k] | s_split[2][k] | s_split[3][k];
  unsigned long long cost = batch_cost(k, t, items, split, p.slots);
  if (target_sixteenths(k) < 16 && !p.two) cost = ~0ull;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) {
    const unsigned long long o = __shfl_xor(cost, off, 64);
    cost = o < cost ? o : cost;
  }
  const int best = __builtin_amdgcn_readfirstlane(static_cast<int>(cost & 0xff));
  const int ns = T ? paged_splits(nb, __builtin_amdgcn_readlane(t, best)) : 1;
  // this sequence's ranges of the work list and of the partials.  (Row ranges
  // of sequences that overlap, which no page map makes, can pass the bounds:
  // the last sequences then have no work.)
  const int len = T ? (p.Hkv * ns + 7) / 8 * 8 * nqg : 0;
  const int ptiles = ns > 1 ? ns * p.Hkv * (rows_pad / kQTile) : 0;   // (four an item at most: no wrap where the items fit)
  int item_end = scan_wave(len, add), tile_end = scan_wave(ptiles, add);
  if (lane == 63) {
    part_items[wave] = item_end;
    part_rows[wave] = tile_end;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    item_end += w < wave ? part_items[w] : 0;
    tile_end += w < wave ? part_rows[w] : 0;
  }
  const long long part_end = static_cast<long long>(tile_end) * kQTile, prows = static_cast<long long>(ptiles) * kQTile;
  const bool fits = item_end <= p.items_cap && part_end <= p.part_cap;
  const int last = last_lane(scan_wave(fits ? item_end : 0, larger));
  if (lane == 0) s_end[wave] = last;
  const int b = blockIdx.x;
  if (tid == b) {
    s_seq = PlanSeq{r0, fits ? T : 0, ns, rows_pad, part_end - prows, {0, 0}};
    s_tree = named ? tr : 0;
    s_L = L;
    s_len = fits ? len : 0;
    s_item0 = item_end - len;
    s_nb0 = first;
  }
  __syncthreads();
  // the pages this sequence will read
  int bad = 0;
  const int sL = s_L;
  if (s_seq.T > 0) {
    const int* row = p.table + static_cast<size_t>(b) * p.max_pages;
    for (int e = (first_pos(sL, p.window) >> p.shift) + tid; e < (sL + P - 1) >> p.shift; e += kPlanThreads) {
      const int id = row[e];
      bad |= id < 0 || id >= p.n_pages;
    }
  }
  bad = __syncthreads_or(bad);
  const int sT = bad ? 0 : s_seq.T;
  const PagedTree& tree = p.trees.t[s_tree];
  const int sns = s_seq.nsplit, sblk = s_nb0;
  const int snb = (sL + s_seq.T + KB - 1) / KB - sblk, sqg = query_groups(s_seq.rows_pad / kQTile);
  const int extra = sT > 0 ? paged_tree_extra(snb, snb - (sL / KB - sblk), sns) : 0;
  PlanItem* const list = reinterpret_cast<PlanItem*>(p.plan + p.items_at) + s_item0;
  // where split c begins: c (snb + extra) / sns, without the product's 33 bits
  const int share = (snb + extra) / sns, rest = (snb + extra) % sns;
  auto begin = [&](int c) { return c * share + c * rest / sns; };
  // the query groups of one (head, split) at a distance of eight: workgroups
  // go to the XCDs in turn, so they share an L2
  for (int i = tid; i < s_len; i += kPlanThreads) {
    const int qg = (i >> 3) % sqg, gc = ((i >> 3) / sqg) * 8 + (i & 7);
    const int g = gc / sns, c = gc % sns;
    PlanItem it;
    it.T = gc < p.Hkv * sns ? sT : 0;
    it.L = sL;
    it.row0 = s_seq.row0;
    it.D = tree.D;
    it.off_mask = tree.off_mask;
    it.off_depth = tree.off_depth;
    it.b = b;
    it.g = g;
    it.qg = qg;
    it.split = c;
    it.nsplit = sns;
    it.blk_lo = sblk + begin(c);
    it.blk_hi = sblk + (c + 1 < sns ? begin(c + 1) : snb);
    it.rows_pad = s_seq.rows_pad;
    it.part_lo = static_cast<uint32_t>(s_seq.part_off);
    it.part_hi = static_cast<uint32_t>(s_seq.part_off >> 32);
    list[i] = it;
  }
  if (tid < sT) p.plan[p.rows_at + s_seq.row0 + tid] = static_cast<uint8_t>(b);
  static_assert(kPlanThreads >= ENTMTP_T_MAX, "one thread per tree row");
  if (tid == 0) {
    PlanSeq q = s_seq;
    q.T = sT;
    reinterpret_cast<PlanSeq*>(p.plan + sizeof(PlanHeader))[b] = q;
    reinterpret_cast<int*>(p.plan + p.topo_at)[b] = sT > 0 ? s_tree : -1;
    if (p.bad) p.bad[b] = bad != 0;
    if (b == 0) {
      PlanHeader h{};
      h.magic = kPlanMagic;
      h.B = p.B;
      h.Hq = p.Hq;
      h.Hkv = p.Hkv;
      h.shift = p.shift;
      h.n_pages = p.n_pages;
      h.max_pages = p.max_pages;
      h.rows_cap = p.rows_cap;
      h.window = p.window;
      h.items = max(max(s_end[0], s_end[1]), max(s_end[2], s_end[3]));
      h.bank_lo = static_cast<uint32_t>(p.trees.bank);
      h.bank_hi = static_cast<uint32_t>(p.trees.bank >> 32);
      *reinterpret_cast<PlanHeader*>(p.plan) = h;
    }
  }
}

// ---------------------------------------------------------------- attend --

struct PagedArgs {
  const uint8_t* plan;
  const uint8_t* arena;
  const int* table;      // [B][max_pages]
  const int* slot_map;   // [rows_cap]
  const float* slopes;   // [Hq] or NULL
  const uint16_t* q;     // [rows_cap][Hq][HD]
  const uint16_t* kt;    // [rows_cap][Hkv][HD]
  const uint16_t* vt;
  uint16_t* kp;          // [n_pages][Hkv][P][HD]
  uint16_t* vp;
  // [part rows][HD]: the split's output, normalised by its sum so that it stays
  // within its values' range, in bf16: in fp32 the whole output's error against
  // 64 bits is 3.4-3.5e-3 instead of 3.7-3.9e-3 (the weights' and the query's
  // roundings stay), and the bytes cost 3-6 % of long prefixes and windows, 15 % of 26
  // nodes at 8192 (21.5 -> 24.7 us)
  uint16_t* part_o;
  float* part_ml;        // [part rows][2]
  uint16_t* out;         // [rows_cap][Hq][HD]
  long long rows_at, items_at;
  uint64_t bank;         // the bank's number
  int B, G, Hq, Hkv, shift, n_pages, max_pages, rows_cap, window;
  float q_scale;     // scale log2(e), or with a cap 2 log2(e) scale / cap: of the rotated query, or the products
  float cap_log2;    // cap log2(e), 0: no cap
  double freq[kRopePairs];   // of the rotation's pairs
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
__device__ __forceinline__ bool plan_is_ours(const PagedArgs& p, const PlanHeader& h) {
  return ((h.magic ^ kPlanMagic) | (h.B ^ p.B) | (h.Hq ^ p.Hq) | (h.Hkv ^ p.Hkv) | (h.shift ^ p.shift) |
          (h.n_pages ^ p.n_pages) | (h.max_pages ^ p.max_pages) | (h.rows_cap ^ p.rows_cap) | (h.window ^ p.window) |
          static_cast<int>(h.bank_lo ^ static_cast<uint32_t>(p.bank)) |
          static_cast<int>(h.bank_hi ^ static_cast<uint32_t>(p.bank >> 32))) == 0;
}

// A pair of bf16 values with those that are not finite as zeros (odd is set).
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool& odd) {
  const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
  odd = odd || lo || hi;
  return w & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
}

// TURN: no rotation, one whose angles keep to the short sine's range, or one
// whose angles may pass it (wide_angles).  MOD: a score cap, distance bias or
// window.
enum Turn { kStill, kNear, kWide };
template <Turn TURN, bool MOD>
__global__ __launch_bounds__(kAttnThreads, 2) void paged_attn_kernel(PagedArgs p) {
  // one LDS object per slot, so that the compiler can tell the slot being
  // read from the slots the copies in flight write to
  __shared__ __attribute__((aligned(16))) uint8_t slot0[kRingSlot];
  __shared__ __attribute__((aligned(16))) uint8_t slot1[kRingSlot];
  __shared__ __attribute__((aligned(16))) uint8_t slot2[kRingSlot];
  __shared__ __attribute__((aligned(16))) uint8_t slot3[kRingSlot];
  __shared__ uint8_t s_depth[ENTMTP_T_MAX];
  __shared__ __attribute__((aligned(8))) uint8_t s_odd[2][KB][8];   // tree values that are not finite, by key and chunk pair
  uint8_t* const ring[4] = {slot0, slot1, slot2, slot3};
  static_assert(kRing == 4, "the ring's slots");
  const int x = static_cast<int>(blockIdx.x);
  const i32x16 head = record(p.plan), item = record(p.plan + p.items_at + static_cast<size_t>(x) * sizeof(PlanItem));
  const PlanHeader h = __builtin_bit_cast(PlanHeader, head);
  const PlanItem it = __builtin_bit_cast(PlanItem, item);
  if (!plan_is_ours(p, h) | (x >= h.items) | (it.T == 0)) return;
  const int T = it.T, L = it.L, row0 = it.row0, D = it.D, b = it.b, g = it.g, qg = it.qg;
  const int split = it.split, nsplit = it.nsplit, blk_lo = it.blk_lo, blk_hi = it.blk_hi;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 31, lh = lane >> 5;
  const int nkeys = L + T, GT = p.G * T, P = 1 << p.shift;
  const int qt = qg * kTilesPerWg + wave;        // this wave's query tile
  const bool live = qt < it.rows_pad / kQTile;   // (uniform per wave)
  const uint32_t* const mask = reinterpret_cast<const uint32_t*>(p.arena + it.off_mask);
  const int* const depth = reinterpret_cast<const int*>(p.arena + it.off_depth);
  const Const<int> pages = as_const<int>(p.table + static_cast<size_t>(b) * p.max_pages);
  const int nb = blk_hi - blk_lo;
  constexpr bool rope = TURN != kStill, WIDE = TURN == kWide;
  // what the products are: exponents of two over the row's reference (REF), bare
  // dot products still to be scaled (!rope), or, with a cap's or bias's turn to
  // come, scaled ones
  constexpr bool REF = rope && !MOD;
  // the first query group's workgroups keep the tree's keys (rotated) and
  // values in their slots of the pool for the steps after this one
  const bool keeper = qg == 0;
  // the split's first np blocks lie wholly in the prefix
  const int np = max(0, min(nb, L / KB - blk_lo));
  // positions before every row's window (their slots may be anyone's by now)
  const int w_lo = MOD ? first_pos(L, p.window) : 0;

  // Copies of prefix block i (past the last: that one again) into a slot:
  // instruction j of wave w fills rows 8 w + 4 j .. + 3 of K and of V, lane l
  // the chunk position l % 16 of row l / 16 among them.  The buffers span the
  // wave's eight rows, which lie in one page; without a prefix block, or with
  // a page outside the pool, they are empty and the copies bring zeros, so
  // that every path carries the same count.
  uint32_t koff[kRingLoads / 2], voffs[kRingLoads / 2];
#pragma unroll
  for (int j = 0; j < kRingLoads / 2; ++j) {
    const int r = 4 * j + (lane >> 4), rb = 8 * wave + r;
    koff[j] = r * 256 + (((lane & 15) ^ k_swz(rb)) << 4);
    voffs[j] = r * 256 + (((lane & 15) ^ v_swz(rb)) << 4);
  }
  static_assert(kRingLoads / 2 == 2 && kAttnThreads == 256, "eight rows a wave");
  auto pos_of = [&](int i) { return (blk_lo + min(i, max(np - 1, 0))) * KB + 8 * wave; };
  auto page_of = [&](int i) { return pages[min(pos_of(i) >> p.shift, p.max_pages - 1)]; };
  auto gload = [&](uint8_t* slot, int i, int page) {
    const int pos = pos_of(i);
    const bool there = np > 0 && static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
    const size_t off = (((static_cast<size_t>(there ? page : 0) * p.Hkv + g) << p.shift) + (pos & (P - 1))) * HD;
    const uint32_t bytes = there ? 8 * HD * 2 : 0;
    const __amdgpu_buffer_rsrc_t kbuf = dma_buffer(p.kp + off, bytes);
    const __amdgpu_buffer_rsrc_t vbuf = dma_buffer(p.vp + off, bytes);
#pragma unroll
    for (int j = 0; j < kRingLoads / 2; ++j) {
      uint8_t* const row = slot + (8 * wave + 4 * j) * 256;
      uint32_t past = 0;   // (past the buffer's end: zeros)
      if constexpr (MOD) past = pos + 4 * j + (lane >> 4) < w_lo ? 1u << 20 : 0u;
      buf_dma16(kbuf, koff[j] + past, row);
      buf_dma16(vbuf, voffs[j] + past, row + kRingK);
    }
  };

  // Blocks that hold tree keys go through registers instead: thread (row
  // tid / 8, cc = tid % 8) takes chunks cc and cc + 8 of its key and value
  // row (the two halves of pairs 8 cc .. 8 cc + 7), rotates a tree key, and
  // the keeper writes it and its value to the pool.  (In the main loop an
  // ordinary load or an LDS store would wait for every copy in flight.)
  auto tab64 = [&](int d) {   // angles at depth d, 16 depths a slot
    return reinterpret_cast<double2*>(d < 16 ? slot2 : slot3) + (d & 15) * kRopePairs;
  };
  static_assert(16 * kRopePairs * sizeof(double2) <= kRingSlot && ENTMTP_D_MAX < 32, "the angles fit in two slots");
  struct TreeRegs {
    u32x4 k0, k1, v0, v1;
    int slot;
    bool there;
  };
  const int trow = tid >> 3, tcc = tid & 7;
  auto tree_key = [&](int i) { return min((blk_lo + min(i, nb - 1)) * KB + trow, nkeys - 1); };
  // the page of a prefix key, the slot of a tree key (the keeper's)
  auto tree_find = [&](TreeRegs& t, int i) {
    const int key = tree_key(i);
    t.slot = -1;
    if (key < L)
      t.slot = p.table[static_cast<size_t>(b) * p.max_pages + (key >> p.shift)];
    else if (keeper)
      t.slot = p.slot_map[row0 + key - L];
  };
  auto tree_load = [&](TreeRegs& t, int i) {
    const int key = tree_key(i);
    const uint16_t *kp, *vp;
    t.there = true;
    if (key < L) {
      t.there = static_cast<unsigned>(t.slot) < static_cast<unsigned>(p.n_pages) && key >= w_lo;
      const size_t off = (((static_cast<size_t>(t.there ? t.slot : 0) * p.Hkv + g) << p.shift) + (key & (P - 1))) * HD;
      kp = p.kp + off;
      vp = p.vp + off;
    } else {
      const size_t own = (static_cast<size_t>(row0 + key - L) * p.Hkv + g) * HD;
      kp = p.kt + own;
      vp = p.vt + own;
    }
    kp += 8 * tcc;
    vp += 8 * tcc;
    t.k0 = *reinterpret_cast<const u32x4*>(kp);
    t.k1 = *reinterpret_cast<const u32x4*>(kp + HD / 2);
    t.v0 = *reinterpret_cast<const u32x4*>(vp);
    t.v1 = *reinterpret_cast<const u32x4*>(vp + HD / 2);
  };
  // A value that is not finite is staged as zero (a zero weight would make it a
  // NaN in every row) and noted, and the rows that see its key become NaN.
  auto tree_stage = [&](uint8_t* slot, TreeRegs& t, int i, int buf) {
    const int key = (blk_lo + i) * KB + trow;
    bool odd = false;
    if (!t.there) t.k0 = t.k1 = t.v0 = t.v1 = u32x4{0u, 0u, 0u, 0u};   // (here: the loads' first use)
    if (key >= L && key < nkeys) {
      if constexpr (rope) rope_pairs(t.k0, t.k1, tab64(s_depth[key - L]) + 8 * tcc, tcc & 7);
      if (t.slot >= 0 && t.slot < p.n_pages << p.shift) {
        const size_t off = (((static_cast<size_t>(t.slot >> p.shift) * p.Hkv + g) << p.shift) + (t.slot & (P - 1))) * HD;
        uint16_t* kd = p.kp + off + 8 * tcc;
        uint16_t* vd = p.vp + off + 8 * tcc;
        *reinterpret_cast<u32x4*>(kd) = t.k0;
        *reinterpret_cast<u32x4*>(kd + HD / 2) = t.k1;
        *reinterpret_cast<u32x4*>(vd) = t.v0;
        *reinterpret_cast<u32x4*>(vd + HD / 2) = t.v1;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      t.v0[e] = finite_pair(t.v0[e], odd);
      t.v1[e] = finite_pair(t.v1[e], odd);
    }
    s_odd[buf][trow][tcc] = odd;
    uint8_t* const row = slot + trow * 256;
    *reinterpret_cast<u32x4*>(row + ((tcc ^ k_swz(trow)) << 4)) = t.k0;
    *reinterpret_cast<u32x4*>(row + (((tcc + 8) ^ k_swz(trow)) << 4)) = t.k1;
    *reinterpret_cast<u32x4*>(row + kRingK + ((tcc ^ v_swz(trow)) << 4)) = t.v0;
    *reinterpret_cast<u32x4*>(row + kRingK + (((tcc + 8) ^ v_swz(trow)) << 4)) = t.v1;
  };

  double freq = rope ? p.freq[tid % kRopePairs] : 0.0;
  int page = page_of(0);
  const int page1 = page_of(1), page2 = page_of(2);
  TreeRegs tregs;
  if (nb > np) tree_find(tregs, np);

  // The small loads go first (this wave's Q fragments, its rows' depths and
  // masks, all unconditional: rows past the tree read row 0 and are never
  // stored): behind the key blocks they would wait for every workgroup's
  // burst.  Query row r of KV head g is (head g * G + r / T, node r % T);
  // chunks s and s + 4 hold the two halves of pairs 16s + 8lh + e.
  u32x4 qf[8];
  const int qrow = qt * kQTile + li;
  const bool qlive = qrow < GT;
  const int qnode = qlive ? qrow % T : 0;
  const int qhead = g * p.G + (qlive ? qrow / T : 0);
  {
    const uint16_t* qp = p.q + (static_cast<size_t>(row0 + qnode) * p.Hq + qhead) * HD + 8 * lh;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s);
  }
  const int qdepth = depth[qnode];
  const int tdepth = depth[min(tid, T - 1)];
  u32x4 mlo = *reinterpret_cast<const u32x4*>(mask + qnode * ENTMTP_MASK_WORDS);
  u32x4 mhi = *reinterpret_cast<const u32x4*>(mask + qnode * ENTMTP_MASK_WORDS + 4);
  static_assert(ENTMTP_MASK_WORDS == 8, "a mask row is two 16-byte loads");
  float slope = 0.f;
  if constexpr (MOD)
    if (p.slopes) slope = p.slopes[qhead] * kLog2e;
  if (nb > np) tree_load(tregs, np);
  gload(ring[0], 0, page);
  gload(ring[1], 1, page1);
  gload(ring[2], 2, page2);
  page = page_of(3);
  static_assert(kRing == 4, "three blocks ahead");
  // the angles, while the blocks arrive: the queries' fp32 table lies in the
  // last slot, free until the loop's first copies
  asm volatile("" : "+v"(freq));   // (the compiler would sink its load below the copies)
  float2* const tab32 = reinterpret_cast<float2*>(slot3);
  static_assert((ENTMTP_D_MAX + 1) * kRopePairs * sizeof(float2) <= kRingSlot, "the angles fit in a slot");
  // (times what the scores are scaled by, so that the products give logits in
  // base 2, or the cap's argument)
  const float qs = p.q_scale;
  auto tab_put = [&](int d, int pr, double2 cs) {
    tab32[d * kRopePairs + (pr ^ (2 * (d & 31)))] = make_float2(static_cast<float>(cs.x) * qs, static_cast<float>(cs.y) * qs);
  };
  if constexpr (rope) rope_table<WIDE>(tid, D, L, freq, tab_put);
  s_depth[tid] = static_cast<uint8_t>(tdepth);
  static_assert(kAttnThreads >= ENTMTP_T_MAX, "one thread per node");
  wait_lds();
  stage_barrier();
  if (!qlive) mlo = mhi = u32x4{~0u, ~0u, ~0u, ~0u};   // padding rows see every key
  if constexpr (rope) {
    const float2* tr = tab32 + qdepth * kRopePairs;
#pragma unroll
    for (int s = 0; s < 4; ++s) rope_pairs_f32(qf[s], qf[s + 4], tr, 16 * s + 8 * lh, 2 * (qdepth & 31));
  }
  const int qpos = L + qdepth;
  const int w_row = MOD && p.window > 0 ? qpos - p.window + 1 : -1;   // the row's first position
  const int w_hi = MOD && p.window > 0 ? L + D - p.window + 1 : -1;   // from here on every row sees the prefix

  // l_run: the sum of this lane's half of the keys (the halves meet at the end)
  float m_run = -INFINITY, l_run = 0.f;
  // REF: a block's products start from minus the row's
  // reference (zero before its first), so that they come out as the exponents
  // themselves; lift: how far a block's largest may pass the reference.
  f32x16 ref;
#pragma unroll
  for (int r = 0; r < 16; ++r) ref[r] = 0.f;
  float lift = -INFINITY;
  f32x16 o[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ct][r] = 0.f;

  // fragment addresses within a slot: K row li, chunk 2 s + lh; the
  // transposing reads of V: row 4 lh + (lane % 16) / 4 of each 8 rows, dims
  // 32 ct + 16 (li / 16) + 4 (lane % 4)
  const int kx = lh ^ k_swz(li);
  const int vrow = 4 * lh + ((lane & 15) >> 2);
  const int vx = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swz(vrow);
  const int voff = kRingK + vrow * 256 + 8 * (lane & 1);

  // S^T = K Q^T of the block in a slot
  auto scores = [&](const uint8_t* slot, f32x16& sacc) {
    if constexpr (REF) {
      sacc = ref;
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(slot + li * 256 + ((kx ^ (2 * s)) << 4));
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf), as_bf16x8(qf[s]), sacc, 0, 0, 0);
    }
  };
  // MOD: the block's products as logits in base 2, key r at distance dist(r).
  // tanh(u) = 1 - 2 / (e^2u + 1) with 2 u / ln 2 from the products: 0 and
  // infinity of the exponential give -1 and 1.
  auto bend = [&](f32x16& sacc, auto dist) {
    if constexpr (!rope) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] *= qs;
    }
    if (p.cap_log2 > 0.f) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        sacc[r] = fmaf(-2.f * p.cap_log2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(sacc[r]) + 1.f), p.cap_log2);
    }
    if (p.slopes) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = fmaf(-slope, static_cast<float>(dist(r)), sacc[r]);
    }
  };
  auto key_of = [&](int r) { return 8 * (r >> 2) + 4 * lh + (r & 3); };   // accumulator r's key of the block
  // the keys noted in buffer buf, a bit each
  auto odd_keys = [&](int buf) {
    const uint2 f = *reinterpret_cast<const uint2*>(s_odd[buf][li]);
    return static_cast<uint32_t>(__ballot((f.x | f.y) != 0u));
  };
  // Keeps the scores of the keys in vis (a bit each), -inf elsewhere; a row
  // that sees a key in odd becomes NaN.
  auto keep = [&](f32x16& sacc, float& l, uint32_t vis, uint32_t odd) {
    if ((vis & odd) != 0u) l = NAN;
    vis >>= 4 * lh;   // bit 8 (r / 4) + r % 4 is accumulator r's key
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int m = static_cast<int>(vis << (31 - (8 * (r >> 2) + (r & 3)))) >> 31;
      sacc[r] = __builtin_bit_cast(float, (m & __builtin_bit_cast(int, static_cast<float>(sacc[r]))) | (~m & INT32_C(-0x800000)));
    }
  };
  // Block i's softmax (lazily raised max) and O^T += V^T P^T from its slot;
  // prefix: every key of the block is in the prefix; ahead: the next block's
  // scores, which move with the reference they started from.
  auto attend = [&](int i, const uint8_t* slot, f32x16& sacc, f32x16& ahead, auto prefix) {
    float bmax = -INFINITY;
    const int kb = (blk_lo + i) * KB;
    if constexpr (decltype(prefix)::value) {
      if constexpr (MOD) {
        bend(sacc, [&](int r) { return qpos - (kb + key_of(r)); });
        if (kb < w_hi) {
          const int out = min(max(w_row - kb, 0), KB);   // keys before the row's window
          keep(sacc, l_run, static_cast<uint32_t>(0xFFFFFFFFull << out), odd_keys(i & 1));
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) bmax = fmaxf(bmax, sacc[r]);
    } else {
      uint32_t vis;
      const int rel = kb - L;
      auto word = [&](int w) {   // (w is uniform)
        uint32_t m = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = w == k ? (k < 4 ? mlo[k & 3] : mhi[k & 3]) : m;
        return m;
      };
      if (rel < 0) {
        const int npre = -rel;
        vis = (0xFFFFFFFFu >> (32 - npre)) | (mlo[0] << npre);
      } else {
        const int wi = rel >> 5, sh = rel & 31;
        const uint32_t lo = word(wi), hi = word(wi + 1);
        vis = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
      }
      if (nkeys - kb < KB) vis &= (1u << (nkeys - kb)) - 1u;
      if constexpr (MOD) {
        // (a tree key's position is that of its depth)
        auto pos_k = [&](int n) {
          const int j = kb + n - L;
          return j < 0 ? kb + n : L + s_depth[min(j, ENTMTP_T_MAX - 1)];
        };
        bend(sacc, [&](int r) { return qpos - pos_k(key_of(r)); });
        if (min(kb, L) < w_hi) {   // (else the window holds the block)
          for (int n = 0; n < KB; ++n)
            if (pos_k(n) < w_row) vis &= ~(1u << n);
        }
      }
      keep(sacc, l_run, vis, odd_keys((i - np) & 1));
#pragma unroll
      for (int r = 0; r < 16; ++r) bmax = fmaxf(bmax, sacc[r]);
    }
    bmax = max_halves(bmax);
    constexpr bool bare = !rope && !MOD;
    if constexpr (bare) bmax *= qs;
    // REF's are relative to m_run, the others are held against it here
    const bool need = REF ? bmax > lift : bmax > m_run + kLazyLog2;
    if (__any(need)) {
      const float mn = !need ? m_run : (!REF || m_run == -INFINITY ? bmax : m_run + bmax);
      const float alpha = !need ? 1.f : (m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - mn));
      l_run *= alpha;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[ct][r] *= alpha;
      m_run = mn;
      if constexpr (REF) {
        const float by = need ? bmax : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sacc[r] -= by;
          ahead[r] -= by;
          ref[r] -= by;
        }
        lift = need ? kLazyLog2 : lift;
      }
    }
    const float mneg = REF || m_run == -INFINITY ? 0.f : -m_run;
    float pr[16];
    float rsum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pr[r] = __builtin_amdgcn_exp2f(REF ? sacc[r] : (bare ? fmaf(sacc[r], qs, mneg) : sacc[r] + mneg));
      rsum += pr[r];
    }
    l_run += rsum;
    bf16x8 pf[2];   // (weights up to 2^8 in bf16, as the products take them: each off by at most 2^-8)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                               (f32x2{pr[8 * u + 2 * e], pr[8 * u + 2 * e + 1]}), bf16x2));
      pf[u] = as_bf16x8(w);
    }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const uint8_t* vp = slot + voff + ((vx ^ (4 * ct)) << 4);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint2 x0 = lds_read_tr(vp + 16 * u * 256);
        const uint2 x1 = lds_read_tr(vp + (16 * u + 8) * 256);
        const u32x4 w = {x0.x, x0.y, x1.x, x1.y};
        o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w), pf[u], o[ct], 0, 0, 0);
      }
    }
  };

  // The prefix's blocks.  Step i takes the scores of block i + 1 ahead of
  // block i's softmax, so that a wave has products to issue beside its
  // exponentials; blocks i + 2 and i + 3 are in flight, the latter's copies
  // going into the slot block i - 1 left, behind the barrier every wave
  // reaches after its products.  Copies past the last block fetch it again,
  // so the count in flight is always the same.
  f32x16 sa, sb;
  wait_vmcnt<(kRing - 2) * kRingLoads>();
  if constexpr (MOD) {
    // At the window's edge some rows of a tile see a prefix key and others do
    // not.  Values there that are not finite are taken as zeros (a zero weight
    // would make them NaNs) and noted, and the rows that see them become NaN.
    // A tree's positions differ by less than a block, so the edge lies in the
    // split's first two blocks; each wave's rows are those that it copied.
    static_assert(ENTMTP_D_MAX < KB, "the edge lies in two blocks");
    if (blk_lo * KB < w_hi) {
      wait_vmcnt<(kRing - 3) * kRingLoads>();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bool odd = false;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32x4* const at = reinterpret_cast<u32x4*>(ring[k] + kRingK + trow * 256 + (((tcc + 8 * c) ^ v_swz(trow)) << 4));
          u32x4 v = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = finite_pair(v[e], odd);
          *at = v;
        }
        s_odd[k][trow][tcc] = odd;
      }
      wait_lds();
    }
  }
  stage_barrier();
  if (live) scores(ring[0], sa);
  int i0 = 0;
  for (; i0 + kRing <= np; i0 += kRing) {
#pragma unroll
    for (int k = 0; k < kRing; ++k) {
      wait_vmcnt<(kRing - 3) * kRingLoads>();
      stage_barrier();
      gload(ring[(k + kRing - 1) % kRing], i0 + k + kRing - 1, page);
      page = page_of(i0 + k + kRing);
      if (live) {
        f32x16& cur = k & 1 ? sb : sa;
        scores(ring[(k + 1) % kRing], k & 1 ? sa : sb);
        attend(i0 + k, ring[k], cur, k & 1 ? sa : sb, std::true_type{});
      }
    }
  }
  // the last np % kRing blocks are in flight (a loop left from within its
  // round would make the compiler add full waits)
  wait_vmcnt<0>();
  stage_barrier();
  if (live) {
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k)
      if (i0 + k < np) {
        f32x16& cur = k & 1 ? sb : sa;
        if (k + 1 < kRing - 1) scores(ring[k + 1], k & 1 ? sa : sb);
        attend(i0 + k, ring[k], cur, k & 1 ? sa : sb, std::true_type{});
      }
  }

  // the blocks that hold tree keys: staged into two of the slots in turn, the
  // next block's loads ahead of this one's products, the keys' fp64 angles in
  // the other two
  if (nb > np) {
    __syncthreads();
    if constexpr (rope) {
      rope_table<WIDE>(tid, D, L, freq, [&](int d, int pr, double2 cs) { tab64(d)[pr ^ ((pr >> 3) & 7)] = cs; });
      __syncthreads();
    }
    for (int i = np; i < nb; ++i) {
      const int buf = (i - np) & 1;
      uint8_t* const slot = buf ? slot1 : slot0;
      tree_stage(slot, tregs, i, buf);
      if (i + 1 < nb) {   // (in flight during this block's products: the barrier waits for the LDS alone)
        tree_find(tregs, i + 1);
        tree_load(tregs, i + 1);
      }
      wait_lds();
      stage_barrier();
      if (live) {
        scores(slot, sa);
        attend(i, slot, sa, sb, std::false_type{});
      }
    }
  }

  // this wave's tile: the output (one split) or its partial.  Lane (query li,
  // half lh) holds dims 32 ct + 8 j + 4 lh + i in o[ct][4 j + i]; the halves
  // trade a chunk so that each stores 16 bytes: lane 0..31 dims 8 j .. 8 j + 7
  // of even j, lane 32..63 of odd j.
  if (!live) return;
  l_run += __shfl_xor(l_run, 32, 64);
  const int row = qt * kQTile + li;
  uint16_t* dst;
  if (nsplit == 1) {
    const int r = row < GT ? row : 0;
    dst = p.out + (static_cast<size_t>(row0 + r % T) * p.Hq + g * p.G + r / T) * HD;
  } else {
    const long long part = static_cast<long long>((static_cast<unsigned long long>(it.part_hi) << 32) | it.part_lo);
    const size_t prow = part + (static_cast<size_t>(split) * p.Hkv + g) * it.rows_pad + row;
    dst = p.part_o + prow * HD;
    if (lh == 0 && row < GT) {
      p.part_ml[prow * 2 + 0] = m_run;
      p.part_ml[prow * 2 + 1] = l_run;
    }
  }
  // (a split may hold no key that the row sees: zeros; a whole row sees its own)
  const float il = l_run == 0.f && nsplit > 1 ? 0.f : 1.f / l_run;
  auto pack = [&](float u, float v) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{u * il, v * il}), bf16x2));
  };
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const f32x16& a = o[ct];
      const auto u = __builtin_amdgcn_permlane32_swap(pack(a[4 * j], a[4 * j + 1]),
                                                      pack(a[4 * j + 4], a[4 * j + 5]), false, false);
      const auto v = __builtin_amdgcn_permlane32_swap(pack(a[4 * j + 2], a[4 * j + 3]),
                                                      pack(a[4 * j + 6], a[4 * j + 7]), false, false);
      if (row < GT) *reinterpret_cast<u32x4*>(dst + 32 * ct + 8 * (j + lh)) = u32x4{u[0], v[0], u[1], v[1]};
    }
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

template <int LANES>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedArgs p) {
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
  const uint16_t* const po = p.part_o + base * HD + 4 * (lane & 31);
  float m[kPairs], l[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) {
    m[k] = -INFINITY;
    l[k] = 0.f;
    if (lane + LANES * k < nsplit) {
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (base + (lane + LANES * k) * stride) * 2);
      m[k] = ml.x;
      l[k] = ml.y;
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
        const uint2 v = c + first + k < nsplit ? ob[k] : uint2{0u, 0u};   // (the last one again may hold infinities)
        acc.x = fmaf(wc, __uint_as_float(v.x << 16), acc.x);
        acc.y = fmaf(wc, __uint_as_float(v.x & 0xffff0000u), acc.y);
        acc.z = fmaf(wc, __uint_as_float(v.y << 16), acc.z);
        acc.w = fmaf(wc, __uint_as_float(v.y & 0xffff0000u), acc.w);
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

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

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
  size_t plan_bytes = 0, workspace = 0;
};

PagedShape paged_shape(const entmtp_bank* bank, int B, int rows_cap, int Hq, int Hkv, long long cap) {
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

bool shape_ok(const entmtp_bank* bank, int B, int rows_cap, int Hq, int Hkv, int max_pages, int page_size) {
  return bank && !bank->desc.empty() && paged_batch(B) && rows_cap >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 &&
         Hq / Hkv <= 32 && Hkv <= kMaxKvHeads && page_shift(page_size) >= 0 && max_pages >= 1 &&
         static_cast<int64_t>(max_pages) * page_size <= INT32_MAX - 1024;
}

int32_t check_batch(int32_t B, int32_t rows_cap, int32_t Hq, int32_t Hkv, int32_t max_pages, int32_t page_size,
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

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" size_t entmtp_tree_attn_paged_plan_bytes(const entmtp_bank* bank, int32_t B, int32_t rows_cap,
                                                    int32_t Hq, int32_t Hkv, int32_t max_pages,
                                                    int32_t page_size) {
  if (!shape_ok(bank, B, rows_cap, Hq, Hkv, max_pages, page_size)) return 0;
  return paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size).plan_bytes;
}

extern "C" size_t entmtp_tree_attn_paged_workspace(const entmtp_bank* bank, int32_t B, int32_t rows_cap, int32_t Hq,
                                                   int32_t Hkv, int32_t d, int32_t max_pages, int32_t page_size) {
  if (!shape_ok(bank, B, rows_cap, Hq, Hkv, max_pages, page_size) || d != HD) return 0;
  return paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size).workspace;
}

extern "C" const int32_t* entmtp_tree_attn_paged_topo(const void* plan, int32_t B) {
  if (!plan || !paged_batch(B)) return nullptr;
  return reinterpret_cast<const int32_t*>(static_cast<const uint8_t*>(plan) + plan_topo_at(B));
}

extern "C" int32_t entmtp_tree_attn_paged_plan(const entmtp_bank* bank, int32_t B, const int32_t* topo,
                                               const int32_t* prefix_len, const int32_t* row_off,
                                               const int32_t* status, const int32_t* block_table, int32_t max_pages,
                                               int32_t page_size, int32_t n_pages, int32_t rows_cap, int32_t Hq,
                                               int32_t Hkv, int32_t window, int32_t* bad, void* plan,
                                               size_t plan_bytes, void* stream) {
  clear_error();
  if (int32_t rc = check_batch(B, rows_cap, Hq, Hkv, max_pages, page_size, n_pages, window)) return rc;
  ENTMTP_CHECK_ARG(topo && prefix_len && row_off && status && block_table && plan, ENTMTP_EINVAL,
                   "topo, prefix_len, row_off, status, block_table and plan must be non-NULL device arrays");
  ENTMTP_CHECK_ARG((reinterpret_cast<uintptr_t>(plan) & 63u) == 0, ENTMTP_EINVAL, "the plan must be 64-byte aligned");
  PlanArgs a{};
  if (int32_t rc = tree_table(bank, &a.trees)) return rc;
  const PagedShape sh = paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size);
  ENTMTP_CHECK_ARG(sh.items < INT32_MAX / 64, ENTMTP_ERANGE, "%d rows of %d heads: too many", rows_cap, Hq);
  ENTMTP_CHECK_ARG(plan_bytes >= sh.plan_bytes, ENTMTP_ENOSPC, "the plan has %zu bytes, needs %zu", plan_bytes,
                   sh.plan_bytes);
  ENTMTP_CHECK_ARG(reinterpret_cast<uintptr_t>(topo) - reinterpret_cast<uintptr_t>(plan) >= sh.plan_bytes, ENTMTP_EINVAL,
                   "topo must not lie in the plan that is made from it");
  a.topo = topo;
  a.len = prefix_len;
  a.row_off = row_off;
  a.status = status;
  a.table = block_table;
  a.bad = bad;
  a.plan = static_cast<uint8_t*>(plan);
  a.topo_at = static_cast<long long>(plan_topo_at(B));
  a.rows_at = static_cast<long long>(plan_rows_at(B));
  a.items_at = static_cast<long long>(plan_items_at(B, rows_cap));
  a.part_cap = sh.part_rows;
  a.B = B;
  a.G = Hq / Hkv;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.shift = page_shift(page_size);
  a.n_pages = n_pages;
  a.max_pages = max_pages;
  a.rows_cap = rows_cap;
  a.window = window;
  a.slots = device_cus() * kWgPerCu;
  a.items_cap = sh.items;
  a.two = sh.two;
  hipLaunchKernelGGL(paged_plan_kernel, dim3(B), dim3(kPlanThreads), 0, static_cast<hipStream_t>(stream), a);
  return launch_status("tree_attn_paged_plan launch");
}

extern "C" int32_t entmtp_tree_attn_paged(const entmtp_bank* bank, int32_t B, const void* plan, size_t plan_bytes,
                                          const entmtp_bf16* q, const entmtp_bf16* k_tree, const entmtp_bf16* v_tree,
                                          entmtp_bf16* k_pool, entmtp_bf16* v_pool, int32_t n_pages,
                                          int32_t page_size, const int32_t* block_table, int32_t max_pages,
                                          const int32_t* slot_map, int32_t rows_cap, int32_t Hq, int32_t Hkv,
                                          int32_t d, float scale, float rope_theta, float softcap, int32_t window,
                                          const float* slopes, entmtp_bf16* out, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  clear_error();
  if (int32_t rc = check_batch(B, rows_cap, Hq, Hkv, max_pages, page_size, n_pages, window)) return rc;
  ENTMTP_CHECK_ARG(plan && q && k_tree && v_tree && k_pool && v_pool && block_table && slot_map && out, ENTMTP_EINVAL,
                   "plan, tensors, block_table and slot_map must be non-NULL");
  ENTMTP_CHECK_ARG(d == HD, ENTMTP_EINVAL, "head dim %d unsupported (built for %d)", d, HD);
  ENTMTP_CHECK_ARG(scale > 0.f && scale < INFINITY, ENTMTP_EINVAL, "scale must be positive");
  ENTMTP_CHECK_ARG(rope_theta >= 0.f && rope_theta < INFINITY, ENTMTP_EINVAL, "rope_theta must be >= 0");
  // (1 - 2 / (e^2u + 1) is off by about 2^-22, the cap times that.  The query
  // carries scale / softcap: past 2^64 ordinary ones would come near bf16's
  // and the products' largest numbers, and infinities of both signs are no tanh.)
  ENTMTP_CHECK_ARG(softcap >= 0.f && softcap <= kMaxCap && (softcap == 0.f || scale / softcap <= 0x1p64f),
                   ENTMTP_EINVAL, "softcap = %g must be 0 or in (0, %g], scale / softcap at most 2^64",
                   static_cast<double>(softcap), static_cast<double>(kMaxCap));
  ENTMTP_CHECK_ARG((reinterpret_cast<uintptr_t>(plan) & 63u) == 0, ENTMTP_EINVAL, "the plan must be 64-byte aligned");
  ENTMTP_CHECK_ARG(aligned16(q) && aligned16(k_tree) && aligned16(v_tree) && aligned16(k_pool) && aligned16(v_pool) &&
                       aligned16(out) && aligned16(workspace),
                   ENTMTP_EINVAL, "tensors, pools and workspace must be 16-byte aligned");
  TreeTable trees;
  if (int32_t rc = tree_table(bank, &trees)) return rc;
  const PagedShape sh = paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size);
  ENTMTP_CHECK_ARG(sh.items < INT32_MAX / 64, ENTMTP_ERANGE, "%d rows of %d heads: too many", rows_cap, Hq);
  ENTMTP_CHECK_ARG(plan_bytes >= sh.plan_bytes, ENTMTP_ENOSPC, "the plan has %zu bytes, needs %zu", plan_bytes,
                   sh.plan_bytes);
  ENTMTP_CHECK_ARG(sh.workspace == 0 || (workspace && workspace_bytes >= sh.workspace), ENTMTP_ENOSPC,
                   "workspace has %zu bytes, needs %zu", workspace ? workspace_bytes : size_t(0), sh.workspace);
  PagedArgs a{};
  a.plan = static_cast<const uint8_t*>(plan);
  a.arena = trees.arena;
  a.bank = trees.bank;
  a.table = block_table;
  a.slot_map = slot_map;
  a.slopes = slopes;
  a.q = q;
  a.kt = k_tree;
  a.vt = v_tree;
  a.kp = k_pool;
  a.vp = v_pool;
  a.part_o = static_cast<uint16_t*>(workspace);
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
  a.q_scale = softcap > 0.f ? 2.f * kLog2e * (scale / softcap) : scale * kLog2e;
  a.cap_log2 = softcap * kLog2e;
  const double theta = static_cast<double>(rope_theta);
  rope_freqs(rope_theta, a.freq);
  // a wavefront a head where they are few, so that long prefixes' many splits
  // take half the round trips: 26 rows of 32 heads at 8192 21.4 us (attention and
  // merge) against 23.9 by half wavefronts, 8 rows of 8 heads at 32000 18.3
  // against 26.4; 4096 heads are level, 32768 take 10 us more by whole ones
  const bool few = static_cast<long long>(rows_cap) * Hq <= 4LL * device_cus();
  const int heads = kMergeThreads / (few ? 64 : 32);
  const long long blocks = static_cast<long long>(rows_cap) * ((Hq + heads - 1) / heads);
  ENTMTP_CHECK_ARG(blocks <= INT32_MAX, ENTMTP_ERANGE, "%d rows of %d heads: too many", rows_cap, Hq);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(sh.items), dim3(kAttnThreads), 0, s, a); };
  const bool mod = softcap > 0.f || window > 0 || slopes != nullptr;
  if (theta == 0.0)
    mod ? go(paged_attn_kernel<kStill, true>) : go(paged_attn_kernel<kStill, false>);
  else if (wide_angles(theta))
    mod ? go(paged_attn_kernel<kWide, true>) : go(paged_attn_kernel<kWide, false>);
  else
    mod ? go(paged_attn_kernel<kNear, true>) : go(paged_attn_kernel<kNear, false>);
  if (int32_t rc = launch_status("tree_attn_paged launch")) return rc;
  if (!sh.splits) return ENTMTP_OK;
  auto merge = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kMergeThreads), 0, s, a);
  };
  few ? merge(paged_merge_kernel<64>) : merge(paged_merge_kernel<32>);
  return launch_status("tree_attn_paged merge launch");
}
