// Tree attention over a page pool whose keys and values are held in 4 bits
// (their form is described in fp4.hpp), for batches of up to 256 sequences.
//
//   s = scale q . k;  s = cap tanh(s / cap) (a score cap);  s = s - slope_h
//   (pos_i - pos_k) (a distance bias);  visible where pos_i - pos_k < window
//   out = softmax(s) V
// over the prefix and the root-to-node path of every tree node.  The queries
// come as they enter the products and the tree's rows lie in the pool already,
// so that a key block of the tree differs from one of the prefix by its mask
// alone.  The work list is that of paged_attn.hip: a workgroup takes a KV head's
// query rows (four tiles of 32) and a range of 32-key blocks.
//  - Keys enter the matrix instruction (32 x 32 x 64, 4-bit by 8-bit: bf16's rate)
//    as they lie in the pool, codes and scale bytes.  A query is the sum of two 8-bit
//    numbers, the second what the first leaves at a scale 2^4 below, under a scale of
//    its group of 32: together they hold bf16's eight bits of every value down to
//    2^-13 of the group's largest, exactly, and of smaller ones all but 2^-21 of that
//    largest, so that a channel which stands out costs the others nothing.  Scores
//    are scaled in fp32.  (Three 6-bit numbers, which share their steps with the
//    group's largest, run at twice the rate, three times over, and took 2-4 % less in
//    large trees; beside a channel 64 times the others' size they were off by more
//    than a rounding to bf16, beside one 1000 times by a third of their values.)
//  - Values become bf16 numbers, exactly, on their way to the LDS, from which the
//    products read them transposed.
//  - Many rows (three or four tiles): the workgroup's wavefronts, a tile each,
//    share the blocks, which come as codes by direct copies three ahead; every
//    wavefront turns a quarter of a block's values into numbers, a block ahead,
//    and takes the next block's scores before this one's softmax.
//  - Few rows: a wavefront streams its blocks by itself, from memory to registers,
//    two ahead, and no barrier joins it to the others: the range is shared by four
//    (two tiles: two), every fourth block each, which meet in the LDS at the end --
//    a few rows' blocks are a chain of products, softmax and products that one
//    wavefront could not walk at memory's rate.
//  - At most 16 rows: the same on 16 columns of queries, half of the products.
// The splits' partial outputs are fp16 with a scale a row; another kernel joins them.
//
// What bounds it (replayed graphs, 32:8 heads): one token at 63 takes 5.3 us, launch
// and one chain of loads and products.  32 tokens at 8192 take 60 us, 5 of them the
// merge: 4.8 TB/s of a plain read's 6.4.  26 nodes at 131000 take 88 us, the merge
// 7: the products (0.63 PFLOP/s; the keys' twice, once for each part of the query),
// in four tiles of which a head group fills 3.25.  Eight 128-node trees at 8192 take
// 154 us (0.90 PFLOP/s; 201 with a score cap): for a block a wavefront keeps the
// matrix pipe for 513 cycles and issues 611 cycles of vector instructions, of which
// 206 run beside each other; it waits 516 of its 2173 cycles, and two wavefronts
// share a SIMD.  Over pages of bf16 rows the four take 7.6, 189-196, 110-113 and
// 160-171 us.  The instance with cap, bias and window does not fit its 256 registers
// (nine are spilled; of the loops over blocks the one beside a window's edge and the
// tree reloads one).
#include <algorithm>
#include <type_traits>

#include "fp4.hpp"
#include "paged_plan.hpp"

namespace entmtp {
namespace {

constexpr int kFp4Ahead = 2;               // blocks in flight per wavefront (few rows)
constexpr int kFp4Ring = 4;                // blocks in the LDS (many rows)
constexpr int kFp4Stage = KB * HD * 2;     // bytes of a block's values in bf16

// A block's rows as they lie in the pool: wavefront w's copies are the keys' (w = 0,
// 1) or the values' (2, 3) 16 rows, codes and scale bytes (16 dwords, then zeros).
struct Fp4Block {
  uint8_t k[KB * HD / 2], v[KB * HD / 2];
  uint32_t s[kAttnThreads / 64][64];
};

struct PagedFp4Args : PagedCall {
  const uint8_t* arena;
  const int* table;      // [B][max_pages]
  const float* slopes;   // [Hq] or NULL
  const uint16_t* q;     // [rows_cap][Hq][HD]
  const uint8_t* kp;     // [n_pages][Hkv][P x 68]
  const uint8_t* vp;
  float q_scale;     // of the products, in fp32: scale log2(e), or with a cap 2 log2(e) scale / cap
  float cap_log2;    // cap log2(e), 0: no cap
};

// Chunk c (16 bytes) of row r of the staged values lies at c ^ stage_swz(r): a
// store takes one chunk of 16 rows, every other one of two, or every fourth of
// four, a transposing read 64 bytes of four rows or 32 of eight; all then cover all
// banks.  (Eight rows on: chunk ^ 1, sixteen: the same.)  Of the keys' codes chunk
// c of row r lies at c ^ (r / 4 % 4).
__device__ __forceinline__ int stage_swz(int r) {
  return 4 * (r & 3) + ((((r >> 3) & 1) | ((r >> 1) & 2)) ^ (r & 3));
}

// The largest of a lane's value and those of the lanes 16, 32 and 48 away.
__device__ __forceinline__ float max_quarters(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// 16 or 4 bytes at byte voff of the buffer (zeros past its end).
__device__ __forceinline__ u32x4 buf_load16(__amdgpu_buffer_rsrc_t buf, uint32_t voff) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, static_cast<int>(voff), 0, 0));
}
__device__ __forceinline__ uint32_t buf_load4(__amdgpu_buffer_rsrc_t buf, uint32_t voff) {
  return __builtin_bit_cast(uint32_t, buf_load(buf, voff));
}

// The larger of a lane's number and that of the lane 32 (16) away.
__device__ __forceinline__ uint32_t top_halves(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(r[0], r[1]);
}
__device__ __forceinline__ uint32_t top_sixteenths(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return max(r[0], r[1]);
}

// A lane's 32 values of a query as the sum of two 8-bit operands of the matrix
// instruction (a sign, 4 bits of exponent, 3 of mantissa), the second at a scale 2^4
// below the first's.
struct Query8 {
  i32x8 part[2];
};

// Scale byte of a group of 32 whose largest magnitude has the bf16 bits top: the
// largest comes to lie in [224, 448) steps; not a number where a value is not finite.
__device__ __forceinline__ uint32_t query_scale(uint32_t top) {
  const int e = static_cast<int>((top + 0x20u) >> 7);   // (the carry is that of a mantissa of 1.75 or more)
  return top >= 0x7f80u ? kFp4NaN : static_cast<uint32_t>(max(e, 12) - 8);
}
__device__ __forceinline__ uint32_t second_scale(uint32_t b) { return b == kFp4NaN ? b : b - 4u; }

// Bytes 16 h .. + 15 of both parts from 16 values (v: their bf16 pairs) of a group
// with scale byte b.
__device__ __forceinline__ void query8(const u32x4 (&v)[2], uint32_t b, int h, Query8& q) {
  const float inv = __uint_as_float((254u - (b == kFp4NaN ? 127u : b)) << 23);
#pragma unroll
  for (int w = 0; w < 4; ++w) {   // (four values to a word)
    float hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t u = v[w >> 1][2 * (w & 1) + (k >> 1)];
      const float x = (k & 1 ? bf16_hi(u) : bf16_lo(u)) * inv;
      // to the smallest steps of the format, then to four bits of mantissa: a number of it
      const float r = (x + 24576.f) - 24576.f;   // 1.5 x 2^23 x 2^-9
      hi[k] = __uint_as_float((__float_as_uint(r) + 0x80000u) & 0xfff00000u);
      lo[k] = (x - hi[k]) * 16.f;
    }
    auto pack = [](const float (&f)[4]) {
      return __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false), true);
    };
    q.part[0][4 * h + w] = pack(hi);
    q.part[1][4 * h + w] = pack(lo);
  }
}

// MOD: a score cap, distance bias or window.
template <bool MOD>
__global__ __launch_bounds__(kAttnThreads, 2) void paged_attn_fp4_kernel(PagedFp4Args p) {
  // (one LDS object per slot, so that the compiler can tell the one being read
  // from those that copies in flight write to)
  __shared__ __attribute__((aligned(16))) Fp4Block raw0;
  __shared__ __attribute__((aligned(16))) Fp4Block raw1;
  __shared__ __attribute__((aligned(16))) Fp4Block raw2;
  __shared__ __attribute__((aligned(16))) Fp4Block raw3;
  __shared__ __attribute__((aligned(16))) uint8_t s_val[kTilesPerWg][kFp4Stage];   // (many rows: two in turn)
  __shared__ float2 s_ml[kTilesPerWg][KB];
  __shared__ uint32_t s_odd[4];   // a block's keys with values that are no numbers, a bit each
  __shared__ uint32_t s_mask[kTilesPerWg][KB][ENTMTP_MASK_WORDS + 1];   // the rows' ancestors, a wavefront's own
  __shared__ uint8_t s_depth[ENTMTP_T_MAX];
  Fp4Block* const ring[kFp4Ring] = {&raw0, &raw1, &raw2, &raw3};
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
  // this workgroup's tiles, the wavefronts that share one, this one's place among them
  const int nt = min(it.rows_pad / kQTile - qg * kTilesPerWg, kTilesPerWg);
  const int ways = nt == 1 ? 4 : (nt == 2 ? 2 : 1);
  const int tile = nt >= 3 ? wave : wave % nt, way = nt >= 3 ? 0 : wave / nt;
  const bool live = tile < nt;   // (uniform per wave)
  const int qt = qg * kTilesPerWg + tile;
  const uint32_t* const mask = reinterpret_cast<const uint32_t*>(p.arena + it.off_mask);
  const int* const depth = reinterpret_cast<const int*>(p.arena + it.off_depth);
  const Const<int> pages = as_const<int>(p.table + static_cast<size_t>(b) * p.max_pages);
  // positions before every row's window (their slots may be anyone's by now)
  const int w_lo = MOD ? first_pos(L, p.window) : 0;
  auto page_at = [&](int pos) { return pages[min(pos >> p.shift, p.max_pages - 1)]; };
  auto head_at = [&](int page) { return (static_cast<size_t>(page) * p.Hkv + g) * static_cast<size_t>(P * kFp4RowBytes); };

  // The query row (row r of KV head g: head g G + r / T, node r % T), its depth
  // and mask, all unconditional: rows past the tree read row 0, see every key
  // and are never stored.  Matrix instruction m of a block takes keys' dims 64 m +
  // 32 lh .. + 31 and queries' 64 m + 16 lh .. + 15 and 64 m + 32 + 16 lh .. + 15
  // (small: the only one 32 lq .. + 31, and 16 lq .. + 15 and 64 + 16 lq .. + 15),
  // and a scale byte of dims 64 m + 32 lh .. + 31 (32 lq .. + 31) of either.
  const bool small = GT <= 16;   // (16 columns of queries: lane % 16, groups of 32 dims: lane / 16)
  const int lc = lane & 15, lq = lane >> 4;
  const int qrow = qt * kQTile + (small ? lc : li);
  const bool qlive = live && qrow < GT;
  const int qnode = qlive ? qrow % T : 0;
  const int qhead = g * p.G + (qlive ? qrow / T : 0);
  u32x4 qf[2][2][2];   // [m][16 values][chunk]
  {
    const uint16_t* qp = p.q + (static_cast<size_t>(row0 + qnode) * p.Hq + qhead) * HD + 16 * (small ? lq : lh);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        qf[m][e >> 1][e & 1] = *reinterpret_cast<const u32x4*>(qp + (small ? 0 : 64 * m) + (small ? 64 : 32) * (e >> 1) + 8 * (e & 1));
  }
  const int qdepth = depth[qnode];
  const int tdepth = depth[min(tid, T - 1)];
  const u32x4 qmask = *reinterpret_cast<const u32x4*>(mask + qnode * ENTMTP_MASK_WORDS + 4 * lh);
  static_assert(ENTMTP_MASK_WORDS == 8, "a mask row is two 16-byte loads");
  float slope = 0.f;
  if constexpr (MOD)
    if (p.slopes) slope = p.slopes[qhead] * kLog2e;

  // l_run: the sum of this lane's half of the keys (the halves meet at the end)
  float m_run = -INFINITY, l_run = 0.f;
  const float to_log2 = MOD ? 1.f : p.q_scale;   // from a block's scores to logits in base 2 (MOD: bend's work)
  const int qpos = L + qdepth;
  const int w_row = MOD && p.window > 0 ? qpos - p.window + 1 : -1;   // the row's first position
  const int w_hi = MOD && p.window > 0 ? L + D - p.window + 1 : -1;   // from here on every row sees the prefix
  auto keep_mask = [&]() __attribute__((always_inline)) {   // (read by the wavefront that writes it)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_mask[wave][small ? lc : li][4 * lh + e] = qlive ? qmask[e] : ~0u;
  };
  // The keys of the block at kb, which reaches into the tree or past it, that the
  // row sees, a bit each.
  auto seen = [&](int kb) __attribute__((always_inline)) {
    const int rel = kb - L;
    const uint32_t* const row = s_mask[wave][small ? lc : li];
    auto word = [&](int w) { return w < ENTMTP_MASK_WORDS ? row[w] : 0u; };   // (w is uniform)
    uint32_t vis = ~0u;
    if (rel + KB > 0) {
      if (rel < 0) {
        const int npre = -rel;
        vis = (0xFFFFFFFFu >> (32 - npre)) | (word(0) << npre);
      } else {
        const int wi = rel >> 5, sh = rel & 31;
        const uint32_t lo = word(wi), hi = word(wi + 1);
        vis = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
      }
    }
    if (nkeys - kb < KB) vis &= (1u << (nkeys - kb)) - 1u;
    return vis;
  };
  // The row's place in the output (one split), or among the partials; of the
  // latter's (max, sum) one lane of the row stores them.
  auto out_row = [&]() __attribute__((always_inline)) {
    const int r = qrow < GT ? qrow : 0;
    return p.out + (static_cast<size_t>(row0 + r % T) * p.Hq + g * p.G + r / T) * HD;
  };
  // (top: the largest magnitude of the row's normalised output; by: what brings it
  // to [2^14, 2^15), where the smaller ones keep fp16's eleven bits)
  auto part_row = [&](float top, float& by) __attribute__((always_inline)) {
    const int e = max(static_cast<int>(__float_as_uint(top) >> 23), 15);
    by = e == 255 ? 1.f : __uint_as_float(static_cast<uint32_t>(268 - e) << 23);
    const float undo = e == 255 ? 1.f : __uint_as_float(static_cast<uint32_t>(e - 14) << 23);
    const long long part = static_cast<long long>((static_cast<unsigned long long>(it.part_hi) << 32) | it.part_lo);
    const size_t prow = part + (static_cast<size_t>(split) * p.Hkv + g) * it.rows_pad + qrow;
    if ((small ? lq : lh) == 0 && qrow < GT) *reinterpret_cast<float4*>(p.part_ml + prow * 4) = make_float4(m_run, l_run, undo, 0.f);
    return static_cast<uint16_t*>(p.part_o) + prow * HD;
  };
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  auto halves = [](float a, float b) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
  };

  if (small) {
    // At most 16 rows: as the few below, with 16 columns of queries (16 x 16 x 128 for
    // the scores of 16 keys, 16 x 16 x 32 for the outputs' 16 dims), half of the
    // products and of the softmax, and copies of whole runs of 16 rows.
    const int nb = max(0, (blk_hi - blk_lo - wave + 3) / 4);
    auto key_at = [&](int i) { return (blk_lo + wave + max(min(i, nb - 1), 0) * 4) * KB; };
    struct Block {
      u32x4 k[2], v[2];
      uint32_t ks[2], vs[2];
    };
    struct Pages {
      int lo, hi;
    };
    auto pages_of = [&](int i) { return Pages{page_at(key_at(i)), page_at(key_at(i) + 16)}; };
    constexpr uint32_t kPast = 1u << 30;   // (past the buffer's end: zeros)
    // (run j of 16 keys; a key's codes by lane (key lc, group lq), a value's by lane
    // (row lane / 4, group lane % 4))
    auto load = [&](Block& s, int i, Pages pg) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int pos = key_at(i) + 16 * j, in = pos & (P - 1), page = j ? pg.hi : pg.lo;
        const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
        const size_t at = head_at(there ? page : 0);
        const __amdgpu_buffer_rsrc_t kb = dma_buffer(p.kp + at, there ? P * kFp4RowBytes : 0);
        const __amdgpu_buffer_rsrc_t vb = dma_buffer(p.vp + at, there ? P * kFp4RowBytes : 0);
        const uint32_t kpast = MOD && pos + lc < w_lo ? kPast : 0, vpast = MOD && pos + (lane >> 2) < w_lo ? kPast : 0;
        s.k[j] = buf_load16(kb, kpast + (in + lc) * (HD / 2) + 16 * lq);
        s.ks[j] = buf_load4(kb, kpast + P * (HD / 2) + 4 * (in + lc));
        s.v[j] = buf_load16(vb, vpast + in * (HD / 2) + 16 * lane);
        s.vs[j] = buf_load4(vb, vpast + P * (HD / 2) + 4 * (in + (lane >> 2)));
      }
    };
    constexpr int kAhead = 2;
    Block blk[kAhead];
    Pages pg[kAhead + 1];
#pragma unroll
    for (int k = 0; k <= kAhead; ++k) pg[k] = pages_of(k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load(blk[k], k, pg[k]);
    Pages next = pg[kAhead];
    s_depth[tid] = static_cast<uint8_t>(tdepth);
    if (MOD) {
      wait_lds();
      stage_barrier();
    }
    keep_mask();
    Query8 qs;
    uint32_t qscale;   // scale bytes of the first part and the second
    {
      const uint32_t b0 = query_scale(top_sixteenths(max(bf16_top(qf[0][0][0]), bf16_top(qf[0][0][1]))));   // dims 32 (lq / 2) .. + 31
      const uint32_t b1 = query_scale(top_sixteenths(max(bf16_top(qf[0][1][0]), bf16_top(qf[0][1][1]))));   // 64 on
      query8(qf[0][0], b0, 0, qs);
      query8(qf[0][1], b1, 1, qs);
      const uint32_t other = static_cast<uint32_t>(__shfl_xor(static_cast<int>(lq < 2 ? b1 : b0), 48, 64));
      const uint32_t mine = lq == 0 ? b0 : (lq == 3 ? b1 : other);   // dims 32 lq .. + 31
      qscale = mine | second_scale(mine) << 8;
    }
    f32x4 out[8];
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) out[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint8_t* const stage = s_val[wave];
    const int wrow = lane >> 2, wsw = stage_swz(wrow);   // (row 16 on: the same)
    const int rrow = 4 * lq + (lc >> 2), rsw = stage_swz(rrow);
    uint8_t* const put = stage + wrow * 256;
    const uint8_t* const get = stage + rrow * 256 + 8 * (lane & 1);
    auto step = [&](Block& s, int i) __attribute__((always_inline)) {
      const int kb = key_at(i);
      f32x4 sc[2];
      uint32_t odd = 0u;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const i32x8 ka = {static_cast<int>(s.k[j][0]), static_cast<int>(s.k[j][1]), static_cast<int>(s.k[j][2]), static_cast<int>(s.k[j][3]), 0, 0, 0, 0};
        const int kscale = static_cast<int>(s.ks[j] >> (8 * lq));
        sc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, qs.part[1], sc[j], 4, 0, 0, kscale, 1, static_cast<int>(qscale));
        sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, qs.part[0], sc[j], 4, 0, 0, kscale, 0, static_cast<int>(qscale));
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t b = s.vs[j] >> (8 * (lane & 3)) & 0xffu;
        const unsigned long long bad = __ballot(b > kFp4Top);
        if (bad != 0ull) {   // (uniform) rows' groups as nibbles, a bit a row
          if (b > kFp4Top) s.v[j] = u32x4{0u, 0u, 0u, 0u};
          unsigned long long m = bad | bad >> 1;
          m |= m >> 2;
#pragma unroll
          for (int r = 0; r < 16; ++r) odd |= static_cast<uint32_t>(m >> (4 * r) & 1ull) << (16 * j + r);
        }
        const float st = fp4_step(b > kFp4Top ? 127u : b);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<u32x4*>(put + 16 * j * 256 + (((4 * (lane & 3) + c) ^ wsw) << 4)) = fp4_values(s.v[j][c], st);
      }
      auto key_of = [&](int j, int r) { return 16 * j + 4 * lq + r; };
      auto bend16 = [&](auto dist) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            sc[j][r] *= p.q_scale;
            if (p.cap_log2 > 0.f)
              sc[j][r] = fmaf(-2.f * p.cap_log2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(sc[j][r]) + 1.f), p.cap_log2);
            if (p.slopes) sc[j][r] = fmaf(-slope, static_cast<float>(dist(key_of(j, r))), sc[j][r]);
          }
      };
      uint32_t vis = ~0u;
      if (kb + KB <= L && !(MOD && kb < w_hi)) {   // (uniform)
        if constexpr (MOD) bend16([&](int n) { return qpos - (kb + n); });
      } else {
        vis = seen(kb);
        if constexpr (MOD) {
          auto pos_k = [&](int n) {
            const int j = kb + n - L;
            return j < 0 ? kb + n : L + s_depth[min(j, ENTMTP_T_MAX - 1)];
          };
          bend16([&](int n) { return qpos - pos_k(n); });
          if (min(kb, L) < w_hi) {
            for (int n = 0; n < KB; ++n)
              if (pos_k(n) < w_row) vis &= ~(1u << n);
          }
        }
        const uint32_t mine = vis >> (4 * lq);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((mine >> (16 * j + r) & 1u) == 0u) sc[j][r] = -INFINITY;
      }
      if (odd != 0u) {   // (uniform)
        if ((vis & odd) != 0u) l_run = NAN;
      }
      float bmax = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                         fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      bmax = max_quarters(bmax) * to_log2;
      const bool need = bmax > m_run + kLazyLog2;
      if (__any(need)) {
        const float mn = need ? bmax : m_run;
        const float alpha = !need ? 1.f : (m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - mn));
        l_run *= alpha;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) out[ct] *= alpha;
        m_run = mn;
      }
      const float mneg = m_run == -INFINITY ? 0.f : -m_run;
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          e[r] = __builtin_amdgcn_exp2f(MOD ? sc[j][r] + mneg : fmaf(sc[j][r], to_log2, mneg));
          l_run += e[r];
        }
        w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{e[0], e[1]}), bf16x2));
        w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{e[2], e[3]}), bf16x2));
      }
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const uint8_t* const at = get + (((2 * ct + ((lane & 3) >> 1)) ^ rsw) << 4);
        const uint2 x0 = lds_read_tr(at), x1 = lds_read_tr(at + 16 * 256);
        out[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4{x0.x, x0.y, x1.x, x1.y}), as_bf16x8(w), out[ct], 0, 0, 0);
      }
    };
    // (whole rounds without a branch, so that a wait for a block leaves the later
    // ones in flight; the last blocks have been asked for by then)
    int i0 = 0;
    for (; i0 + kAhead <= nb; i0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        step(blk[k], i0 + k);
        load(blk[k], i0 + k + kAhead, next);
        next = pages_of(i0 + k + kAhead + 1);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead - 1; ++k)
      if (i0 + k < nb) step(blk[k], i0 + k);
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    // the four wavefronts' sums meet
    for (int half = 2; half >= 1; half >>= 1) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
        f32x4* const at = reinterpret_cast<f32x4*>(s_val[wave - half]);
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) at[ct * 64 + lane] = out[ct];
        if (lq == 0) s_ml[wave - half][lc] = make_float2(m_run, l_run);
      }
      __syncthreads();
      if (wave < half) {
        const f32x4* const at = reinterpret_cast<const f32x4*>(s_val[wave]);
        const float2 ml = s_ml[wave][lc];
        const float mn = fmaxf(m_run, ml.x);
        // (no key seen: max -inf, nothing to add; a NaN of the sum stays)
        const float a0 = m_run == mn ? 1.f : __builtin_amdgcn_exp2f(m_run - mn);
        const float a1 = ml.x == mn ? 1.f : __builtin_amdgcn_exp2f(ml.x - mn);
        m_run = mn;
        l_run = l_run * a0 + ml.y * a1;
#pragma unroll
        for (int ct = 0; ct < 8; ++ct) {
          const f32x4 v = at[ct * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) out[ct][e] = out[ct][e] * a0 + v[e] * a1;
        }
      }
    }
    if (wave > 0) return;
    if (nsplit > 1) {
      // (a split may hold no key that the row sees: zeros)
      const float il = l_run == 0.f ? 0.f : 1.f / l_run;
      float top = 0.f, by;
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          out[ct][e] *= il;
          top = fmaxf(top, fabsf(out[ct][e]));
        }
      uint16_t* const dst = part_row(max_quarters(top), by);
      if (qrow < GT) {
#pragma unroll
        for (int ct = 0; ct < 8; ++ct)
          *reinterpret_cast<uint2*>(dst + 16 * ct + 4 * lq) =
              uint2{halves(out[ct][0] * by, out[ct][1] * by), halves(out[ct][2] * by, out[ct][3] * by)};
      }
      return;
    }
    const float il = 1.f / l_run;   // (a whole row sees its own key)
    uint16_t* const dst = out_row();
    if (qrow < GT) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        const uint2 v = {__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{out[ct][0] * il, out[ct][1] * il}), bf16x2)),
                         __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{out[ct][2] * il, out[ct][3] * il}), bf16x2))};
        *reinterpret_cast<uint2*>(dst + 16 * ct + 4 * lq) = v;
      }
    }
    return;
  }

  f32x16 o[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ct][r] = 0.f;
  Query8 qs[2];
  uint32_t qsc = 0u;   // scale bytes of the first part for m = 0, 1, and the second's
  auto settle = [&]() __attribute__((always_inline)) {   // (behind the loads of the first blocks)
    keep_mask();
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t b[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        b[k] = query_scale(top_halves(max(bf16_top(qf[m][k][0]), bf16_top(qf[m][k][1]))));
        query8(qf[m][k], b[k], k, qs[m]);
      }
      const uint32_t mine = lh ? b[1] : b[0];
      qsc |= (mine | second_scale(mine) << 16) << (8 * m);
    }
  };

  // the transposing reads of the values: row 4 lh + (lane % 16) / 4 of each 8
  // rows, dims 32 ct + 16 (li / 16) + 4 (lane % 4)
  const int vrow = 4 * lh + ((lane & 15) >> 2);
  const int vx = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ stage_swz(vrow);   // (rows 8 on: chunk ^ 1)
  const int voff = vrow * 256 + 8 * (lane & 1);

  // S^T = K Q^T of a block: row li's codes of dims 64 m + 32 lh .. + 31 and its scale bytes
  auto scores = [&](const u32x4& k0, const u32x4& k1, uint32_t ks, f32x16& sacc) __attribute__((always_inline)) {
    const i32x8 ka = {static_cast<int>(k0[0]), static_cast<int>(k0[1]), static_cast<int>(k0[2]), static_cast<int>(k0[3]), 0, 0, 0, 0};
    const i32x8 kc = {static_cast<int>(k1[0]), static_cast<int>(k1[1]), static_cast<int>(k1[2]), static_cast<int>(k1[3]), 0, 0, 0, 0};
    const int kscale = static_cast<int>(lh ? ks >> 8 : ks), qscale = static_cast<int>(qsc);
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qs[0].part[1], sacc, 4, 0, 0, kscale, 2, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kc, qs[1].part[1], sacc, 4, 0, 2, kscale, 3, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qs[0].part[0], sacc, 4, 0, 0, kscale, 0, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kc, qs[1].part[0], sacc, 4, 0, 2, kscale, 1, qscale);
  };
  auto key_of = [&](int r) { return 8 * (r >> 2) + 4 * lh + (r & 3); };   // accumulator r's key of the block
  // MOD: the block's products as logits in base 2, key r at
  // distance dist(r).  tanh(u) = 1 - 2 / (e^2u + 1) with 2 u / ln 2 from the
  // products: 0 and infinity of the exponential give -1 and 1.
  auto bend = [&](f32x16& sacc, auto dist) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] *= p.q_scale;
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
  // The softmax of the block at key kb (lazily raised maximum) and O^T += V^T P^T
  // from its staged values; odd: its keys whose values are no numbers; prefix: the
  // caller knows that every row sees every key.
  auto attend = [&](int kb, const uint8_t* stage, uint32_t odd, f32x16& sacc, auto prefix) __attribute__((always_inline)) {
    uint32_t vis = ~0u;
    if (decltype(prefix)::value || (kb + KB <= L && !(MOD && kb < w_hi))) {   // (uniform)
      if constexpr (MOD) bend(sacc, [&](int r) { return qpos - (kb + key_of(r)); });
    } else {
      vis = seen(kb);
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
      const uint32_t mine = vis >> (4 * lh);   // bit 8 (r / 4) + r % 4 is accumulator r's key
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = static_cast<int>(mine << (31 - (8 * (r >> 2) + (r & 3)))) >> 31;
        sacc[r] = __builtin_bit_cast(float, (m & __builtin_bit_cast(int, static_cast<float>(sacc[r]))) | (~m & INT32_C(-0x800000)));
      }
    }
    if (odd != 0u) {   // (uniform)
      if ((vis & odd) != 0u) l_run = NAN;
    }
    float bmax = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) bmax = fmaxf(bmax, sacc[r]);
    bmax = max_halves(bmax) * to_log2;
    const bool need = bmax > m_run + kLazyLog2;
    if (__any(need)) {
      const float mn = need ? bmax : m_run;
      const float alpha = !need ? 1.f : (m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - mn));
      l_run *= alpha;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[ct][r] *= alpha;
      m_run = mn;
    }
    const float mneg = m_run == -INFINITY ? 0.f : -m_run;
    float pr[16];
    float rsum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pr[r] = __builtin_amdgcn_exp2f(MOD ? sacc[r] + mneg : fmaf(sacc[r], to_log2, mneg));
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
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint2 x0 = lds_read_tr(stage + voff + 16 * u * 256 + ((vx ^ (4 * ct)) << 4));
        const uint2 x1 = lds_read_tr(stage + voff + (16 * u + 8) * 256 + ((vx ^ (4 * ct) ^ 1) << 4));
        const u32x4 w = {x0.x, x0.y, x1.x, x1.y};
        o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w), pf[u], o[ct], 0, 0, 0);
      }
  };

  if (nt >= 3) {
    // Many rows.  Round i waits for the codes of block i + 1, turns its values into
    // numbers and takes its scores, then attends to block i; copies of block i + 4
    // take block i's place, which no one reads behind the barrier.
    const int nb = blk_hi - blk_lo;
    const int np = max(0, min(nb, L / KB - blk_lo));   // blocks wholly in the prefix
    const int n0 = MOD ? min(np, max(0, (w_hi + KB - 1) / KB - blk_lo)) : 0;   // of these, at the window's edge
    auto pos_of = [&](int i) { return (blk_lo + min(i, nb - 1)) * KB + 16 * (wave & 1); };   // of this wavefront's copies
    const int crow = lane >> 2, cchunk = wave < 2 ? (lane & 3) ^ ((crow >> 2) & 3) : lane & 3;
    auto copy = [&](Fp4Block* to, int i, int page) __attribute__((always_inline)) {
      const int pos = pos_of(i), in = pos & (P - 1);
      const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
      const __amdgpu_buffer_rsrc_t buf =
          dma_buffer((wave < 2 ? p.kp : p.vp) + head_at(there ? page : 0), there ? P * kFp4RowBytes : 0);
      constexpr uint32_t kPast = 1u << 30;   // (past the buffer's end: zeros)
      const uint32_t codes = MOD && pos + crow < w_lo ? kPast : (in + crow) * (HD / 2) + 16 * cchunk;
      const uint32_t bytes = lane >= 16 || (MOD && pos + lane < w_lo) ? kPast : P * (HD / 2) + 4 * (in + lane);
      buf_dma16(buf, codes, (wave < 2 ? to->k : to->v) + 1024 * (wave & 1));
      buf_dma4(buf, bytes, to->s[wave]);
    };
    constexpr int kCopies = 2;
    // thread (row tid / 8, eighth tid % 8 of it) turns 16 values into numbers;
    // groups that are no numbers, or hold infinities as bf16 numbers, into zeros (a
    // zero weight would make them NaNs in every row), and their keys are noted
    const int trow = tid >> 3, tsw = stage_swz(trow);
    auto turn = [&](const Fp4Block* from, uint8_t* stage, int i) __attribute__((always_inline)) {
      const uint2 c = *reinterpret_cast<const uint2*>(from->v + 8 * tid);
      const uint32_t sb = from->s[2 + (trow >> 4)][trow & 15] >> (8 * ((tid & 7) >> 1)) & 0xffu;
      const bool none = sb > kFp4Top;
      const unsigned long long bad = __ballot(none);
      if (bad != 0ull) {
        if (none) atomicOr(&s_odd[i & 3], 1u << trow);
      }
      const float step = none ? 0.f : fp4_step(sb);
      const u32x4 lo = fp4_values(none ? 0u : c.x, step), hi = fp4_values(none ? 0u : c.y, step);
      uint8_t* const row = stage + trow * 256;
      *reinterpret_cast<u32x4*>(row + (((2 * (tid & 7)) ^ tsw) << 4)) = lo;
      *reinterpret_cast<u32x4*>(row + (((2 * (tid & 7) + 1) ^ tsw) << 4)) = hi;
    };
    auto score = [&](const Fp4Block* from, f32x16& sacc) __attribute__((always_inline)) {
      const int sw = (li >> 2) & 3;
      const u32x4 k0 = *reinterpret_cast<const u32x4*>(from->k + li * (HD / 2) + ((lh ^ sw) << 4));
      const u32x4 k1 = *reinterpret_cast<const u32x4*>(from->k + li * (HD / 2) + (((2 + lh) ^ sw) << 4));
      scores(k0, k1, from->s[li >> 4][li & 15], sacc);
    };
    int page[kFp4Ring];
#pragma unroll
    for (int k = 0; k < kFp4Ring; ++k) page[k] = page_at(pos_of(k));
#pragma unroll
    for (int k = 0; k < kFp4Ring; ++k) copy(ring[k], k, page[k]);
    int next = page_at(pos_of(kFp4Ring));
    if (tid < 4) s_odd[tid] = 0u;
    s_depth[tid] = static_cast<uint8_t>(tdepth);
    static_assert(kAttnThreads >= ENTMTP_T_MAX, "one thread per node");
    settle();
    f32x16 sa, sb;
    wait_vmcnt<(kFp4Ring - 1) * kCopies>();
    stage_barrier();
    turn(ring[0], s_val[0], 0);
    if (live) score(ring[0], sa);
    // (the odd keys' words: block i's is read in round i, cleared in the next and
    // written again two rounds later)
    auto round = [&](int i, auto kc, auto prefix) __attribute__((always_inline)) {
      constexpr int k = decltype(kc)::value;
      stage_barrier();
      copy(ring[k], i + kFp4Ring, next);
      next = page_at(pos_of(i + kFp4Ring + 1));
      if (tid == 0) s_odd[(k + 3) & 3] = 0u;
      if (live) {
        f32x16& cur = k & 1 ? sb : sa;
        f32x16& ahead = k & 1 ? sa : sb;
        score(ring[(k + 1) % kFp4Ring], ahead);
        const uint32_t odd = __builtin_amdgcn_readfirstlane(s_odd[k]);
        attend((blk_lo + i) * KB, s_val[k & 1], odd, cur, prefix);
      }
      turn(ring[(k + 1) % kFp4Ring], s_val[(k + 1) & 1], k + 1);
    };
    int i0 = 0;
    if (n0 == 0)
      for (; i0 + kFp4Ring <= np; i0 += kFp4Ring) {
        wait_vmcnt<(kFp4Ring - 2) * kCopies>();
        round(i0, std::integral_constant<int, 0>{}, std::true_type{});
        wait_vmcnt<(kFp4Ring - 2) * kCopies>();
        round(i0 + 1, std::integral_constant<int, 1>{}, std::true_type{});
        wait_vmcnt<(kFp4Ring - 2) * kCopies>();
        round(i0 + 2, std::integral_constant<int, 2>{}, std::true_type{});
        wait_vmcnt<(kFp4Ring - 2) * kCopies>();
        round(i0 + 3, std::integral_constant<int, 3>{}, std::true_type{});
      }
    for (; i0 < nb; i0 += kFp4Ring) {
      wait_vmcnt<(kFp4Ring - 2) * kCopies>();
      round(i0, std::integral_constant<int, 0>{}, std::false_type{});
      if (i0 + 1 >= nb) break;
      wait_vmcnt<(kFp4Ring - 2) * kCopies>();
      round(i0 + 1, std::integral_constant<int, 1>{}, std::false_type{});
      if (i0 + 2 >= nb) break;
      wait_vmcnt<(kFp4Ring - 2) * kCopies>();
      round(i0 + 2, std::integral_constant<int, 2>{}, std::false_type{});
      if (i0 + 3 >= nb) break;
      wait_vmcnt<(kFp4Ring - 2) * kCopies>();
      round(i0 + 3, std::integral_constant<int, 3>{}, std::false_type{});
    }
    wait_vmcnt<0>();   // (copies of blocks past the last)
  } else {
    // Few rows: this wavefront's blocks, number i at blk_lo + way + i ways (past the
    // last the last one again); a block's two runs of 16 keys lie in a page each.
    const int nb = max(0, (blk_hi - blk_lo - way + ways - 1) / ways);
    auto key_at = [&](int i) { return (blk_lo + way + max(min(i, nb - 1), 0) * ways) * KB; };
    struct Block {
      u32x4 k0, k1, v0, v1;
      uint32_t ks, vs;
      bool there;   // this lane's page lies in the pool
    };
    struct Pages {
      int lo, hi;
    };
    auto pages_of = [&](int i) { return Pages{page_at(key_at(i)), page_at(key_at(i) + 16)}; };
    auto load = [&](Block& s, int i, Pages pg) {
      const int key = key_at(i) + li;
      const int page = li < 16 ? pg.lo : pg.hi;
      s.there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
      if (MOD && key < w_lo) s.there = false;
      const size_t base = head_at(s.there ? page : 0);
      const int in = key & (P - 1);
      const uint8_t *kr = p.kp + base, *vr = p.vp + base;
      // key codes of dims 64 m + 32 lh .. + 31, value codes of dims 64 lh .. + 63
      s.k0 = *reinterpret_cast<const u32x4*>(kr + in * (HD / 2) + 16 * lh);
      s.k1 = *reinterpret_cast<const u32x4*>(kr + in * (HD / 2) + 16 * lh + 32);
      s.ks = *reinterpret_cast<const uint32_t*>(kr + P * (HD / 2) + in * 4);
      s.v0 = *reinterpret_cast<const u32x4*>(vr + in * (HD / 2) + 32 * lh);
      s.v1 = *reinterpret_cast<const u32x4*>(vr + in * (HD / 2) + 32 * lh + 16);
      s.vs = *reinterpret_cast<const uint32_t*>(vr + P * (HD / 2) + in * 4);
    };
    Block blk[kFp4Ahead];
    Pages pg[kFp4Ahead + 1];
#pragma unroll
    for (int k = 0; k <= kFp4Ahead; ++k) pg[k] = pages_of(k);
#pragma unroll
    for (int k = 0; k < kFp4Ahead; ++k) load(blk[k], k, pg[k]);
    Pages next = pg[kFp4Ahead];
    s_depth[tid] = static_cast<uint8_t>(tdepth);
    if (MOD) {
      wait_lds();
      stage_barrier();
    }
    settle();
    uint8_t* const stage = s_val[wave];
    uint8_t* const srow = stage + li * 256;
    const int sx = stage_swz(li);
    auto step = [&](Block& s, int i) __attribute__((always_inline)) {
      uint32_t ks = s.ks, vs = s.vs;
      if (!__all(s.there)) {   // (a page outside the pool: zeros)
        if (!s.there) {
          s.k0 = s.k1 = s.v0 = s.v1 = u32x4{0u, 0u, 0u, 0u};
          ks = vs = 0x7f7f7f7fu;
        }
      }
      f32x16 sacc;
      scores(s.k0, s.k1, ks, sacc);
      // the values to the LDS; groups that are no numbers as zeros (a zero weight
      // would make them NaNs in every row) and their keys noted
      const uint32_t v2 = lh ? vs >> 16 : vs;   // groups 2 lh and 2 lh + 1
      const uint32_t va = v2 & 0xffu, vb = v2 >> 8 & 0xffu;
      const unsigned long long bad = __ballot(va > kFp4Top || vb > kFp4Top);
      const uint32_t odd = static_cast<uint32_t>(bad) | static_cast<uint32_t>(bad >> 32);
      if (odd != 0u) {   // (uniform)
        if (va > kFp4Top) s.v0 = u32x4{0u, 0u, 0u, 0u};
        if (vb > kFp4Top) s.v1 = u32x4{0u, 0u, 0u, 0u};
      }
      const float sa = fp4_step(va > kFp4Top ? 127u : va), sb = fp4_step(vb > kFp4Top ? 127u : vb);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t w = c < 4 ? s.v0[c & 3] : s.v1[c & 3];
        *reinterpret_cast<u32x4*>(srow + (((8 * lh + c) ^ sx) << 4)) = fp4_values(w, c < 4 ? sa : sb);
      }
      attend(key_at(i), stage, odd, sacc, std::false_type{});
    };
    for (int i = 0; i < nb; i += kFp4Ahead) {
#pragma unroll
      for (int k = 0; k < kFp4Ahead; ++k) {
        if (i + k < nb) {   // (uniform)
          step(blk[k], i + k);
          load(blk[k], i + k + kFp4Ahead, next);
          next = pages_of(i + k + kFp4Ahead + 1);
        }
      }
    }
  }

  // wavefronts that share a tile: each hands its sums to one of a lower place,
  // halving their number
  l_run += __shfl_xor(l_run, 32, 64);
  for (int half = ways >> 1; half >= 1; half >>= 1) {
    __syncthreads();
    const int slot = tile + nt * (way % half);   // (below four: half * nt <= 2)
    if (way >= half && way < 2 * half) {
      f32x4* const at = reinterpret_cast<f32x4*>(s_val[2 * slot]);   // (16 KB: two stages)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          at[(4 * ct + j) * 64 + lane] = f32x4{o[ct][4 * j], o[ct][4 * j + 1], o[ct][4 * j + 2], o[ct][4 * j + 3]};
      if (lh == 0) s_ml[slot][li] = make_float2(m_run, l_run);
    }
    __syncthreads();
    if (way < half) {
      const f32x4* const at = reinterpret_cast<const f32x4*>(s_val[2 * slot]);
      const float2 ml = s_ml[slot][li];
      const float mn = fmaxf(m_run, ml.x);
      // (no key seen: max -inf, nothing to add; a NaN of the sum stays)
      const float a0 = m_run == mn ? 1.f : __builtin_amdgcn_exp2f(m_run - mn);
      const float a1 = ml.x == mn ? 1.f : __builtin_amdgcn_exp2f(ml.x - mn);
      m_run = mn;
      l_run = l_run * a0 + ml.y * a1;
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 v = at[(4 * ct + j) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[ct][4 * j + e] = o[ct][4 * j + e] * a0 + v[e] * a1;
        }
    }
  }
  if (!live || way > 0) return;

  // this wave's tile: the output (one split) or its partial.  Lane (query li,
  // half lh) holds dims 32 ct + 8 j + 4 lh + i in o[ct][4 j + i].
  // The halves trade a chunk so that each stores 16 bytes: lane 0..31 dims 8 j ..
  // 8 j + 7 of even j, lane 32..63 of odd j.
  // (a split may hold no key that the row sees: zeros; a whole row sees its own)
  const float il = l_run == 0.f && nsplit > 1 ? 0.f : 1.f / l_run;
  uint16_t* dst;
  float by = 1.f;
  const bool whole = nsplit == 1;   // (uniform)
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ct][r] *= il;
  if (whole) {
    dst = out_row();
  } else {
    float top = 0.f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(o[ct][r]));
    dst = part_row(max_halves(top), by);
  }
  auto pack = [&](float u, float v) {
    return whole ? __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{u, v}), bf16x2)) : halves(u * by, v * by);
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
      if (qrow < GT) *reinterpret_cast<u32x4*>(dst + 32 * ct + 8 * (j + lh)) = u32x4{u[0], v[0], u[1], v[1]};
    }
}

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" size_t entmtp_tree_attn_paged_fp4_plan_bytes(const entmtp_bank* bank, int32_t B, int32_t rows_cap,
                                                        int32_t Hq, int32_t Hkv, int32_t max_pages,
                                                        int32_t page_size) {
  return entmtp_tree_attn_paged_plan_bytes(bank, B, rows_cap, Hq, Hkv, max_pages, page_size);
}

extern "C" size_t entmtp_tree_attn_paged_fp4_workspace(const entmtp_bank* bank, int32_t B, int32_t rows_cap,
                                                       int32_t Hq, int32_t Hkv, int32_t d, int32_t max_pages,
                                                       int32_t page_size) {
  if (!shape_ok(bank, B, rows_cap, Hq, Hkv, max_pages, page_size) || d != HD) return 0;
  return fp4_workspace(paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size));
}

extern "C" int32_t entmtp_tree_attn_paged_fp4_plan(const entmtp_bank* bank, int32_t B, const int32_t* topo,
                                                   const int32_t* prefix_len, const int32_t* row_off,
                                                   const int32_t* status, const int32_t* block_table,
                                                   int32_t max_pages, int32_t page_size, int32_t n_pages,
                                                   int32_t rows_cap, int32_t Hq, int32_t Hkv, int32_t window,
                                                   int32_t* bad, void* plan, size_t plan_bytes, void* stream) {
  return launch_paged_plan(true, bank, B, topo, prefix_len, row_off, status, block_table, max_pages, page_size,
                           n_pages, rows_cap, Hq, Hkv, window, bad, plan, plan_bytes, stream);
}

extern "C" int32_t entmtp_tree_attn_paged_fp4(const entmtp_bank* bank, int32_t B, const void* plan, size_t plan_bytes,
                                              const entmtp_bf16* q, const uint8_t* k_pool, const uint8_t* v_pool,
                                              int32_t n_pages, int32_t page_size, const int32_t* block_table,
                                              int32_t max_pages, int32_t rows_cap, int32_t Hq, int32_t Hkv, int32_t d,
                                              float scale, float softcap, int32_t window, const float* slopes,
                                              entmtp_bf16* out, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  if (int32_t rc = check_batch(B, rows_cap, Hq, Hkv, max_pages, page_size, n_pages, window)) return rc;
  ENTMTP_CHECK_ARG(plan && q && k_pool && v_pool && block_table && out, ENTMTP_EINVAL,
                   "plan, tensors and block_table must be non-NULL");
  ENTMTP_CHECK_ARG(d == HD, ENTMTP_EINVAL, "head dim %d unsupported (built for %d)", d, HD);
  ENTMTP_CHECK_ARG(scale > 0.f && scale < INFINITY, ENTMTP_EINVAL, "scale must be positive");
  // (as for bf16 pools: 1 - 2 / (e^2u + 1) is off by about 2^-22, the cap times that)
  ENTMTP_CHECK_ARG(softcap >= 0.f && softcap <= kMaxCap && (softcap == 0.f || scale / softcap <= 0x1p64f),
                   ENTMTP_EINVAL, "softcap = %g must be 0 or in (0, %g], scale / softcap at most 2^64",
                   static_cast<double>(softcap), static_cast<double>(kMaxCap));
  ENTMTP_CHECK_ARG((reinterpret_cast<uintptr_t>(plan) & 63u) == 0, ENTMTP_EINVAL, "the plan must be 64-byte aligned");
  ENTMTP_CHECK_ARG(aligned16(q) && aligned16(k_pool) && aligned16(v_pool) && aligned16(out) && aligned16(workspace),
                   ENTMTP_EINVAL, "q, pools, out and workspace must be 16-byte aligned");
  TreeTable trees;
  if (int32_t rc = tree_table(bank, &trees)) return rc;
  const PagedShape sh = paged_shape(bank, B, rows_cap, Hq, Hkv, static_cast<long long>(max_pages) * page_size);
  ENTMTP_CHECK_ARG(sh.items < INT32_MAX / 64, ENTMTP_ERANGE, "%d rows of %d heads: too many", rows_cap, Hq);
  ENTMTP_CHECK_ARG(plan_bytes >= sh.plan_bytes, ENTMTP_ENOSPC, "the plan has %zu bytes, needs %zu", plan_bytes,
                   sh.plan_bytes);
  const size_t need = fp4_workspace(sh);
  ENTMTP_CHECK_ARG(need == 0 || (workspace && workspace_bytes >= need), ENTMTP_ENOSPC,
                   "workspace has %zu bytes, needs %zu", workspace ? workspace_bytes : size_t(0), need);
  ENTMTP_CHECK_ARG(merge_blocks(rows_cap, Hq) <= INT32_MAX, ENTMTP_ERANGE, "%d rows of %d heads: too many", rows_cap, Hq);
  PagedFp4Args a{};
  fill_call(a, trees, sh, plan, B, n_pages, page_size, max_pages, rows_cap, Hq, Hkv, window, out, workspace,
            kPlanMagicFp4);
  a.arena = trees.arena;
  a.table = block_table;
  a.slopes = slopes;
  a.q = q;
  a.kp = k_pool;
  a.vp = v_pool;
  a.q_scale = softcap > 0.f ? 2.f * kLog2e * (scale / softcap) : scale * kLog2e;
  a.cap_log2 = softcap * kLog2e;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(sh.items), dim3(kAttnThreads), 0, s, a); };
  softcap > 0.f || window > 0 || slopes != nullptr ? go(paged_attn_fp4_kernel<true>) : go(paged_attn_fp4_kernel<false>);
  if (int32_t rc = launch_status("tree_attn_paged_fp4 launch")) return rc;
  if (!sh.splits) return ENTMTP_OK;
  return launch_merge<true>(a, s);
}
