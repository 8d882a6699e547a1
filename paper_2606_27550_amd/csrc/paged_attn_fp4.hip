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
//  - A wavefront streams its blocks by itself, from memory to registers, three
//    ahead, and no barrier joins it to the others.  Where the rows fill one tile
//    (or two) its wavefronts share the range, every fourth (second) block each,
//    and meet in the LDS at the end: a few rows' blocks are a chain of products,
//    softmax and products that one wavefront could not walk at memory's rate.
//  - Keys enter the matrix instruction (32 x 32 x 64, 4-bit by 8-bit) as they lie
//    in the pool, codes and scale bytes; the queries as two 8-bit numbers of four
//    bits of mantissa each, which hold a bf16 number's eight, so that the scores
//    are those of the bf16 query (one below 2^-14 of the largest of its 32 to
//    within 2^-22 of that).
//  - Values become bf16 numbers, exactly, on their way to the wavefront's part of
//    the LDS, from which the products read them transposed.
#include <algorithm>
#include <type_traits>

#include "fp4.hpp"
#include "paged_plan.hpp"

namespace entmtp {
namespace {

constexpr int kFp4Ahead = 3;               // blocks in flight per wavefront
constexpr int kFp4Stage = KB * HD * 2;     // bytes of a block's values in bf16

struct PagedFp4Args : PagedCall {
  const uint8_t* arena;
  const int* table;      // [B][max_pages]
  const float* slopes;   // [Hq] or NULL
  const uint16_t* q;     // [rows_cap][Hq][HD]
  const uint8_t* kp;     // [n_pages][Hkv][P x 68]
  const uint8_t* vp;
  float q_scale;     // of the products: scale log2(e), or with a cap 2 log2(e) scale / cap
  float cap_log2;    // cap log2(e), 0: no cap
};

// Chunk c (16 bytes) of row r of the staged values lies at c ^ stage_swz(r): a
// store takes one chunk of eight rows, a transposing read 32 lanes' 64 bytes of
// four rows; both then cover all banks.
__device__ __forceinline__ int stage_swz(int r) { return 4 * (r & 3) + ((r >> 2) & 3); }

// Two 8-bit operands of 16 bf16 values times inv (a power of two).
__device__ __forceinline__ void query8(u32x4 a, u32x4 b, float inv, i32x8& hi, i32x8& lo, int at) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w0 = j < 2 ? a[2 * (j & 1)] : b[2 * (j & 1)], w1 = j < 2 ? a[2 * (j & 1) + 1] : b[2 * (j & 1) + 1];
    const float x0 = bf16_lo(w0) * inv, x1 = bf16_hi(w0) * inv, x2 = bf16_lo(w1) * inv, x3 = bf16_hi(w1) * inv;
    int h = 0, l = 0;
    h = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, h, false);
    h = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, h, true);
    const auto y = __builtin_amdgcn_cvt_pk_f32_fp8(h, false), z = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
    l = __builtin_amdgcn_cvt_pk_fp8_f32((x0 - y[0]) * 32.f, (x1 - y[1]) * 32.f, l, false);
    l = __builtin_amdgcn_cvt_pk_fp8_f32((x2 - z[0]) * 32.f, (x3 - z[1]) * 32.f, l, true);
    hi[at + j] = h;
    lo[at + j] = l;
  }
}

// MOD: a score cap, distance bias or window.
template <bool MOD>
__global__ __launch_bounds__(kAttnThreads, 2) void paged_attn_fp4_kernel(PagedFp4Args p) {
  __shared__ __attribute__((aligned(16))) uint8_t s_val[kTilesPerWg][kFp4Stage];
  __shared__ float2 s_ml[kTilesPerWg][KB];
  __shared__ uint8_t s_depth[ENTMTP_T_MAX];
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

  // this wavefront's blocks: number i is blk_lo + way + i ways; past the last
  // the last one again
  const int nb = live ? max(0, (blk_hi - blk_lo - way + ways - 1) / ways) : 0;
  auto key_at = [&](int i) { return (blk_lo + way + max(min(i, nb - 1), 0) * ways) * KB; };
  // a block's two runs of 16 keys lie in a page each
  struct Block {
    u32x4 k0, k1, v0, v1;
    uint32_t ks, vs;
    bool there;   // this lane's page lies in the pool
  };
  struct Pages {
    int lo, hi;
  };
  auto pages_of = [&](int i) {
    const int kb = key_at(i);
    return Pages{pages[min(kb >> p.shift, p.max_pages - 1)], pages[min((kb + 16) >> p.shift, p.max_pages - 1)]};
  };
  auto load = [&](Block& s, int i, Pages pg) {
    const int key = key_at(i) + li;
    const int page = li < 16 ? pg.lo : pg.hi;
    s.there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
    if (MOD && key < w_lo) s.there = false;
    const size_t base = (static_cast<size_t>(s.there ? page : 0) * p.Hkv + g) * static_cast<size_t>(P * kFp4RowBytes);
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
  // the query row (row r of KV head g: head g G + r / T, node r % T), its depth
  // and mask, all unconditional: rows past the tree read row 0, see every key
  // and are never stored
  const int qrow = qt * kQTile + li;
  const bool qlive = live && qrow < GT;
  const int qnode = qlive ? qrow % T : 0;
  const int qhead = g * p.G + (qlive ? qrow / T : 0);
  u32x4 qf[8];   // dims 64 m + 32 c + 16 lh .. + 15 (m, c in 0, 1) in qf[4 m + 2 c], [.. + 1]
  {
    const uint16_t* qp = p.q + (static_cast<size_t>(row0 + qnode) * p.Hq + qhead) * HD + 16 * lh;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const u32x4*>(qp + 32 * (s >> 1) + 8 * (s & 1));
  }
  const int qdepth = depth[qnode];
  const int tdepth = depth[min(tid, T - 1)];
  u32x4 mlo = *reinterpret_cast<const u32x4*>(mask + qnode * ENTMTP_MASK_WORDS);
  u32x4 mhi = *reinterpret_cast<const u32x4*>(mask + qnode * ENTMTP_MASK_WORDS + 4);
  static_assert(ENTMTP_MASK_WORDS == 8, "a mask row is two 16-byte loads");
  float slope = 0.f;
  if constexpr (MOD)
    if (p.slopes) slope = p.slopes[qhead] * kLog2e;
#pragma unroll
  for (int k = 0; k < kFp4Ahead; ++k) load(blk[k], k, pg[k]);
  Pages next = pg[kFp4Ahead];
  s_depth[tid] = static_cast<uint8_t>(tdepth);
  static_assert(kAttnThreads >= ENTMTP_T_MAX, "one thread per node");
  if (MOD) {
    wait_lds();
    stage_barrier();
  }
  if (!qlive) mlo = mhi = u32x4{~0u, ~0u, ~0u, ~0u};
  i32x8 qh[2], ql[2];
  uint32_t qsc = 0u;   // scale bytes of this half's blocks: of hi for m = 0, 1, then of lo
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t sc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const u32x4 u = qf[4 * m + 2 * c], w = qf[4 * m + 2 * c + 1];
      uint32_t top = max(bf16_top(u), bf16_top(w));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32, 64)));
      const int e = static_cast<int>(top >> 7), s = e < 14 ? 7 : e - 7;   // largest below 2^8
      query8(u, w, __uint_as_float(static_cast<uint32_t>(254 - s) << 23), qh[m], ql[m], 4 * c);
      sc[c] = top >= 0x7f80u ? kFp4NaN | kFp4NaN << 16 : static_cast<uint32_t>(s) | static_cast<uint32_t>(s - 5) << 16;
    }
    qsc |= (lh ? sc[1] : sc[0]) << (8 * m);
  }
  const float qs = p.q_scale;
  const int qpos = L + qdepth;
  const int w_row = MOD && p.window > 0 ? qpos - p.window + 1 : -1;   // the row's first position
  const int w_hi = MOD && p.window > 0 ? L + D - p.window + 1 : -1;   // from here on every row sees the prefix

  // l_run: the sum of this lane's half of the keys (the halves meet at the end)
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 o[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ct][r] = 0.f;

  // The values' part of the LDS: row li's chunks, and the transposing reads:
  // row 4 lh + (lane % 16) / 4 of each 8 rows, dims 32 ct + 16 (li / 16) + 4 (lane % 4)
  uint8_t* const stage = s_val[wave];
  uint8_t* const srow = stage + li * 256;
  const int sx = stage_swz(li);
  const int vrow = 4 * lh + ((lane & 15) >> 2);
  const int vx = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ stage_swz(vrow);   // (rows 8 on: chunk ^ 2)
  const uint8_t* const vbase = stage + vrow * 256 + 8 * (lane & 1);

  auto key_of = [&](int r) { return 8 * (r >> 2) + 4 * lh + (r & 3); };   // accumulator r's key of the block
  // The block's products as logits in base 2 (with MOD; else they are scaled in
  // the exponent's fused multiply-add), key r at distance dist(r).
  // tanh(u) = 1 - 2 / (e^2u + 1) with 2 u / ln 2 from the products: 0 and
  // infinity of the exponential give -1 and 1.
  auto bend = [&](f32x16& sacc, auto dist) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] *= qs;
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

  auto attend = [&](Block& s, int i) {
    const int kb = key_at(i);
    // keys of this half's dims: group 2 m + lh of matrix instruction m
    uint32_t ks = s.ks, vs = s.vs;
    if (!__all(s.there)) {   // (a page outside the pool: zeros)
      if (!s.there) {
        s.k0 = s.k1 = s.v0 = s.v1 = u32x4{0u, 0u, 0u, 0u};
        ks = vs = 0x7f7f7f7fu;
      }
    }
    ks = lh ? ks >> 8 : ks;
    f32x16 sacc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
    const i32x8 ka = {static_cast<int>(s.k0[0]), static_cast<int>(s.k0[1]), static_cast<int>(s.k0[2]), static_cast<int>(s.k0[3]), 0, 0, 0, 0};
    const i32x8 kc = {static_cast<int>(s.k1[0]), static_cast<int>(s.k1[1]), static_cast<int>(s.k1[2]), static_cast<int>(s.k1[3]), 0, 0, 0, 0};
    const int kscale = static_cast<int>(ks), qscale = static_cast<int>(qsc);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, ql[0], sacc, 4, 0, 0, kscale, 2, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kc, ql[1], sacc, 4, 0, 2, kscale, 3, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qh[0], sacc, 4, 0, 0, kscale, 0, qscale);
    sacc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kc, qh[1], sacc, 4, 0, 2, kscale, 1, qscale);
    // the values to the LDS; groups that are no numbers as zeros (a zero weight
    // would make them NaNs in every row) and their keys noted
    const uint32_t v2 = lh ? vs >> 16 : vs;   // groups 2 lh and 2 lh + 1
    const uint32_t va = v2 & 0xffu, vb = v2 >> 8 & 0xffu;
    const unsigned long long bad = __ballot(va == kFp4NaN || vb == kFp4NaN);
    const uint32_t odd = static_cast<uint32_t>(bad) | static_cast<uint32_t>(bad >> 32);
    const float sa = va == kFp4NaN ? 0.f : fp4_step(va), sb = vb == kFp4NaN ? 0.f : fp4_step(vb);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t w = c < 4 ? s.v0[c & 3] : s.v1[c & 3];
      *reinterpret_cast<u32x4*>(srow + (((8 * lh + c) ^ sx) << 4)) = fp4_values(w, c < 4 ? sa : sb);
    }

    // what every row sees of the block
    uint32_t vis = ~0u;
    const bool whole = kb + KB <= L && !(MOD && kb < w_hi);   // (uniform)
    if (whole) {
      if constexpr (MOD) bend(sacc, [&](int r) { return qpos - (kb + key_of(r)); });
    } else {
      const int rel = kb - L;
      auto word = [&](int w) {   // (w is uniform)
        uint32_t m = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = w == k ? (k < 4 ? mlo[k & 3] : mhi[k & 3]) : m;
        return m;
      };
      if (rel + KB <= 0) {
        vis = ~0u;
      } else if (rel < 0) {
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
      const uint32_t mine = vis >> (4 * lh);   // bit 8 (r / 4) + r % 4 is accumulator r's key
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = static_cast<int>(mine << (31 - (8 * (r >> 2) + (r & 3)))) >> 31;
        sacc[r] = __builtin_bit_cast(float, (m & __builtin_bit_cast(int, static_cast<float>(sacc[r]))) | (~m & INT32_C(-0x800000)));
      }
    }
    if ((vis & odd) != 0u) l_run = NAN;
    float bmax = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) bmax = fmaxf(bmax, sacc[r]);
    bmax = max_halves(bmax);
    if constexpr (!MOD) bmax *= qs;
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
      pr[r] = __builtin_amdgcn_exp2f(MOD ? sacc[r] + mneg : fmaf(sacc[r], qs, mneg));
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
        const uint2 x0 = lds_read_tr(vbase + 16 * u * 256 + ((vx ^ (4 * ct)) << 4));
        const uint2 x1 = lds_read_tr(vbase + (16 * u + 8) * 256 + ((vx ^ (4 * ct) ^ 2) << 4));
        const u32x4 w = {x0.x, x0.y, x1.x, x1.y};
        o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w), pf[u], o[ct], 0, 0, 0);
      }
  };

  for (int i = 0; i < nb; i += kFp4Ahead) {
#pragma unroll
    for (int k = 0; k < kFp4Ahead; ++k) {
      if (i + k < nb) {   // (uniform)
        attend(blk[k], i + k);
        load(blk[k], i + k + kFp4Ahead, next);
        next = pages_of(i + k + kFp4Ahead + 1);
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
  // half lh) holds dims 32 ct + 8 j + 4 lh + i in o[ct][4 j + i]; the halves
  // trade a chunk so that each stores 16 bytes: lane 0..31 dims 8 j .. 8 j + 7
  // of even j, lane 32..63 of odd j.
  uint16_t* dst;
  if (nsplit == 1) {
    const int r = qrow < GT ? qrow : 0;
    dst = p.out + (static_cast<size_t>(row0 + r % T) * p.Hq + g * p.G + r / T) * HD;
  } else {
    const long long part = static_cast<long long>((static_cast<unsigned long long>(it.part_hi) << 32) | it.part_lo);
    const size_t prow = part + (static_cast<size_t>(split) * p.Hkv + g) * it.rows_pad + qrow;
    dst = p.part_o + prow * HD;
    if (lh == 0 && qrow < GT) {
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
  return entmtp_tree_attn_paged_workspace(bank, B, rows_cap, Hq, Hkv, d, max_pages, page_size);
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
  ENTMTP_CHECK_ARG(sh.workspace == 0 || (workspace && workspace_bytes >= sh.workspace), ENTMTP_ENOSPC,
                   "workspace has %zu bytes, needs %zu", workspace ? workspace_bytes : size_t(0), sh.workspace);
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
  return launch_merge(a, s);
}
