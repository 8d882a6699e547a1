// New rows on their way into the page pool: queries and keys normed per head
// and turned to their positions, keys and values written to their slots, in
// bf16 or in 4 bits; and the positions of a step's tree rows.
//
// With x the d values of a head, w the norm's weights and a_c = pos
// theta^(-2c/d):
//   y = x / sqrt(mean(x^2) + eps) w
//   y_c cos a_c - y_{c+d/2} sin a_c,  y_{c+d/2} cos a_c + y_c sin a_c
// rounded to bf16.  All of it is computed in fp64 (angles, the sum of squares,
// which in fp32 passes the range from values of 2^60 on and below 2^-63, and the
// products) and rounded by way of fp32, as a tensor of 64-bit numbers is
// converted, so that a program that computes its keys in tensors finds the same
// bytes in the pool (one value of 2^17 is off by a unit of bf16 from the rounding
// at once that the attention kernels give the keys that they append).  Queries
// in fp32 took 0 to 4 % less time (6476 rows as below 40.6-42.6 us against 42.0-43.2).
//
// Eight threads hold a head (thread cc the chunks cc and cc + 8 of eight values,
// so both halves of eight pairs), a wavefront eight heads at a time.  A wavefront
// works alone: lane c computes the angle of pair c of its row, 40 fp64
// instructions, and leaves it in the wavefront's part of the LDS.
//
// Bytes bound it: 6476 rows of prompts (32:8 heads, norm) into 4-bit pages 42-43 us
// (3.9 TB/s), 3852 (40:40, no norm) into bf16 pages 67 us (4.7 TB/s; a large copy
// 4.9).  The tree rows of a step (208) take 5.5 us, one row 5.3: a launch and
// two round trips; their positions, a kernel of their own once a step, 2.7.  (The
// next group's loads ahead of this one's stores: level.)
#include "attn_tile.hpp"
#include "fp4.hpp"
#include "paged.hpp"

namespace entmtp {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / 64;

struct AppendArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  long long q_stride, k_stride, v_stride;
  const int* pos;        // [rows]
  const int* slot_map;   // [rows]
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  uint16_t* q_out;
  void* kp;
  void* vp;
  uint16_t* k_out;
  uint16_t* v_out;
  int rows, Hq, Hkv, shift, n_slots;
  int parts;             // wavefronts that share a row's groups of eight heads
  int qg, groups;        // groups of queries, of all
  int turn;
  float eps;
  double freq[kRopePairs];
};

// The norm's factor on the 16 values of a thread's chunks; no number where the
// head holds one that is not finite (the sum of 128 finite squares of bf16 numbers
// stays finite: below 2^263).
__device__ __forceinline__ double head_rsqrt(u32x4 lo, u32x4 hi, float eps) {
  double s = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double a = bf16_lo(lo[e]), b = bf16_hi(lo[e]), c = bf16_lo(hi[e]), d = bf16_hi(hi[e]);
    s = a * a + s;
    s = b * b + s;
    s = c * c + s;
    s = d * d + s;
  }
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) s += __shfl_xor(s, off, 8);
  return s < INFINITY ? 1.0 / sqrt(s / HD + static_cast<double>(eps)) : static_cast<double>(NAN);
}

// A head's chunks normed (w: its 16 weights, or null) and turned.
template <bool TURN>
__device__ __forceinline__ void norm_turn(u32x4& lo, u32x4& hi, const uint16_t* w, int cc, float eps, const double2* t) {
#pragma clang fp contract(off)
  double r = 1;
  u32x4 wl = {0u, 0u, 0u, 0u}, wh = wl;
  if (w) {
    wl = *reinterpret_cast<const u32x4*>(w + 8 * cc);
    wh = *reinterpret_cast<const u32x4*>(w + 8 * cc + HD / 2);
    r = head_rsqrt(lo, hi, eps);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t nl = 0u, nh = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      double x = h ? bf16_hi(lo[e]) : bf16_lo(lo[e]), y = h ? bf16_hi(hi[e]) : bf16_lo(hi[e]);
      if (w) {
        x = x * r * static_cast<double>(h ? bf16_hi(wl[e]) : bf16_lo(wl[e]));
        y = y * r * static_cast<double>(h ? bf16_hi(wh[e]) : bf16_lo(wh[e]));
      }
      double a = x, b = y;
      if constexpr (TURN) {
        const double2 cs = t[(2 * e + h) ^ cc];
        a = x * cs.x - y * cs.y;
        b = y * cs.x + x * cs.y;
      }
      nl |= static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(static_cast<float>(a)))) << (16 * h);
      nh |= static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(static_cast<float>(b)))) << (16 * h);
    }
    lo[e] = nl;
    hi[e] = nh;
  }
}

// The pool's row of head g at a slot.
template <bool FP4>
__device__ __forceinline__ void store_row(const AppendArgs& p, void* pool, uint16_t* out, u32x4 lo, u32x4 hi, int row,
                                          int g, int slot, int cc, bool live) {
  const size_t head = static_cast<size_t>(slot >> p.shift) * p.Hkv + g;
  const int in = slot & ((1 << p.shift) - 1);
  const bool there = live && slot >= 0 && slot < p.n_slots;
  if constexpr (FP4) {
    // (both halves' groups are four threads wide; the shuffles are every thread's)
    uint32_t tl = bf16_top(lo), th = bf16_top(hi);
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
      tl = max(tl, static_cast<uint32_t>(__shfl_xor(static_cast<int>(tl), off, 4)));
      th = max(th, static_cast<uint32_t>(__shfl_xor(static_cast<int>(th), off, 4)));
    }
    const uint32_t bl = fp4_scale(tl), bh = fp4_scale(th);
    const uint32_t wl = fp4_codes(lo, bl), wh = fp4_codes(hi, bh);
    // thread 0 has groups 0 and 2, thread 4 groups 1 and 3
    const uint32_t mine = bl | bh << 16, other = static_cast<uint32_t>(__shfl_xor(static_cast<int>(mine), 4, 8));
    if (there) {
      uint8_t* const base = static_cast<uint8_t*>(pool) + (head << p.shift) * kFp4RowBytes;
      uint32_t* const codes = reinterpret_cast<uint32_t*>(base + in * (HD / 2));
      codes[cc] = wl;
      codes[cc + 8] = wh;
      if (cc == 0) reinterpret_cast<uint32_t*>(base + (HD / 2 << p.shift))[in] = mine | other << 8;
    }
    if (out && live) {
      auto value = [](uint32_t w, uint32_t b) {
        u32x4 v = fp4_values(w, fp4_step(b == kFp4NaN ? 127u : b));
        return b == kFp4NaN ? u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u} : v;
      };
      lo = value(wl, bl);
      hi = value(wh, bh);
    }
  } else {
    if (there) {
      uint16_t* const at = static_cast<uint16_t*>(pool) + ((head << p.shift) + in) * HD + 8 * cc;
      *reinterpret_cast<u32x4*>(at) = lo;
      *reinterpret_cast<u32x4*>(at + HD / 2) = hi;
    }
  }
  if (out && live) {
    uint16_t* const at = out + (static_cast<size_t>(row) * p.Hkv + g) * HD + 8 * cc;
    *reinterpret_cast<u32x4*>(at) = lo;
    *reinterpret_cast<u32x4*>(at + HD / 2) = hi;
  }
}

template <bool FP4, bool TURN, bool WIDE>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs p) {
  __shared__ __attribute__((aligned(16))) double2 s_angle[kAppendWaves][kRopePairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long unit = static_cast<long long>(blockIdx.x) * kAppendWaves + wave;
  const int row = static_cast<int>(unit / p.parts), part = static_cast<int>(unit % p.parts);
  if (row >= p.rows) return;
  const int pos = p.pos[row], slot = p.slot_map[row];
  if (pos < 0) return;
  double2* const t = s_angle[wave];
  if constexpr (TURN) {
    const double x = static_cast<double>(pos) * p.freq[lane];
    double2 cs;
    if constexpr (WIDE)
      sincos(x, &cs.y, &cs.x);
    else
      cs = cos_sin(x);
    t[lane ^ ((lane >> 3) & 7)] = cs;
    wait_lds();   // (a wavefront's own: its stores are seen by its loads)
  }
  const int cc = lane & 7, sub = lane >> 3;
  const double2* const mine = t + 8 * cc;
  const int kg = (p.Hkv + 7) / 8;
  for (int g = part; g < p.groups; g += p.parts) {
    // (a group is of one kind; a head past the last is the last one again, not stored)
    const int kind = g < p.qg ? 0 : (g < p.qg + kg ? 1 : 2);
    const int at = 8 * (g - (kind == 0 ? 0 : (kind == 1 ? p.qg : p.qg + kg))) + sub;
    const int H = kind == 0 ? p.Hq : p.Hkv, h = min(at, H - 1);
    const bool live = at < H;
    const uint16_t* const src = (kind == 0 ? p.q + row * p.q_stride : (kind == 1 ? p.k + row * p.k_stride : p.v + row * p.v_stride)) +
                                static_cast<size_t>(h) * HD + 8 * cc;
    u32x4 lo = *reinterpret_cast<const u32x4*>(src), hi = *reinterpret_cast<const u32x4*>(src + HD / 2);
    if (kind == 0) {
      norm_turn<TURN>(lo, hi, p.q_norm, cc, p.eps, mine);
      if (live) {
        uint16_t* const out = p.q_out + (static_cast<size_t>(row) * p.Hq + h) * HD + 8 * cc;
        *reinterpret_cast<u32x4*>(out) = lo;
        *reinterpret_cast<u32x4*>(out + HD / 2) = hi;
      }
    } else if (kind == 1) {
      norm_turn<TURN>(lo, hi, p.k_norm, cc, p.eps, mine);
      store_row<FP4>(p, p.kp, p.k_out, lo, hi, row, h, slot, cc, live);
    } else {
      store_row<FP4>(p, p.vp, p.v_out, lo, hi, row, h, slot, cc, live);
    }
  }
}

// A workgroup a sequence, and one for the rows that lie in no sequence's range.
struct PositionArgs {
  TreeTable trees;
  const int* topo;
  const int* len;
  const int* row_off;   // [B + 1]
  int* pos;
  int B, rows;
};

__global__ __launch_bounds__(ENTMTP_T_MAX) void tree_positions_kernel(PositionArgs p) {
  __shared__ int s_off[kPagedSeqs + 1];
  const int b = blockIdx.x, tid = threadIdx.x;
  // (offsets of any size: as far as there are rows, counted in 64 bits)
  auto clear = [&](long long first, long long end) {
    for (long long r = first + tid; r < end; r += ENTMTP_T_MAX) p.pos[r] = -1;
  };
  auto within = [&](int r) { return min(max(r, 0), p.rows); };
  if (b == p.B) {
    // offsets that never fall leave the rows before the first and behind the last;
    // others (none that entmtp_page_map makes) are looked up row by row
    static_assert(ENTMTP_T_MAX >= kPagedSeqs, "a thread per sequence");
    const int off = p.row_off[min(tid, p.B - 1)], end = p.row_off[min(tid, p.B - 1) + 1];
    if (tid < p.B) s_off[tid] = off;
    if (tid == p.B - 1) s_off[p.B] = end;
    if (__syncthreads_and(off <= end)) {
      clear(0, within(s_off[0]));
      clear(within(s_off[p.B]), p.rows);
      return;
    }
    for (long long r = tid; r < p.rows; r += ENTMTP_T_MAX) {
      bool held = false;
      for (int k = 0; k < p.B; ++k) held = held || (s_off[k] <= r && r < s_off[k + 1]);
      if (!held) p.pos[r] = -1;
    }
    return;
  }
  const int tr = p.topo[b], L = p.len[b], r0 = p.row_off[b], r1 = within(p.row_off[b + 1]);
  const bool named = tr >= 0 && tr < p.trees.n;
  const PagedTree& tree = p.trees.t[named ? tr : 0];
  const int* const depth = reinterpret_cast<const int*>(p.trees.arena + tree.off_depth);
  // (r1 - r0 above -2^31: both are at least zero)
  const int T = named && r0 >= 0 && tree.T <= r1 - r0 && L >= 0 && L <= INT32_MAX - ENTMTP_T_MAX ? tree.T : 0;
  for (int i = tid; i < T; i += ENTMTP_T_MAX) p.pos[r0 + i] = L + depth[i];
  clear(static_cast<long long>(max(r0, 0)) + T, r1);
}

template <bool FP4>
int32_t append(const entmtp_bf16* q, int64_t q_stride, const entmtp_bf16* k, int64_t k_stride, const entmtp_bf16* v,
               int64_t v_stride, int32_t rows, int32_t Hq, int32_t Hkv, int32_t d, const int32_t* pos,
               const int32_t* slot_map, const entmtp_bf16* q_norm, const entmtp_bf16* k_norm, float eps,
               float rope_theta, entmtp_bf16* q_out, void* k_pool, void* v_pool, int32_t n_pages, int32_t page_size,
               entmtp_bf16* k_out, entmtp_bf16* v_out, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(k && v && pos && slot_map && k_pool && v_pool, ENTMTP_EINVAL,
                   "k, v, pos, slot_map and pools must be non-NULL");
  ENTMTP_CHECK_ARG((q == nullptr) == (q_out == nullptr), ENTMTP_EINVAL, "q and q_out go together");
  ENTMTP_CHECK_ARG(q || !q_norm, ENTMTP_EINVAL, "q_norm without q");
  ENTMTP_CHECK_ARG(d == HD, ENTMTP_EINVAL, "head dim %d unsupported (built for %d)", d, HD);
  ENTMTP_CHECK_ARG(rows >= 1 && Hkv >= 1 && (!q || Hq >= 1), ENTMTP_EINVAL, "rows = %d, Hq = %d, Hkv = %d must be >= 1",
                   rows, Hq, Hkv);
  ENTMTP_CHECK_ARG(Hkv <= 65536 && (!q || Hq <= 65536), ENTMTP_ERANGE, "%d or %d heads: too many", Hq, Hkv);
  if (int32_t rc = check_pool(n_pages, page_size)) return rc;
  ENTMTP_CHECK_ARG(eps >= 0.f && eps < INFINITY, ENTMTP_EINVAL, "eps must be >= 0");
  ENTMTP_CHECK_ARG(rope_theta >= 0.f && rope_theta < INFINITY, ENTMTP_EINVAL, "rope_theta must be >= 0");
  constexpr int64_t kFar = int64_t{1} << 40;
  ENTMTP_CHECK_ARG((!q || (q_stride >= static_cast<int64_t>(Hq) * d && q_stride % 8 == 0 && q_stride <= kFar)) &&
                       k_stride >= static_cast<int64_t>(Hkv) * d && k_stride % 8 == 0 && k_stride <= kFar &&
                       v_stride >= static_cast<int64_t>(Hkv) * d && v_stride % 8 == 0 && v_stride <= kFar,
                   ENTMTP_EINVAL, "row strides must hold their heads and be multiples of 8");
  ENTMTP_CHECK_ARG(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(q_out) && aligned16(k_pool) &&
                       aligned16(v_pool) && aligned16(k_out) && aligned16(v_out) && aligned16(q_norm) && aligned16(k_norm),
                   ENTMTP_EINVAL, "tensors and pools must be 16-byte aligned");
  AppendArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.pos = pos;
  a.slot_map = slot_map;
  a.q_norm = q_norm;
  a.k_norm = k_norm;
  a.q_out = q_out;
  a.kp = k_pool;
  a.vp = v_pool;
  a.k_out = k_out;
  a.v_out = v_out;
  a.rows = rows;
  a.Hq = q ? Hq : 0;
  a.Hkv = Hkv;
  a.shift = page_shift(page_size);
  a.n_slots = n_pages * page_size;
  a.qg = (a.Hq + 7) / 8;
  a.groups = a.qg + 2 * ((Hkv + 7) / 8);
  a.eps = eps;
  rope_freqs(rope_theta, a.freq);
  // few rows: a wavefront a group, so that they are in flight together
  const long long room = 16LL * device_cus();   // wavefronts
  a.parts = static_cast<int>(std::max<long long>(1, std::min<long long>(a.groups, room / rows)));
  const long long blocks = (static_cast<long long>(rows) * a.parts + kAppendWaves - 1) / kAppendWaves;
  ENTMTP_CHECK_ARG(blocks <= INT32_MAX, ENTMTP_ERANGE, "%d rows: too many", rows);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kAppendThreads), 0,
                       static_cast<hipStream_t>(stream), a);
  };
  if (rope_theta == 0.f)
    go(kv_append_kernel<FP4, false, false>);
  else if (wide_angles(rope_theta))
    go(kv_append_kernel<FP4, true, true>);
  else
    go(kv_append_kernel<FP4, true, false>);
  return launch_status("kv_append_paged launch");
}

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" int32_t entmtp_tree_positions(const entmtp_bank* bank, int32_t B, const int32_t* topo,
                                         const int32_t* prefix_len, const int32_t* row_off, int32_t rows, int32_t* pos,
                                         void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(topo && prefix_len && row_off && pos, ENTMTP_EINVAL,
                   "topo, prefix_len, row_off and pos must be non-NULL device arrays");
  ENTMTP_CHECK_ARG(rows >= 1, ENTMTP_EINVAL, "rows = %d < 1", rows);
  PositionArgs a{};
  if (int32_t rc = tree_table(bank, &a.trees)) return rc;
  a.topo = topo;
  a.len = prefix_len;
  a.row_off = row_off;
  a.pos = pos;
  a.B = B;
  a.rows = rows;
  hipLaunchKernelGGL(tree_positions_kernel, dim3(B + 1), dim3(ENTMTP_T_MAX), 0, static_cast<hipStream_t>(stream), a);
  return launch_status("tree_positions launch");
}

extern "C" int32_t entmtp_kv_append_paged(const entmtp_bf16* q, int64_t q_stride, const entmtp_bf16* k,
                                          int64_t k_stride, const entmtp_bf16* v, int64_t v_stride, int32_t rows,
                                          int32_t Hq, int32_t Hkv, int32_t d, const int32_t* pos,
                                          const int32_t* slot_map, const entmtp_bf16* q_norm,
                                          const entmtp_bf16* k_norm, float eps, float rope_theta, entmtp_bf16* q_out,
                                          entmtp_bf16* k_pool, entmtp_bf16* v_pool, int32_t n_pages, int32_t page_size,
                                          entmtp_bf16* k_out, entmtp_bf16* v_out, void* stream) {
  return append<false>(q, q_stride, k, k_stride, v, v_stride, rows, Hq, Hkv, d, pos, slot_map, q_norm, k_norm, eps,
                       rope_theta, q_out, k_pool, v_pool, n_pages, page_size, k_out, v_out, stream);
}

extern "C" int32_t entmtp_kv_append_paged_fp4(const entmtp_bf16* q, int64_t q_stride, const entmtp_bf16* k,
                                              int64_t k_stride, const entmtp_bf16* v, int64_t v_stride, int32_t rows,
                                              int32_t Hq, int32_t Hkv, int32_t d, const int32_t* pos,
                                              const int32_t* slot_map, const entmtp_bf16* q_norm,
                                              const entmtp_bf16* k_norm, float eps, float rope_theta,
                                              entmtp_bf16* q_out, uint8_t* k_pool, uint8_t* v_pool, int32_t n_pages,
                                              int32_t page_size, entmtp_bf16* k_out, entmtp_bf16* v_out,
                                              void* stream) {
  return append<true>(q, q_stride, k, k_stride, v, v_stride, rows, Hq, Hkv, d, pos, slot_map, q_norm, k_norm, eps,
                      rope_theta, q_out, k_pool, v_pool, n_pages, page_size, k_out, v_out, stream);
}
