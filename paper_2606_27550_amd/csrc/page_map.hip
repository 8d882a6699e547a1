// Page map of a batch: where every tree row of a step lies.
//
// Sequences share a pool of pages of P slots; row b of the block table names
// the pages of sequence b in order, so position p of it is slot
// table[b][p / P] * P + p % P.  Before a step's attention a tree of T nodes
// needs slots for positions L .. L + T - 1: the entries L / P ..
// (L + T - 1) / P, of which those below zero are missing and are taken from
// the top of a stack of free pages, sequence after sequence, in order.
//
// With d_b missing entries of sequence b and D_b = d_0 + .. + d_b, the k-th
// missing entry of sequence b is page free[n_free - 1 - (D_b - d_b) - k], and
// the sequence is served when D_b <= n_free; D never falls, so the served
// ones that take pages come first and the stack shrinks by the largest D_b
// among them.  Row offsets are the running sum of the node counts.
//
// One workgroup: two scans over at most 256 sequences (a thread each), then a
// thread per tree row.  It is bound by its memory round trips (entries, trees,
// table, free list), so each of them asks for all it needs at once: 3.8 us for
// one sequence, 9.0 for 256 of up to 128 nodes.
#include "paged.hpp"

namespace entmtp {
namespace {

constexpr int kMapThreads = 1024;
constexpr int kEntries = ENTMTP_T_MAX / 16 + 1;   // pages of 16 slots that a tree's positions fall into
static_assert(kPagedSeqs == 256, "four wavefronts hold a thread per sequence");

struct MapArgs {
  TreeTable trees;
  const int* topo;
  const int* len;
  int* table;          // [B][max_pages]
  const int* free;     // [free_cap], or NULL
  int* n_free;
  int* row_off;        // [B + 1]
  int* slot_map;       // [rows_cap]
  int* status;         // [B]
  int B, max_pages, shift, n_pages, free_cap, rows_cap;
};

// Inclusive sum over threads 0 .. 255 (four whole wavefronts call it).
__device__ __forceinline__ int scan256(int v, int* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = scan_wave(v, add);
  if (wave < 4 && lane == 63) part[wave] = v;
  __syncthreads();
  for (int w = 0; w < 3; ++w)
    if (w < wave) v += part[w];
  return v;
}

__global__ __launch_bounds__(kMapThreads) void page_map_kernel(MapArgs p) {
  __shared__ int s_off[kPagedSeqs + 1], s_len[kPagedSeqs], s_ok[kPagedSeqs];
  __shared__ int s_page[kEntries][kPagedSeqs];   // pages of the trees' positions
  __shared__ int part_rows[4], part_take[4];
  __shared__ int s_taken;
  const int tid = threadIdx.x;
  const int P = 1 << p.shift;
  if (tid == 0) s_taken = 0;
  int tr = -1, L = 0;
  const bool mine = tid < p.B;
  int free_n = 0;
  if (mine) {
    tr = p.topo[tid];
    L = p.len[tid];
  }
  if (p.free) {
    free_n = *p.n_free;
    free_n = free_n < 0 ? 0 : (free_n > p.free_cap ? p.free_cap : free_n);
  }
  const bool named = mine && tr >= 0 && tr < p.trees.n;
  const int T = named ? p.trees.t[named ? tr : 0].T : 0;
  const int end = scan256(T, part_rows);
  int status = named ? ENTMTP_PAGE_OK : ENTMTP_PAGE_NONE;
  if (named && (end > p.rows_cap || L < 0 ||
                static_cast<long long>(L) + T > static_cast<long long>(p.max_pages) * P))
    status = ENTMTP_PAGE_RANGE;
  // the entries the tree's positions fall into (all requested at once)
  int* const row = p.table + static_cast<size_t>(mine ? tid : 0) * p.max_pages;
  const int p0 = L >> p.shift;
  const int n = status == ENTMTP_PAGE_OK ? ((L + T - 1) >> p.shift) - p0 + 1 : 0;
  int id[kEntries];
#pragma unroll
  for (int k = 0; k < kEntries; ++k) id[k] = k < n ? row[p0 + k] : 0;
  int lack = 0;
  bool bad = n > 0 && id[0] < 0 && (L & (P - 1)) != 0;   // its page holds prefix slots
#pragma unroll
  for (int k = 0; k < kEntries; ++k) {
    bad = bad || id[k] >= p.n_pages;
    lack += id[k] < 0;
  }
  if (bad) {
    status = ENTMTP_PAGE_BAD;
    lack = 0;
  }
  const int upto = scan256(lack, part_take);
  if (lack > 0) {
    if (upto > free_n) {
      status = ENTMTP_PAGE_FULL;
    } else {
      atomicMax(&s_taken, upto);
      const int* top = p.free + (free_n - 1 - (upto - lack));
      int take[kEntries];
#pragma unroll
      for (int k = 0; k < kEntries; ++k) take[k] = k < lack ? top[-k] : 0;
#pragma unroll
      for (int k = 0; k < kEntries; ++k) bad = bad || take[k] < 0 || take[k] >= p.n_pages;
      if (bad) {
        status = ENTMTP_PAGE_BAD;
      } else {
#pragma unroll
        for (int k = 0; k < kEntries; ++k)   // the j-th missing entry takes the j-th page
          if (id[k] < 0) {
            id[k] = take[0];
            row[p0 + k] = take[0];
#pragma unroll
            for (int j = 0; j + 1 < kEntries; ++j) take[j] = take[j + 1];
          }
      }
    }
  }
  if (mine) {
#pragma unroll
    for (int k = 0; k < kEntries; ++k)
      if (k < n) s_page[k][tid] = id[k];
  }
  if (mine) {
    p.status[tid] = status;
    s_len[tid] = L;
    s_ok[tid] = status == ENTMTP_PAGE_OK;
    s_off[tid + 1] = min(end, p.rows_cap);
    p.row_off[tid + 1] = min(end, p.rows_cap);
  }
  if (tid == 0) {
    s_off[0] = 0;
    p.row_off[0] = 0;
  }
  __syncthreads();   // (and every thread has read *n_free)
  if (tid == 0 && p.free) *p.n_free = free_n - s_taken;
  const int rows = s_off[p.B];
#pragma unroll 4   // (the searches' LDS round trips overlap)
  for (int r = tid; r < rows; r += kMapThreads) {
    int b = 0;   // the last sequence that starts at or before r
#pragma unroll
    for (int step = kPagedSeqs / 2; step >= 1; step >>= 1)
      if (s_off[min(b + step, p.B)] <= r && b + step < p.B) b += step;
    const int pos = s_len[b] + (r - s_off[b]);
    p.slot_map[r] = s_ok[b] ? (s_page[(pos >> p.shift) - (s_len[b] >> p.shift)][b] << p.shift) + (pos & (P - 1)) : -1;
  }
}

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" int32_t entmtp_page_map(const entmtp_bank* bank, int32_t B, const int32_t* topo,
                                   const int32_t* prefix_len, int32_t* block_table, int32_t max_pages,
                                   int32_t page_size, int32_t n_pages, const int32_t* free_pages,
                                   int32_t free_cap, int32_t* n_free, int32_t rows_cap, int32_t* row_off,
                                   int32_t* slot_map, int32_t* status, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(paged_batch(B), ENTMTP_EINVAL, "B = %d outside [1, %d]", B, ENTMTP_PAGED_B_MAX);
  ENTMTP_CHECK_ARG(topo && prefix_len && block_table && row_off && slot_map && status, ENTMTP_EINVAL,
                   "topo, prefix_len, block_table, row_off, slot_map and status must be non-NULL device arrays");
  ENTMTP_CHECK_ARG((free_pages == nullptr) == (n_free == nullptr), ENTMTP_EINVAL,
                   "free_pages and n_free go together");
  ENTMTP_CHECK_ARG(free_pages == nullptr || free_cap >= 1, ENTMTP_EINVAL, "free_cap = %d < 1", free_cap);
  ENTMTP_CHECK_ARG(rows_cap >= 1, ENTMTP_EINVAL, "rows_cap = %d < 1", rows_cap);
  if (int32_t rc = check_pool(n_pages, page_size)) return rc;
  if (int32_t rc = check_pages(max_pages, page_size)) return rc;
  MapArgs a{};
  if (int32_t rc = tree_table(bank, &a.trees)) return rc;
  a.topo = topo;
  a.len = prefix_len;
  a.table = block_table;
  a.free = free_pages;
  a.n_free = n_free;
  a.row_off = row_off;
  a.slot_map = slot_map;
  a.status = status;
  a.B = B;
  a.max_pages = max_pages;
  a.shift = page_shift(page_size);
  a.n_pages = n_pages;
  a.free_cap = free_cap;
  a.rows_cap = rows_cap;
  hipLaunchKernelGGL(page_map_kernel, dim3(1), dim3(kMapThreads), 0, static_cast<hipStream_t>(stream), a);
  return launch_status("page_map launch");
}
