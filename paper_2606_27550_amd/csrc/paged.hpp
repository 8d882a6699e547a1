// What the operators over a shared page pool have in common: the bank's trees
// as kernel arguments, and where a row of a batch lies.
//
// A batch's choices (tree indices, prefix lengths, row offsets) are device
// arrays that the host never reads, so every kernel checks the entries it
// uses: a tree index against the bank, a row against the sequence's range and
// the rows there are, a pool slot against the pool.
#pragma once

#include "common.hpp"

namespace entmtp {

constexpr int kPagedSeqs = ENTMTP_PAGED_B_MAX;
constexpr int kPagedTrees = 32;   // bank trees a call can name (kernel arguments)

struct PagedTree {
  int T, D;
  int off_mask, off_depth, off_path;   // bytes into the bank's arena
};

struct TreeTable {
  const uint8_t* arena;
  uint64_t bank;   // its number
  int n;
  PagedTree t[kPagedTrees];
};

// The bank's trees as kernel arguments; an error status where the bank is not
// on the current device or holds more trees than a call can name.
inline int32_t tree_table(const entmtp_bank* bank, TreeTable* out) {
  if (int32_t rc = check_device_bank(bank, 0)) return rc;
  int dev = -1;
  if (int32_t rc = hip_status(hipGetDevice(&dev), "hipGetDevice")) return rc;
  ENTMTP_CHECK_ARG(dev == bank->device, ENTMTP_EINVAL, "the bank lies on device %d, the current one is %d",
                   bank->device, dev);
  ENTMTP_CHECK_ARG(static_cast<int>(bank->desc.size()) <= kPagedTrees, ENTMTP_ERANGE,
                   "a device-planned batch names at most %d bank trees (bank has %zu)", kPagedTrees,
                   bank->desc.size());
  out->arena = bank->arena;
  out->bank = bank->number;
  out->n = static_cast<int>(bank->desc.size());
  for (int k = 0; k < out->n; ++k) {
    const TopoDesc& td = bank->desc[k];
    ENTMTP_CHECK_ARG(td.off_path <= INT32_MAX, ENTMTP_ERANGE, "bank arena offsets past 2 GiB");
    out->t[k] = PagedTree{td.T, td.D, static_cast<int>(td.off_mask), static_cast<int>(td.off_depth),
                          static_cast<int>(td.off_path)};
  }
  return ENTMTP_OK;
}

// Compute units of the current device.
inline int device_cus() {
  static int cus[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  if (cus[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cus[dev] = n;
  }
  return cus[dev];
}

inline bool paged_batch(int B) { return B >= 1 && B <= kPagedSeqs; }

// log2 of a page size (16, 32, 64, 128 or 256 slots), or -1.
inline int page_shift(int page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

// Checks of a pool that every entry point makes.
inline int32_t check_pool(int32_t n_pages, int32_t page_size) {
  ENTMTP_CHECK_ARG(page_shift(page_size) >= 0, ENTMTP_EINVAL,
                   "page_size = %d must be 16, 32, 64, 128 or 256", page_size);
  ENTMTP_CHECK_ARG(n_pages >= 1, ENTMTP_EINVAL, "n_pages = %d < 1", n_pages);
  ENTMTP_CHECK_ARG(static_cast<int64_t>(n_pages) * page_size <= INT32_MAX, ENTMTP_ERANGE,
                   "%d pages of %d slots: slots are 32-bit numbers", n_pages, page_size);
  return ENTMTP_OK;
}

// Positions of a sequence of max_pages pages: 32-bit numbers, with room for a
// tree and a tile past the last one.
inline int32_t check_pages(int32_t max_pages, int32_t page_size) {
  ENTMTP_CHECK_ARG(max_pages >= 1 && static_cast<int64_t>(max_pages) * page_size <= INT32_MAX - 1024, ENTMTP_ERANGE,
                   "max_pages = %d of %d slots: positions are 32-bit numbers", max_pages, page_size);
  return ENTMTP_OK;
}

// Inclusive sum (or, of values not below zero, maximum) over a wavefront's
// lanes, by DPP: within rows of 16, then from row to row.
template <typename F>
__device__ __forceinline__ int scan_wave(int v, F f) {
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));   // row_shr:1
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));   // lane 15 to the next row
  return f(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));   // lane 31 to the upper half
}
__device__ __forceinline__ int add(int a, int b) { return a + b; }
__device__ __forceinline__ int larger(int a, int b) { return max(a, b); }
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

// The sequence whose rows [row_off[b], row_off[b + 1]) hold row r: the number
// of sequences that end at or before it (B: none).  Called by whole
// wavefronts with r uniform; the loads go out together.
__device__ __forceinline__ int seq_of_row(const int* __restrict__ row_off, int B, int r) {
  const int lane = threadIdx.x & 63;
  int end[kPagedSeqs / 64];
#pragma unroll
  for (int k = 0; k < kPagedSeqs / 64; ++k) {
    if (64 * k >= B) break;   // (uniform)
    end[k] = row_off[min(64 * k + lane, B - 1) + 1];
  }
  int b = 0;
#pragma unroll
  for (int k = 0; k < kPagedSeqs / 64; ++k) {
    if (64 * k >= B) break;
    b += __popcll(__ballot(64 * k + lane < B && end[k] <= r));
  }
  return b;
}

}  // namespace entmtp
