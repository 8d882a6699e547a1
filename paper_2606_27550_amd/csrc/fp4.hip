// bf16 rows to 4-bit codes and scale bytes (the form is described in fp4.hpp).
#include <algorithm>

#include "fp4.hpp"

namespace entmtp {
namespace {

constexpr int kQuantThreads = 256;

// A thread takes eight values, four threads a group, whose largest magnitude
// goes round by two exchanges.  It moves 2.53 bytes a value and computes a dozen
// instructions for eight: bytes bound it (32000 rows of 4096 values 58 us, 5.7 TB/s), once for a model's
// weights.
__global__ __launch_bounds__(kQuantThreads) void quantize_fp4_kernel(const uint16_t* __restrict__ x, long long chunks,
                                                                     uint32_t* __restrict__ codes,
                                                                     uint8_t* __restrict__ scales) {
  const long long step = static_cast<long long>(gridDim.x) * kQuantThreads;
  for (long long i = static_cast<long long>(blockIdx.x) * kQuantThreads + threadIdx.x; i < chunks; i += step) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(x + 8 * i);
    uint32_t top = bf16_top(v);   // (the four of a group are all there: chunks is a multiple of four)
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1, 4)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2, 4)));
    const uint32_t b = fp4_scale(top);
    codes[i] = fp4_codes(v, b);
    if ((i & 3) == 0) scales[i >> 2] = static_cast<uint8_t>(b);
  }
}

}  // namespace
}  // namespace entmtp

using namespace entmtp;

extern "C" int32_t entmtp_quantize_fp4(const entmtp_bf16* x, int64_t rows, int32_t n, uint8_t* codes,
                                       uint8_t* scales, void* stream) {
  clear_error();
  ENTMTP_CHECK_ARG(x && codes && scales, ENTMTP_EINVAL, "x, codes and scales must be non-NULL");
  ENTMTP_CHECK_ARG(rows >= 1 && n >= kFp4Group && n % kFp4Group == 0, ENTMTP_EINVAL,
                   "rows = %lld must be >= 1, n = %d a multiple of %d", static_cast<long long>(rows), n, kFp4Group);
  ENTMTP_CHECK_ARG(rows <= (int64_t{1} << 62) / n, ENTMTP_EINVAL, "%lld rows of %d values: too many",
                   static_cast<long long>(rows), n);
  ENTMTP_CHECK_ARG(aligned16(x) && (reinterpret_cast<uintptr_t>(codes) & 3u) == 0, ENTMTP_EINVAL,
                   "x must be 16-byte aligned, codes 4-byte");
  const long long chunks = static_cast<long long>(rows) * (n / 8);
  const long long blocks = std::min<long long>((chunks + kQuantThreads - 1) / kQuantThreads, 1 << 16);
  hipLaunchKernelGGL(quantize_fp4_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kQuantThreads), 0,
                     static_cast<hipStream_t>(stream), x, chunks, reinterpret_cast<uint32_t*>(codes), scales);
  return launch_status("quantize_fp4 launch");
}
