// The paged cache's attention over 8-bit rows (the kernel is in ssd_paged_decode.cuh).
#include "ssd_paged_decode.cuh"

namespace ssd {

cudaError_t launch_paged_decode_8(const PagedDecodeParams& p, int head_dim, int sms, cudaStream_t st) {
  if (p.bf16)
    return head_dim == 128 ? paged::launch_paged_format<128, kPagedE4m3>(p, sms, st) : paged::launch_paged_format<64, kPagedE4m3>(p, sms, st);
  return head_dim == 128 ? paged::launch_paged_format<128, kPagedE4m3Fine>(p, sms, st) : paged::launch_paged_format<64, kPagedE4m3Fine>(p, sms, st);
}

}  // namespace ssd
