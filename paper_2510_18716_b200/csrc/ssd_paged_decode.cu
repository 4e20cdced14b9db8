// The paged cache's attention over 16-bit rows (the kernel is in ssd_paged_decode.cuh).
#include "ssd_paged_decode.cuh"

namespace ssd {

size_t paged_max_workers(int sms) { return (size_t)sms * (paged::kWarps8 > paged::kWarps16 ? paged::kWarps8 : paged::kWarps16); }

cudaError_t launch_paged_decode_16(const PagedDecodeParams& p, int head_dim, int sms, cudaStream_t st) {
  if (p.bf16)
    return head_dim == 128 ? paged::launch_paged_format<128, kPagedBf16>(p, sms, st) : paged::launch_paged_format<64, kPagedBf16>(p, sms, st);
  return head_dim == 128 ? paged::launch_paged_format<128, kPagedFp16>(p, sms, st) : paged::launch_paged_format<64, kPagedFp16>(p, sms, st);
}

}  // namespace ssd
