// Paged decode kernels, bf16 tensors: pages of elements, 8-bit and 4-bit codes.
#include "thk_paged_decode_impl.h"

namespace thk {
hipError_t launch_paged_decode_bf16(int bits, const PagedDecodeArgs &a, hipStream_t st) {
  return bits == 0 ? paged::launch<THK_BF16, 0>(a, st) : bits == 4 ? paged::launch<THK_BF16, 4>(a, st) : paged::launch<THK_BF16, 8>(a, st);
}
}  // namespace thk
