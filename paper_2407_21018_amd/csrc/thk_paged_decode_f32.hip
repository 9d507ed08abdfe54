// Paged decode kernels, fp32 tensors: pages of elements, 8-bit and 4-bit codes.
#include "thk_paged_decode_impl.h"

namespace thk {
hipError_t launch_paged_decode_f32(int bits, const PagedDecodeArgs &a, hipStream_t st) {
  return bits == 0 ? paged::launch<THK_F32, 0>(a, st) : bits == 4 ? paged::launch<THK_F32, 4>(a, st) : paged::launch<THK_F32, 8>(a, st);
}
}  // namespace thk
