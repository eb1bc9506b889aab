// The walks over whole sequences for bfloat16 tensors: products on the bf16 MFMA, 64 tokens per chunk;
// up to 64 k-features: forward pass and dv.
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_forward_bf16_64(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_forward_dk<linear::Tile16BF16, 64>(a, stream); }
hipError_t launch_linear_values_bf16_64(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_values_dk<linear::Tile16BF16, 64>(a, stream); }
}  // namespace gka
