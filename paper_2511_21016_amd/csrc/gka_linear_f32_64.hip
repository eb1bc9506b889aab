// The walks over whole sequences for float32 tensors: products on the float32 MFMA, 32 tokens per chunk;
// up to 64 k-features: forward pass and dv.
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_forward_f32_64(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_forward_dk<linear::Tile16F32, 64>(a, stream); }
hipError_t launch_linear_values_f32_64(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_values_dk<linear::Tile16F32, 64>(a, stream); }
}  // namespace gka
