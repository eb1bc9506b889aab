// The walk over whole sequences for float32 tensors: products on the float32 MFMA, 32 tokens per chunk;
// up to 256 k-features.
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_walk_f32_256(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_walk_dk<linear::Tile16F32, 256>(a, stream); }
}  // namespace gka
