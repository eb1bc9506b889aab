// The walk over whole sequences for bfloat16 tensors: products on the bf16 MFMA, 64 tokens per chunk;
// up to 64 k-features.
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_walk_bf16_64(const LinearWalkArgs &a, hipStream_t stream) { return linear::launch_walk_dk<linear::Tile16BF16, 64>(a, stream); }
}  // namespace gka
