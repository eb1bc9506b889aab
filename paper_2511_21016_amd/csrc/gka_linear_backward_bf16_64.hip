// The walks of the backward pass for bfloat16 tensors: products on the bf16 MFMA, 64 tokens per chunk;
// up to 64 v-features (the k-features of the walks of dq and dk).
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_backward_bf16_64(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream)
{
    return linear::launch_backward_dk<linear::Tile16BF16, 64>(dq, dk, dv, dv_alike, stream);
}
}  // namespace gka
