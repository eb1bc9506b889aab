// The walks of the backward pass for float32 tensors: products on the float32 MFMA, 32 tokens per chunk;
// up to 128 v-features (the k-features of the walks of dq and dk).
#include "gka_linear_walk.hpp"

namespace gka {
hipError_t launch_linear_backward_f32_128(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream)
{
    return linear::launch_backward_dk<linear::Tile16F32, 128>(dq, dk, dv, dv_alike, stream);
}
}  // namespace gka
