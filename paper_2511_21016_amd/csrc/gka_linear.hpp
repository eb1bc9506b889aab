// Linear attention with a decay for each head: argument blocks and launchers of its kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gka {

// A tensor of rows [B, T, heads, d]: element strides of batch, token and head; the d elements of a row are contiguous.
struct RowTensor {
    const void *p;
    int64_t sb, st, sh;
};

// Gates up to exp(-100) (to float32's last bits there) wipe the state. Small ones are those that the gradient of the decays is not divided
// by (gka_linear_gradient.hip).
constexpr float kWipingGate = 3.8e-44f, kSmallGate = 0.0625f;
__device__ __forceinline__ bool small_gate(float gate) { return gate > kWipingGate && gate < kSmallGate; }

// One walk over whole sequences: y_t = S_t q_t, S_t = gate_t S_{t-1} + sum over the sources v_t k_t^T, with S [dv, dk].
// With other tensors in the roles of q, k, v it is the forward pass and each of the three gradients (the tensors' own names
// on the right):
//   y   q -> q   k -> k   v -> v    forwards           dq  q -> dy  k -> v   v -> k    forwards, S transposed
//   dv  q -> k   k -> q   v -> dy   reverse            dk  q -> v   k -> dy  v -> q    reverse, S transposed
// A state belongs to one of the H_kv heads; n_q queries or n_src sources of a token share it (one of the two is 1).
// reverse: from the last token to the first, the gate of a token being that of the one behind it (of the last: 1). The chunks are the
// same, counted from the first token.
struct LinearWalkArgs {
    RowTensor q, k, v;            // heads: H_kv n_q, H_kv n_src, H_kv n_src; features dk, dk, dv
    RowTensor y;                  // H_kv n_q heads, dv features (written)
    const float *gate;            // [B, T, H_kv], or [H_kv] with gate_per_head
    int gate_per_head, reverse;
    int B, T, Hkv, n_q, n_src;
    int dk, dv;                   // multiples of 16 up to 256
    const float *init;            // [B / share, H_kv, dv, dk] or nullptr (zero)
    int share;                    // consecutive sequences with one initial state
    int transposed;               // init, final and state_dot_with are stored [dk, dv]
    float *final;                 // [B, H_kv, dv, dk] or nullptr: the state behind the last token
    int final_times_gate;         // ... times the gate of the tensors' token 0 (the gradient at the initial state)
    // what the gradient of the decays is made of (written where the pointers are not null, in the order [slices, B, H_kv, ...]):
    RowTensor dot_with;           // like y: dot_out [slices, B, H_kv, n_q, T] = dot_with . y, y before it is rounded
    double *dot_out;
    const float *state_dot_with;  // [B, H_kv, dv, dk]: state_dot_out [slices, B, H_kv] = its product with the last state
    double *state_dot_out;
    // ... and at small gates, with dot_out: the state before each chunk that holds one (in the order of seg_states, with chunks from the
    // front in the segments' place), and by the forward walk [B, H_kv, chunks] which ones those are
    float *chunk_states;
    int *small_gates;
    // plan
    int n_segs, seg_chunks;       // segments of the walk, chunks each
    int scanned;                  // a launch between turns what the segments add into the states that they start from (else each
                                  // segment adds up those before it)
    int slices;                   // of dv, a workgroup takes one
    float *seg_states;            // [B, H_kv, slices, n_segs, slice, DK] in the kernel's order: what each segment adds, then the
                                  // state that it starts from
    float *seg_decay;             // [B, H_kv, n_segs]; negative: wiped
    int seg_turned[3];            // not 0: seg_states are those of the walk with transposed states: its waves, tiles a wave, slices
};

// Tokens of a chunk, features of a slice and padded dk of the kernels for these sizes; floats of a segment's state.
struct LinearShape {
    int chunk, slice, padded_dk, slices;
    int64_t state_floats;
};
LinearShape linear_shape(bool bf16, int dk, int dv);
// The forward pass, and the three walks of the backward pass, with the summaries of their segments. dk's and dv's have the same
// segments; those of dv need seg_states and seg_decay of dk's.
hipError_t launch_linear_forward(const LinearWalkArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_linear_backward(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool bf16, hipStream_t stream);
// ... by type and padded_dk
hipError_t launch_linear_forward_bf16_64(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_bf16_64(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_bf16_64(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);
hipError_t launch_linear_forward_bf16_128(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_bf16_128(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_bf16_128(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);
hipError_t launch_linear_forward_bf16_256(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_bf16_256(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_bf16_256(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);
hipError_t launch_linear_forward_f32_64(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_f32_64(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_f32_64(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);
hipError_t launch_linear_forward_f32_128(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_f32_128(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_f32_128(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);
hipError_t launch_linear_forward_f32_256(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_values_f32_256(const LinearWalkArgs &a, hipStream_t stream);
hipError_t launch_linear_backward_f32_256(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream);

// The gradient of the decays, and the sum of gradients at shared initial states.
struct LinearGateArgs {
    const double *q_dq;           // [q_slices, B, H_kv, G, T]
    const double *k_dk;           // [k_slices, B, H_kv, T]
    const double *state_dot;      // [q_slices, B, H_kv] or nullptr
    int q_slices, k_slices, G;
    const float *gate;
    float *dgate;                 // [B, T, H_kv], or [H_kv] with gate_per_head
    int gate_per_head;
    int B, T, Hkv;
    // chunks with small gates
    RowTensor q, k, v, dy;
    int dk, dv, chunk;            // features; tokens of a chunk
    const int *small_gates;       // [B, H_kv, chunks]
    const float *S_chunk, *dS_chunk;   // [B, H_kv, slices, chunks] states: before the chunk's first token, dS behind its last one
    int state_slice, state_dk;    // of those: k-features of a slice (of all d_k), padded d_v
    double *part_sums, *per_part; // (carved from the workspace by the launcher)
    double *chunk_first, *per_chunk;
    int *part_open;
};
size_t linear_gate_workspace_bytes(int64_t pairs, int T, int chunk);
hipError_t launch_linear_small_gates(const LinearGateArgs &a, bool bf16, hipStream_t stream);
hipError_t launch_linear_gate(const LinearGateArgs &a, bool bf16, void *workspace, hipStream_t stream);
hipError_t launch_linear_state_sum(const float *per_sequence, float *out, int groups, int share, int64_t state_floats,
                                   hipStream_t stream);

// T tokens of the recurrence on stored states.
struct LinearDecodeArgs {
    const float *S_in;            // [B / share, H_kv, dv, dk]
    float *S_out;                 // [B, H_kv, dv, dk]; S_in's own buffer with share = 1
    RowTensor q, k, v, y;
    const float *gate;            // [B, T, H_kv] or [H_kv]
    int gate_per_head, share, B, T, Hkv, G, dk, dv;
};
hipError_t launch_linear_decode(const LinearDecodeArgs &a, bool bf16, hipStream_t stream);

// One token of sequences that continue a shared prefix.
struct LinearSharedArgs {
    const float *S;               // [B / share, H_kv, dv, dk]
    RowTensor q, k, v, y;         // one token per sequence (st unused)
    const float *gate;            // [B, H_kv] or [H_kv]
    void *k_cache, *v_cache;      // [B, N, H_kv, dk], [B, N, H_kv, dv]
    float *gate_cache;            // [B, N, H_kv], nullptr with gate_per_head
    const int32_t *lengths;       // [B]
    int gate_per_head, share, B, N, Hkv, G, dk, dv;
};
hipError_t launch_linear_shared(const LinearSharedArgs &a, bool bf16, hipStream_t stream);

}  // namespace gka
