// Linear attention with a decay for each head, the ends of the backward pass: the gradient of the decays from the dot products
// that the walks leave, and the gradient at an initial state that several sequences share.
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace {

// dL/dlog(gate_t) is what the tokens from t on read of the states before t:
//   L_t = x_t + L_{t+1},  x_t = sum_g q_t . dq_t - k_t . dk_t,  L_T = <dS_final, S_T>;   dgate_t = L_t / gate_t.
// A gate of at most exp(-100) wipes the state (L_t = 0 there): the sum starts anew before it and its own gradient is
// written as 0. One workgroup to a (sequence, kv head): a thread sums a run of consecutive tokens, runs are joined by a scan
// over the threads, all in float64.
constexpr int kThreads = 256;
__global__ __launch_bounds__(kThreads) void linear_gate_kernel(LinearGateArgs a)
{
    __shared__ double sum[2][kThreads];
    __shared__ int open[2][kThreads];
    const int pair = blockIdx.x, n_pairs = a.B * a.Hkv;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    const int tid = threadIdx.x;
    const int run = (a.T + kThreads - 1) / kThreads;
    const int t0 = min(tid * run, a.T), t1 = min(t0 + run, a.T);
    const float wiped = 3.8e-44f;                  // exp(-100) to float32's last bits there
    auto gate_at = [&](int t) { return a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + t) * a.Hkv + h]; };
    auto x_at = [&](int t) {
        double x = 0.0;
        for (int s = 0; s < a.q_slices; ++s)
            for (int i = 0; i < a.G; ++i) x += (double)a.q_dq[(((int64_t)s * n_pairs + pair) * a.G + i) * a.T + t];
        for (int s = 0; s < a.k_slices; ++s) x -= (double)a.k_dk[((int64_t)s * n_pairs + pair) * a.T + t];
        return x;
    };
    // a run takes what comes from behind, c, to sum + (open ? c : 0)
    double mine = 0.0;
    int mine_open = 1;
    for (int t = t1 - 1; t >= t0; --t) {
        mine += x_at(t);
        if (!(gate_at(t) > wiped)) {
            mine = 0.0;
            mine_open = 0;
        }
    }
    sum[0][tid] = mine;
    open[0][tid] = mine_open;
    __syncthreads();
    int from = 0;
    for (int off = 1; off < kThreads; off *= 2) {
        double s = sum[from][tid];
        int o = open[from][tid];
        if (o && tid + off < kThreads) {
            s += sum[from][tid + off];
            o = open[from][tid + off];
        }
        sum[1 - from][tid] = s;
        open[1 - from][tid] = o;
        from = 1 - from;
        __syncthreads();
    }
    double end = 0.0;
    if (a.state_dot)
        for (int s = 0; s < a.q_slices; ++s) end += (double)a.state_dot[(int64_t)s * n_pairs + pair];
    double c = end;
    if (tid + 1 < kThreads) c = sum[from][tid + 1] + (open[from][tid + 1] ? end : 0.0);
    double total = 0.0;
    for (int t = t1 - 1; t >= t0; --t) {
        const float gate = gate_at(t);
        c += x_at(t);
        double d = c / (double)gate;
        if (!(gate > wiped)) c = d = 0.0;
        if (!a.gate_per_head) a.dgate[((int64_t)b * a.T + t) * a.Hkv + h] = (float)d;
        total += d;
    }
    if (a.gate_per_head) {
        __syncthreads();
        sum[0][tid] = total;
        __syncthreads();
        for (int off = kThreads / 2; off > 0; off /= 2) {
            if (tid < off) sum[0][tid] += sum[0][tid + off];
            __syncthreads();
        }
        if (tid == 0) a.per_pair[pair] = sum[0][0];
    }
}

__global__ __launch_bounds__(64) void linear_gate_heads_kernel(LinearGateArgs a)
{
    const int h = blockIdx.x * 64 + threadIdx.x;
    if (h >= a.Hkv) return;
    double x = 0.0;
    for (int b = 0; b < a.B; ++b) x += a.per_pair[(int64_t)b * a.Hkv + h];
    a.dgate[h] = (float)x;
}

__global__ __launch_bounds__(256) void linear_state_sum_kernel(const float *per_sequence, float *out, int share, int64_t state_floats)
{
    const int64_t blocks = (state_floats + 1023) / 1024;
    const int64_t group = blockIdx.x / blocks, at = (blockIdx.x % blocks * 256 + threadIdx.x) * 4;
    if (at >= state_floats) return;
    const float *p = per_sequence + group * share * state_floats + at;
    f32x4 x = *(const f32x4 *)p;
    for (int i = 1; i < share; ++i) x += *(const f32x4 *)(p + i * state_floats);
    *(f32x4 *)(out + group * state_floats + at) = x;
}

}  // namespace

hipError_t launch_linear_gate(const LinearGateArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(linear_gate_kernel, dim3(a.B * a.Hkv), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.gate_per_head) return e;
    hipLaunchKernelGGL(linear_gate_heads_kernel, dim3((a.Hkv + 63) / 64), dim3(64), 0, stream, a);
    return hipGetLastError();
}

// state_floats: of all heads of a sequence, a multiple of 4
hipError_t launch_linear_state_sum(const float *per_sequence, float *out, int groups, int share, int64_t state_floats, hipStream_t stream)
{
    const int64_t blocks = groups * ((state_floats + 1023) / 1024);
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(linear_state_sum_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, per_sequence, out, share, state_floats);
    return hipGetLastError();
}

}  // namespace gka
