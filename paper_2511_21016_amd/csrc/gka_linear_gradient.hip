// Linear attention with a decay for each head, the ends of the backward pass: the gradient of the decays from the dot products
// that the walks leave, and the gradient at an initial state that several sequences share.
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace {

// The gradient of a gate is <dS_t, S_{t-1}>. Times the gate it is what the tokens from t on read of the states before t,
//   gate_t dgate_t = L_t = x_t + L_{t+1},  x_t = sum_g q_t . dq_t - k_t . dk_t,  L_T = <dS_final, S_T>,
// a sum over numbers that the walks leave anyhow. But it is a difference of terms of any size whose error, float32's, L_t / gate_t
// multiplies: a gate of 1e-8 would get 182 for a derivative of 6.1. So this form serves gates from kSmallGate = 2^-4 on (and its error
// grows 16 times at most); the tokens of a chunk that holds a smaller one, which no error may be divided by, get the inner
// product from the states around the chunk (gka_linear_small_gates.hip), and the sum of L starts anew before it with theirs.
// A gate of at most exp(-100) wipes the state: its own gradient is written as 0, and L_t is 0 there.
//
// L: a workgroup takes up to 4096 tokens of a (sequence, kv head), four consecutive ones to a thread, joined by a scan over
// the threads in float64; of longer sequences a first launch (SUMS) leaves what each part adds up to. 64 heads x 4096 tokens: 14 us for
// 6 MiB, bound by the latency of one chain (gates and results of a head lie H_kv apart).
constexpr int kThreads = 1024, kRun = 4, kPart = kThreads * kRun;

template <bool SUMS>
__global__ __launch_bounds__(kThreads) void linear_gate_kernel(LinearGateArgs a)
{
    // a run of tokens takes what comes from behind it, c, to sum + (open ? c : 0)
    __shared__ double wave_sums[kThreads / 64];
    __shared__ int wave_open[kThreads / 64];
    const int pair = blockIdx.x % (a.B * a.Hkv), part = blockIdx.x / (a.B * a.Hkv), n_pairs = a.B * a.Hkv;
    const int parts = (a.T + kPart - 1) / kPart;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int t0 = part * kPart + tid * kRun;
    // (a thread's tokens lie in one chunk)
    const int64_t chunk = (int64_t)pair * ((a.T + a.chunk - 1) / a.chunk) + min(t0, a.T - 1) / a.chunk;
    const bool small = t0 < a.T && a.small_gates[chunk] != 0;
    // (tokens behind the last one read it again, so that all reads are under way at once, and are then left out)
    float gate[kRun];
    double x[kRun];
    int at[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        at[i] = min(t0 + i, a.T - 1);
        gate[i] = a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + at[i]) * a.Hkv + h];
        x[i] = 0.0;
    }
    for (int s = 0; s < a.q_slices; ++s)
        for (int g = 0; g < a.G; ++g)
#pragma unroll
            for (int i = 0; i < kRun; ++i) x[i] += a.q_dq[(((int64_t)s * n_pairs + pair) * a.G + g) * a.T + at[i]];
    for (int s = 0; s < a.k_slices; ++s)
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] -= a.k_dk[((int64_t)s * n_pairs + pair) * a.T + at[i]];
#pragma unroll
    for (int i = 0; i < kRun; ++i)
        if (t0 + i >= a.T) {
            gate[i] = 1.0f;
            x[i] = 0.0;
        }
    double sum = 0.0;
    int open = 1;
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        sum += x[i];
        if (!(gate[i] > kWipingGate)) {
            sum = 0.0;
            open = 0;
        }
    }
    if (small) {
        sum = t0 % a.chunk == 0 ? a.chunk_first[chunk] : 0.0;
        open = 0;
    }
    // this thread's run with those of the threads behind it in the wave
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const double s = __shfl_down(sum, off, 64);
        const int o = __shfl_down(open, off, 64);
        if (lane + off < 64 && open) {
            sum += s;
            open = o;
        }
    }
    if (lane == 0) {
        wave_sums[w] = sum;
        wave_open[w] = open;
    }
    __syncthreads();
    if constexpr (SUMS) {
        if (tid == 0) {
            double all = 0.0;
            int through = 1;
            for (int i = kThreads / 64 - 1; i >= 0; --i) {
                all = wave_sums[i] + (wave_open[i] ? all : 0.0);
                through &= wave_open[i];
            }
            a.part_sums[(int64_t)pair * parts + part] = all;
            a.part_open[(int64_t)pair * parts + part] = through;
        }
        return;
    }
    // what comes from behind this wave
    double c = 0.0;
    if (a.state_dot)
        for (int s = 0; s < a.q_slices; ++s) c += a.state_dot[(int64_t)s * n_pairs + pair];
    for (int i = parts - 1; i > part; --i) {
        const int64_t at = (int64_t)pair * parts + i;
        c = a.part_sums[at] + (a.part_open[at] ? c : 0.0);
    }
    for (int i = kThreads / 64 - 1; i > w; --i) c = wave_sums[i] + (wave_open[i] ? c : 0.0);
    // ... and behind this thread
    const double s1 = __shfl_down(sum, 1, 64);
    const int o1 = __shfl_down(open, 1, 64);
    if (lane < 63) c = s1 + (o1 ? c : 0.0);
    double total = 0.0;
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        const int t = t0 + i;
        if (t >= a.T || small) continue;
        c += x[i];
        double d = c / (double)gate[i];
        if (!(gate[i] > kWipingGate)) c = d = 0.0;
        if (!a.gate_per_head) a.dgate[((int64_t)b * a.T + t) * a.Hkv + h] = (float)d;
        total += d;
    }
    if (a.gate_per_head) {
#pragma unroll
        for (int off = 32; off > 0; off /= 2) total += __shfl_xor(total, off, 64);
        __syncthreads();
        if (lane == 0) wave_sums[w] = total;
        __syncthreads();
        if (tid == 0) {
            double all = 0.0;
            for (int i = 0; i < kThreads / 64; ++i) all += wave_sums[i];
            a.per_part[(int64_t)pair * parts + part] = all;
        }
    }
}

__global__ __launch_bounds__(64) void linear_gate_heads_kernel(LinearGateArgs a)
{
    const int h = blockIdx.x * 64 + threadIdx.x;
    if (h >= a.Hkv) return;
    const int parts = (a.T + kPart - 1) / kPart;
    const int chunks = (a.T + a.chunk - 1) / a.chunk;
    const bool small = small_gate(a.gate[h]);      // (of all chunks)
    const int n = small ? chunks : parts;
    const double *from = small ? a.per_chunk : a.per_part;
    double x = 0.0;
    for (int b = 0; b < a.B; ++b)
        for (int i = 0; i < n; ++i) x += from[((int64_t)b * a.Hkv + h) * n + i];
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

size_t linear_gate_workspace_bytes(int64_t pairs, int T, int chunk)
{
    const int64_t parts = ((int64_t)T + kPart - 1) / kPart, chunks = ((int64_t)T + chunk - 1) / chunk;
    return (size_t)(pairs * parts) * (2 * sizeof(double) + sizeof(int)) + (size_t)(pairs * chunks) * 2 * sizeof(double);
}

hipError_t launch_linear_gate(const LinearGateArgs &a0, bool bf16, void *workspace, hipStream_t stream)
{
    LinearGateArgs a = a0;
    const int64_t pairs = (int64_t)a.B * a.Hkv, parts = ((int64_t)a.T + kPart - 1) / kPart, chunks = ((int64_t)a.T + a.chunk - 1) / a.chunk;
    if (pairs * parts > 0x7fffffff) return hipErrorInvalidValue;
    a.part_sums = (double *)workspace;
    a.per_part = a.part_sums + pairs * parts;
    a.chunk_first = a.per_part + pairs * parts;
    a.per_chunk = a.chunk_first + pairs * chunks;
    a.part_open = (int *)(a.per_chunk + pairs * chunks);
    hipError_t e = launch_linear_small_gates(a, bf16, stream);
    if (e != hipSuccess) return e;
    if (parts > 1) {
        hipLaunchKernelGGL(linear_gate_kernel<true>, dim3((unsigned)(pairs * parts)), dim3(kThreads), 0, stream, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(linear_gate_kernel<false>, dim3((unsigned)(pairs * parts)), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
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
