// Linear attention with a decay for each head, backward pass: gradients of the gates in chunks that hold a small one.
//
// The gradient is <dS_t, S_{t-1}>. With S the state before the chunk's first token, D = dS behind its last one, and reader C - the
// end of the chunk - and source -1 - its start - beside the tokens,
//   dgate_t = sum_{s < t <= u} (gate_{s+1} .. gate_{t-1}) A[u, s] (gate_{t+1} .. gate_u),
//   A[u, s] = sum_g (q_u . k_s)(dy_u . v_s),   A[u, -1] = sum_g dy_u^T S q_u,   A[C, s] = v_s^T D k_s,   A[C, -1] = <D, S>:
// nothing is divided by gate_t. From the last token on X_t[s] = A[t, s] + gate_{t+1} X_{t+1}[s] collects the readers, a lane to each
// source. Gates that wipe leave out what lies on their other side, whatever it is.
//
// The walks leave S and D of these chunks alone, in the order in which they hold them. bf16 tensors: products on the bf16 MFMA, rows as
// they are, states in three pieces; float32: on the float32 MFMA. A workgroup, one to a CU, looks at every gridDim-th chunk;
// where none has small gates, the launch takes 4 us (1024 workgroups, four rounds of them: 12). Bound by one chunk's chain of reads, products and readers, 15 us (bf16, d 128: staging and A[u, s]
// 3 us, the states 7, the readers 5) with one workgroup on a CU; all chunks of 64 heads x 4096 tokens: 390 us. Rows of q, k, v,
// dy come through LDS: read where they are needed, 32 bytes of 16 rows at a time, they took three times as long.
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace {

// Features with padding, and bytes from row to row in LDS (16 more: neighbouring rows lie in other banks).
__host__ __device__ __forceinline__ int padded_features(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
__host__ __device__ __forceinline__ int small_gates_pitch(const LinearGateArgs &a, int element)
{
    return padded_features(a.dk > a.dv ? a.dk : a.dv) * element + 16;
}

template <bool BF16>
__global__ __launch_bounds__(512) void linear_small_gates_kernel(LinearGateArgs a)
{
    typedef std::conditional_t<BF16, IOBF16, IOF32> IO;
    typedef typename IO::type elem_t;
    typedef std::conditional_t<BF16, u16x8, f32x4> piece_t;       // 16 bytes of a row
    constexpr int C = BF16 ? 64 : 32, TB = C / 16, WAVES = 8, ROW = C + 1, E = BF16 ? 8 : 4;
    __shared__ float sA[C * ROW];                  // A[u, s], then what source s adds to dgate_u
    __shared__ float sRead[WAVES][C], sSource[WAVES][C], sStart[C];       // the waves' parts of A[u, -1] and A[C, s]; what source -1 adds
    __shared__ double sStates[WAVES], sPart[WAVES][64], sPartStart[WAVES], sThrough[WAVES];
    __shared__ uint64_t sFound[WAVES];
    // rows of k, v and of a head's q, dy, padded with zeros to whole tiles and to C tokens
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int pitch = small_gates_pitch(a, sizeof(elem_t));
    unsigned char *sK = smem, *sV = sK + C * pitch, *sQ = sV + C * pitch, *sDy = sQ + C * pitch;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int chunks = (a.T + C - 1) / C;
    const int64_t total = (int64_t)a.B * a.Hkv * chunks;
    const int NW = a.state_slice / 16, NJ = a.state_dk / 16;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    auto mma_f32 = [](f32x4 x, f32x4 y, f32x4 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    };

    auto gradients = [&](int64_t at) {
        const int64_t pair = at / chunks;
        const int b = (int)(pair / a.Hkv), h = (int)(pair % a.Hkv), chunk = (int)(at % chunks), t0 = chunk * C;
        const int count = min(C, a.T - t0);
        // two tensors' rows of a head, all reads under way at once
        auto stage = [&](const RowTensor &x, int dx, unsigned char *to_x, const RowTensor &y, int dy, unsigned char *to_y, int head) {
            constexpr int MOST = C * 256 / E / 512;
            piece_t p[2][MOST];
            auto each = [&](auto use) {
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const int shift = __builtin_ctz(padded_features(side ? dy : dx) / E);
#pragma unroll
                    for (int i = 0; i < MOST; ++i) {
                        const int at = tid + 512 * i;
                        if (at < C << shift) use(side, i, at >> shift, at & ((1 << shift) - 1));
                    }
                }
            };
            each([&](int side, int i, int t, int column) {
                const RowTensor &from = side ? y : x;
                p[side][i] = piece_t{};
                if (t < count && E * column < (side ? dy : dx))
                    p[side][i] = *(const piece_t *)((const elem_t *)from.p + b * from.sb + (int64_t)(t0 + t) * from.st + head * from.sh + E * column);
            });
            each([&](int side, int i, int t, int column) { *(piece_t *)((side ? to_y : to_x) + t * pitch + 16 * column) = p[side][i]; });
        };
        // sum over the features of rows u and s, 16 of each: rows u on the accumulator's rows
        auto products = [&](const unsigned char *u, const unsigned char *s, int d) {
            f32x4 c = zero;
            for (int f = 0; f < d; f += 4 * E) {
                const piece_t x = *(const piece_t *)(u + n * pitch + (f + E * kg) * sizeof(elem_t));
                const piece_t y = *(const piece_t *)(s + n * pitch + (f + E * kg) * sizeof(elem_t));
                if constexpr (BF16) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
                else c = mma_f32(x, y, c);
            }
            return c;
        };
        // adds up over the features (left^T state)(right) of every token, of the state's column tile j. Tile (j, i): d_k features
        // 16 j + n, d_v features 16 i + 4 kg + r; FLY at a time. `with`: the other state, whose product with this one is added up, too
        constexpr int FLY = 4;
        double states = 0.0;
        auto through = [&](const float *state, const float *with, const unsigned char *left, const unsigned char *right, int j,
                           float (&part)[TB][4]) {
            f32x4 z[TB];
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) z[tb] = zero;
#pragma unroll 1
            for (int i0 = 0; 16 * i0 < a.dv; i0 += FLY) {           // (tiles behind d_v: the state's padding, zeros)
                f32x4 x[FLY];
#pragma unroll
                for (int i = 0; i < FLY; ++i) x[i] = *(const f32x4 *)(state + (i0 + i) * 256);
                if (with) {
                    f32x4 y[FLY];
#pragma unroll
                    for (int i = 0; i < FLY; ++i) y[i] = *(const f32x4 *)(with + (i0 + i) * 256);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < FLY; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) states += (double)x[i][e] * (double)y[i][e];
                }
                const unsigned char *rows = left + n * pitch + (16 * i0 + 4 * kg) * sizeof(elem_t);
#pragma unroll
                for (int i = 0; i < FLY; i += 2) {
                    if constexpr (BF16) {
                        float rest[8] = {x[i][0], x[i][1], x[i][2], x[i][3], x[i + 1][0], x[i + 1][1], x[i + 1][2], x[i + 1][3]}, back[8];
                        bf16x8 f[3];
#pragma unroll
                        for (int piece = 0; piece < 3; ++piece) {
                            f[piece] = MmaBF16::pack(rest);
                            MmaBF16::unpack(f[piece], back);
#pragma unroll
                            for (int e = 0; e < 8; ++e) rest[e] -= back[e];
                        }
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) {
                            const unsigned char *row = rows + 16 * tb * pitch + 32 * i;
                            const u16x4 lo = *(const u16x4 *)row, hi = *(const u16x4 *)(row + 32);
                            const u16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
                            for (int piece = 0; piece < 3; ++piece)
                                z[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, both), f[piece], z[tb], 0, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int tb = 0; tb < TB; ++tb)
                                z[tb] = mma_f32(*(const f32x4 *)(rows + 16 * tb * pitch + 64 * (i + half)), x[i + half], z[tb]);
                    }
                }
            }
#pragma unroll
            for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    part[tb][r] += z[tb][r] * IO::load(right + (16 * tb + 4 * kg + r) * pitch, 16 * j + n);
        };
        // ---- A[u, s] for s <= u, 16 x 16 of them to a wave at a time; A[u, -1], A[C, s] and A[C, -1], a wave's column tiles
        constexpr int UNITS = TB * (TB + 1) / 2, MINE = (UNITS + WAVES - 1) / WAVES;
        f32x4 sum[MINE];
#pragma unroll
        for (int i = 0; i < MINE; ++i) sum[i] = zero;
        float read[TB][4] = {}, source[TB][4] = {};
        auto block_of = [](int unit) { return unit < 1 ? 0 : unit < 3 ? 1 : unit < 6 ? 2 : 3; };
        for (int g = 0; g < a.G; ++g) {
            if (g == 0) stage(a.k, a.dk, sK, a.v, a.dv, sV, h);
            else __syncthreads();
            stage(a.q, a.dk, sQ, a.dy, a.dv, sDy, h * a.G + g);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                const int unit = w + WAVES * i;
                if (unit >= UNITS) break;
                const int ub = block_of(unit), sb = unit - ub * (ub + 1) / 2;
                sum[i] += products(sQ + 16 * ub * pitch, sK + 16 * sb * pitch, a.dk) * products(sDy + 16 * ub * pitch, sV + 16 * sb * pitch, a.dv);
            }
            for (int j = w; 16 * j < a.dk; j += WAVES) {
                const int64_t tiles = ((pair * a.q_slices + j / NW) * chunks + chunk) * NW * NJ * 256 + ((j % NW) * NJ * 64 + lane) * 4;
                const float *S = a.S_chunk + tiles;
                if (g == 0) through(a.dS_chunk + tiles, S, sV, sK, j, source);
                through(S, nullptr, sDy, sQ, j, read);
            }
        }
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int unit = w + WAVES * i;
            if (unit >= UNITS) break;
            const int ub = block_of(unit), sb = unit - ub * (ub + 1) / 2;
#pragma unroll
            for (int r = 0; r < 4; ++r) sA[(16 * ub + 4 * kg + r) * ROW + 16 * sb + n] = sum[i][r];
        }
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = sum_over_lanes<16>(read[tb][r]), y = sum_over_lanes<16>(source[tb][r]);
                if (n == 0) sRead[w][16 * tb + 4 * kg + r] = x;
                if (n == 0) sSource[w][16 * tb + 4 * kg + r] = y;
            }
        states = lane63_f64(wave_inclusive_scan_f64(states));
        if (lane == 0) sStates[w] = states;
        __syncthreads();

        // ---- the readers from the last token on, lane s: source s. A wave takes PART tokens: what its own readers come to, then, with what
        // the waves behind it have, the sums themselves
        constexpr int PART = C / WAVES;
        auto gate_of = [&](int t) { return a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + t0 + t) * a.Hkv + h]; };
        auto broadcast = [&](double x, int from) {
            return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), from), __builtin_amdgcn_readlane(__double2loint(x), from));
        };
        const int s = lane < C ? lane : C - 1;
        const float gate = lane < count ? gate_of(lane) : 1.0f;
        const double G = wave_inclusive_scan_f64(log2_gate_f64(gate));
        const uint64_t wiping = __ballot(!(gate > kWipingGate));
        float behind = __shfl_down(gate, 1, 64);   // the gate of the token behind lane's; 0: nothing comes through
        if (lane >= count - 1) behind = lane == count - 1 && t0 + count < a.T ? gate_of(count) : 1.0f;
        if (!(behind > kWipingGate)) behind = 0.0f;
        double reads = 0.0, from_source = 0.0, from_start = 0.0, through_part = 1.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) reads += sRead[i][s];
        float row[PART];
#pragma unroll
        for (int i = PART - 1; i >= 0; --i) {
            const int t = w * PART + i;
            const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(behind), t));
            row[i] = sA[t * ROW + s];
            from_source = (g != 0.0f ? g * from_source : 0.0) + row[i];
            from_start = (g != 0.0f ? g * from_start : 0.0) + broadcast(reads, t);
            through_part *= g;
        }
        sPart[w][lane] = from_source;
        if (lane == 0) sPartStart[w] = from_start;
        if (lane == 0) sThrough[w] = through_part;
        __syncthreads();
        from_source = from_start = 0.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            from_source += sSource[i][s];
            from_start += sStates[i];
        }
        for (int i = WAVES - 1; i > w; --i) {
            const double g = sThrough[i];
            from_source = (g != 0.0 ? g * from_source : 0.0) + sPart[i][lane];
            from_start = (g != 0.0 ? g * from_start : 0.0) + sPartStart[i];
        }
#pragma unroll
        for (int i = PART - 1; i >= 0; --i) {
            const int t = w * PART + i;
            const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(behind), t));
            from_source = (g != 0.0f ? g * from_source : 0.0) + row[i];
            from_start = (g != 0.0f ? g * from_start : 0.0) + broadcast(reads, t);
            const uint64_t before = wiping & ((1ull << t) - 1);
            const int first = before ? 63 - __builtin_clzll(before) : -1;        // the sources that the tokens before t have left
            const double G1 = t > 0 ? broadcast(G, t > 0 ? t - 1 : 0) : 0.0;
            const float weight = __builtin_amdgcn_exp2f((float)(G1 - G));
            if (lane < C) sA[t * ROW + lane] = lane >= first && lane < t ? (float)(from_source * weight) : 0.0f;
            if (lane == 0) sStart[t] = first < 0 ? (float)(from_start * __builtin_amdgcn_exp2f((float)G1)) : 0.0f;
        }
        __syncthreads();
        if (w == 0) {
            double sum = 0.0;
            if (lane < count && gate > kWipingGate) {
                sum = sStart[lane];
#pragma unroll 16
                for (int i = 0; i < C; ++i) sum += sA[s * ROW + i];
            }
            if (!a.gate_per_head && lane < count) a.dgate[((int64_t)b * a.T + t0 + lane) * a.Hkv + h] = (float)sum;
            if (lane == 0) a.chunk_first[at] = sum * gate;
            sum = lane63_f64(wave_inclusive_scan_f64(sum));
            if (lane == 0) a.per_chunk[at] = sum;
        }
        __syncthreads();
    };

    for (int64_t base = blockIdx.x; base < total; base += (int64_t)64 * WAVES * gridDim.x) {
        const int64_t mine = base + (int64_t)tid * gridDim.x;
        const uint64_t found = __ballot(mine < total && a.small_gates[mine] != 0);
        if (lane == 0) sFound[w] = found;
        __syncthreads();
        for (int i = 0; i < WAVES; ++i)
            for (uint64_t left = sFound[i]; left != 0; left &= left - 1)
                gradients(base + (int64_t)(64 * i + __builtin_ctzll(left)) * gridDim.x);
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_linear_small_gates(const LinearGateArgs &a, bool bf16, hipStream_t stream)
{
    const int64_t chunks = (int64_t)a.B * a.Hkv * (((int64_t)a.T + a.chunk - 1) / a.chunk);
    const dim3 grid((unsigned)(chunks < kComputeUnits ? chunks : kComputeUnits));
    const size_t lds = (size_t)4 * a.chunk * small_gates_pitch(a, bf16 ? 2 : 4);
    static bool raised[kMaxLdsDevices] = {};
    constexpr size_t most = (size_t)4 * 64 * (256 * 2 + 16);       // (float32: 32 rows of 256 x 4 + 16 bytes, less)
    const hipError_t e = raise_lds_limits(raised, {{(const void *)linear_small_gates_kernel<true>, most}, {(const void *)linear_small_gates_kernel<false>, most}});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(bf16 ? linear_small_gates_kernel<true> : linear_small_gates_kernel<false>, grid, dim3(512), lds, stream, a);
    return hipGetLastError();
}

}  // namespace gka
