// Linear attention with a decay for each head, single tokens:
//   decode  a few tokens (usually one) of S_t = gate_t S_{t-1} + v_t k_t^T, y_t = S_t q_t on stored states;
//   shared  one token of each of many sequences that continue a common prefix. The prefix is one state S for all of them; the
//           n tokens behind it lie in a cache of the sequence's own keys, values and gates:
//             y = zeta S q + sum_j M_j (k_j . q) v_j,   M_j = gate_{j+1} .. gate_n,   zeta = gate_1 .. gate_n.
// Both are bound by the bytes that they have to move: decode 8 dk dv for a state in and out, shared the cached rows
// (a state is read by every workgroup of a prefix, from the L2 cache after the first).
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// ---- decode ----------------------------------------------------------------------------------------------------------
// A row of the state (one v-feature) lies across LPR lanes, four k-features on each; a thread holds NR rows, a workgroup
// (256 / LPR) NR of them. The state crosses memory once, whatever the number of tokens.
template <bool BF16, int LPR, int NR>
__global__ __launch_bounds__(256) void linear_decode_kernel(LinearDecodeArgs a)
{
    typedef std::conditional_t<BF16, IOBF16, IOF32> IO;
    typedef typename IO::type elem_t;
    constexpr int RP = 256 / LPR;                  // rows a workgroup covers at once
    const int blocks = (a.dv + RP * NR - 1) / (RP * NR);
    const int64_t pair = blockIdx.x / blocks;
    const int row0 = (int)(blockIdx.x % blocks) * RP * NR + (int)(threadIdx.x / LPR);
    const int b = (int)(pair / a.Hkv), h = (int)(pair % a.Hkv);
    const int l = threadIdx.x % LPR, col = 4 * l;
    const bool col_in = col < a.dk;
    const float *S0 = a.S_in + ((int64_t)(b / a.share) * a.Hkv + h) * a.dv * a.dk;
    f32x4 S[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = row0 + i * RP;
        S[i] = col_in && row < a.dv ? *(const f32x4 *)(S0 + (int64_t)row * a.dk + col) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int t = 0; t < a.T; ++t) {
        const elem_t *k = (const elem_t *)a.k.p + b * a.k.sb + t * a.k.st + h * a.k.sh;
        const elem_t *v = (const elem_t *)a.v.p + b * a.v.sb + t * a.v.st + h * a.v.sh;
        const float gate = a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + t) * a.Hkv + h];
        const f32x4 k4 = col_in ? IO::load4(k, col) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int row = row0 + i * RP;
            const float x = row < a.dv ? IO::load(v, row) : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) S[i][e] = gate * S[i][e] + x * k4[e];
        }
        for (int s = 0; s < a.G; ++s) {
            const int head = h * a.G + s;
            const elem_t *q = (const elem_t *)a.q.p + b * a.q.sb + t * a.q.st + head * a.q.sh;
            elem_t *y = (elem_t *)const_cast<void *>(a.y.p) + b * a.y.sb + t * a.y.st + head * a.y.sh;
            const f32x4 q4 = col_in ? IO::load4(q, col) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            float p[NR];
#pragma unroll
            for (int i = 0; i < NR; ++i) p[i] = (S[i][0] * q4[0] + S[i][1] * q4[1]) + (S[i][2] * q4[2] + S[i][3] * q4[3]);
            // sums over the LPR lanes of a row: while a lane holds several rows, the two lanes of an exchange keep a half each
            int n = NR;
#pragma unroll
            for (int off = LPR / 2; off > 0; off >>= 1) {
                if (n > 1) {
                    const bool upper = (l & off) != 0;
#pragma unroll
                    for (int i = 0; i < NR / 2; ++i) {
                        if (i >= n / 2) break;
                        const float send = upper ? p[i] : p[i + n / 2], keep = upper ? p[i + n / 2] : p[i];
                        p[i] = keep + __shfl_xor(send, off, 64);
                    }
                    n /= 2;
                } else {
                    p[0] += __shfl_xor(p[0], off, 64);
                }
            }
            constexpr int HELD = NR > LPR ? NR / LPR : 1, TWINS = NR > LPR ? 1 : LPR / NR;   // rows a lane holds, lanes that hold a row
            if (l % TWINS == 0) {
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    const int row = row0 + (l / TWINS * HELD + i) * RP;
                    if (row < a.dv) IO::store1(y, row, p[i]);
                }
            }
        }
    }
    float *S1 = a.S_out + pair * a.dv * a.dk;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = row0 + i * RP;
        if (col_in && row < a.dv) *(f32x4 *)(S1 + (int64_t)row * a.dk + col) = S[i];
    }
}

// ---- shared ----------------------------------------------------------------------------------------------------------
// A workgroup takes up to `ncol` columns of one (prefix, kv head): a column is a query head of a sequence, G of them to a
// sequence, one behind the other. First S q of all its columns on the matrix cores (S cut into two bf16 pieces, or float32),
// then each wave the cached tokens of its columns, up to four of one sequence at a time.
constexpr int kSharedCols = 32, kSharedHeads = 4;

template <bool BF16>
__global__ __launch_bounds__(256) void linear_shared_kernel(LinearSharedArgs a, int ncol, int lk, int lv)
{
    typedef std::conditional_t<BF16, IOBF16, IOF32> IO;
    typedef typename IO::type elem_t;
    constexpr int E = BF16 ? 8 : 4;                // elements of a 16-byte piece
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int ys = a.dv + 4;                       // floats of a column of S q
    float *sY = (float *)smem;
    float *sS = sY + ncol * ys;                    // [waves][kSharedHeads][64]
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, g = lane >> 5;
    const int64_t cols = (int64_t)a.share * a.G;
    const int tiles = (int)((cols + ncol - 1) / ncol);
    const int tile = blockIdx.x % tiles;
    const int h = blockIdx.x / tiles % a.Hkv;
    const int prefix = blockIdx.x / tiles / a.Hkv;
    const int64_t col0 = (int64_t)tile * ncol;
    const int my_cols = (int)(cols - col0 < ncol ? cols - col0 : ncol);
    const float *S = a.S + ((int64_t)prefix * a.Hkv + h) * a.dv * a.dk;
    auto row_of = [&](const RowTensor &x, int b, int head) { return (const elem_t *)x.p + b * x.sb + head * x.sh; };

    // ---- S q: wave w takes the 32-row blocks w, w + 4, ..
    {
        const int c = n < my_cols ? n : 0;         // (columns that do not exist repeat the first; their results are not read)
        const int64_t col = col0 + c;
        const elem_t *q = row_of(a.q, prefix * a.share + (int)(col / a.G), h * a.G + (int)(col % a.G));
        for (int rb = w; 32 * rb < a.dv; rb += 4) {
            f32x16 acc = zero16();
            const int row = 32 * rb + n;
            const bool in = row < a.dv;
            const float *s = S + (int64_t)(in ? row : 0) * a.dk;
            if constexpr (BF16) {
#pragma unroll 4
                for (int k0 = 0; k0 < a.dk; k0 += 16) {
                    const f32x4 x0 = *(const f32x4 *)(s + k0 + 8 * g), x1 = *(const f32x4 *)(s + k0 + 8 * g + 4);
                    const u32x4_t qv = *(const u32x4_t *)(q + k0 + 8 * g);
                    float x[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]}, back[8];
                    const bf16x8 hi = MmaBF16::pack(x), qf = __builtin_bit_cast(bf16x8, qv);
                    MmaBF16::unpack(hi, back);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] -= back[e];
                    acc = MmaBF16::mma(hi, qf, acc);
                    acc = MmaBF16::mma(MmaBF16::pack(x), qf, acc);
                }
            } else {
#pragma unroll 4
                for (int k0 = 0; k0 < a.dk; k0 += 8) {
                    const f32x4 x = *(const f32x4 *)(s + k0 + 4 * g), qv = *(const f32x4 *)(q + k0 + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc = MmaF32::mma(x[e], qv[e], acc);
                }
            }
            if (n < my_cols) {
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    if (32 * rb + 8 * q4 < a.dv)
                        *(f32x4 *)(sY + n * ys + 32 * rb + 8 * q4 + 4 * g) =
                            f32x4{acc[4 * q4], acc[4 * q4 + 1], acc[4 * q4 + 2], acc[4 * q4 + 3]};
            }
        }
    }
    __syncthreads();

    // ---- the cached tokens
    float *score = sS + w * kSharedHeads * 64;
    const int kl = lane % lk, kr = lane / lk, krows = 64 / lk;     // pieces of a key row across lk lanes
    const int vl = lane % lv, vr = lane / lv, vrows = 64 / lv;
    const bool k_in = E * kl < a.dk, v_in = E * vl < a.dv;
    const int per_wave = (ncol + 3) / 4;
    int c = w * per_wave;
    const int c_end = c + per_wave < my_cols ? c + per_wave : my_cols;
    while (c < c_end) {
        const int64_t col = col0 + c;
        const int b = prefix * a.share + (int)(col / a.G), head0 = (int)(col % a.G);
        int m = a.G - head0;                       // columns of this sequence, taken together
        m = m < c_end - c ? m : c_end - c;
        m = m < kSharedHeads ? m : kSharedHeads;
        const int len = a.lengths[b];
        if (len < 0 || len >= a.N) {               // an idle row of the batch: nothing of it is touched
            c += m;
            continue;
        }
        const elem_t *k_new = row_of(a.k, b, h), *v_new = row_of(a.v, b, h);
        const float gate_new = a.gate_per_head ? a.gate[h] : a.gate[(int64_t)b * a.Hkv + h];
        const int64_t cache_row = (int64_t)b * a.N * a.Hkv + h;     // + j Hkv: row of token j
        elem_t *kc = (elem_t *)a.k_cache + cache_row * a.dk, *vc = (elem_t *)a.v_cache + cache_row * a.dv;
        const int64_t kc_step = (int64_t)a.Hkv * a.dk, vc_step = (int64_t)a.Hkv * a.dv;
        if (head0 == 0) {                          // (once for a sequence: the new token goes into the cache)
            if (kr == 0 && k_in) *(u32x4_t *)(kc + len * kc_step + E * kl) = *(const u32x4_t *)(k_new + E * kl);
            if (vr == 0 && v_in) *(u32x4_t *)(vc + len * vc_step + E * vl) = *(const u32x4_t *)(v_new + E * vl);
            if (!a.gate_per_head && lane == 0) a.gate_cache[cache_row + (int64_t)len * a.Hkv] = gate_new;
        }
        float q[kSharedHeads][E], y[kSharedHeads][E];
#pragma unroll
        for (int i = 0; i < kSharedHeads; ++i) {
            const elem_t *row = row_of(a.q, b, h * a.G + head0 + (i < m ? i : 0));
#pragma unroll
            for (int e = 0; e < E; ++e) y[i][e] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const f32x4 x = k_in ? IO::load4(row, E * kl + e) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 4; ++j) q[i][e + j] = x[j];
            }
        }
        double behind = 0.0;                       // log2 decay over the tokens behind the tile
        for (int j0 = len / 64 * 64; j0 >= 0; j0 -= 64) {
            const int count = len + 1 - j0 < 64 ? len + 1 - j0 : 64;
            double lg = 0.0;
            if (lane < count) {
                const float gate = a.gate_per_head || j0 + lane == len ? gate_new : a.gate_cache[cache_row + (int64_t)(j0 + lane) * a.Hkv];
                lg = (double)log2_gate(gate);
            }
            const double G = wave_inclusive_scan_f64(lg), total = lane63_f64(G);
            const float weight = lane < count ? exp2f((float)(behind + (total - G))) : 0.0f;
            behind += total;
#pragma unroll 4
            for (int r = 0; r < count; r += krows) {
                const int j = j0 + r + kr;
                const elem_t *row = j < len ? kc + j * kc_step : k_new;
                const bool in = k_in && r + kr < count;
                float x[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f32x4 u = in ? IO::load4(row, E * kl + e) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[e + i] = u[i];
                }
#pragma unroll
                for (int i = 0; i < kSharedHeads; ++i) {
                    if (i >= m) break;
                    float dot = 0.0f;
#pragma unroll
                    for (int e = 0; e < E; ++e) dot += x[e] * q[i][e];
                    for (int off = lk / 2; off > 0; off >>= 1) dot += __shfl_xor(dot, off, 64);
                    if (kl == 0 && r + kr < 64) score[i * 64 + r + kr] = dot;
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the wave's own scores)
#pragma unroll
            for (int i = 0; i < kSharedHeads; ++i)
                if (i < m) score[i * 64 + lane] = lane < count ? score[i * 64 + lane] * weight : 0.0f;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 4
            for (int r = 0; r < count; r += vrows) {
                const int j = j0 + r + vr;
                const elem_t *row = j < len ? vc + j * vc_step : v_new;
                const bool in = v_in && r + vr < count;
                float x[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f32x4 u = in ? IO::load4(row, E * vl + e) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[e + i] = u[i];
                }
#pragma unroll
                for (int i = 0; i < kSharedHeads; ++i) {
                    if (i >= m) break;
                    const float s = score[i * 64 + ((r + vr) & 63)];
#pragma unroll
                    for (int e = 0; e < E; ++e) y[i][e] += s * x[e];
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (read before the next tile's are written)
        }
        const float zeta = exp2f((float)behind);
#pragma unroll
        for (int i = 0; i < kSharedHeads; ++i) {
            if (i >= m) break;
#pragma unroll
            for (int e = 0; e < E; ++e)
                for (int off = lv; off < 64; off <<= 1) y[i][e] += __shfl_xor(y[i][e], off, 64);
            if (vr == 0 && v_in) {
                elem_t *out = const_cast<elem_t *>(row_of(a.y, b, h * a.G + head0 + i)) + E * vl;
                const float *s = sY + (c + i) * ys + E * vl;
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    IO::store4(out, e, zeta * s[e] + y[i][e], zeta * s[e + 1] + y[i][e + 1], zeta * s[e + 2] + y[i][e + 2],
                               zeta * s[e + 3] + y[i][e + 3]);
            }
        }
        c += m;
    }
}

int pow2_at_least(int x)
{
    int p = 1;
    while (p < x) p *= 2;
    return p;
}

template <bool BF16, int LPR>
hipError_t launch_decode_rows(const LinearDecodeArgs &a, hipStream_t stream)
{
    constexpr int RP = 256 / LPR;
    const int64_t pairs = (int64_t)a.B * a.Hkv;
    // as many rows to a thread as leave four workgroups to a CU
    const auto blocks = [&](int nr) { return pairs * ((a.dv + RP * nr - 1) / (RP * nr)); };
    if (blocks(8) >= 1024)
        hipLaunchKernelGGL((linear_decode_kernel<BF16, LPR, 8>), dim3((unsigned)blocks(8)), dim3(256), 0, stream, a);
    else if (blocks(4) >= 1024)
        hipLaunchKernelGGL((linear_decode_kernel<BF16, LPR, 4>), dim3((unsigned)blocks(4)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((linear_decode_kernel<BF16, LPR, 1>), dim3((unsigned)blocks(1)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16>
hipError_t launch_decode(const LinearDecodeArgs &a, hipStream_t stream)
{
    switch (pow2_at_least(a.dk / 4)) {
    case 4: return launch_decode_rows<BF16, 4>(a, stream);
    case 8: return launch_decode_rows<BF16, 8>(a, stream);
    case 16: return launch_decode_rows<BF16, 16>(a, stream);
    case 32: return launch_decode_rows<BF16, 32>(a, stream);
    default: return launch_decode_rows<BF16, 64>(a, stream);
    }
}

}  // namespace

hipError_t launch_linear_decode(const LinearDecodeArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? launch_decode<true>(a, stream) : launch_decode<false>(a, stream);
}

hipError_t launch_linear_shared(const LinearSharedArgs &a, bool bf16, hipStream_t stream)
{
    const int e = bf16 ? 8 : 4;
    const int64_t cols = (int64_t)a.share * a.G, groups = (int64_t)(a.B / a.share) * a.Hkv;
    int ncol = kSharedCols;
    while (ncol > 4 && groups * ((cols + ncol - 1) / ncol) < 512) ncol /= 2;
    const int64_t blocks = groups * ((cols + ncol - 1) / ncol);
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const size_t lds = ((size_t)ncol * (a.dv + 4) + 4 * kSharedHeads * 64) * sizeof(float);
    if (bf16)
        hipLaunchKernelGGL(linear_shared_kernel<true>, dim3((unsigned)blocks), dim3(256), lds, stream, a, ncol, pow2_at_least(a.dk / e),
                           pow2_at_least(a.dv / e));
    else
        hipLaunchKernelGGL(linear_shared_kernel<false>, dim3((unsigned)blocks), dim3(256), lds, stream, a, ncol, pow2_at_least(a.dk / e),
                           pow2_at_least(a.dv / e));
    return hipGetLastError();
}

}  // namespace gka
