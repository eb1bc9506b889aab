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
// A row of the state (one v-feature) lies across LPR lanes, 4 J k-features on each (runs of four, 4 LPR apart); a thread holds NR
// rows, a workgroup (256 / LPR) NR of them. Few lanes to a row: a token costs each of its G heads a sum over them. The state
// crosses memory once, whatever the number of tokens. Rows of q, k, v and gates come through LDS, as many tokens at a time as
// fit, so that their latency is paid once and beside the state's. Bound by HBM: 8192 states of d 128 in 192 us, 5.6 TB/s (a large copy:
// 5.3); 384 states of 4 tokens x 4 heads, 16 us, by the sums over a row's lanes.
constexpr int kDecodeQueries = 32;                 // q rows of a pass through LDS, or those of one token in parts of as many
constexpr int kDecodeTokens = 16;                  // tokens of a pass at most

template <bool BF16, int LPR, int J, int NR>
__global__ __launch_bounds__(256) void linear_decode_kernel(LinearDecodeArgs a, int tokens)
{
    typedef std::conditional_t<BF16, IOBF16, IOF32> IO;
    typedef typename IO::type elem_t;
    constexpr int RP = 256 / LPR;                  // rows a workgroup covers at once
    constexpr int DKP = 4 * LPR * J;               // k-features with padding
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int queries = a.G < kDecodeQueries ? a.G : kDecodeQueries;       // heads of a token in LDS at once
    float *sk = lds, *sv = sk + tokens * DKP, *sg = sv + tokens * RP * NR, *sq = sg + kDecodeTokens;
    const int blocks = (a.dv + RP * NR - 1) / (RP * NR);
    const int64_t pair = blockIdx.x / blocks;
    const int row_first = (int)(blockIdx.x % blocks) * RP * NR;
    const int tid = threadIdx.x, row0 = row_first + tid / LPR;
    const int b = (int)(pair / a.Hkv), h = (int)(pair % a.Hkv);
    const int l = tid % LPR;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const float *S0 = a.S_in + ((int64_t)(b / a.share) * a.Hkv + h) * a.dv * a.dk;
    f32x4 S[NR][J];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row0 + i * RP, col = 4 * (l + LPR * j);
            S[i][j] = col < a.dk && row < a.dv ? *(const f32x4 *)(S0 + (int64_t)row * a.dk + col) : zero;
        }
    auto row_of = [&](const RowTensor &x, int t, int head) { return (const elem_t *)x.p + b * x.sb + t * x.st + head * x.sh; };
    // `count` rows of q or k, the i-th given by where(i), into LDS
    auto load_rows = [&](float *to, int count, auto where) {
        for (int i = tid; i < count * (DKP / 4); i += 256) {
            const int col = 4 * (i % (DKP / 4));
            *(f32x4 *)(to + 4 * i) = col < a.dk ? IO::load4(where(i / (DKP / 4)), col) : zero;
        }
    };
    for (int t0 = 0; t0 < a.T; t0 += tokens) {
        const int count = a.T - t0 < tokens ? a.T - t0 : tokens;
        if (t0 > 0) __syncthreads();
        load_rows(sk, count, [&](int i) { return row_of(a.k, t0 + i, h); });
        load_rows(sq, count * queries, [&](int i) { return row_of(a.q, t0 + i / queries, h * a.G + i % queries); });
        for (int i = tid; i < count * RP * NR; i += 256) {
            const int row = row_first + i % (RP * NR);
            sv[i] = row < a.dv ? IO::load(row_of(a.v, t0 + i / (RP * NR), h), row) : 0.0f;
        }
        if (tid < count) sg[tid] = a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + t0 + tid) * a.Hkv + h];
        __syncthreads();
        for (int t = 0; t < count; ++t) {
            float gate = sg[t];
            if (!(gate > kWipingGate)) {           // (nothing of the state before comes through, whatever it holds)
                gate = 0.0f;
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j) S[i][j] = zero;
            }
            float x[NR];
#pragma unroll
            for (int i = 0; i < NR; ++i) x[i] = sv[t * RP * NR + i * RP + tid / LPR];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const f32x4 k4 = *(const f32x4 *)(sk + t * DKP + 4 * (l + LPR * j));
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[i][j][e] = gate * S[i][j][e] + x[i] * k4[e];
            }
            elem_t *y = const_cast<elem_t *>(row_of(a.y, t0 + t, h * a.G)) + row0;
            for (int head0 = 0; head0 < a.G; head0 += queries) {
                const int heads = a.G - head0 < queries ? a.G - head0 : queries;
                if (head0 > 0) {                   // (more heads than LDS has room for: one token a pass, part by part)
                    __syncthreads();
                    load_rows(sq, heads, [&](int i) { return row_of(a.q, t0 + t, h * a.G + head0 + i); });
                    __syncthreads();
                }
                const float *q = sq + t * queries * DKP + 4 * l;
                for (int s = 0; s < heads; ++s) {
                    float p[NR];
#pragma unroll
                    for (int i = 0; i < NR; ++i) p[i] = 0.0f;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const f32x4 q4 = *(const f32x4 *)(q + s * DKP + 4 * LPR * j);
#pragma unroll
                        for (int i = 0; i < NR; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) p[i] += S[i][j][e] * q4[e];
                    }
                    float mine = 0.0f;             // lane i of a row's lanes: row i of the thread's
#pragma unroll
                    for (int i = 0; i < NR; ++i) {
                        const float all = sum_over_lanes<LPR>(p[i]);
                        mine = l == i ? all : mine;
                    }
                    if (l < NR && row0 + l * RP < a.dv) IO::store1(y + (head0 + s) * a.y.sh, l * RP, mine);
                }
            }
        }
    }
    float *S1 = a.S_out + pair * a.dv * a.dk;
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row0 + i * RP, col = 4 * (l + LPR * j);
            if (col < a.dk && row < a.dv) *(f32x4 *)(S1 + (int64_t)row * a.dk + col) = S[i][j];
        }
}

// ---- shared ----------------------------------------------------------------------------------------------------------
// A workgroup takes up to 16 columns of one (prefix, kv head): a column is a query head of a sequence, G of them to a
// sequence, one behind the other. First S q of its columns on the matrix cores (16 x 16 tiles: 16 rows of S to a wave; S cut into
// three bf16 pieces, which hold all its bits, or float32), then each wave the cached tokens of its columns, two at most, together
// where they are heads of one sequence, LR lanes to a row of 16-byte pieces.
// Bound by the latency of a wave's reads, one batch after the other: 256 samples of 4 prefixes, 32 heads of d 128, up to 128 tokens:
// 67 us for 262 MiB (4.1 TB/s) from HBM. One head alone leaves registers for 16 reads in flight instead of 8 (72 us). Waves that take the
// columns by falling length instead of in their order: 1 per cent, not kept. Two heads with room for no more than two (no wave has more): 8 heads
// of d 64 to a state, 512 samples of 8 prefixes, 67 us; with the registers for four 102.
constexpr int kSharedCols = 16, kSharedWaves = 8, kSharedHeads = kSharedCols / kSharedWaves;

template <bool BF16, int LR, int HEADS>
__global__ __launch_bounds__(64 * kSharedWaves) void linear_shared_kernel(LinearSharedArgs a, int ncol)
{
    typedef std::conditional_t<BF16, IOBF16, IOF32> IO;
    typedef typename IO::type elem_t;
    constexpr int E = BF16 ? 8 : 4;                // elements of a 16-byte piece
    constexpr int RP = 64 / LR;                    // rows a wave reads at once
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int ys = a.dv + 4;                       // floats of a column of S q
    float *sY = (float *)smem;
    float *sS = sY + ncol * ys;                    // [waves][kSharedHeads][64]
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t cols = (int64_t)a.share * a.G;
    const int tiles = (int)((cols + ncol - 1) / ncol);
    const int tile = blockIdx.x % tiles;
    const int h = blockIdx.x / tiles % a.Hkv;
    const int prefix = blockIdx.x / tiles / a.Hkv;
    const int64_t col0 = (int64_t)tile * ncol;
    const int my_cols = (int)(cols - col0 < ncol ? cols - col0 : ncol);
    const float *S = a.S + ((int64_t)prefix * a.Hkv + h) * a.dv * a.dk;
    auto row_of = [&](const RowTensor &x, int b, int head) { return (const elem_t *)x.p + b * x.sb + head * x.sh; };

    // ---- S q: wave w takes the rows 16 w .. + 15, 16 (w + 8) .. + 15
    {
        const int n = lane & 15, kg = lane >> 4;
        const int c = n < my_cols ? n : 0;         // (columns that do not exist repeat the first; their results are not kept)
        const int64_t col = col0 + c;
        const elem_t *q = row_of(a.q, prefix * a.share + (int)(col / a.G), h * a.G + (int)(col % a.G));
        for (int rb = w; 16 * rb < a.dv; rb += kSharedWaves) {
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
            const float *s = S + (int64_t)(16 * rb + n) * a.dk;
            // 32 k-features a step, four steps' rows in flight (features that do not exist: zeros on both sides)
            constexpr int KSTEPS = E * LR / 32 > 0 ? E * LR / 32 : 1, FLY = KSTEPS < 4 ? KSTEPS : 4;
            const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int s0 = 0; s0 < KSTEPS; s0 += FLY) {
                f32x4 x0[FLY], x1[FLY];
                u32x4_t q0[FLY], q1[FLY];
#pragma unroll
                for (int i = 0; i < FLY; ++i) {
                    const int k0 = 32 * (s0 + i) + 8 * kg;
                    const bool in = k0 < a.dk;
                    x0[i] = in ? *(const f32x4 *)(s + k0) : zero;
                    x1[i] = in ? *(const f32x4 *)(s + k0 + 4) : zero;
                    q0[i] = in ? *(const u32x4_t *)(q + k0) : u32x4_t{0, 0, 0, 0};
                    if constexpr (!BF16) q1[i] = in ? *(const u32x4_t *)(q + k0 + 4) : u32x4_t{0, 0, 0, 0};
                }
#pragma unroll
                for (int i = 0; i < FLY; ++i) {
                    if constexpr (BF16) {
                        float x[8] = {x0[i][0], x0[i][1], x0[i][2], x0[i][3], x1[i][0], x1[i][1], x1[i][2], x1[i][3]}, back[8];
                        const bf16x8 qf = __builtin_bit_cast(bf16x8, q0[i]);
#pragma unroll
                        for (int piece = 0; piece < 3; ++piece) {
                            const bf16x8 f = MmaBF16::pack(x);
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf, acc, 0, 0, 0);
                            MmaBF16::unpack(f, back);
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] -= back[e];
                        }
                    } else {
                        const f32x4 qa = __builtin_bit_cast(f32x4, q0[i]), qb = __builtin_bit_cast(f32x4, q1[i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x0[i][e], qa[e], acc, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x1[i][e], qb[e], acc, 0, 0, 0);
                    }
                }
            }
            if (n < my_cols) *(f32x4 *)(sY + n * ys + 16 * rb + 4 * kg) = acc;
        }
    }
    __syncthreads();

    // ---- the cached tokens
    float *score = sS + w * kSharedHeads * 64;
    const int l = lane % LR, r = lane / LR;        // piece of a row, row of a read
    const bool k_in = E * l < a.dk, v_in = E * l < a.dv;
    const int per_wave = (ncol + kSharedWaves - 1) / kSharedWaves;
    int c = w * per_wave;
    const int c_end = c + per_wave < my_cols ? c + per_wave : my_cols;
    while (c < c_end) {
        const int64_t col = col0 + c;
        const int b = prefix * a.share + (int)(col / a.G), head0 = (int)(col % a.G);
        int m = a.G - head0;                       // columns of this sequence, taken together
        m = m < c_end - c ? m : c_end - c;
        m = m < HEADS ? m : HEADS;
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
            if (r == 0 && k_in) *(u32x4_t *)(kc + len * kc_step + E * l) = *(const u32x4_t *)(k_new + E * l);
            if (r == 0 && v_in) *(u32x4_t *)(vc + len * vc_step + E * l) = *(const u32x4_t *)(v_new + E * l);
            if (!a.gate_per_head && lane == 0) a.gate_cache[cache_row + (int64_t)len * a.Hkv] = gate_new;
        }
        float q[HEADS][E], y[HEADS][E];
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const elem_t *row = row_of(a.q, b, h * a.G + head0 + (i < m ? i : 0));
#pragma unroll
            for (int e = 0; e < E; ++e) y[i][e] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const f32x4 x = k_in ? IO::load4(row, E * l + e) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 4; ++j) q[i][e + j] = x[j];
            }
        }
        // a row's piece as floats (zeros: not one of the tile's tokens, or beyond the features)
        typedef struct { u32x4_t bits; } piece;
        auto fetch = [&](const elem_t *cache, int64_t step, const elem_t *newest, int j, bool in) {
            return piece{in ? *(const u32x4_t *)((j < len ? cache + j * step : newest) + E * l) : u32x4_t{0, 0, 0, 0}};
        };
        auto floats = [](piece p, float (&x)[E]) {
            if constexpr (BF16) {
                MmaBF16::unpack(__builtin_bit_cast(bf16x8, p.bits), x);
            } else {
                const f32x4 u = __builtin_bit_cast(f32x4, p.bits);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = u[e];
            }
        };
        constexpr int MOST = HEADS == 1 ? 16 : 8, FLY = LR < MOST ? LR : MOST;    // reads in flight
        double behind = 0.0;                       // log2 decay over the tokens behind the tile
        bool wiped = false;                        // nothing before that tile comes through
        for (int j0 = len / 64 * 64; j0 >= 0 && !wiped; j0 -= 64) {
            const int count = len + 1 - j0 < 64 ? len + 1 - j0 : 64;
            double lg = 0.0;
            bool wipes = false;
            if (lane < count) {
                const float gate = a.gate_per_head || j0 + lane == len ? gate_new : a.gate_cache[cache_row + (int64_t)(j0 + lane) * a.Hkv];
                lg = log2_gate_f64(gate);
                wipes = !(gate > kWipingGate);
            }
            const uint64_t wiping = __ballot(wipes);
            const int first = wiping != 0 ? 63 - __builtin_clzll(wiping) : 0;        // the first token of the tile that counts
            for (int s0 = 0; s0 < count; s0 += FLY * RP) {
                piece p[FLY];
#pragma unroll
                for (int i = 0; i < FLY; ++i) p[i] = fetch(kc, kc_step, k_new, j0 + s0 + i * RP + r, k_in && s0 + i * RP + r < count);
#pragma unroll
                for (int i = 0; i < FLY; ++i) {
                    float x[E];
                    floats(p[i], x);
#pragma unroll
                    for (int g = 0; g < HEADS; ++g) {
                        if (g < m) {
                            float dot = 0.0f;
#pragma unroll
                            for (int e = 0; e < E; ++e) dot += x[e] * q[g][e];
                            dot = sum_over_lanes<LR>(dot);
                            if (l == 0) score[g * 64 + s0 + i * RP + r] = dot;
                        }
                    }
                }
            }
            const double G = wave_inclusive_scan_f64(lg), total = lane63_f64(G);
            const bool counts = lane >= first && lane < count;
            const float weight = counts ? __builtin_amdgcn_exp2f((float)(behind + (total - G))) : 0.0f;
            behind += total;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the wave's own scores)
#pragma unroll
            for (int g = 0; g < HEADS; ++g)
                if (g < m) score[g * 64 + lane] = counts ? score[g * 64 + lane] * weight : 0.0f;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            for (int s0 = 0; s0 < count; s0 += FLY * RP) {
                piece p[FLY];
#pragma unroll
                for (int i = 0; i < FLY; ++i) {
                    const int token = s0 + i * RP + r;
                    p[i] = fetch(vc, vc_step, v_new, j0 + token, v_in && token >= first && token < count);
                }
#pragma unroll
                for (int i = 0; i < FLY; ++i) {
                    float x[E];
                    floats(p[i], x);
#pragma unroll
                    for (int g = 0; g < HEADS; ++g) {
                        if (g < m) {
                            const float s = score[g * 64 + s0 + i * RP + r];
#pragma unroll
                            for (int e = 0; e < E; ++e) y[g][e] += s * x[e];
                        }
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (read before the next tile's are written)
            wiped = wiping != 0;
        }
        const float zeta = wiped ? 0.0f : __builtin_amdgcn_exp2f((float)behind);
#pragma unroll
        for (int g = 0; g < HEADS; ++g) {
            if (g >= m) continue;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int off = LR; off < 64; off <<= 1) y[g][e] += __shfl_xor(y[g][e], off, 64);
            if (r == 0 && v_in) {
                elem_t *out = const_cast<elem_t *>(row_of(a.y, b, h * a.G + head0 + g)) + E * l;
                const float *s = sY + (c + g) * ys + E * l;
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f32x4 x = wiped ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : *(const f32x4 *)(s + e);
                    IO::store4(out, e, zeta * x[0] + y[g][e], zeta * x[1] + y[g][e + 1], zeta * x[2] + y[g][e + 2], zeta * x[3] + y[g][e + 3]);
                }
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

template <bool BF16, int LPR, int J, int NR>
hipError_t launch_decode_kernel(const LinearDecodeArgs &a, hipStream_t stream)
{
    constexpr int ROWS = 256 / LPR * NR;           // of a workgroup
    const int64_t blocks = (int64_t)a.B * a.Hkv * ((a.dv + ROWS - 1) / ROWS);
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    // tokens of a pass through LDS: as many as all of whose q rows have room
    int tokens = a.G >= kDecodeQueries ? 1 : kDecodeQueries / a.G;
    tokens = tokens < kDecodeTokens ? tokens : kDecodeTokens;
    tokens = tokens < a.T ? tokens : a.T;
    const int queries = a.G < kDecodeQueries ? tokens * a.G : kDecodeQueries;
    const size_t lds = ((size_t)(tokens + queries) * 4 * LPR * J + tokens * ROWS + kDecodeTokens) * sizeof(float);
    hipLaunchKernelGGL((linear_decode_kernel<BF16, LPR, J, NR>), dim3((unsigned)blocks), dim3(256), lds, stream, a, tokens);
    return hipGetLastError();
}

template <bool BF16, int DK>
hipError_t launch_decode_dk(const LinearDecodeArgs &a, hipStream_t stream)
{
    const int64_t pairs = (int64_t)a.B * a.Hkv;
    const auto fills = [&](int rows) { return pairs * ((a.dv + rows - 1) / rows) >= 1024; };   // four workgroups to a CU
    // One or two query heads to a state: a row lies across as many lanes as it has runs, in one stretch of memory, and a thread takes
    // eight rows where enough workgroups remain (8192 states of d 128, one token: 187 us against 193, 16 states: 4.2 us against
    // 4.8). More heads: fewer lanes (384 states, 4 tokens of 4 heads: 17.0 us against 22.2). The number of tokens has no part in
    // this: several tokens in a call give the same bits as one after the other.
    if (a.G <= 2)
        return fills(8 * 256 / (DK / 4)) ? launch_decode_kernel<BF16, DK / 4, 1, (DK < 32 ? DK / 4 : 8)>(a, stream)
                                         : launch_decode_kernel<BF16, DK / 4, 1, 1>(a, stream);
    constexpr int LPR = DK <= 16 ? 4 : DK <= 128 ? 8 : 16, J = DK / 4 / LPR;
    return fills(2 * 256 / LPR) ? launch_decode_kernel<BF16, LPR, J, 2>(a, stream) : launch_decode_kernel<BF16, LPR, J, 1>(a, stream);
}

template <bool BF16>
hipError_t launch_decode(const LinearDecodeArgs &a, hipStream_t stream)
{
    if (a.dk <= 16) return launch_decode_dk<BF16, 16>(a, stream);
    if (a.dk <= 32) return launch_decode_dk<BF16, 32>(a, stream);
    if (a.dk <= 64) return launch_decode_dk<BF16, 64>(a, stream);
    if (a.dk <= 128) return launch_decode_dk<BF16, 128>(a, stream);
    return launch_decode_dk<BF16, 256>(a, stream);
}

template <bool BF16, int LR, int HEADS>
hipError_t launch_shared_heads(const LinearSharedArgs &a, hipStream_t stream)
{
    const int64_t cols = (int64_t)a.share * a.G, groups = (int64_t)(a.B / a.share) * a.Hkv;
    // two workgroups to a CU, with fewer columns to each where there are not so many (four instead: 75 us against 63, 64 samples of 4
    // prefixes, 32 heads)
    int ncol = kSharedCols;
    while (ncol > 1 && groups * ((cols + ncol - 1) / ncol) < 512) ncol /= 2;
    const int64_t blocks = groups * ((cols + ncol - 1) / ncol);
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const size_t lds = ((size_t)ncol * (a.dv + 4) + kSharedWaves * kSharedHeads * 64) * sizeof(float);
    hipLaunchKernelGGL((linear_shared_kernel<BF16, LR, HEADS>), dim3((unsigned)blocks), dim3(64 * kSharedWaves), lds, stream, a, ncol);
    return hipGetLastError();
}

template <bool BF16, int LR>
hipError_t launch_shared(const LinearSharedArgs &a, hipStream_t stream)
{
    return a.G == 1 ? launch_shared_heads<BF16, LR, 1>(a, stream) : launch_shared_heads<BF16, LR, kSharedHeads>(a, stream);
}

template <bool BF16>
hipError_t launch_shared_rows(const LinearSharedArgs &a, hipStream_t stream)
{
    switch (pow2_at_least((a.dk > a.dv ? a.dk : a.dv) / (BF16 ? 8 : 4))) {
    case 2: if constexpr (BF16) return launch_shared<true, 2>(a, stream); else return hipErrorInvalidValue;
    case 4: return launch_shared<BF16, 4>(a, stream);
    case 8: return launch_shared<BF16, 8>(a, stream);
    case 16: return launch_shared<BF16, 16>(a, stream);
    case 32: return launch_shared<BF16, 32>(a, stream);
    default: if constexpr (!BF16) return launch_shared<false, 64>(a, stream); else return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_linear_decode(const LinearDecodeArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? launch_decode<true>(a, stream) : launch_decode<false>(a, stream);
}

hipError_t launch_linear_shared(const LinearSharedArgs &a, bool bf16, hipStream_t stream)
{
    return bf16 ? launch_shared_rows<true>(a, stream) : launch_shared_rows<false>(a, stream);
}

}  // namespace gka
