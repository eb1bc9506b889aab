// Linear attention with a decay for each head over whole sequences:
//   S_t = gate_t S_{t-1} + v_t k_t^T,   y_t = S_t q_t       (S [dv, dk] in float32, one for each sequence and kv head)
// chunk by chunk (C tokens, G_t the cumulative log2 decay inside the chunk, zeta_t = 2^G_t, M[t, s] = 2^(G_t - G_s), s <= t):
//   y_t = zeta_t S_[n] q_t + sum_{s <= t} M[t, s] (k_s . q_t) v_s,     S_[n+1] = zeta_C S_[n] + sum_s 2^(G_C - G_s) v_s k_s^T.
// The same walk with other tensors in the roles of q, k, v gives the three gradients (LinearWalkArgs).
//
// A workgroup walks the chunks of one segment of one (sequence, kv head), for a slice of up to 128 of the dv features, with the
// state in registers: wave w holds features 32 w .. 32 w + 31 of the slice for all k-features, accumulator tile jb element
// [32 jb + kidx(r, g)][32 w + n] on lane (n, g), register r. A tile converts in place into the A operand of S q. Segments
// start from states that a summary launch (SUMMARY: the updates alone) and a scan over the segments leave in the workspace.
//
// Precision. bf16 tensors enter the products as they are; what is computed in float32 (states, masked products, weighted
// v) is cut into bf16 pieces of 8 bits each: two where the product ends in a bf16 output (17 bits against the output's 8), three
// where it ends in float32: in the state itself, and in the dot products behind the gradient of the decays, a long sum of
// differences. float32 tensors use the float32 MFMA. Decays are summed in float64 and kept as two floats: a difference of
// two of them is then exact to float32 wherever a sequence is wiped by a gate of 0 (2^-144 each) before.
#pragma once
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace linear {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// MMA: MmaBF16 (64 tokens per chunk) or MmaF32 (32). DK: padded features of q and k. NW: waves, 32 features of v each.
template <class MMA, int DK, int NW>
struct Shape {
    static constexpr bool BF16 = MMA::VEC == 8;
    static constexpr int TB = BF16 ? 2 : 1;        // 32-token blocks
    static constexpr int C = 32 * TB;
    static constexpr int NT = 64 * NW;
    static constexpr int NBK = DK / 32;
    static constexpr int E = BF16 ? 8 : 4;         // elements of a 16-byte piece
    static constexpr int RSQ = DK + (BF16 ? 8 : 4);
    static constexpr int RSK = DK + (BF16 ? 16 : 4);
    static constexpr int RSV = 32 * NW + (BF16 ? 16 : 4);
    static constexpr int PK = C * DK / E / NT;     // 16-byte pieces of a chunk's q or k rows per thread
    static constexpr int PV = C * 32 / E / 64;     // ... of its v rows
    static constexpr int TILES = TB == 2 ? 3 : 1;  // causal 32 x 32 tiles of the masked products
    static constexpr int ES = sizeof(typename MMA::elem_t);
    static constexpr size_t q_bytes = (size_t)C * RSQ * ES, k_bytes = (size_t)C * RSK * ES, v_bytes = (size_t)C * RSV * ES;
    // masked products: bf16 fragments of up to three pieces; float32: what each wave adds to the one tile
    static constexpr size_t p_bytes(int pieces) { return BF16 ? (size_t)TILES * 2 * 64 * 16 * pieces : (size_t)NW * 1024 * 4; }
    static constexpr size_t tab_bytes = 3 * 64 * sizeof(float);
    static constexpr size_t lds_bytes(int pieces, bool summary)
    {
        return (summary ? 0 : q_bytes + p_bytes(pieces)) + k_bytes + v_bytes + tab_bytes;
    }
};

struct RowsAt {
    int rs;
    __device__ __forceinline__ int operator()(int row, int col) const { return row * rs + col; }
};

// Operand fragment of step `st` of 32-feature block `blk`: a row of a row-major tile, its features in kidx order ...
__device__ __forceinline__ bf16x8 row_frag(const uint16_t *row, int blk, int st, int g)
{
    const uint16_t *p = row + 32 * blk + 16 * st + 4 * g;
    const u32x2_t a = *(const u32x2_t *)p, b = *(const u32x2_t *)(p + 8);
    const u32x4_t u = {a[0], a[1], b[0], b[1]};
    return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ float row_frag(const float *row, int blk, int st, int g)
{
    const f32x4 x = *(const f32x4 *)(row + 32 * blk + 8 * (st >> 2) + 4 * g);
    return x[st & 3];
}
// ... or its columns col0 .. col0 + 31, the rows (tokens) of 32-block `blk` in kidx order.
__device__ __forceinline__ bf16x8 col_frag(const uint16_t *tile, int rs, int col0, int blk, int st, int lane)
{
    const int t0 = 32 * blk + 16 * st + 4 * (lane >> 5);
    return gather_transposed_bf16(tile, RowsAt{rs}, col0 + 16 * ((lane >> 4) & 1), lane, t0, t0 + 8);
}
__device__ __forceinline__ float col_frag(const float *tile, int rs, int col0, int blk, int st, int lane)
{
    return tile[(32 * blk + kidx(st, lane >> 5)) * rs + col0 + (lane & 31)];
}

// VEC floats as pieces of operand precision; all of them together hold 8 bits per piece (float32 operands: one piece, exact).
template <class MMA, int N>
__device__ __forceinline__ void cut(const float *x, typename MMA::frag (&f)[N])
{
    float rest[MMA::VEC];
#pragma unroll
    for (int e = 0; e < MMA::VEC; ++e) rest[e] = x[e];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f[i] = MMA::pack(rest);
        if (i + 1 < N) {
            float back[MMA::VEC];
            MMA::unpack(f[i], back);
#pragma unroll
            for (int e = 0; e < MMA::VEC; ++e) rest[e] -= back[e];
        }
    }
}

// Float `i` of the state of segment `seg` of (pair, slice), as the scan and the walks address it: tile (w, jb), register r, lane.
__device__ __forceinline__ int64_t seg_state_at(const LinearWalkArgs &a, int64_t pair, int slice, int seg, int64_t state_floats)
{
    return ((pair * a.slices + slice) * a.n_segs + seg) * state_floats;
}

// A caller's state [dv, dk] (or stored [dk, dv]) as a raw buffer: rows and columns of the padding read as zeros, writes to them are
// dropped. Lane (n, g) of the wave whose first v-feature is `row0`: run(jb, q4) is its elements [32 jb + 8 q4 + 4 g ..+3][row0 + n].
struct StateAt {
    buffer_rsrc state;
    int lane_offset, dk, pitch;                    // pitch: bytes from one k-feature to the next
    bool transposed;
    __device__ __forceinline__ StateAt(const float *states, int64_t index, const LinearWalkArgs &a, int row0, int lane)
    {
        const int row = row0 + (lane & 31), g = lane >> 5;
        state = __builtin_amdgcn_make_buffer_rsrc((void *)(states + index * a.dv * a.dk), 0, a.dv * a.dk * 4, 0x00020000);
        transposed = a.transposed != 0;
        pitch = transposed ? 4 * a.dv : 4;
        dk = a.dk;
        lane_offset = row < a.dv ? row * (transposed ? 4 : 4 * a.dk) + 4 * g * pitch : (int)0x80000000;
    }
    // (dk is a multiple of 16: whether a run exists depends on the pair of runs alone)
    __device__ __forceinline__ bool exists(int jb, int q4) const { return 32 * jb + 16 * (q4 >> 1) < dk; }
    __device__ __forceinline__ f32x4 load(int jb, int q4) const
    {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        if (!exists(jb, q4)) return x;
        const int at = lane_offset + (32 * jb + 8 * q4) * pitch;
        if (!transposed) return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(state, at, 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(state, at + e * pitch, 0, 0));
        return x;
    }
    __device__ __forceinline__ void store(int jb, int q4, f32x4 x) const
    {
        if (!exists(jb, q4)) return;
        const int at = lane_offset + (32 * jb + 8 * q4) * pitch;
        if (!transposed) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), state, at, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[e]), state, at + e * pitch, 0, 0);
        }
    }
};

// One chunk's rows of one head as a raw buffer: reads of tokens and features that do not exist give zeros and writes to them are
// dropped by the buffer's bounds, without a branch. `lane` offsets (chunk_row below) count from the first row of the buffer.
struct ChunkRows {
    buffer_rsrc rows;
    int top;                                       // byte offset of the walk's first token of the chunk
};
// ES: bytes of an element. Rows are at most 2^23 elements apart, so that a chunk's bytes stay below 2^30.
template <int C, int ES>
__device__ __forceinline__ ChunkRows chunk_rows(const RowTensor &x, int b, int head, int tau0, int T, int reverse)
{
    const int left = T - tau0;                     // tokens of the walk from here on
    const int count = left < C ? left : C;
    const int lowest = reverse ? left - count : tau0;
    const char *base = (const char *)x.p + (b * x.sb + lowest * x.st + head * x.sh) * ES;
    const int pitch = (int)x.st * ES;
    return {__builtin_amdgcn_make_buffer_rsrc((void *)base, 0, count * pitch, 0x00020000), reverse ? (count - 1) * pitch : 0};
}
// Offset of feature `col` of the chunk's row `row` but for ChunkRows::top; far outside for a feature that does not exist. A token
// behind the last one lies behind the buffer's end or, in reverse, at a negative offset, which counts as one of 2^31 or more.
template <int ES>
__device__ __forceinline__ int chunk_offset(const RowTensor &x, int row, int col, bool exists, int reverse)
{
    const int pitch = (int)x.st * ES;
    return exists ? (reverse ? -row : row) * pitch + col * ES : (int)0x80000000;
}

enum Group { kOne, kQueries, kSources };           // n_q = n_src = 1; several queries; several sources of a token

// PIECES: of states and masked products in the readout (float32 tensors: 1). DOT: dot_out is wanted.
template <class MMA, int DK, int NW, int PIECES, bool DOT, bool SUMMARY, Group GROUP>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(DK > 128 ? 1 : 2, DK > 128 ? 1 : 2)))
void linear_walk_kernel(LinearWalkArgs a)
{
    typedef Shape<MMA, DK, NW> SH;
    typedef typename MMA::frag frag;
    typedef typename MMA::elem_t elem_t;
    constexpr bool BF16 = SH::BF16;
    constexpr int C = SH::C, TB = SH::TB, NT = SH::NT, NBK = SH::NBK, E = SH::E, PK = SH::PK, PV = SH::PV, HS = MMA::HS, ES = SH::ES;
    constexpr int RSQ = SH::RSQ, RSK = SH::RSK, RSV = SH::RSV;
    constexpr int VW = BF16 ? 3 : 1;               // pieces of the weighted v (they end in the float32 state)
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    elem_t *sK = (elem_t *)smem;
    elem_t *sV = (elem_t *)(smem + SH::k_bytes);
    float *sHi = (float *)(smem + SH::k_bytes + SH::v_bytes), *sLo = sHi + 64, *sW = sLo + 64;
    elem_t *sQ = (elem_t *)(sW + 64);
    frag *sP = (frag *)((unsigned char *)sQ + SH::q_bytes);

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, g = lane >> 5;
    const int n_pairs = a.B * a.Hkv;
    const int pair = blockIdx.x % n_pairs;
    const int slice = blockIdx.x / n_pairs % a.slices;
    const int seg = blockIdx.x / n_pairs / a.slices;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    const int n_chunks = (a.T + C - 1) / C;
    const int chunk_begin = seg * a.seg_chunks;
    const int chunk_end = min(chunk_begin + a.seg_chunks, n_chunks);
    const int steps = GROUP == kQueries ? a.n_q : GROUP == kSources ? a.n_src : 1;
    const int v0 = slice * 32 * NW;                // first feature of the slice
    const int64_t state_floats = (int64_t)32 * NW * DK;

    // ---- the state that the segment starts from
    f32x16 acc[NBK];
#pragma unroll
    for (int jb = 0; jb < NBK; ++jb) acc[jb] = zero16();
    if constexpr (!SUMMARY) {
        if (a.n_segs > 1) {
            const float *s = a.seg_states + seg_state_at(a, pair, slice, seg, state_floats) + w * NBK * 1024;
#pragma unroll
            for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 x = *(const f32x4 *)(s + (jb * 4 + q4) * 256 + 4 * lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[jb][4 * q4 + e] = x[e];
                }
        } else if (a.init) {
            const StateAt S(a.init, (int64_t)(b / a.share) * a.Hkv + h, a, v0 + 32 * w, lane);
#pragma unroll
            for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 x = S.load(jb, q4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[jb][4 * q4 + e] = x[e];
                }
        }
    }

    // ---- rows of a chunk: memory -> registers (a step ahead) -> LDS
    struct Rows {
        u32x4_t q[SUMMARY ? 1 : PK], k[PK], v[PV];
        float gate;
    };
    constexpr int KROW = DK / E, VROW = 32 * NW / E;          // pieces of a row
    const int krow = tid / KROW, kcol = E * (tid % KROW);     // (a thread's pieces all lie in one column)
    const int vrow = tid / VROW, vcol = E * (tid % VROW);
    const bool k_in = kcol < a.dk, v_in = v0 + vcol < a.dv;
    const int q_off = chunk_offset<ES>(a.q, krow, kcol, k_in, a.reverse);
    const int k_off = chunk_offset<ES>(a.k, krow, kcol, k_in, a.reverse);
    const int v_off = chunk_offset<ES>(a.v, vrow, v0 + vcol, v_in, a.reverse);
    auto fetch_rows = [&](auto &to, const RowTensor &x, int head, int tau0, int offset, int rows_per) {
        const ChunkRows r = chunk_rows<C, ES>(x, b, head, tau0, a.T, a.reverse);
        const int step = chunk_offset<ES>(x, rows_per, 0, true, a.reverse);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(to) / 16); ++i)
            to[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r.rows, offset + (r.top + i * step), 0, 0));
    };
    auto fetch = [&](Rows &f, int c, int s) {
        if constexpr (!SUMMARY)
            if (GROUP == kQueries || s == 0) fetch_rows(f.q, a.q, GROUP == kQueries ? h * steps + s : h, c * C, q_off, NT / KROW);
        if (GROUP == kSources || s == 0) {
            const int head = GROUP == kSources ? h * steps + s : h;
            fetch_rows(f.k, a.k, head, c * C, k_off, NT / KROW);
            fetch_rows(f.v, a.v, head, c * C, v_off, NT / VROW);
        }
        if (s == 0) {
            const int tau = c * C + lane;
            f.gate = 1.0f;
            if (lane < C && tau < a.T && !(a.reverse && tau == 0))
                f.gate = a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + (a.reverse ? a.T - tau : tau)) * a.Hkv + h];
        }
    };
    auto stage = [&](const Rows &f, int s) {
        if constexpr (!SUMMARY)
            if (GROUP == kQueries || s == 0) {
#pragma unroll
                for (int i = 0; i < PK; ++i) *(u32x4_t *)(sQ + (krow + i * (NT / KROW)) * RSQ + kcol) = f.q[i];
            }
        if (GROUP == kSources || s == 0) {
#pragma unroll
            for (int i = 0; i < PK; ++i) *(u32x4_t *)(sK + (krow + i * (NT / KROW)) * RSK + kcol) = f.k[i];
#pragma unroll
            for (int i = 0; i < PV; ++i) *(u32x4_t *)(sV + (vrow + i * (NT / VROW)) * RSV + vcol) = f.v[i];
        }
    };

    float seg_decay = 1.0f;
    Rows rows;
    fetch(rows, chunk_begin, 0);
    for (int c = chunk_begin; c < chunk_end; ++c) {
        // ---- decays of the chunk (every wave for itself): lane j holds token j
        const double G = wave_inclusive_scan_f64((double)log2_gate(rows.gate));
        const double Gtot = lane63_f64(G);
        const float g_hi = (float)G, g_lo = (float)(G - (double)g_hi);
        const float zeta_C = __builtin_amdgcn_exp2f((float)Gtot);
        const float w_j = c * C + lane < a.T ? __builtin_amdgcn_exp2f((float)(Gtot - G)) : 0.0f;   // of token j in the state after the chunk
        seg_decay *= zeta_C;
        f32x16 y[TB];
        for (int s = 0; s < steps; ++s) {
            lds_barrier();                         // the tiles of the step before have been read
            stage(rows, s);
            if (s == 0 && w == 0) {
                sHi[lane] = g_hi;
                sLo[lane] = g_lo;
                sW[lane] = w_j;
            }
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < steps) fetch(rows, c, s + 1);
            else if (c + 1 < chunk_end) fetch(rows, c + 1, 0);
            lds_barrier();                         // (no wait for the rows in flight)
            __builtin_amdgcn_sched_barrier(0);

            if constexpr (!SUMMARY) {
                // ---- products K Q^T of the causal tiles (key block sb, token block tb)
                // M[t, s] on register r of lane (n, g): token 32 tb + n, key 32 sb + kidx(r, g)
                auto masked = [&](const f32x16 &x, int sb, int tb, float (&m)[16]) {
                    const float hi = sHi[32 * tb + n], lo = sLo[32 * tb + n];
                    const int t = 32 * (tb - sb) + n;          // (in the tile below the diagonal: above every key)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        const int s0 = 32 * sb + 8 * q4 + 4 * g;
                        const f32x4 h4 = *(const f32x4 *)(sHi + s0), l4 = *(const f32x4 *)(sLo + s0);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            m[4 * q4 + e] = 8 * q4 + 4 * g + e <= t
                                                ? x[4 * q4 + e] * __builtin_amdgcn_exp2f((hi - h4[e]) + (lo - l4[e]))
                                                : 0.0f;
                    }
                };
                if constexpr (BF16) {
                    // a tile to a wave; masked, cut into pieces and left as operand fragments
                    for (int tile = w; tile < 3; tile += NW) {
                        const int sb = tile >> 1, tb = (tile + 1) >> 1;
                        f32x16 x = zero16();
                        const elem_t *krow_p = sK + (32 * sb + n) * RSK, *qrow_p = sQ + (32 * tb + n) * RSQ;
#pragma unroll
                        for (int st = 0; st < NBK * HS; ++st)
                            x = MMA::mma(row_frag(krow_p, st / HS, st % HS, g), row_frag(qrow_p, st / HS, st % HS, g), x);
                        float m[16];
                        masked(x, sb, tb, m);
#pragma unroll
                        for (int st = 0; st < HS; ++st) {
                            frag f[PIECES];
                            cut<MMA, PIECES>(m + MMA::VEC * st, f);
#pragma unroll
                            for (int i = 0; i < PIECES; ++i) sP[((i * 3 + tile) * HS + st) * 64 + lane] = f[i];
                        }
                    }
                } else {
                    // the one tile: every wave adds the products of its share of the features
                    f32x16 x = zero16();
#pragma unroll
                    for (int j = 0; j < (NBK + NW - 1) / NW; ++j) {
                        const int jb = j * NW + w;
                        if (jb < NBK)
#pragma unroll
                            for (int st = 0; st < HS; ++st)
                                x = MMA::mma(row_frag(sK + n * RSK, jb, st, g), row_frag(sQ + n * RSQ, jb, st, g), x);
                    }
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4)
                        *(f32x4 *)((float *)sP + w * 1024 + q4 * 256 + 4 * lane) = f32x4{x[4 * q4], x[4 * q4 + 1], x[4 * q4 + 2], x[4 * q4 + 3]};
                }
                __builtin_amdgcn_sched_barrier(0);

                // ---- zeta_t S_[n] q_t: the state's tiles are the A operand
                if (GROUP == kQueries || s == 0) {
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) y[tb] = zero16();
#pragma unroll
                    for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                        for (int st = 0; st < HS; ++st) {
                            float x[MMA::VEC];
#pragma unroll
                            for (int e = 0; e < MMA::VEC; ++e) x[e] = acc[jb][MMA::VEC * st + e];
                            frag f[PIECES];
                            cut<MMA, PIECES>(x, f);
#pragma unroll
                            for (int tb = 0; tb < TB; ++tb) {
                                const frag qf = row_frag(sQ + (32 * tb + n) * RSQ, jb, st, g);
#pragma unroll
                                for (int i = 0; i < PIECES; ++i) y[tb] = MMA::mma(f[i], qf, y[tb]);
                            }
                        }
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) {
                        const float zeta = __builtin_amdgcn_exp2f(sHi[32 * tb + n]);
#pragma unroll
                        for (int r = 0; r < 16; ++r) y[tb][r] *= zeta;
                    }
                }
                lds_barrier();                     // the masked products are there
                __builtin_amdgcn_sched_barrier(0);
            }

            frag vt[TB][HS];                       // v, features on the lanes, tokens in kidx order
#pragma unroll
            for (int sb = 0; sb < TB; ++sb)
#pragma unroll
                for (int st = 0; st < HS; ++st) vt[sb][st] = col_frag(sV, RSV, 32 * w, sb, st, lane);

            if constexpr (!SUMMARY) {
                // ---- + sum_s v_s M[t, s] (k_s . q_t)
                if constexpr (BF16) {
#pragma unroll
                    for (int tile = 0; tile < 3; ++tile) {
                        const int sb = tile == 2 ? 1 : 0, tb = tile == 0 ? 0 : 1;
#pragma unroll
                        for (int st = 0; st < HS; ++st)
#pragma unroll
                            for (int i = 0; i < PIECES; ++i)
                                y[tb] = MMA::mma(vt[sb][st], sP[((i * 3 + tile) * HS + st) * 64 + lane], y[tb]);
                    }
                } else {
                    f32x16 x = zero16();
#pragma unroll
                    for (int i = 0; i < NW; ++i)
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4) {
                            const f32x4 part = *(const f32x4 *)((const float *)sP + i * 1024 + q4 * 256 + 4 * lane);
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[4 * q4 + e] += part[e];
                        }
                    const float hi = sHi[n], lo = sLo[n];
                    float m[16];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        const f32x4 h4 = *(const f32x4 *)(sHi + 8 * q4 + 4 * g), l4 = *(const f32x4 *)(sLo + 8 * q4 + 4 * g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            m[4 * q4 + e] = 8 * q4 + 4 * g + e <= n ? x[4 * q4 + e] * __builtin_amdgcn_exp2f((hi - h4[e]) + (lo - l4[e])) : 0.0f;
                    }
#pragma unroll
                    for (int st = 0; st < HS; ++st) y[0] = MMA::mma(vt[0][st], m[st], y[0]);
                }
                // ---- out: lane (n, g) holds features v0 + 32 w + kidx(r, g) of token 32 tb + n
                if (GROUP == kQueries || s + 1 == steps) {
                    const int head = GROUP == kQueries ? h * steps + s : h;
                    if constexpr (DOT) {
                        float *sDot = (float *)sP; // [NW][C], in place of the masked products
                        const ChunkRows r = chunk_rows<C, ES>(a.dot_with, b, head, c * C, a.T, a.reverse);
                        lds_barrier();
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) {
                            float dot = 0.0f;
#pragma unroll
                            for (int q4 = 0; q4 < 4; ++q4) {
                                const int col = v0 + 32 * w + 8 * q4 + 4 * g;
                                const int at = chunk_offset<ES>(a.dot_with, 32 * tb + n, col, col < a.dv, a.reverse) + r.top;
                                f32x4 x;
                                if constexpr (BF16)
                                    x = IOBF16::cvt4(__builtin_bit_cast(u16x4, __builtin_amdgcn_raw_buffer_load_b64(r.rows, at, 0, 0)));
                                else
                                    x = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r.rows, at, 0, 0));
#pragma unroll
                                for (int e = 0; e < 4; ++e) dot += x[e] * y[tb][4 * q4 + e];
                            }
                            dot += __shfl_xor(dot, 32, 64);
                            if (g == 0) sDot[w * C + 32 * tb + n] = dot;
                        }
                        lds_barrier();
                        if (w == 0 && lane < C && c * C + lane < a.T) {
                            float dot = 0.0f;
#pragma unroll
                            for (int i = 0; i < NW; ++i) dot += sDot[i * C + lane];
                            const int tau = c * C + lane;
                            a.dot_out[((((int64_t)slice * n_pairs + pair) * a.n_q) + (GROUP == kQueries ? s : 0)) * a.T + (a.reverse ? a.T - 1 - tau : tau)] = dot;
                        }
                    }
                    const ChunkRows out = chunk_rows<C, ES>(a.y, b, head, c * C, a.T, a.reverse);
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) {
                        if constexpr (BF16) {
                            // (the halves of the wave exchange runs, so that a lane stores eight features at once)
                            u32x2_t x[4];
#pragma unroll
                            for (int q4 = 0; q4 < 4; ++q4) {
                                const u16x4 o = {f32_to_bf16_bits(y[tb][4 * q4]), f32_to_bf16_bits(y[tb][4 * q4 + 1]),
                                                 f32_to_bf16_bits(y[tb][4 * q4 + 2]), f32_to_bf16_bits(y[tb][4 * q4 + 3])};
                                x[q4] = __builtin_bit_cast(u32x2_t, o);
                            }
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                const auto r0 = __builtin_amdgcn_permlane32_swap(x[2 * p][0], x[2 * p + 1][0], false, false);
                                const auto r1 = __builtin_amdgcn_permlane32_swap(x[2 * p][1], x[2 * p + 1][1], false, false);
                                const int col = v0 + 32 * w + 16 * p + 8 * g;
                                __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{r0[0], r1[0], r0[1], r1[1]}, out.rows,
                                                                       chunk_offset<ES>(a.y, 32 * tb + n, col, col < a.dv, a.reverse) + out.top, 0, 0);
                            }
                        } else {
#pragma unroll
                            for (int q4 = 0; q4 < 4; ++q4) {
                                const int col = v0 + 32 * w + 8 * q4 + 4 * g;
                                const f32x4 x = {y[tb][4 * q4], y[tb][4 * q4 + 1], y[tb][4 * q4 + 2], y[tb][4 * q4 + 3]};
                                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), out.rows,
                                                                       chunk_offset<ES>(a.y, 32 * tb + n, col, col < a.dv, a.reverse) + out.top, 0, 0);
                            }
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }

            // ---- S <- zeta_C S + sum_s w_s v_s k_s^T
            if (GROUP == kSources ? s == 0 : s + 1 == steps) {
#pragma unroll
                for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[jb][r] *= zeta_C;
            }
            if (GROUP == kSources || s + 1 == steps) {
#pragma unroll
                for (int sb = 0; sb < TB; ++sb)
#pragma unroll
                    for (int st = 0; st < HS; ++st) {
                        float x[MMA::VEC];
                        MMA::unpack(vt[sb][st], x);
                        if constexpr (BF16) {
                            const int t0 = 32 * sb + 16 * st + 4 * g;
                            const f32x4 w0 = *(const f32x4 *)(sW + t0), w1 = *(const f32x4 *)(sW + t0 + 8);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] *= w0[e];
                                x[4 + e] *= w1[e];
                            }
                        } else {
                            x[0] *= sW[kidx(st, g)];
                        }
                        frag f[VW];
                        cut<MMA, VW>(x, f);
#pragma unroll
                        for (int jb = 0; jb < NBK; ++jb) {
                            const frag kt = col_frag(sK, RSK, 32 * jb, sb, st, lane);
#pragma unroll
                            for (int i = 0; i < VW; ++i) acc[jb] = MMA::mma(kt, f[i], acc[jb]);
                        }
                    }
            }
        }
    }

    if constexpr (SUMMARY) {
        float *s = a.seg_states + seg_state_at(a, pair, slice, seg, state_floats) + w * NBK * 1024;
#pragma unroll
        for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *(f32x4 *)(s + (jb * 4 + q4) * 256 + 4 * lane) =
                    f32x4{acc[jb][4 * q4], acc[jb][4 * q4 + 1], acc[jb][4 * q4 + 2], acc[jb][4 * q4 + 3]};
        if (tid == 0 && slice == 0) a.seg_decay[(int64_t)pair * a.n_segs + seg] = seg_decay;
    } else if (seg == a.n_segs - 1) {
        if (a.state_dot_out) {
            const StateAt S(a.state_dot_with, pair, a, v0 + 32 * w, lane);
            float dot = 0.0f;
#pragma unroll
            for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 x = S.load(jb, q4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dot += x[e] * acc[jb][4 * q4 + e];
                }
            dot = wave_sum(dot);
            lds_barrier();
            if (lane == 0) sHi[w] = dot;
            lds_barrier();
            if (tid == 0) {
                float all = 0.0f;
#pragma unroll
                for (int i = 0; i < NW; ++i) all += sHi[i];
                a.state_dot_out[(int64_t)slice * n_pairs + pair] = all;
            }
        }
        if (a.final) {
            const StateAt S(a.final, pair, a, v0 + 32 * w, lane);
            float scale = 1.0f;
            if (a.final_times_gate) scale = __builtin_amdgcn_exp2f(log2_gate(a.gate_per_head ? a.gate[h] : a.gate[(int64_t)b * a.T * a.Hkv + h]));
#pragma unroll
            for (int jb = 0; jb < NBK; ++jb)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
                    S.store(jb, q4, f32x4{acc[jb][4 * q4], acc[jb][4 * q4 + 1], acc[jb][4 * q4 + 2], acc[jb][4 * q4 + 3]} * scale);
        }
    }
}

// What the segments add -> the states that they start from, in place: a thread carries four floats of a state over the segments.
template <int DK, int NW>
__global__ __launch_bounds__(256) void linear_scan_kernel(LinearWalkArgs a)
{
    constexpr int NBK = DK / 32;
    constexpr int64_t state_floats = (int64_t)32 * NW * DK;
    constexpr int BLOCKS = (int)(state_floats / 1024);         // workgroups for a state of a slice
    const int part = blockIdx.x % BLOCKS;
    const int slice = blockIdx.x / BLOCKS % a.slices;
    const int pair = blockIdx.x / BLOCKS / a.slices;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    const int at = (part * 256 + threadIdx.x) * 4;             // ((w NBK + jb) 4 + q4) 256 + 4 lane
    float *s = a.seg_states + seg_state_at(a, pair, slice, 0, state_floats) + at;
    f32x4 run = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.init) {
        const int lane = at / 4 % 64, q4 = at / 256 % 4, jb = at / 1024 % NBK, w = at / 1024 / NBK;
        const StateAt S(a.init, (int64_t)(b / a.share) * a.Hkv + h, a, slice * 32 * NW + 32 * __builtin_amdgcn_readfirstlane(w), lane);
        run = S.load(__builtin_amdgcn_readfirstlane(jb), __builtin_amdgcn_readfirstlane(q4));
    }
    const float *decay = a.seg_decay + (int64_t)pair * a.n_segs;
    f32x4 next = *(const f32x4 *)s;
    for (int seg = 0; seg < a.n_segs; ++seg) {
        const f32x4 adds = next;
        if (seg + 2 < a.n_segs) next = *(const f32x4 *)(s + (seg + 1) * state_floats);
        *(f32x4 *)(s + seg * state_floats) = run;
        if (seg + 1 < a.n_segs) run = run * decay[seg] + adds;
    }
}

template <class MMA, int DK, int NW, int PIECES, bool DOT, bool SUMMARY, Group GROUP>
hipError_t launch_kernel(const LinearWalkArgs &a, int workgroups, hipStream_t stream)
{
    typedef Shape<MMA, DK, NW> SH;
    constexpr size_t lds = SH::lds_bytes(PIECES, SUMMARY);
    static bool raised[kMaxLdsDevices] = {};
    const hipError_t e = raise_lds_limits(raised, {{(const void *)linear_walk_kernel<MMA, DK, NW, PIECES, DOT, SUMMARY, GROUP>, lds}});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((linear_walk_kernel<MMA, DK, NW, PIECES, DOT, SUMMARY, GROUP>), dim3(workgroups), dim3(SH::NT), lds, stream, a);
    return hipGetLastError();
}

template <class MMA, int DK, int NW, Group GROUP>
hipError_t launch_walk(const LinearWalkArgs &a, hipStream_t stream)
{
    constexpr bool BF16 = Shape<MMA, DK, NW>::BF16;
    const int n = a.B * a.Hkv * a.slices;
    if (a.n_segs > 1) {
        hipError_t e = launch_kernel<MMA, DK, NW, 1, false, true, GROUP == kSources ? kSources : kOne>(a, n * (a.n_segs - 1), stream);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((linear_scan_kernel<DK, NW>), dim3(n * (32 * NW * DK / 1024)), dim3(256), 0, stream, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return a.dot_out ? launch_kernel<MMA, DK, NW, BF16 ? 3 : 1, true, false, GROUP>(a, n * a.n_segs, stream)
                     : launch_kernel<MMA, DK, NW, BF16 ? 2 : 1, false, false, GROUP>(a, n * a.n_segs, stream);
}

template <class MMA, int DK>
hipError_t launch_walk_dk(const LinearWalkArgs &a, hipStream_t stream)
{
    const bool narrow = a.dv <= 64;
    if (a.n_q > 1) return narrow ? launch_walk<MMA, DK, 2, kQueries>(a, stream) : launch_walk<MMA, DK, 4, kQueries>(a, stream);
    if (a.n_src > 1) return narrow ? launch_walk<MMA, DK, 2, kSources>(a, stream) : launch_walk<MMA, DK, 4, kSources>(a, stream);
    return narrow ? launch_walk<MMA, DK, 2, kOne>(a, stream) : launch_walk<MMA, DK, 4, kOne>(a, stream);
}

}  // namespace linear
}  // namespace gka
