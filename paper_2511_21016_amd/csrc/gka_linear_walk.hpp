// Linear attention with a decay for each head over whole sequences:
//   S_t = gate_t S_{t-1} + v_t k_t^T,   y_t = S_t q_t       (S [dv, dk] in float32, one for each sequence and kv head)
// chunk by chunk (C tokens, G_t the cumulative log2 decay inside the chunk, zeta_t = 2^G_t, M[t, s] = 2^(G_t - G_s), s <= t):
//   y_t = zeta_t S_[n] q_t + sum_{s <= t} M[t, s] (k_s . q_t) v_s,     S_[n+1] = zeta_C S_[n] + sum_s 2^(G_C - G_s) v_s k_s^T.
// The same walk with other tensors in the roles of q, k, v gives the three gradients (LinearWalkArgs).
//
// A workgroup walks the chunks of one segment of one (sequence, kv head), for a slice of up to 128 of the dv features, with the
// state in registers. Everything is built from 16 x 16 MFMA tiles: lane 16 kg + n of an accumulator holds rows 4 kg + r (r = 0..3)
// of column n. Wave w holds v-features 16 w .. + 15 of the slice for all k-features: tile j is S^T's rows (k-features) 16 j .. and
// columns (v-features) 16 w ... Two tiles convert in place into one A operand of S q, whose contraction index is then
// enumerated 4 kg .. + 3, 16 + 4 kg .. + 3 within each 32 (bf16; float32: tile by tile); q rows lie in LDS in that order, and
// the masked products of two key tiles are an operand of the product with v without leaving their lanes. Few registers a wave
// (128: four waves on a SIMD) matter more here than operand reuse: a chunk is a chain of short phases with barriers between.
// Segments start from states that a summary launch (SUMMARY: the updates alone) leaves in the workspace.
//
// Bound by the phases of a chunk, with two workgroups on a CU to fill each other's waits: 64 states of d 128 x 4096 tokens (bf16), walk 86
// us, summary 34 us (120 MiB of reads, 3.7 TB/s); the walk's matrix pipe is busy 39 per cent of the time, vector instructions take 51,
// LDS 36 (1/7 of that bank conflicts). The backward pass's three walks: 290 us, 37, 54 and 35 per cent. Slices of 64 features with four
// waves took 10 per cent more for the pass; tiles of 32 features a wave would need 256 registers, two waves on a SIMD.
//
// Precision. bf16 tensors enter the products as they are; what is computed in float32 (states, masked products, weighted
// v) is cut into three bf16 pieces, which hold all of its 24 bits. (Two pieces in the readout round one in 400 of the bf16 outputs
// the other way than its exact value, and take 13 per cent less: 64 states of d 128 x 4096 tokens, 107 us the pass against 120.)
// float32 tensors use the float32 MFMA. Decays are summed in float64 and kept as two floats: a difference of two of them is then
// exact to float32 wherever a sequence is wiped by a gate of 0 (2^-144 each) before.
#pragma once
#include "gka_device.hpp"
#include "gka_linear.hpp"

namespace gka {
namespace linear {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// Products of 16 x 16 tiles. STEPS: MFMAs for a contraction over 32; VEC: operand elements per lane of each.
struct Tile16BF16 {
    static constexpr bool BF16 = true;
    static constexpr int VEC = 8, STEPS = 1, PIECES = 3;       // (of a float32 operand)
    typedef bf16x8 frag;
    typedef uint16_t elem_t;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ frag pack(const float *x) { return MmaBF16::pack(x); }
    static __device__ __forceinline__ void unpack(frag f, float *x) { MmaBF16::unpack(f, x); }
};
struct Tile16F32 {
    static constexpr bool BF16 = false;
    static constexpr int VEC = 1, STEPS = 8, PIECES = 1;
    typedef float frag;
    typedef float elem_t;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ frag pack(const float *x) { return x[0]; }
    static __device__ __forceinline__ void unpack(frag f, float *x) { x[0] = f; }
};

// Row-major LDS tiles, D elements a row. Padded: the lanes of a read fall into different banks for bf16 transpose reads, 32 bytes of
// 8 rows (32 bytes of padding), and float32 reads of 16 columns of 4 rows that are 4 apart (16). Everything but a lane's own
// base is then an offset known when compiling.
template <int D, int ES, int PAD>
struct PaddedTile16 {
    static constexpr int ROW = D * ES + PAD;
    // byte offset of 16-byte piece `piece` of row `row`
    static __device__ __forceinline__ int at(int row, int piece) { return row * ROW + piece * 16; }
    // `pieces` further in the same row
    static __device__ __forceinline__ int further(int offset, int pieces) { return offset + pieces * 16; }
};
// Swizzled (bf16): no padding, a row's pieces permuted by a XOR. A 16-byte read of 16 rows and two neighbouring pieces runs in groups
// of 16 lanes, rows 0-3 and 12-15 of one piece with rows 4-11 of the other; a transpose read in halves of 8 rows by 32 bytes. Rows
// 0-7 are given different pairs of pieces and rows 8-15 the other members of the pairs, in such an order that both reads meet
// every bank once. (Padded rows instead, d = 128: 24 and 8 cycles for the reads of k rows and q rows, 8 and 4 without conflicts.)
template <int D>
struct SwizzledTile16 {
    static constexpr int PIECES = D / 8, ROW = 2 * D;
    static __device__ __forceinline__ int swizzle(int row)
    {
        if constexpr (PIECES >= 16) return ((row & 7) ^ (row >> 1 & 4)) << 1 | (row >> 3 & 1);
        else return ((row >> 1 & 3) ^ (row >> 2 & 2)) << 1 | (row >> 3 & 1);
    }
    static __device__ __forceinline__ int at(int row, int piece) { return row * ROW + (piece ^ swizzle(row)) * 16; }
    // (where `pieces` has no bits in common with the piece of `offset`)
    static __device__ __forceinline__ int further(int offset, int pieces) { return offset ^ pieces * 16; }
};

// Place of a piece of row `row` + `pass` ROWS: a fixed distance on where ROWS is a multiple of 16, after which the swizzle repeats.
template <class T, int ROWS>
__device__ __forceinline__ int row_of_pass(int row, int piece, int pass)
{
    if constexpr (ROWS % 16 == 0) return T::at(row, piece) + pass * ROWS * T::ROW;
    else return T::at(row + pass * ROWS, piece);
}

// The value again, as one that the compiler does not know: what is computed from it inside a loop is not kept in registers across
// it (some thirty offsets into the swizzled tiles, one XOR each, spilled otherwise).
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Fragments of step `st` of the contraction over a 32-block `blk`, from the lane's own place in the tile (the functions *_place).
// Rows row0 + n of q: its LDS tile holds the features of each 32 in the order of the operands (bf16: piece kg of the block is
// features 4 kg .. + 3 and 16 + 4 kg .. + 3) ...
template <class T>
__device__ __forceinline__ int q_place(int lane) { return T::at(lane & 15, lane >> 4); }
template <class M, class T>
__device__ __forceinline__ typename M::frag q_frag(const unsigned char *tile, int place, int row0, int blk, int st)
{
    if constexpr (M::BF16) return __builtin_bit_cast(bf16x8, *(const u32x4_t *)(tile + T::further(place, 4 * blk) + row0 * T::ROW));
    else return (*(const f32x4 *)(tile + T::further(place, 8 * blk + 4 * (st >> 2)) + row0 * T::ROW))[st & 3];
}
// ... rows row0 + n of k: theirs lie in natural order, for the transpose reads ...
template <class M, class T>
__device__ __forceinline__ int k_place(int lane)
{
    if constexpr (M::BF16) return T::at(lane & 15, lane >> 5) + 8 * (lane >> 4 & 1);
    else return q_place<T>(lane);
}
template <class M, class T>
__device__ __forceinline__ typename M::frag k_frag(const unsigned char *tile, int place, int row0, int blk, int st)
{
    if constexpr (M::BF16) {
        const u32x2_t a = *(const u32x2_t *)(tile + T::further(place, 4 * blk) + row0 * T::ROW);
        const u32x2_t b = *(const u32x2_t *)(tile + T::further(place, 4 * blk + 2) + row0 * T::ROW);
        const u32x4_t u = {a[0], a[1], b[0], b[1]};
        return __builtin_bit_cast(bf16x8, u);
    } else {
        return q_frag<M, T>(tile, place, row0, blk, st);
    }
}
// ... and columns 16 c16 .. + 15, contraction over the 32 rows (tokens) of block `blk`. bf16: within 16 lanes, lane i supplies the
// address of row i / 4 at columns 4 (i % 4) .. and receives four rows of its own column.
template <class M, class T>
__device__ __forceinline__ int col_place(int lane)
{
    const int kg = lane >> 4, i = lane & 15;
    if constexpr (M::BF16) return T::at(4 * kg + (i >> 2), i >> 1 & 1) + 8 * (i & 1);
    else return T::at(4 * kg, i >> 2) + 4 * (i & 3);
}
template <class M, class T>
__device__ __forceinline__ typename M::frag col_frag(const unsigned char *tile, int place, int c16, int blk, int st)
{
    if constexpr (M::BF16) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const unsigned char *p = tile + T::further(place, 2 * c16) + 32 * blk * T::ROW;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 16 * T::ROW));
        const s16x8 r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        return __builtin_bit_cast(bf16x8, r);
    } else {
        return *(const float *)(tile + T::further(place, 4 * c16) + (32 * blk + 16 * (st >> 2) + (st & 3)) * T::ROW);
    }
}

// VEC floats as pieces of operand precision; all of them together hold 8 bits per piece (float32 operands: one piece, exact). What a
// piece leaves over is x - piece, exact in float32: one dot product of the packed pair with (-1, 0) or (0, -1), added to x, instead
// of an unpacking and a subtraction for each element. (The factors come from registers: as a literal, (0, -1) has the bits of
// the inline constant -1.0, which the instruction reads otherwise. As assembly, because the compiler only knows the form that
// overwrites x and copies x first. Waits: other instructions may read a dot product's result three states later, hence the
// s_nop; none is needed where x comes from a matrix instruction, because the packing before has read the same registers.)
template <class M, int N>
__device__ __forceinline__ void cut(const float *x, typename M::frag (&f)[N])
{
    if constexpr (!M::BF16) {
        static_assert(N == 1, "float32 operands are not cut");
        f[0] = x[0];
    } else {
        uint32_t first = 0x0000bf80u, second = 0xbf800000u;
        asm("" : "+s"(first), "+s"(second));
        float rest[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f[i] = M::pack(rest);
            if (i + 1 < N) {
                const u32x4_t pairs = __builtin_bit_cast(u32x4_t, f[i]);
                float left[8];
                asm("v_dot2_f32_bf16 %0, %8, %12, %14\n\tv_dot2_f32_bf16 %1, %8, %13, %15\n\t"
                    "v_dot2_f32_bf16 %2, %9, %12, %16\n\tv_dot2_f32_bf16 %3, %9, %13, %17\n\t"
                    "v_dot2_f32_bf16 %4, %10, %12, %18\n\tv_dot2_f32_bf16 %5, %10, %13, %19\n\t"
                    "v_dot2_f32_bf16 %6, %11, %12, %20\n\tv_dot2_f32_bf16 %7, %11, %13, %21\n\ts_nop 2"
                    : "=&v"(left[0]), "=&v"(left[1]), "=&v"(left[2]), "=&v"(left[3]), "=&v"(left[4]), "=&v"(left[5]), "=&v"(left[6]),
                      "=&v"(left[7])
                    : "v"(pairs[0]), "v"(pairs[1]), "v"(pairs[2]), "v"(pairs[3]), "s"(first), "s"(second), "v"(rest[0]), "v"(rest[1]),
                      "v"(rest[2]), "v"(rest[3]), "v"(rest[4]), "v"(rest[5]), "v"(rest[6]), "v"(rest[7]));
#pragma unroll
                for (int e = 0; e < 8; ++e) rest[e] = left[e];
            }
        }
    }
}

// Whether a wave's v fragments hold infinities or NaN.
template <class M, int SB>
__device__ __forceinline__ bool any_nonfinite(const typename M::frag (&v)[SB][M::STEPS])
{
    // (0 unless one of them is infinite or NaN)
    float zero = 0.0f;
#pragma unroll
    for (int sb = 0; sb < SB; ++sb)
#pragma unroll
        for (int st = 0; st < M::STEPS; ++st) {
            if constexpr (M::BF16) {
                typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
                const u32x4_t u = __builtin_bit_cast(u32x4_t, v[sb][st]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t pair = u[e];
                    zero = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, pair), __builtin_bit_cast(pair_t, 0u), zero, false);
                }
            } else {
                zero = __builtin_fmaf(v[sb][st], 0.0f, zero);
            }
        }
    return __ballot(!(zero == 0.0f)) != 0;
}

// The fragments with zeros for infinities and NaN; returns the chunk's tokens that have one in feature lane % 16, a bit each.
template <class M, int SB>
__device__ __forceinline__ uint64_t clear_nonfinite(typename M::frag (&v)[SB][M::STEPS], int lane)
{
    uint64_t bad = 0;
#pragma unroll
    for (int sb = 0; sb < SB; ++sb)
#pragma unroll
        for (int st = 0; st < M::STEPS; ++st) {
            if constexpr (M::BF16) {
                u32x4_t u = __builtin_bit_cast(u32x4_t, v[sb][st]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t exponent = e & 1 ? 0x7f800000u : 0x7f80u;
                    if ((u[e / 2] & exponent) == exponent) {
                        bad |= 1ull << (32 * sb + 16 * (e >> 2) + (e & 3) + 4 * (lane >> 4));
                        u[e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
                    }
                }
                v[sb][st] = __builtin_bit_cast(typename M::frag, u);
            } else if ((__float_as_uint(v[sb][st]) & 0x7f800000u) == 0x7f800000u) {
                bad |= 1ull << (32 * sb + 16 * (st >> 2) + (st & 3) + 4 * (lane >> 4));
                v[sb][st] = 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
    for (int lanes = 16; lanes <= 32; lanes *= 2) {
        const uint32_t lo = __shfl_xor((uint32_t)bad, lanes, 64), hi = __shfl_xor((uint32_t)(bad >> 32), lanes, 64);
        bad |= (uint64_t)hi << 32 | lo;
    }
    return bad;
}

// The fragments with zeros for the tokens before `first`.
template <class M, int SB>
__device__ __forceinline__ void clear_before(typename M::frag (&v)[SB][M::STEPS], int first, int lane)
{
#pragma unroll
    for (int sb = 0; sb < SB; ++sb)
#pragma unroll
        for (int st = 0; st < M::STEPS; ++st) {
            const int token = 32 * sb + 4 * (lane >> 4);
            if constexpr (M::BF16) {
                u32x4_t u = __builtin_bit_cast(u32x4_t, v[sb][st]);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (token + 16 * (e >> 2) + (e & 3) < first) u[e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
                v[sb][st] = __builtin_bit_cast(typename M::frag, u);
            } else if (token + 16 * (st >> 2) + (st & 3) < first) {
                v[sb][st] = 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
}

// DK: padded features of q and k. NW: waves, 16 features of v each.
template <class M, int DK, int NW>
struct Shape {
    static constexpr int ES = sizeof(typename M::elem_t);
    static constexpr int C = M::BF16 ? 64 : 32;    // tokens of a chunk
    static constexpr int TB = C / 16, SB = C / 32; // blocks of 16 tokens, of 32 keys
    static constexpr int NT = 64 * NW, NJ = DK / 16, KB = DK / 32;
    static constexpr int E = 16 / ES;              // elements of a 16-byte piece
    static constexpr int PK = (C * DK / E + NT - 1) / NT;     // pieces of a chunk's q or k rows per thread
    static constexpr int PV = C * 16 / E / 64;     // ... of its v rows
    static constexpr int UNITS = M::BF16 ? 6 : 2;  // (token block, 32 keys at or before it)
    typedef std::conditional_t<M::BF16, SwizzledTile16<DK>, PaddedTile16<DK, ES, 16>> QT;
    typedef QT KT;
    typedef PaddedTile16<16 * NW, ES, M::BF16 ? 32 : 16> VT;
    static constexpr size_t q_bytes = (size_t)C * QT::ROW, k_bytes = (size_t)C * KT::ROW, v_bytes = (size_t)C * VT::ROW;
    static constexpr size_t unit_bytes = M::STEPS * 64 * sizeof(typename M::frag);
    static constexpr size_t tables = 2 * 5 * 64 * sizeof(float);
    static constexpr size_t dot_bytes = (size_t)NW * C * sizeof(double);
    static constexpr size_t p_bytes = UNITS * unit_bytes * M::PIECES;
    static constexpr size_t lds_bytes(bool summary, bool dot)
    {
        return k_bytes + v_bytes + tables + (summary ? 0 : q_bytes + p_bytes + (dot ? dot_bytes : 0));
    }
    static_assert((C * DK / E) % NT == 0 && NT % (DK / E) == 0, "a thread's pieces lie in one column");
};

__device__ __forceinline__ int64_t seg_state_at(const LinearWalkArgs &a, int64_t pair, int slice, int seg, int64_t state_floats)
{
    return ((pair * a.slices + slice) * a.n_segs + seg) * state_floats;
}

// The segments' states as wave w of a slice reads them: its own tile j (written by the same wave of a summary), or, where they are
// those of the walk with transposed states (seg_turned: waves, tiles a wave and slices of that walk), the lane's elements of the
// tile with rows and columns exchanged.
template <bool TURNED>
struct SegStates {
    const float *p;
    int64_t step;                                  // floats from a segment to the next
    int row_block, waves, tiles, slices, n_segs;
    __device__ __forceinline__ SegStates(const LinearWalkArgs &a, int64_t pair, int slice, int w, int lane, int NW, int NJ)
    {
        if constexpr (!TURNED) {
            step = (int64_t)NW * NJ * 256;
            p = a.seg_states + seg_state_at(a, pair, slice, 0, step) + (w * NJ * 64 + lane) * 4;
        } else {
            waves = a.seg_turned[0];
            tiles = a.seg_turned[1];
            slices = a.seg_turned[2];
            n_segs = a.n_segs;
            step = (int64_t)waves * tiles * 256;
            row_block = slice * NW + w;            // its 16 v-features are that walk's k-features of this tile
            p = a.seg_states + pair * slices * n_segs * step + (16 * ((lane & 15) >> 2) + 4 * (lane >> 4)) * 4 + (lane & 3);
        }
    }
    __device__ __forceinline__ f32x4 load(int seg, int j) const
    {
        if constexpr (!TURNED) return *(const f32x4 *)(p + seg * step + j * 256);
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        const int slice = j / waves, w = j % waves;
        if (row_block >= tiles || slice >= slices) return x;
        const float *from = p + ((int64_t)slice * n_segs + seg) * step + (w * tiles + row_block) * 256;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = from[4 * r];
        return x;
    }
};

// A caller's state [dv, dk] (or stored [dk, dv]) as a raw buffer: rows and columns of the padding read as zeros, writes to them are
// dropped. Lane 16 kg + n of the wave whose first v-feature is `row0`: run j is its elements [16 j + 4 kg .. + 3][row0 + n].
struct StateAt {
    buffer_rsrc state;
    int lane_offset, dk, pitch;                    // pitch: bytes from one k-feature to the next
    bool transposed;
    __device__ __forceinline__ StateAt(const float *states, int64_t index, const LinearWalkArgs &a, int row0, int lane)
    {
        const int row = row0 + (lane & 15), kg = lane >> 4;
        state = __builtin_amdgcn_make_buffer_rsrc((void *)(states + index * a.dv * a.dk), 0, a.dv * a.dk * 4, 0x00020000);
        transposed = a.transposed != 0;
        pitch = transposed ? 4 * a.dv : 4;
        dk = a.dk;
        lane_offset = row < a.dv ? row * (transposed ? 4 : 4 * a.dk) + 4 * kg * pitch : (int)0x80000000;
    }
    // (dk is a multiple of 16: a run exists for all lanes or for none)
    __device__ __forceinline__ f32x4 load(int j) const
    {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        if (16 * j >= dk) return x;
        const int at = lane_offset + 16 * j * pitch;
        if (!transposed) return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(state, at, 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(state, at + e * pitch, 0, 0));
        return x;
    }
    __device__ __forceinline__ void store(int j, f32x4 x) const
    {
        if (16 * j >= dk) return;
        const int at = lane_offset + 16 * j * pitch;
        if (!transposed) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), state, at, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[e]), state, at + e * pitch, 0, 0);
        }
    }
};

// The rows of one head chunk by chunk, each chunk's a raw buffer: reads of tokens and features that do not exist give zeros and writes
// to them are dropped by the buffer's bounds, without a branch. `lane` offsets (chunk_offset below) count from the first row of
// the buffer. Rows are below 2^23 elements apart, so that a chunk's bytes stay below 2^30. Both directions have the same chunks, of C
// tokens counted from the first one: in reverse it is the walk's first chunk whose rows may be fewer, those that it meets last.
template <int C, int ES>
struct ChunkRows {
    const char *base;                              // the chunk's lowest token
    int pitch;                                     // bytes
    // chunk: from the front
    __device__ __forceinline__ ChunkRows(const RowTensor &x, int b, int head, int chunk)
    {
        pitch = (int)x.st * ES;
        base = (const char *)x.p + (b * x.sb + head * x.sh) * ES + (int64_t)chunk * C * pitch;
    }
    __device__ __forceinline__ void next(int reverse) { base += (int64_t)(reverse ? -C : C) * pitch; }
    // count: tokens of the chunk (0: an empty buffer); head: bytes to a further head
    __device__ __forceinline__ buffer_rsrc rows(int count, int64_t head = 0) const
    {
        return __builtin_amdgcn_make_buffer_rsrc((void *)(base + head), 0, count * pitch, 0x00020000);
    }
    // byte offset of the walk's first token of a whole chunk
    __device__ __forceinline__ int top(int reverse) const { return reverse ? (C - 1) * pitch : 0; }
};
// Offset of feature `col` of the chunk's row `row` but for ChunkRows::top(); far outside for a feature that does not exist. A token
// behind the last one lies behind the buffer's end.
template <int ES>
__device__ __forceinline__ int chunk_offset(const RowTensor &x, int row, int col, bool exists, int reverse)
{
    const int pitch = (int)x.st * ES;
    return exists ? (reverse ? -row : row) * pitch + col * ES : (int)0x80000000;
}

// use(0), .., use(N - 1), each after load(i) into one of two buffers, the next load issued before: LDS reads travel while the products
// of the ones before run. (Left to itself the compiler puts every read right in front of its product and waits for it.)
template <int I, int N, class Buffer, class Load, class Use>
__device__ __forceinline__ void in_flight_step(Buffer (&buffer)[2], Load load, Use use)
{
    if constexpr (I < N) {
        if constexpr (I + 1 < N) load(std::integral_constant<int, I + 1>{}, buffer[(I + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
        use(std::integral_constant<int, I>{}, buffer[I & 1]);
        __builtin_amdgcn_sched_barrier(0);
        in_flight_step<I + 1, N>(buffer, load, use);
    }
}
template <int N, class Buffer, class Load, class Use>
__device__ __forceinline__ void in_flight(Load load, Use use)
{
    Buffer buffer[2];
    load(std::integral_constant<int, 0>{}, buffer[0]);
    in_flight_step<0, N>(buffer, load, use);
}

enum Group { kOne, kQueries, kSources };           // n_q = n_src = 1; several queries; several sources of a token

// Waves on a SIMD that a kernel's registers are limited for: two workgroups of a CU's LDS, one with 256 k-features.
constexpr int walk_waves(int dk, int nw) { return nw == 8 && dk <= 128 ? 4 : 2; }

// DOT: dot_out is wanted. TURNED: see SegStates.
template <class M, int DK, int NW, bool DOT, bool SUMMARY, Group GROUP, bool TURNED = false>
__device__ __forceinline__ void walk(const LinearWalkArgs &a, int workgroup)
{
    typedef Shape<M, DK, NW> SH;
    typedef typename SH::QT QT;
    typedef typename SH::KT KT;
    typedef typename SH::VT VT;
    typedef typename M::frag frag;
    constexpr bool BF16 = M::BF16;
    constexpr int C = SH::C, TB = SH::TB, SB = SH::SB, NT = SH::NT, NJ = SH::NJ, KB = SH::KB, E = SH::E, ES = SH::ES, PK = SH::PK,
                  PV = SH::PV, STEPS = M::STEPS, VEC = M::VEC, PIECES = M::PIECES;
    constexpr bool ROOMY = walk_waves(DK, NW) == 2;
    constexpr int LOOKAHEAD = ROOMY ? 4 : GROUP == kSources ? 1 : 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char *sK = smem, *sV = smem + SH::k_bytes;
    float *tables = (float *)(sV + SH::v_bytes);   // [2][5][64]: log2 decay (two floats), weight in the state, zeta of a token (both with the state's factor); see decays
    unsigned char *sQ = (unsigned char *)tables + SH::tables, *sP = sQ + SH::q_bytes;
    double *sDot = (double *)(sP + SH::p_bytes);        // [NW][C]: the waves' parts of the dot products (DOT)

    const int tid = threadIdx.x;
    const int lane0 = tid & 63, lane = lane0;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n_pairs = a.B * a.Hkv;
    const int pair = workgroup % n_pairs;
    const int slice = workgroup / n_pairs % a.slices;
    const int seg = workgroup / n_pairs / a.slices;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    const int n_chunks = (a.T + C - 1) / C;
    // chunk c of the walk is chunk `from_front(c)` of the tensors; the last of those has `last_count` tokens
    const auto from_front = [&](int c) { return a.reverse ? n_chunks - 1 - c : c; };
    const int last_count = a.T - (n_chunks - 1) * C;
    const int chunk_begin = seg * a.seg_chunks;
    const int chunk_end = min(chunk_begin + a.seg_chunks, n_chunks);
    const int steps = GROUP == kQueries ? a.n_q : GROUP == kSources ? a.n_src : 1;
    const int v0 = slice * 16 * NW;                // first feature of the slice
    constexpr int64_t state_floats = (int64_t)16 * NW * DK;

    // ---- rows of a chunk: memory -> registers (a step ahead) -> LDS
    struct Rows {
        u32x4_t q[SUMMARY ? 1 : PK], k[PK], v[PV];
    };
    constexpr int KROW = DK / E, VROW = 16 * NW / E;          // pieces of a row
    // (a thread's pieces all lie in one column)
    const int q_off = chunk_offset<ES>(a.q, tid / KROW, E * (tid % KROW), E * (tid % KROW) < a.dk, a.reverse);
    const int k_off = chunk_offset<ES>(a.k, tid / KROW, E * (tid % KROW), E * (tid % KROW) < a.dk, a.reverse);
    const int v_off = chunk_offset<ES>(a.v, tid / VROW, v0 + E * (tid % VROW), v0 + E * (tid % VROW) < a.dv, a.reverse);
    // (chunks behind the segment: an empty buffer, zeros without a read. Every path writes the registers, so that they are not
    // held from where they are staged to where the next rows are asked for.)
    typedef ChunkRows<C, ES> Tokens;
    Tokens q_rows(a.q, b, h * (GROUP == kQueries ? steps : 1), from_front(chunk_begin));
    Tokens k_rows(a.k, b, h * (GROUP == kSources ? steps : 1), from_front(chunk_begin));
    Tokens v_rows(a.v, b, h * (GROUP == kSources ? steps : 1), from_front(chunk_begin));
    auto count_of = [&](int c) { return c >= chunk_end ? 0 : from_front(c) == n_chunks - 1 ? last_count : C; };
    auto fetch_rows = [&](auto &to, const Tokens &x, int64_t head, int count, int offset, int rows_per) {
        const buffer_rsrc rows = x.rows(count, head);
        const int top = x.top(a.reverse), step = (a.reverse ? -rows_per : rows_per) * x.pitch;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(to) / 16); ++i)
            to[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rows, offset + (top + i * step), 0, 0));
    };
    auto no_rows = [&](auto &to) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(to) / 16); ++i) to[i] = u32x4_t{0, 0, 0, 0};
    };
    // (of the chunk that q_rows, k_rows and v_rows stand at)
    auto fetch = [&](Rows &f, int count, int s) {
        if constexpr (!SUMMARY) {
            if (GROUP == kQueries || s == 0) fetch_rows(f.q, q_rows, GROUP == kQueries ? s * a.q.sh * ES : 0, count, q_off, NT / KROW);
            else no_rows(f.q);
        }
        if (GROUP == kSources || s == 0) {
            fetch_rows(f.k, k_rows, GROUP == kSources ? s * a.k.sh * ES : 0, count, k_off, NT / KROW);
            fetch_rows(f.v, v_rows, GROUP == kSources ? s * a.v.sh * ES : 0, count, v_off, NT / VROW);
        } else {
            no_rows(f.k);
            no_rows(f.v);
        }
    };
    auto stage = [&](const Rows &f, int s) {
        const int thread = anew(tid);
        const int krow = thread / KROW, kpiece = thread % KROW;
        if constexpr (!SUMMARY)
            if (GROUP == kQueries || s == 0) {
                const int j = kpiece & 3, to = kpiece & ~3, half = 8 * (j >> 1);
#pragma unroll
                for (int i = 0; i < PK; ++i) {
                    if constexpr (BF16) {
                        *(u32x2_t *)(sQ + row_of_pass<QT, NT / KROW>(krow, to + (2 * j & 3), i) + half) = u32x2_t{f.q[i][0], f.q[i][1]};
                        *(u32x2_t *)(sQ + row_of_pass<QT, NT / KROW>(krow, to + (2 * j & 3) + 1, i) + half) = u32x2_t{f.q[i][2], f.q[i][3]};
                    } else {
                        *(u32x4_t *)(sQ + row_of_pass<QT, NT / KROW>(krow, kpiece, i)) = f.q[i];
                    }
                }
            }
        if (GROUP == kSources || s == 0) {
#pragma unroll
            for (int i = 0; i < PK; ++i) *(u32x4_t *)(sK + row_of_pass<KT, NT / KROW>(krow, kpiece, i)) = f.k[i];
#pragma unroll
            for (int i = 0; i < PV; ++i) *(u32x4_t *)(sV + row_of_pass<VT, NT / VROW>(thread / VROW, thread % VROW, i)) = f.v[i];
        }
    };
    const int q_lane = q_place<QT>(lane), k_lane = k_place<M, KT>(lane), kt_lane = col_place<M, KT>(lane);
    const int v_lane = VT::further(col_place<M, VT>(lane), w * (16 * ES / 16));

    // ---- decays: the last wave leaves those of the next chunk in the tables, lane j those of token j. The state is kept up to a
    // factor, `scale`, which takes up the chunks' decays; only where it gets small are the registers multiplied by it, instead of all
    // of them in every chunk. Table[256]: by what they are multiplied in this chunk (1: not), [257] the factor behind the chunk, [258]
    // before it, [259] (DOT) whether the chunk holds a small gate, [260], [261] its tokens whose gates wipe the state, a bit each: what
    // lies before the last of those is left out by selections, in the few chunks that hold one, so that nothing of it comes through.
    float gate = 1.0f, seg_decay = 1.0f, scale = 1.0f;
    uint64_t small_gates = 0;                      // tokens of the chunk whose decays were formed last that have one
    auto fetch_gate = [&](int c) {
        const int token = a.reverse ? (n_chunks - c) * C - lane : c * C + lane;       // whose gate it is (reverse: of the one behind)
        gate = 1.0f;
        if (lane < C && token >= 0 && token < a.T) gate = a.gate_per_head ? a.gate[h] : a.gate[((int64_t)b * a.T + token) * a.Hkv + h];
    };
    auto decays = [&](int c) {
        const double G = wave_inclusive_scan_f64(log2_gate_f64(gate)), total = lane63_f64(G);
        const float hi = (float)G, zeta_C = __builtin_amdgcn_exp2f((float)total);
        const uint64_t wiping = __ballot(!(gate > kWipingGate));
        if constexpr (DOT) small_gates = __ballot(small_gate(gate));
        const float before = scale, after = scale * zeta_C;
        const bool small = wiping != 0 || after < 0x1p-16f;
        float *t = tables + (c & 1) * 320 + lane;
        t[0] = hi;
        t[64] = (float)(G - (double)hi);
        t[128] = __builtin_amdgcn_exp2f((float)(total - G)) * (small ? 1.0f : 1.0f / after);
        t[192] = __builtin_amdgcn_exp2f(hi) * scale;
        scale = small ? 1.0f : after;
        t[256] = lane == 0 ? (small ? after : 1.0f) : lane == 2 ? before : lane < 4 ? scale : __uint_as_float((uint32_t)(lane == 4 ? wiping : wiping >> 32));
        seg_decay = wiping != 0 || seg_decay < 0.0f ? -1.0f : seg_decay * zeta_C;
    };

    Rows rows;
    fetch(rows, count_of(chunk_begin), 0);
    if (w == NW - 1) fetch_gate(chunk_begin);

    // ---- the state that the segment starts from
    f32x4 acc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (!SUMMARY) {
        const SegStates<TURNED> states(a, pair, slice, w, lane, NW, NJ);
        if (a.n_segs > 1 && a.scanned) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[j] = states.load(seg, j);
        } else {
            if (a.init) {
                const StateAt S(a.init, (int64_t)(b / a.share) * a.Hkv + h, a, v0 + 16 * w, lane);
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[j] = S.load(j);
            }
            // (the next segment's in flight while one is added)
            f32x4 next[NJ];
            if (seg > 0) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) next[j] = states.load(0, j);
            }
            for (int before = 0; before < seg; ++before) {
                const float decay = a.seg_decay[(int64_t)pair * a.n_segs + before];
                if (decay < 0.0f) {                // (wiped)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const f32x4 adds = next[j];
                    next[j] = states.load(before + 1 < seg ? before + 1 : before, j);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][r] = decay * acc[j][r] + adds[r];
                }
            }
        }
    }

    // dot products of chunk c (query s), whose parts lie in LDS since the step before: the same barriers serve both. A wave without decays
    // and with the fewest masked products does this.
    auto add_dots = [&](int c, int s) {
        const int lane = anew(lane0), token = from_front(c) * C + (a.reverse ? C - 1 - lane : lane);
        if (w != NW - 2 || lane >= C || token >= a.T) return;
        double dot = 0.0;
#pragma unroll
        for (int i = 0; i < NW; ++i) dot += sDot[i * C + lane];
        a.dot_out[(((int64_t)slice * n_pairs + pair) * a.n_q + s) * a.T + token] = dot;
    };

    Tokens y_rows(a.y, b, h * (GROUP == kQueries ? steps : 1), from_front(chunk_begin));
    Tokens dot_rows(a.dot_with, b, h * (GROUP == kQueries ? steps : 1), from_front(chunk_begin));
    if (w == NW - 1) {
        decays(chunk_begin);
        fetch_gate(chunk_begin + 1);
    }
    for (int c = chunk_begin; c < chunk_end; ++c) {
        const float *sHi = tables + (c & 1) * 320, *sLo = sHi + 64, *sW = sHi + 128, *sZ = sHi + 192;
        const int count = count_of(c);
        uint64_t wiping = 0;
        auto wiping_tokens = [&] {
            return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(__float_as_int(sHi[261])) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane(__float_as_int(sHi[260]));
        };
        f32x4 y[TB];
        for (int s = 0; s < steps; ++s) {
            lds_barrier();                         // the tiles of the step before have been read
            if constexpr (DOT) {
                if (GROUP == kQueries && s > 0) add_dots(c, s - 1);
                else if (s == 0 && c > chunk_begin) add_dots(c - 1, GROUP == kQueries ? steps - 1 : 0);
            }
            stage(rows, s);
            auto fetch_next = [&] {
                const bool more = GROUP != kOne && s + 1 < steps;
                if (!more) {
                    q_rows.next(a.reverse);
                    k_rows.next(a.reverse);
                    v_rows.next(a.reverse);
                }
                fetch(rows, count_of(more ? c : c + 1), more ? s + 1 : 0);
            };
            if (SUMMARY || ROOMY) fetch_next();
            lds_barrier();                         // (no wait for the rows in flight)
            __builtin_amdgcn_sched_barrier(0);
            if (w == NW - 1 && s == 0) {
                if constexpr (DOT) {
                    // (in reverse the gate of the chunk's first token is the first one of the walk's next chunk)
                    const bool any = a.reverse ? (small_gates & ~1ull) != 0 || (__ballot(small_gate(gate)) & 1) != 0 : small_gates != 0;
                    if (lane == 0) {
                        tables[(c & 1) * 320 + 259] = any ? 1.0f : 0.0f;
                        if (!a.reverse && slice == 0) a.small_gates[(int64_t)pair * n_chunks + c] = any;
                    }
                }
                if (c + 1 < chunk_end) {
                    decays(c + 1);                 // (its gates were asked for a chunk ago)
                    fetch_gate(c + 2);
                }
            }

            if constexpr (!SUMMARY) {
                wiping = wiping_tokens();
                // ---- masked products M[t, s] (k_s . q_t): a unit is a block of 16 tokens and 32 keys, left as operand fragments
                const int k_at = anew(k_lane);
                int q_at = anew(q_lane);
                const int lane = anew(lane0), n = lane & 15, kg = lane >> 4;
                for (int unit = w; unit < SH::UNITS; unit += NW) {
                    const int tb = unit < 2 ? unit : 1 + unit / 2, sb = unit < 2 ? 0 : unit & 1;
                    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    f32x4 x[2];
                    constexpr int PB = !BF16 ? 1 : KB < LOOKAHEAD ? KB : LOOKAHEAD;        // 32-blocks of features in flight
                    frag qf[PB][STEPS], kf[2][PB][STEPS];
#pragma unroll
                    for (int k0 = 0; k0 < KB; k0 += PB) {
#pragma unroll
                        for (int kb = 0; kb < PB; ++kb)
#pragma unroll
                            for (int st = 0; st < STEPS; ++st) {
                                qf[kb][st] = q_frag<M, QT>(sQ, q_at, 16 * tb, k0 + kb, st);
                                kf[0][kb][st] = k_frag<M, KT>(sK, k_at, 32 * sb, k0 + kb, st);
                                kf[1][kb][st] = k_frag<M, KT>(sK, k_at, 32 * sb + 16, k0 + kb, st);
                            }
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int kb = 0; kb < PB; ++kb)
#pragma unroll
                            for (int st = 0; st < STEPS; ++st) {
                                x[0] = M::mma(kf[0][kb][st], qf[kb][st], k0 + kb + st == 0 ? zero : x[0]);
                                x[1] = M::mma(kf[1][kb][st], qf[kb][st], k0 + kb + st == 0 ? zero : x[1]);
                            }
                    }
                    // register r: key 32 sb + 16 half + 4 kg + r, token 16 tb + n
                    const float hi = sHi[16 * tb + n], lo = sLo[16 * tb + n];
                    float m[8];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int s0 = 32 * sb + 16 * half + 4 * kg, below = tb - 2 * sb - half;
                        const f32x4 d = (hi - *(const f32x4 *)(sHi + s0)) + (lo - *(const f32x4 *)(sLo + s0));
                        // (keys behind the token are left out by a selection: they may hold anything)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float product = x[half][r] * __builtin_amdgcn_exp2f(d[r]);
                            m[4 * half + r] = below < 0 || (below == 0 && 4 * kg + r > n) ? 0.0f : product;
                        }
                    }
                    if (__builtin_expect(wiping != 0, 0)) {
                        const uint64_t up_to = wiping & ((2ull << (16 * tb + n)) - 1);
                        const int first = up_to != 0 ? 63 - __builtin_clzll(up_to) : 0;        // (the first key that the token sees)
#pragma unroll
                        for (int e = 0; e < 8; ++e) m[e] = 32 * sb + 16 * (e >> 2) + 4 * kg + (e & 3) < first ? 0.0f : m[e];
                    }
#pragma unroll
                    for (int st = 0; st < STEPS; ++st) {
                        frag f[PIECES];
                        cut<M, PIECES>(m + VEC * st, f);
#pragma unroll
                        for (int i = 0; i < PIECES; ++i) ((frag *)sP)[((i * SH::UNITS + unit) * STEPS + st) * 64 + lane] = f[i];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);

                // ---- zeta_t S_[n] q_t: pairs of the state's tiles are the A operand
                q_at = anew(q_at);
                if (GROUP == kQueries || s == 0) {
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        // (the reads travel while the state is cut)
                        frag qf[TB][STEPS];
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                            for (int st = 0; st < STEPS; ++st) qf[tb][st] = q_frag<M, QT>(sQ, q_at, 16 * tb, kb, st);
                        __builtin_amdgcn_sched_barrier(0);
                        const f32x4 lo = acc[2 * kb], hi = acc[2 * kb + 1];
                        const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
                        for (int st = 0; st < STEPS; ++st) {
                            frag f[PIECES];
                            cut<M, PIECES>(x + VEC * st, f);
#pragma unroll
                            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                                for (int tb = 0; tb < TB; ++tb)
                                    y[tb] = M::mma(f[i], qf[tb][st], kb == 0 && st == 0 && i == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : y[tb]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) {
                        const float zeta = sZ[16 * tb + n];
#pragma unroll
                        for (int r = 0; r < 4; ++r) y[tb][r] *= zeta;
                    }
                    if (__builtin_expect(wiping != 0, 0)) {
                        const int seen = __builtin_ctzll(wiping);                              // (tokens that see the state)
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
                            for (int r = 0; r < 4; ++r) y[tb][r] = 16 * tb + n < seen ? y[tb][r] : 0.0f;
                    }
                }
            }
            frag vt[SB][STEPS];                    // v, features on the lanes, contraction over the tokens
#pragma unroll
            for (int sb = 0; sb < SB; ++sb)
#pragma unroll
                for (int st = 0; st < STEPS; ++st) vt[sb][st] = col_frag<M, VT>(sV, v_lane, 0, sb, st);

            if constexpr (!SUMMARY) {
                // Infinities and NaN in v reach the tokens from their own on, in their feature; a product with the zeros of the tokens before
                // would carry them there too. They leave these products and are put in below, where there are any.
                const bool nonfinite = any_nonfinite<M>(vt);
                if (__builtin_expect(nonfinite, 0)) clear_nonfinite<M>(vt, lane0);
                // (rows of the dot products: before the next chunk's, which are not waited for with them)
                std::conditional_t<BF16, u32x2_t, u32x4_t> dot_row[DOT ? TB : 1];
                if constexpr (DOT) {
                    if (GROUP == kQueries || s + 1 == steps) {
                        const int lane = anew(lane0), n = lane & 15, kg = lane >> 4;
                        const buffer_rsrc with = dot_rows.rows(count, (GROUP == kQueries ? s : 0) * a.dot_with.sh * ES);
                        const int top = dot_rows.top(a.reverse);
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) {
                            const int at = chunk_offset<ES>(a.dot_with, 16 * tb + n, v0 + 16 * w + 4 * kg, v0 + 16 * w < a.dv, a.reverse) + top;
                            if constexpr (BF16) dot_row[tb] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(with, at, 0, 0));
                            else dot_row[tb] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(with, at, 0, 0));
                        }
                    }
                }
                // (asked for only now where registers are few: half a chunk ahead, with none of them held through the products before)
                if (!ROOMY) fetch_next();
                lds_barrier();                     // the masked products are there
                __builtin_amdgcn_sched_barrier(0);
                // ---- + sum_s v_s M[t, s] (k_s . q_t)
                const int products = anew(lane0);
                struct Products {
                    frag f[!BF16 ? 8 : ROOMY ? 3 : LOOKAHEAD];
                };
                constexpr int BATCH = sizeof(Products) / sizeof(frag);
                in_flight<PIECES * SH::UNITS * STEPS / BATCH, Products>(
                    [&](auto i, Products &p) {
#pragma unroll
                        for (int e = 0; e < BATCH; ++e) p.f[e] = ((const frag *)sP)[(i * BATCH + e) * 64 + products];
                    },
                    [&](auto i, const Products &p) {
#pragma unroll
                        for (int e = 0; e < BATCH; ++e) {
                            const int at = i * BATCH + e, st = at % STEPS, unit = at / STEPS % SH::UNITS;
                            const int tb = unit < 2 ? unit : 1 + unit / 2, sb = unit < 2 ? 0 : unit & 1;
                            y[tb] = M::mma(vt[sb][st], p.f[e], y[tb]);
                        }
                    });
                if (__builtin_expect(nonfinite, 0)) {
                    const int lane = anew(lane0);
#pragma unroll
                    for (int sb = 0; sb < SB; ++sb)
#pragma unroll
                        for (int st = 0; st < STEPS; ++st) vt[sb][st] = col_frag<M, VT>(sV, v_lane, 0, sb, st);
                    const uint64_t bad = clear_nonfinite<M>(vt, lane);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint64_t of_feature = (uint64_t)__shfl((uint32_t)(bad >> 32), 4 * (lane >> 4) + r, 64) << 32 | __shfl((uint32_t)bad, 4 * (lane >> 4) + r, 64);
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) {
                            const uint64_t up_to = (2ull << (16 * tb + (lane & 15))) - 1, wiped = wiping & up_to;
                            const uint64_t before = wiped != 0 ? (1ull << (63 - __builtin_clzll(wiped))) - 1 : 0;
                            y[tb][r] = (of_feature & up_to & ~before) != 0 ? __builtin_nanf("") : y[tb][r];
                        }
                    }
#pragma unroll
                    for (int sb = 0; sb < SB; ++sb)
#pragma unroll
                        for (int st = 0; st < STEPS; ++st) vt[sb][st] = col_frag<M, VT>(sV, v_lane, 0, sb, st);
                }
                // ---- out: register r holds feature v0 + 16 w + 4 kg + r of token 16 tb + n
                if (GROUP == kQueries || s + 1 == steps) {
                    const int lane = anew(lane0), n = lane & 15, kg = lane >> 4;
                    const int64_t to_head = GROUP == kQueries ? s : 0;
                    const int col = v0 + 16 * w + 4 * kg;
                    const bool in = v0 + 16 * w < a.dv;
                    if constexpr (DOT) {
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb) {
                            f32x4 x;
                            if constexpr (BF16) x = IOBF16::cvt4(__builtin_bit_cast(u16x4, dot_row[tb]));
                            else x = __builtin_bit_cast(f32x4, dot_row[tb]);
                            double dot = 0.0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) dot += (double)x[e] * (double)y[tb][e];
                            dot = sum_over_kg_f64(dot);
                            if (kg == 0) sDot[w * C + 16 * tb + n] = dot;
                        }
                    }
                    const buffer_rsrc out = y_rows.rows(count, to_head * a.y.sh * ES);
                    const int out_top = y_rows.top(a.reverse);
                    if constexpr (BF16) {
                        // (lanes of neighbouring kg exchange runs of two token blocks, so that a lane stores eight features at once)
#pragma unroll
                        for (int tb = 0; tb < TB; tb += 2) {
                            u32x2_t x[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const u16x4 o = {f32_to_bf16_bits(y[tb + i][0]), f32_to_bf16_bits(y[tb + i][1]), f32_to_bf16_bits(y[tb + i][2]),
                                                 f32_to_bf16_bits(y[tb + i][3])};
                                x[i] = __builtin_bit_cast(u32x2_t, o);
                            }
                            const auto r0 = __builtin_amdgcn_permlane16_swap(x[0][0], x[1][0], false, false);
                            const auto r1 = __builtin_amdgcn_permlane16_swap(x[0][1], x[1][1], false, false);
                            // even kg: features 4 kg .. + 7 of block tb; odd kg: 4 (kg - 1) .. + 7 of block tb + 1
                            const int at = chunk_offset<ES>(a.y, 16 * (tb + (kg & 1)) + n, v0 + 16 * w + 4 * (kg & 2), in, a.reverse) + out_top;
                            __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{r0[0], r1[0], r0[1], r1[1]}, out, at, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int tb = 0; tb < TB; ++tb)
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, y[tb]), out,
                                                                   chunk_offset<ES>(a.y, 16 * tb + n, col, in, a.reverse) + out_top, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }

            // ---- S <- zeta_C S + sum_s w_s v_s k_s^T
            if (GROUP == kSources ? s == 0 : s + 1 == steps) {
                if constexpr (DOT) {
                    // (the state before the chunk, for the gradients of its small gates)
                    if (__builtin_amdgcn_readfirstlane(__float_as_uint(sHi[259])) != 0) {
                        const float before = sHi[258];
                        const int64_t at = (((int64_t)pair * a.slices + slice) * n_chunks + from_front(c)) * state_floats;
                        float *to = a.chunk_states + at + (w * NJ * 64 + anew(lane0)) * 4;
#pragma unroll
                        for (int j = 0; j < NJ; ++j) *(f32x4 *)(to + j * 256) = acc[j] * before;
                    }
                }
                if constexpr (SUMMARY) wiping = wiping_tokens();
                const float factor = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(sHi[256])));
                if (__builtin_expect(wiping != 0, 0)) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                } else if (factor != 1.0f) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j) acc[j] *= factor;
                }
            }
            if (GROUP == kSources || s + 1 == steps) {
                const int kt_at = anew(kt_lane), kg = anew(lane0) >> 4;
                if (__builtin_expect(wiping > 1, 0)) {
                    // The tokens before the last wiping one add nothing, whatever they hold. (Every wave clears all their k rows, which no
                    // other product of this step reads any more: what it then reads are zeros, its own or another wave's.)
                    const int first = 63 - __builtin_clzll(wiping);
                    clear_before<M>(vt, first, lane0);
                    for (int i = lane0; i < first * KROW; i += 64) *(u32x4_t *)(sK + KT::at(i / KROW, i % KROW)) = u32x4_t{0, 0, 0, 0};
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
                // BATCH tiles of the state at a time, the steps of the contraction over the tokens on the outside
                constexpr int BATCH = !BF16 ? (NJ < 8 ? NJ : 8) : LOOKAHEAD, PARTS = NJ / BATCH;
                struct Keys {
                    frag f[BATCH];
                };
                frag f[PIECES];
                in_flight<SB * STEPS * PARTS, Keys>(
                    [&](auto i, Keys &k) {
                        constexpr int part = i % PARTS, st = i / PARTS % STEPS, sb = i / PARTS / STEPS;
#pragma unroll
                        for (int e = 0; e < BATCH; ++e) k.f[e] = col_frag<M, KT>(sK, kt_at, part * BATCH + e, sb, st);
                    },
                    [&](auto i, const Keys &k) {
                        constexpr int part = i % PARTS, st = i / PARTS % STEPS, sb = i / PARTS / STEPS;
                        if constexpr (part == 0) {
                            float x[VEC];
                            M::unpack(vt[sb][st], x);
                            if constexpr (BF16) {
                                const f32x4 w0 = *(const f32x4 *)(sW + 32 * sb + 4 * kg), w1 = *(const f32x4 *)(sW + 32 * sb + 16 + 4 * kg);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    x[e] *= w0[e];
                                    x[4 + e] *= w1[e];
                                }
                            } else {
                                x[0] *= sW[32 * sb + 16 * (st >> 2) + 4 * kg + (st & 3)];
                            }
                            cut<M, PIECES>(x, f);
                        }
#pragma unroll
                        for (int n_piece = 0; n_piece < PIECES; ++n_piece)
#pragma unroll
                            for (int e = 0; e < BATCH; ++e) acc[part * BATCH + e] = M::mma(k.f[e], f[n_piece], acc[part * BATCH + e]);
                    });
            }
        }
        if constexpr (!SUMMARY) y_rows.next(a.reverse);
        if constexpr (DOT) dot_rows.next(a.reverse);
    }

    if constexpr (DOT) {
        lds_barrier();
        add_dots(chunk_end - 1, GROUP == kQueries ? steps - 1 : 0);
    }
    {
        const float factor = tables[((chunk_end - 1) & 1) * 320 + 257];
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] *= factor;
    }
    if constexpr (SUMMARY) {
        float *s = a.seg_states + seg_state_at(a, pair, slice, seg, state_floats) + (w * NJ * 64 + lane) * 4;
#pragma unroll
        for (int j = 0; j < NJ; ++j) *(f32x4 *)(s + j * 256) = acc[j];
        if (w == NW - 1 && lane == 0 && slice == 0) a.seg_decay[(int64_t)pair * a.n_segs + seg] = seg_decay;
    } else if (seg == a.n_segs - 1) {
        if (a.state_dot_out) {
            const StateAt S(a.state_dot_with, pair, a, v0 + 16 * w, lane);
            double dot = 0.0;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const f32x4 x = S.load(j);
#pragma unroll
                for (int e = 0; e < 4; ++e) dot += (double)x[e] * (double)acc[j][e];
            }
            dot = lane63_f64(wave_inclusive_scan_f64(dot));
            lds_barrier();
            if (lane == 0) ((double *)tables)[w] = dot;
            lds_barrier();
            if (tid == 0) {
                double all = 0.0;
#pragma unroll
                for (int i = 0; i < NW; ++i) all += ((const double *)tables)[i];
                a.state_dot_out[(int64_t)slice * n_pairs + pair] = all;
            }
        }
        if (a.final) {
            const StateAt S(a.final, pair, a, v0 + 16 * w, lane);
            float scale = 1.0f;
            if (a.final_times_gate) scale = a.gate_per_head ? a.gate[h] : a.gate[(int64_t)b * a.T * a.Hkv + h];
#pragma unroll
            for (int j = 0; j < NJ; ++j) S.store(j, scale > kWipingGate ? acc[j] * scale : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
        }
    }
}

template <class M, int DK, int NW, bool SUMMARY, Group GROUP, bool TURNED>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(walk_waves(DK, NW), walk_waves(DK, NW))))
void linear_walk_kernel(LinearWalkArgs a)
{
    walk<M, DK, NW, false, SUMMARY, GROUP, TURNED>(a, blockIdx.x);
}

// The walks of the backward pass in one launch, `walks` of them (dq, dk, dv; SUMMARY: dq, dk), groups of eight workgroups of each in
// turn: workgroups go round the eight XCDs, so that the walks of a pair's segment meet in one L2 and share its rows, and the
// GPU runs empty once instead of three times.
struct LinearBackwardArgs {
    LinearWalkArgs walk[3];
    int workgroups;                                // of each
};
template <class M, int DK, int NW, bool SUMMARY, bool GROUPED, int WALKS>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(walk_waves(DK, NW), walk_waves(DK, NW))))
void linear_backward_kernel(LinearBackwardArgs a)
{
    const int role = blockIdx.x / 8 % WALKS, workgroup = blockIdx.x / (8 * WALKS) * 8 + blockIdx.x % 8;
    if (workgroup >= a.workgroups) return;
    if (!GROUPED && role <= 1) walk<M, DK, NW, !SUMMARY, SUMMARY, kOne>(a.walk[role], workgroup);
    else if (role == 0) walk<M, DK, NW, !SUMMARY, SUMMARY, GROUPED && !SUMMARY ? kQueries : kOne>(a.walk[0], workgroup);
    else if (role == 1) walk<M, DK, NW, !SUMMARY, SUMMARY, GROUPED ? kSources : kOne>(a.walk[1], workgroup);
    else if constexpr (WALKS == 3) walk<M, DK, NW, false, false, GROUPED ? kSources : kOne, true>(a.walk[2], workgroup);
}

// What the segments add -> the states that they start from, in place, of walk blockIdx.y: a thread carries four floats of a state over
// the segments, sixteen of which it asks for at a time (8 states of 32 KiB x 21 segments, two walks: 6 us,
// against 2 x 9.5 us with one ahead and a launch for each).
template <int DK, int NW>
__global__ __launch_bounds__(64) void linear_scan_kernel(LinearBackwardArgs walks)
{
    constexpr int NJ = DK / 16, AHEAD = 16;
    constexpr int64_t state_floats = (int64_t)16 * NW * DK;
    constexpr int TILES = (int)(state_floats / 256);           // workgroups for a state of a slice; tile: w NJ + j
    const LinearWalkArgs &a = walks.walk[blockIdx.y];
    const int tile = blockIdx.x % TILES, lane = threadIdx.x;
    const int slice = blockIdx.x / TILES % a.slices;
    const int pair = blockIdx.x / TILES / a.slices;
    const int b = pair / a.Hkv, h = pair % a.Hkv;
    float *s = a.seg_states + seg_state_at(a, pair, slice, 0, state_floats) + (tile * 64 + lane) * 4;
    f32x4 run = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.init) run = StateAt(a.init, (int64_t)(b / a.share) * a.Hkv + h, a, slice * 16 * NW + 16 * (tile / NJ), lane).load(tile % NJ);
    const float *decay = a.seg_decay + (int64_t)pair * a.n_segs;
    const int last = a.n_segs - 1;                 // (nothing starts from what it would add: its place only takes a state)
    for (int seg = 0; seg <= last; seg += AHEAD) {
        f32x4 adds[AHEAD];
        float factor[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int at = min(seg + i, last - 1);
            adds[i] = *(const f32x4 *)(s + at * state_floats);
            factor[i] = decay[at];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (seg + i > last) break;
            *(f32x4 *)(s + (seg + i) * state_floats) = run;
            if (factor[i] < 0.0f) run = f32x4{0.0f, 0.0f, 0.0f, 0.0f};     // (wiped)
            run = run * factor[i] + adds[i];
        }
    }
}

template <class Kernel, class Args>
hipError_t launch_kernel(Kernel kernel, bool (&raised)[kMaxLdsDevices], int workgroups, int threads, size_t lds, const Args &a, hipStream_t stream)
{
    const hipError_t e = raise_lds_limits(raised, {{(const void *)kernel, lds}});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(threads), lds, stream, a);
    return hipGetLastError();
}

template <class M, int DK, int NW, bool SUMMARY, Group GROUP, bool TURNED = false>
hipError_t launch_one(const LinearWalkArgs &a, hipStream_t stream)
{
    typedef Shape<M, DK, NW> SH;
    static_assert(SH::lds_bytes(false, true) <= (size_t)160 << 10, "LDS of a CU");
    static bool raised[kMaxLdsDevices] = {};
    return launch_kernel(linear_walk_kernel<M, DK, NW, SUMMARY, GROUP, TURNED>, raised,
                         a.B * a.Hkv * a.slices * (SUMMARY ? a.n_segs - 1 : a.n_segs), SH::NT, SH::lds_bytes(SUMMARY, false), a, stream);
}

template <int DK, int NW>
hipError_t launch_scan(const LinearBackwardArgs &walks, int n, hipStream_t stream)
{
    const LinearWalkArgs &a = walks.walk[0];
    hipLaunchKernelGGL((linear_scan_kernel<DK, NW>), dim3(a.B * a.Hkv * a.slices * (NW * DK / 16), n), dim3(64), 0, stream, walks);
    return hipGetLastError();
}

// The forward pass.
template <class M, int DK, int NW, Group GROUP>
hipError_t launch_forward(const LinearWalkArgs &a, hipStream_t stream)
{
    if (a.n_segs > 1) {
        hipError_t e = launch_one<M, DK, NW, true, kOne>(a, stream);
        if (e == hipSuccess && a.scanned) e = launch_scan<DK, NW>({{a}, 0}, 1, stream);
        if (e != hipSuccess) return e;
    }
    return launch_one<M, DK, NW, false, GROUP>(a, stream);
}
template <class M, int DK>
hipError_t launch_forward_dk(const LinearWalkArgs &a, hipStream_t stream)
{
    const bool narrow = a.dv <= 64;
    if (a.n_q > 1) return narrow ? launch_forward<M, DK, 4, kQueries>(a, stream) : launch_forward<M, DK, 8, kQueries>(a, stream);
    return narrow ? launch_forward<M, DK, 4, kOne>(a, stream) : launch_forward<M, DK, 8, kOne>(a, stream);
}

// The backward pass: dq and dk have states of one shape. dv's, the same as dk's but transposed, start from what dk's segments left;
// where they are of the same padded shape, the three walks are one launch.
template <class M, int DK, int NW, bool GROUPED>
hipError_t launch_backward(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream)
{
    typedef Shape<M, DK, NW> SH;
    LinearBackwardArgs a = {{dq, dk, dv}, 0};
    const int pairs = dq.B * dq.Hkv * dq.slices;
    const auto grid = [&](int walks) { return (a.workgroups + 7) / 8 * 8 * walks; };
    hipError_t e = hipSuccess;
    if (dq.n_segs > 1) {
        static bool raised[kMaxLdsDevices] = {};
        a.workgroups = pairs * (dq.n_segs - 1);
        e = launch_kernel(linear_backward_kernel<M, DK, NW, true, GROUPED, 2>, raised, grid(2), SH::NT, SH::lds_bytes(true, false), a, stream);
        if (e == hipSuccess && dq.scanned) e = launch_scan<DK, NW>(a, 2, stream);
        if (e != hipSuccess) return e;
    }
    a.workgroups = pairs * dq.n_segs;
    if (dv_alike) {
        static bool raised[kMaxLdsDevices] = {};
        return launch_kernel(linear_backward_kernel<M, DK, NW, false, GROUPED, 3>, raised, grid(3), SH::NT, SH::lds_bytes(false, true), a, stream);
    }
    static bool raised[kMaxLdsDevices] = {};
    return launch_kernel(linear_backward_kernel<M, DK, NW, false, GROUPED, 2>, raised, grid(2), SH::NT, SH::lds_bytes(false, true), a, stream);
}
template <class M, int DK>
hipError_t launch_backward_dk(const LinearWalkArgs &dq, const LinearWalkArgs &dk, const LinearWalkArgs &dv, bool dv_alike, hipStream_t stream)
{
    const bool narrow = dq.dv <= 64, grouped = dq.n_q > 1;
    if (grouped) return narrow ? launch_backward<M, DK, 4, true>(dq, dk, dv, dv_alike, stream) : launch_backward<M, DK, 8, true>(dq, dk, dv, dv_alike, stream);
    return narrow ? launch_backward<M, DK, 4, false>(dq, dk, dv, dv_alike, stream) : launch_backward<M, DK, 8, false>(dq, dk, dv, dv_alike, stream);
}
// dv alone
template <class M, int DK>
hipError_t launch_values_dk(const LinearWalkArgs &a, hipStream_t stream)
{
    const bool narrow = a.dv <= 64;
    if (a.n_src > 1) return narrow ? launch_one<M, DK, 4, false, kSources, true>(a, stream)
                                  : launch_one<M, DK, 8, false, kSources, true>(a, stream);
    return narrow ? launch_one<M, DK, 4, false, kOne, true>(a, stream)
                                  : launch_one<M, DK, 8, false, kOne, true>(a, stream);
}

}  // namespace linear
}  // namespace gka
