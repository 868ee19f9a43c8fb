// Products of few rows with 4-bit weights (cascade_w4_gemm), and the layout of the weights (cascade_w4_pack).
//
// What bounds it: every weight is used for a handful of rows, so a launch is as long as streaming the codes from HBM, half a byte
// each.  The 8 wavefronts of a workgroup are column groups by parts of the reduction; each reads the codes of its columns straight
// into matrix operands, a ring of pieces ahead of their use.  X, which all of them need, comes through LDS in the
// order of the operands: whole where it fits, in two halves in turn where not (every wavefront reading its own X from L2: 4 rows of
// 4096x14336 with SwiGLU 31 us instead of 17, since a CU loads some 43 KB a microsecond from L2).
//
// Measured (us a call among others; floor: bytes at the rate of a large copy): 1 row of 4096x4096 6 (1.7: start, X, one round of
// codes and end are a chain of latencies), 4 rows of 4096x14336 with SwiGLU, group 64, 16.9 (12.7), 32 int8 rows of 8192x28672 42.8
// (24.2; instructions, one workgroup a CU, 224 of 256 CUs), 64 rows of 14336x4096 24 (6.5; X is staged for 5, the loop takes 9.5, the 16
// slices' sums out and in 7), 1 row of 4096x128256 61 (53).
//
// Packed layout.  Codes: blocks of 16 columns by 128 reduction elements, 1 KB each, blocks of a column side by side along the
// reduction.  In a block, lane (column l, quarter g) of a wavefront finds its 16 bytes at (16 g + l) * 16: word s holds elements
// 32 s + 8 g .. + 7, which is the operand of one 16x16x32 product, and in a word nibble p < 4 holds element 2p, nibble p + 4
// element 2p + 1.  So two nibbles 16 bits apart become a pair of bf16 numbers by a shift, a mask and an or: 0x4180 | code << 3 is
// 16 + code.  What that adds, and the zero points, come off once per group: scale * (sum x (16 + code) - (16 + zero) * sum x), where
// the sums of X come from one more product per step, with ones, for all columns of the wavefront (fp32 rows: off each code).  INT8 rows
// take codes as bytes (three operations for 8), all in whole numbers up to the scales.  Behind the codes: scales and zeros, [column blocks][groups][16].
#include <algorithm>
#include <type_traits>
#include "common.h"
#include "device_utils.h"
#include "epilogue.h"

namespace {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;
constexpr int NW = 8;                                      // wavefronts of a workgroup (parts of the reduction)
constexpr int BLOCK = 128;                                 // reduction elements of a block of codes

enum XType { X_BF16, X_F32, X_E4M3, X_INT8 };

struct W4Params {
    const char *codes[2], *scales[2], *zeros[2];           // the weights, and EPI_SWIGLU's up weights
    const char *X;
    const float *x_scale;
    const void *bias, *residual;
    void *Y;
    float *planes;                                         // [slices][matrices][row blocks][col blocks][64][4] sums, where the reduction is cut
    int64_t ldx, ldres, ldy;                               // elements
    int32_t M, N, K;
    int32_t blocks, groups;                                // of the reduction
    int32_t row_blocks, col_blocks;                        // of 16
    int32_t group_shift, x_group_shift, x_groups;          // log2 of the elements of a scale (x_group_shift 31: the row)
    int32_t has_zeros, flags;
    int32_t cols_log2;                                     // column groups of a workgroup; 8 >> cols_log2 parts of the reduction
    int32_t slices, slice_blocks;                          // parts of the reduction over workgroups
    int32_t chunk, chunks_held;                            // blocks of X that enter LDS at once; how many chunks LDS has room for
};

template <int XT> constexpr int x_bytes() { return XT == X_BF16 ? 2 : XT == X_F32 ? 4 : 1; }
template <int XT> constexpr int unit_bytes() { return XT == X_F32 ? 48 : XT == X_INT8 ? 8 : 16; }   // 8 columns of a row in LDS
constexpr int MAX_UNITS = 4;                               // of a thread and chunk: chunk * rows * 16 / 512

// 8 columns of X as they came, and in LDS: bf16 numbers (three sets of them for fp32, which add up to it exactly), or bytes in the
// order of the codes' bytes
template <int XT> struct XRaw { u32x4 v; };
template <> struct XRaw<X_F32> { u32x4 v, w; };
template <> struct XRaw<X_E4M3> { u32x2 v; };
template <> struct XRaw<X_INT8> { u32x2 v; };
template <int XT>
__device__ __forceinline__ XRaw<XT> load_x(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    XRaw<XT> x;
    if constexpr (XT == X_E4M3 || XT == X_INT8) x.v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
    else x.v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
    if constexpr (XT == X_F32) x.w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 16, 0));
    return x;
}
template <int XT>
__device__ __forceinline__ void store_x(const XRaw<XT> &x, char *to) {
    if constexpr (XT == X_INT8) {
        *(u32x2 *)to = u32x2{__builtin_amdgcn_perm(x.v[1], x.v[0], 0x05010400u), __builtin_amdgcn_perm(x.v[1], x.v[0], 0x07030602u)};
    } else if constexpr (XT == X_BF16) {
        *(u32x4 *)to = x.v;
    } else {
        float f[8];
        if constexpr (XT == X_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(float, e < 4 ? x.v[e] : x.w[e - 4]);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(x.v[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x.v[h], true);
                f[4 * h] = a[0]; f[4 * h + 1] = a[1]; f[4 * h + 2] = b[0]; f[4 * h + 3] = b[1];
            }
        }
#pragma unroll
        for (int i = 0; i < (XT == X_F32 ? 3 : 1); ++i) {
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = (bf16_t)f[e];
                f[e] -= (float)v[e];
            }
            *(bf16x8 *)(to + 16 * i) = v;
        }
    }
}

// 8 codes of a word as 16 + code
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t w) {
    constexpr uint32_t MASK = 0x00780078u, BASE = 0x41804180u;
    const u32x4 v = {((w << 3) & MASK) | BASE, ((w >> 1) & MASK) | BASE, ((w >> 5) & MASK) | BASE, ((w >> 9) & MASK) | BASE};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ int64_t codes_int8(uint32_t w) {
    const u32x2 v = {w & 0x0f0f0f0fu, (w >> 4) & 0x0f0f0f0fu};
    return __builtin_bit_cast(int64_t, v);
}

template <int XT> using Sum = typename std::conditional<XT == X_INT8, i32x4, f32x4>::type;
// 8 columns of X as an operand (three of them for fp32)
template <int XT> struct XOperand { bf16x8 v[XT == X_F32 ? 3 : 1]; };
template <> struct XOperand<X_INT8> { int64_t v; };
template <int XT>
__device__ __forceinline__ XOperand<XT> operand(const char *x) {
    XOperand<XT> o;
    if constexpr (XT == X_INT8) o.v = *(const int64_t *)x;
    else {
#pragma unroll
        for (int l = 0; l < (XT == X_F32 ? 3 : 1); ++l) o.v[l] = *(const bf16x8 *)(x + 16 * l);
    }
    return o;
}
// The operands of a step's codes, and of ones
template <int XT> using WOperand = typename std::conditional<XT == X_INT8, int64_t, bf16x8>::type;
template <int XT>
__device__ __forceinline__ WOperand<XT> codes(uint32_t w) {
    if constexpr (XT == X_INT8) return codes_int8(w);
    else return codes_bf16(w);
}
// 8 codes less the zero point (whole numbers of four bits and a sign)
__device__ __forceinline__ bf16x8 codes_less(uint32_t w, float zero_16) {
    u32x4 v = __builtin_bit_cast(u32x4, codes_bf16(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __builtin_bit_cast(float, v[i] << 16) - zero_16, b = __builtin_bit_cast(float, v[i] & 0xffff0000u) - zero_16;
        v[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, v);
}
template <int XT>
__device__ __forceinline__ WOperand<XT> ones_operand() {
    if constexpr (XT == X_INT8) return 0x0101010101010101ll;
    else return __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
}
// acc + x w over STEPS steps.  Two steps of bytes go into one 16x16x64 product, which has twice the rate of 16x16x32; in which order
// a lane's 16 elements stand is free, as long as it is the same on both sides.
template <int XT, int STEPS, int STRIDE>
__device__ __forceinline__ Sum<XT> product(const XOperand<XT> *x, const WOperand<XT> *w, Sum<XT> acc) {
    if constexpr (XT == X_INT8 && STEPS > 1) {
        typedef __attribute__((ext_vector_type(2))) int64_t i64x2;
#pragma unroll
        for (int s = 0; s < STEPS; s += 2)
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, i64x2{x[s * STRIDE].v, x[(s + 1) * STRIDE].v}),
                                                        __builtin_bit_cast(i32x4, i64x2{w[s], w[s + 1]}), acc, 0, 0, 0);
    } else if constexpr (XT == X_INT8) {
        acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(x[0].v, w[0], acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int l = 0; l < (XT == X_F32 ? 3 : 1); ++l) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s * STRIDE].v[l], w[s], acc, 0, 0, 0);
    }
    return acc;
}

// A row's outputs of 16 columns from the formula, term by term, in 64 bits: column l16 in every quarter's lanes.  The products above give
// NaN where a row holds an infinity (16 + code and 16 + zero meet it with opposite signs; in fp32 its further parts are none), and fp32
// values next to the largest leave the range of the first of their parts.  The whole wavefront walks along the reduction, a block of
// codes a step: one such row among 32 of 28672x8192 makes a call 0.25 ms instead of 0.04 (a lane for each output alone: 4.2 ms).  With the
// next step's requests under way 0.22, but then kernels that have no use for it spill.
template <int XT, bool F32>
__device__ __forceinline__ float plain_outputs(const W4Params &p, int which, int m, int block) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const char *x_row = p.X + m * p.ldx * x_bytes<XT>();
    struct Step {
        u32x4 words;
        XRaw<XT> x[4];
        float scale[4], x_scale[4];
        int zero[4];
    };
    auto request = [&](int b) {                            // of the last block's columns behind K the last ones
        Step c;
        c.words = *(const u32x4 *)(p.codes[which] + ((int64_t)block * p.blocks + b) * 1024 + lane * 16);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = min(b * BLOCK + 32 * s, p.K - 32) + 8 * g;
            const int64_t at = ((int64_t)block * p.groups + (k >> p.group_shift)) * 16 + l16;
            c.scale[s] = F32 ? ((const float *)p.scales[which])[at] : (float)((const bf16_t *)p.scales[which])[at];
            c.zero[s] = p.has_zeros ? ((const uint8_t *)p.zeros[which])[at] : 8;
            c.x[s].v = *(const decltype(c.x[s].v) *)(x_row + k * x_bytes<XT>());
            if constexpr (XT == X_F32) c.x[s].w = *(const u32x4 *)(x_row + k * 4 + 16);
            if constexpr (XT == X_E4M3 || XT == X_INT8) c.x_scale[s] = p.x_scale[(int64_t)m * p.x_groups + (k >> p.x_group_shift)];
        }
        return c;
    };
    double sum = 0.0;
    for (int b = 0; b < p.blocks; ++b) {
        const Step c = request(b);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (b * BLOCK + 32 * s >= p.K) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                double x;
                if constexpr (XT == X_BF16) x = __builtin_bit_cast(float, j & 1 ? c.x[s].v[j >> 1] & 0xffff0000u : c.x[s].v[j >> 1] << 16);
                else if constexpr (XT == X_F32) x = __builtin_bit_cast(float, j < 4 ? c.x[s].v[j] : c.x[s].w[j - 4]);
                else if constexpr (XT == X_E4M3) x = __builtin_amdgcn_cvt_f32_fp8(c.x[s].v[j >> 2] >> (8 * (j & 3)), 0) * (double)c.x_scale[s];
                else x = (double)(int8_t)(c.x[s].v[j >> 2] >> (8 * (j & 3))) * c.x_scale[s];
                const int code = (int)(c.words[s] >> (4 * ((j >> 1) + 4 * (j & 1))) & 15u);
                sum = fma(x, (double)c.scale[s] * (code - c.zero[s]), sum);
            }
        }
        // where every column has met a NaN, they stay
        uint64_t none = __ballot(sum != sum);
        none |= none >> 32;
        if (((none | none >> 16) & 0xffff) == 0xffff) break;
    }
    sum += __shfl_xor(sum, 16, WAVE);
    return (float)(sum + __shfl_xor(sum, 32, WAVE));
}

// Behind the sums: scales of whole rows, the formula where a sum is no number, bias, activation, residual.  For whole wavefronts whose
// quarters have a row each, of the same 16 columns; is: whether the lane's output exists.
template <int XT, bool F32, bool SWIGLU>
__device__ __forceinline__ void finish(const W4Params &p, float (&v)[2], int row, int n, bool is) {
    typedef typename std::conditional<F32, float, bf16_t>::type T;
#pragma unroll 1                                            // (one copy of what is formed again: registers)
    for (int u = 0; u < (SWIGLU ? 2 : 1); ++u) {
        if ((XT == X_E4M3 || XT == X_INT8) && p.x_groups == 1 && is) v[u] *= p.x_scale[row];
        const bool mend = is && !(fabsf(v[u]) < __builtin_inff());
        const uint64_t rows = __ballot(mend);
        if (__builtin_expect(rows != 0, 0)) {
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                if (!(rows >> (16 * q) & 0xffff)) continue;
                const float formed = plain_outputs<XT, F32>(p, u, __builtin_amdgcn_readlane(row, 16 * q), __builtin_amdgcn_readfirstlane(n) >> 4);
                if (mend && (threadIdx.x >> 4 & 3) == q) v[u] = formed;
            }
        }
    }
    if (!is) return;
    float y = v[0];
    if (p.flags & CASCADE_EPI_BIAS) y += (float)((const T *)p.bias)[n];
    if (SWIGLU) y = silu_f(y) * v[1];
    else y = F32 ? apply_act(y, p.flags) : apply_act_bf16(y, p.flags);
    if (p.flags & CASCADE_EPI_RESIDUAL) y += (float)((const T *)p.residual)[row * p.ldres + n];
    ((T *)p.Y)[row * p.ldy + n] = (T)y;
}

// Up to 16 rows that fit whole leave registers for two workgroups on a CU, but not E4M3 rows over 32 columns: held to 128 registers they
// spill what the ring has requested, and wait for it (8 rows of 8192x28672 51 us; one workgroup, no spills: 41).
constexpr bool two_resident(bool e4m3, int tm, int tn, bool whole) { return tm == 1 && whole && !(e4m3 && tn == 2); }

// TM: 16-row blocks.  TN: 16-column blocks of a wavefront (SWIGLU: gate and up of the same columns).
// FOLD: 32-element steps that share all scales, 1, 2 or 4.
// WHOLE: the slice's X fits into LDS and enters it once; else it comes in chunks of two pieces a wavefront, into halves in turn.
// F32: scales, bias, residual and Y in fp32, else bf16.
template <int XT, bool F32, int TM, int TN, bool SWIGLU, int FOLD, bool WHOLE>
__global__ __launch_bounds__(NW * 64, two_resident(XT == X_E4M3, TM, TN, WHOLE) ? 4 : 2) void w4_kernel(W4Params p) {
    static_assert(!SWIGLU || TN == 2, "gate and up");
    typedef typename std::conditional<F32, float, bf16_t>::type T;
    constexpr bool X8 = XT == X_E4M3 || XT == X_INT8;
    constexpr int TNO = SWIGLU ? 1 : TN, D = 4, UB = unit_bytes<XT>(), MATS = SWIGLU ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cols = 1 << p.cols_log2, parts = NW >> p.cols_log2, cg = wave & (cols - 1), part = wave >> p.cols_log2;
    const int row0 = blockIdx.z * (TM * 16), rows = min(p.M - row0, TM * 16);
    const int tile0 = blockIdx.x * cols * TNO;             // 16-column blocks: of the workgroup,
    // of the wavefront, and how many there are.  Those behind the last column read the first block, or the one beside them, instead, and are
    // not stored: whatever a range check makes of scalar offsets, they stay inside the weights.
    const int left_blocks = p.col_blocks - tile0 - cg * TNO, block0 = __builtin_amdgcn_readfirstlane(left_blocks > 0 ? tile0 + cg * TNO : 0);
    const int n_blocks = __builtin_amdgcn_readfirstlane(left_blocks > 0 ? min(left_blocks, TNO) : 1);
    const int first = blockIdx.y * p.slice_blocks, n_pieces = min(p.blocks - first, p.slice_blocks);

    // LDS: chunks of X, and the scales of its 32-column steps where there are several
    const int row_units = rows | 1;                        // odd: neighbouring units of a row lie in different banks
    const int chunk_bytes = p.chunk * 16 * row_units * UB, chunk_scales = p.chunk * 4 * TM * 16;
    float *xscales = (float *)(lds + p.chunks_held * chunk_bytes);

    __amdgpu_buffer_rsrc_t rw[MATS], rs[MATS], rz[MATS];
#pragma unroll
    for (int i = 0; i < MATS; ++i) {
        const int64_t at = block0, entries = at * p.groups * 16;
        rw[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.codes[i]) + at * p.blocks * 1024, 0, (uint32_t)(n_blocks * p.blocks) * 1024u, 0x00020000);
        rs[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.scales[i]) + entries * sizeof(T), 0, (uint32_t)(n_blocks * p.groups * 16 * sizeof(T)), 0x00020000);
        rz[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.zeros[i]) + entries, 0, (uint32_t)(n_blocks * p.groups * 16), 0x00020000);
    }
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(p.X) + row0 * p.ldx * x_bytes<XT>(), 0, (uint32_t)(((rows - 1) * p.ldx + p.K) * x_bytes<XT>()), 0x00020000);
    const __amdgpu_buffer_rsrc_t rxs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(X8 ? p.x_scale + (int64_t)row0 * p.x_groups : nullptr), 0,
                                                                         X8 ? (uint32_t)(rows * p.x_groups * 4) : 0u, 0x00020000);

    // Unit u of a chunk: columns 8 sg .. of piece (u >> 4) / rows, row (u >> 4) % rows.  f(k, piece, row) for a thread's units, which
    // are 32 rows apart.
    const int sg = tid & 15, units = p.chunk * rows * 16, piece_step = 32 / rows, row_step = 32 % rows;
    auto each_unit = [&](int u, int most, int &piece, int &row, auto f) {
#pragma unroll
        for (int k = 0; k < most; ++k, u += NW * 64) {
            if (u - tid >= units) break;
            f(k, piece, row, u < units);
            piece += piece_step;
            row += row_step;
            if (row >= rows) {
                row -= rows;
                ++piece;
            }
        }
    };
    const int piece0 = (tid >> 4) / rows, row_0 = (tid >> 4) % rows;
    const bool scaled_steps = X8 && p.x_groups > 1;
    struct Unit {
        XRaw<XT> x;
        uint32_t scale;
    };
    auto request_x = [&](int chunk, int piece, int row, bool is) {
        const int q = chunk * p.chunk + piece, col = (first + q) * BLOCK + 8 * sg;
        is = is && q < n_pieces && col < p.K;
        Unit u;
        u.x = load_x<XT>(rx, is ? (uint32_t)(row * p.ldx + col) * x_bytes<XT>() : OUT_OF_RANGE);
        if constexpr (X8) u.scale = __builtin_amdgcn_raw_buffer_load_b32(rxs, is && scaled_steps ? (uint32_t)(row * p.x_groups + (col >> p.x_group_shift)) * 4u : OUT_OF_RANGE, 0, 0);
        return u;
    };
    auto store_unit = [&](int held, int piece, int row, bool is, const Unit &u) {
        if (!is) return;
        store_x<XT>(u.x, lds + held * chunk_bytes + ((piece * 16 + sg) * row_units + row) * UB);
        if (scaled_steps && (sg & 3) == 0) xscales[held * chunk_scales + (piece * 4 + (sg >> 2)) * (TM * 16) + row] = __builtin_bit_cast(float, u.scale);
    };

    struct Piece {
        u32x4 w[TN];
        uint32_t scale[TN], zero[TN];                      // of the fold that this lane's quarter stands for
    } ring[D];
    constexpr int FOLDS = 4 / FOLD;                        // of a piece
    const int my_pieces = (n_pieces - part + parts - 1) / parts;
    // Offsets of the lanes; those of a piece are scalars.  A lane whose fold lies behind the last group of a block that ends early
    // reads out of range there.
    const int group_log2 = p.group_shift, my_group = (g & (FOLDS - 1)) * FOLD * 32 >> group_log2, block_groups = BLOCK >> group_log2;
    const uint32_t scale_off = (uint32_t)(my_group * 16 + l16), tail = (p.blocks - 1) * block_groups + my_group < p.groups ? 0u : OUT_OF_RANGE;
    const uint32_t no_zeros = p.has_zeros ? 0u : OUT_OF_RANGE;
    auto request = [&](Piece &c, int j) {                  // the wavefront's j-th piece
        const int at = min(first + part + parts * j, p.blocks - 1);
        const uint32_t past = j < my_pieces ? 0u : OUT_OF_RANGE, late = past | (at == p.blocks - 1 ? tail : 0u);
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            const int i = SWIGLU ? t : 0, b = SWIGLU ? 0 : min(t, n_blocks - 1), entry = (b * p.groups + at * block_groups) * 16;
            c.w[t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw[i], (uint32_t)lane * 16 | past, (b * p.blocks + at) * 1024, 0));
            if constexpr (F32) c.scale[t] = __builtin_amdgcn_raw_buffer_load_b32(rs[i], scale_off * 4 | late, entry * 4, 0);
            else c.scale[t] = __builtin_amdgcn_raw_buffer_load_b16(rs[i], scale_off * 2 | late, entry * 2, 0);
            c.zero[t] = __builtin_amdgcn_raw_buffer_load_b8(rz[i], scale_off | late | no_zeros, entry, 0);
        }
    };

    f32x4 total[TM][TN];                                   // row 16 i + 4 g + r, column 16 t + l16
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t) total[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};

    int x_row[TM];                                         // rows behind the last one read it again, and are not stored
#pragma unroll
    for (int i = 0; i < TM; ++i) x_row[i] = min(16 * i + l16, rows - 1) * UB;
    auto use = [&](const Piece &c, int held, int piece) {  // piece of the chunk
        const char *x = lds + held * chunk_bytes + (piece * 16 + g) * row_units * UB;
        const float *xsc = xscales + held * chunk_scales + piece * 4 * (TM * 16) + 4 * g;
        // all of the piece's operands are under way before the first is waited for (left to itself, the compiler asks for one at a
        // time), where there is room for them: 64 rows of bf16 with it spill, 30.7 -> 32 us
        constexpr bool AHEAD = XT != X_F32 && (TM <= 2 || (XT == X_INT8 && FOLD > 1));
        // fp32 X: the zero point comes off each code.  That costs three operations more a pair, saves the products with ones and leaves
        // smaller sums to round: errors against 64 bits 1.1e-7 instead of 5.2e-7 at the same time (10 rows of 4096x4096: 11.3 us)
        constexpr bool CENTRED = XT == X_F32;
        XOperand<XT> xo[4][TM];
        auto read_x = [&](int s) {
#pragma unroll
            for (int i = 0; i < TM; ++i) xo[s][i] = operand<XT>(x + 4 * s * row_units * UB + x_row[i]);
        };
        if constexpr (AHEAD) {
#pragma unroll
            for (int s = 0; s < 4; ++s) read_x(s);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int f = 0; f < FOLDS; ++f) {
            Sum<XT> acc[TM][TN], ones[TM];
            float scale[TN];
            uint32_t zero[TN];
            const int from = f * 16 + l16;
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                uint32_t sc = c.scale[t], z = c.zero[t];
                if (FOLDS > 1) {
                    sc = __shfl((int)sc, from, WAVE);
                    z = __shfl((int)z, from, WAVE);
                }
                zero[t] = p.has_zeros ? z : 8;
                scale[t] = __builtin_bit_cast(float, F32 ? sc : sc << 16);
            }
            constexpr int STEPS = XT == X_INT8 && FOLD > 1 ? 2 : 1;
#pragma unroll
            for (int s = f * FOLD; s < (f + 1) * FOLD; s += STEPS) {
                WOperand<XT> w[TN][STEPS], one[STEPS];
#pragma unroll
                for (int k = 0; k < STEPS; ++k) {
                    if constexpr (!AHEAD) read_x(s + k);
                    one[k] = ones_operand<XT>();
#pragma unroll
                    for (int t = 0; t < TN; ++t) {
                        if constexpr (CENTRED) w[t][k] = codes_less(c.w[t][s + k], (float)(zero[t] + 16));
                        else w[t][k] = codes<XT>(c.w[t][s + k]);
                    }
                }
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    if constexpr (!CENTRED) ones[i] = product<XT, STEPS, TM>(&xo[s][i], one, s == f * FOLD ? Sum<XT>{0, 0, 0, 0} : ones[i]);
#pragma unroll
                    for (int t = 0; t < TN; ++t) acc[i][t] = product<XT, STEPS, TM>(&xo[s][i], w[t], s == f * FOLD ? Sum<XT>{0, 0, 0, 0} : acc[i][t]);
                }
            }
            if constexpr (!CENTRED) {
#pragma unroll
                for (int t = 0; t < TN; ++t) {
                    const float minus_zero = -(float)(zero[t] + 16);
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if constexpr (XT == X_INT8) acc[i][t][r] -= __mul24((int)zero[t], ones[i][r]);
                            else acc[i][t][r] = fmaf(minus_zero, ones[i][r], acc[i][t][r]);
                        }
                }
            }
            if (X8 && p.x_groups > 1) {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const f32x4 xs = *(const f32x4 *)(xsc + f * FOLD * (TM * 16) + 16 * i);
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[i][t][r] = fmaf((float)acc[i][t][r], xs[r] * scale[t], total[i][t][r]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[i][t][r] = fmaf((float)acc[i][t][r], scale[t], total[i][t][r]);
            }
        }
    };

    // Loads arrive in the order of their requests: what is needed first is asked for first
    auto fill_ring = [&] {
#pragma unroll
        for (int d = 0; d < D; ++d) request(ring[d], d);
    };
    if constexpr (WHOLE) {
        constexpr int BATCH = XT == X_F32 ? 2 : TM == 1 ? 4 : 8;     // requests of a thread under way
        int piece = piece0, row = row_0;
        auto stage = [&](int u, auto between) {
            Unit x[BATCH];
            int piece_too = piece, row_too = row;
            each_unit(u, BATCH, piece, row, [&](int k, int q, int r, bool is) { x[k] = request_x(0, q, r, is); });
            between();
            each_unit(u, BATCH, piece_too, row_too, [&](int k, int q, int r, bool is) { store_unit(0, q, r, is, x[k]); });
        };
        stage(tid, fill_ring);
        for (int u = tid + BATCH * NW * 64; u - tid < units; u += BATCH * NW * 64) stage(u, [] {});
        __syncthreads();
        for (int j0 = 0; j0 < my_pieces; j0 += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (j0 + d < my_pieces) use(ring[d], 0, (j0 + d) * parts + part);
                request(ring[d], j0 + d + D);
            }
        }
    } else {
        static_assert(D == 4, "two chunks of two pieces");
        const int chunks = (n_pieces + p.chunk - 1) / p.chunk;
        Unit start[MAX_UNITS], ahead[MAX_UNITS];
        auto request_chunk = [&](int chunk, Unit *to) {
            int piece = piece0, row = row_0;
            each_unit(tid, MAX_UNITS, piece, row, [&](int k, int q, int r, bool is) { to[k] = request_x(chunk, q, r, is); });
        };
        auto store_chunk = [&](int held, const Unit *from) {
            int piece = piece0, row = row_0;
            each_unit(tid, MAX_UNITS, piece, row, [&](int k, int q, int r, bool is) { store_unit(held, q, r, is, from[k]); });
        };
        request_chunk(0, start);
        request_chunk(1, ahead);
        fill_ring();
        store_chunk(0, start);
        __syncthreads();
        for (int c0 = 0; c0 < chunks; c0 += 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // the other half has been read before the last barrier; waiting for its X leaves the newest codes under way
                store_chunk(1 - h, ahead);
                request_chunk(c0 + h + 2, ahead);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int j = 2 * (c0 + h) + t;
                    if (j < my_pieces) use(ring[2 * h + t], h, t * parts + part);
                    request(ring[2 * h + t], j + D);
                }
                __syncthreads();
            }
        }
    }

    // Sums stay in the order of the products' results: a lane has four rows of a column.  Those of a cut reduction go out as they
    // are, 1 KB a block, and where no other wavefront of the workgroup has a share in them straight from the registers (turned to
    // rows through LDS first: 7.5 us of a 64-row workgroup instead of 0.5).
    const int row_blocks = (rows + 15) >> 4;
    auto plane = [&](int u, int i, int block) {
        return (f32x4 *)p.planes + ((((int64_t)blockIdx.y * MATS + u) * p.row_blocks + row0 / 16 + i) * p.col_blocks + block) * 64 + lane;
    };
    if (__builtin_expect(p.slices > 1 && parts == 1, 0)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
                if (i < row_blocks && (SWIGLU ? 0 : t) < left_blocks) *plane(SWIGLU ? t : 0, i, block0 + (SWIGLU ? 0 : t)) = total[i][t];
        return;
    }
    f32x4 (*meet)[TM][TN][64] = (f32x4 (*)[TM][TN][64])lds;                      // [wavefront][row block][block][lane]
    if constexpr (WHOLE) __syncthreads();                  // X has been read
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t) meet[wave][i][t][lane] = total[i][t];
    __syncthreads();
    if (__builtin_expect(p.slices > 1, 0)) {               // blocks over wavefronts
        for (int job = wave; job < row_blocks * TNO << p.cols_log2; job += NW) {
            const int c = job & (cols - 1), at = job >> p.cols_log2, t = at & (TNO - 1), i = at / TNO, block = tile0 + c * TNO + t;
            if (block >= p.col_blocks) continue;
#pragma unroll
            for (int u = 0; u < MATS; ++u) {
                f32x4 v = meet[c][i][t + u][lane];
                for (int w = 1; w < parts; ++w) {
                    const f32x4 more = meet[c + (w << p.cols_log2)][i][t + u][lane];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += more[k];
                }
                *plane(u, i, block) = v;
            }
        }
        return;
    }
    // every fourth row of a block over wavefronts, a row's blocks over different ones (they share what a row with an infinity costs)
    const int jobs_log2 = p.cols_log2 + TNO - 1;           // of a row
    for (int job = wave; job < row_blocks * 4 << jobs_log2; job += NW) {
        const int c = job & (cols - 1), t = job >> p.cols_log2 & (TNO - 1), r = job >> jobs_log2 & 3, i = job >> (jobs_log2 + 2);
        const int row = 16 * i + 4 * g + r, n = (tile0 + c * TNO + t) * 16 + l16;
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w >= parts) break;
#pragma unroll
            for (int u = 0; u < MATS; ++u) v[u] += ((const float *)&meet[c + (w << p.cols_log2)][i][t + u][lane])[r];
        }
        finish<XT, F32, SWIGLU>(p, v, row0 + row, n, row < rows && n < p.N);
    }
}

// Adds the slices' sums in their order
template <int XT, bool F32, bool SWIGLU>
__global__ __launch_bounds__(256) void w4_finish_kernel(W4Params p) {
    constexpr int MATS = SWIGLU ? 2 : 1;
    const int64_t plane = (int64_t)p.row_blocks * p.col_blocks * 64;                 // lanes
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < plane; e += (int64_t)gridDim.x * 256) {
        const int lane = (int)(e & 63), n = (int)((e >> 6) % p.col_blocks) * 16 + (lane & 15);
        const int row = (int)((e >> 6) / p.col_blocks) * 16 + (lane >> 4) * 4;
        f32x4 sum[MATS] = {};
#pragma unroll 4
        for (int s = 0; s < p.slices; ++s)
#pragma unroll
            for (int u = 0; u < MATS; ++u) {
                const f32x4 v = ((const f32x4 *)p.planes)[(s * MATS + u) * plane + e];
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[u][k] += v[k];
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[2] = {sum[0][r], sum[MATS - 1][r]};
            finish<XT, F32, SWIGLU>(p, v, row + r, n, n < p.N && row + r < p.M);
        }
    }
}

// How a product is cut.  One choice for the workspace and the launch: the cheapest by a model of what was measured.  Few columns and
// a long reduction want slices (16 rows of 14336x4096: 8 slices 16 us, 2 slices 18, none 20), many columns none (32 int8 rows of
// 8192x28672: none 43, 4 slices 46); a wavefront's columns are 32 where X is shared by more of them that way (1 row of 4096x128256: 61
// against 62 to 67 with 16), 16 where there are few workgroups (1 row of 4096x4096: 6.1 against 7.8).
struct Cut {
    int tm, tn, fold, cols_log2, slices, slice_blocks, chunk, held;
    size_t lds;
};
constexpr size_t LDS_MOST = 160 * 1024;

Cut cut_of(const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    const bool swiglu = d->epilogue & CASCADE_EPI_SWIGLU, x32 = !d->x_format && w->dtype == CASCADE_F32;
    Cut c;
    const int most_tm = x32 ? 2 : 4;
    c.tm = d->rows <= 16 ? 1 : d->rows <= 32 ? 2 : most_tm;
    const int rows = std::min(d->rows, c.tm * 16), unit = x32 ? 48 : d->x_format == CASCADE_Q8_INT8 ? 8 : 16;
    const int blocks = (w->k + BLOCK - 1) / BLOCK, col_blocks = (w->n_out + 15) / 16;
    c.tn = swiglu || c.tm > 1 || col_blocks > 256 ? 2 : 1;
    const int units = (col_blocks + (swiglu ? 1 : c.tn) - 1) / (swiglu ? 1 : c.tn);      // of a wavefront's columns
    const int x_group = d->x_format ? d->x_group : 0;
    // fp32 results take scales step by step: 56 variants less.  It costs 8-bit rows time (folded: 32 int8 rows of 8192x28672
    // 66 -> 43 us, 16 of 4096x4096 9.1 -> 8.3, 8 E4M3 rows of 8192x28672 40 -> 33; groups of 32 the same), not fp32 rows, which do not fold.
    c.fold = w->dtype == CASCADE_F32 ? 1 : std::min(w->group, x_group ? std::min(x_group, BLOCK) : BLOCK) / 32;
    auto lds_of = [&](int chunk, int held) { return (size_t)held * chunk * (16 * (rows | 1) * unit + (d->x_format ? 4 * c.tm * 16 * 4 : 0)); };
    const int row_tiles = (d->rows + c.tm * 16 - 1) / (c.tm * 16);
    double best = 1e30;
    for (int lg = 0; lg <= 3; ++lg) {
        const int parts = NW >> lg, chunk = 2 * parts;
        const int64_t tiles = (units + (1 << lg) - 1) >> lg;
        for (int slices = 1; slices <= 32; ++slices) {
            const int per = ((blocks + slices - 1) / slices + parts - 1) / parts * parts;
            const int64_t groups = tiles * slices * row_tiles;
            if (slices > 1 && (per < 2 * parts || groups > 1024)) break;         // no more slices either: the host's time counts, too
            if (slices > 1 && (int64_t)per * (slices - 1) >= blocks) continue;
            const bool whole = lds_of(std::min(per, blocks), 1) <= LDS_MOST;
            if (!whole && chunk * rows * 16 > MAX_UNITS * NW * 64) continue;
            const size_t lds = std::max(whole ? lds_of(std::min(per, blocks), 1) : lds_of(chunk, 2), (size_t)NW * c.tm * c.tn * 1024);
            if (lds > LDS_MOST) continue;
            const int resident = two_resident(d->x_format == CASCADE_Q8_E4M3, c.tm, c.tn, whole) && lds <= LDS_MOST / 2 ? 2 : 1;
            // microseconds: rounds of workgroups, each a start and its pieces at the rate that the resident ones share
            const int64_t full = groups / (256 * resident), rest = groups - full * 256 * resident;
            // eight wavefronts' pieces at 20 KB a microsecond and CU, or at their products' pace; X at twice that rate
            const double turn = std::max(8 * 1.024 * c.tn / 20.0, 0.17 * c.tm * c.tn);
            const double turns = (double)((per + parts - 1) / parts), x = per * 16.0 * rows * unit / 40e3;
            const double bytes = (full * resident + (rest + 255) / 256) * (turns * turn + x), start = 2.5 * (full + (rest ? 1 : 0));
            const double planes = slices > 1 ? 3.0 + 2.0 * slices * d->rows * (double)w->n_out * 4 * (swiglu ? 2 : 1) / 6e6 : 0.0;
            const double cost = bytes + start + planes;
            if (cost < best) {
                best = cost;
                c.cols_log2 = lg; c.slices = slices; c.slice_blocks = per; c.chunk = whole ? std::min(per, blocks) : chunk;
                c.held = whole ? 1 : 2; c.lds = lds;
            }
        }
    }
    return c;
}

size_t planes_bytes(const Cut &c, const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    if (c.slices == 1) return 0;
    return (size_t)c.slices * ((d->rows + 15) / 16) * ((w->n_out + 15) / 16) * 1024 * (d->epilogue & CASCADE_EPI_SWIGLU ? 2 : 1);
}

template <int XT, bool F32, int TM, int TN, bool SWIGLU, int FOLD, bool WHOLE>
int32_t launch(const W4Params &p, const Cut &c, hipStream_t s) {
    static std::atomic<uint64_t> done{0};
    const void *kernel = (const void *)w4_kernel<XT, F32, TM, TN, SWIGLU, FOLD, WHOLE>;
    CASCADE_HIP_TRY(ensure_dynamic_lds(kernel, (int)LDS_MOST, done));
    const int cols = (SWIGLU ? 1 : TN) << c.cols_log2;
    const dim3 grid((unsigned)((p.col_blocks + cols - 1) / cols), (unsigned)p.slices, (unsigned)((p.M + TM * 16 - 1) / (TM * 16)));
    hipLaunchKernelGGL((w4_kernel<XT, F32, TM, TN, SWIGLU, FOLD, WHOLE>), grid, dim3(NW * 64), c.lds, s, p);
    if (p.slices > 1)
        hipLaunchKernelGGL((w4_finish_kernel<XT, F32, SWIGLU>), dim3((unsigned)std::min<int64_t>(((int64_t)p.row_blocks * p.col_blocks + 3) / 4, 1 << 16)), dim3(256), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}
template <int XT, bool F32, int TM, int TN, bool SWIGLU>
int32_t launch_held(const W4Params &p, const Cut &c, hipStream_t s) {
    if constexpr (!F32) {
        if (c.fold == 4) return c.held == 1 ? launch<XT, F32, TM, TN, SWIGLU, 4, true>(p, c, s) : launch<XT, F32, TM, TN, SWIGLU, 4, false>(p, c, s);
        if (c.fold == 2) return c.held == 1 ? launch<XT, F32, TM, TN, SWIGLU, 2, true>(p, c, s) : launch<XT, F32, TM, TN, SWIGLU, 2, false>(p, c, s);
    }
    return c.held == 1 ? launch<XT, F32, TM, TN, SWIGLU, 1, true>(p, c, s) : launch<XT, F32, TM, TN, SWIGLU, 1, false>(p, c, s);
}
template <int XT, bool F32, int TM>
int32_t launch_rows(const W4Params &p, const Cut &c, hipStream_t s) {
    if (p.flags & CASCADE_EPI_SWIGLU) return launch_held<XT, F32, TM, 2, true>(p, c, s);
    if constexpr (TM == 1)
        if (c.tn == 1) return launch_held<XT, F32, 1, 1, false>(p, c, s);
    return launch_held<XT, F32, TM, 2, false>(p, c, s);
}
template <int XT, bool F32>
int32_t launch_x(const W4Params &p, const Cut &c, hipStream_t s) {
    if (c.tm == 1) return launch_rows<XT, F32, 1>(p, c, s);
    if constexpr (XT != X_F32)
        if (c.tm == 4) return launch_rows<XT, F32, 4>(p, c, s);
    return launch_rows<XT, F32, 2>(p, c, s);
}

// ---------------------------------------------------------------------------- layout
struct PackParams {
    const uint8_t *codes, *zeros;
    const void *scales;
    char *out, *out_scales, *out_zeros;
    int32_t N, K, blocks, groups;
};

// One wavefront per block of codes, each lane its 16 bytes; columns and elements past the end get code 0 (with scale 0)
__global__ __launch_bounds__(256) void w4_pack_kernel(PackParams p) {
    const int64_t n_blocks = (int64_t)((p.N + 15) / 16) * p.blocks;
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    for (int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); b < n_blocks; b += (int64_t)gridDim.x * 4) {
        const int n = (int)(b / p.blocks) * 16 + l16, k0 = (int)(b % p.blocks) * BLOCK + 8 * g;
        u32x4 v = {0, 0, 0, 0};
        if (n < p.N)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (k0 + 32 * s < p.K) {
                    const uint8_t *c = p.codes + (int64_t)n * p.K + k0 + 32 * s;
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[s] |= (uint32_t)(c[j] & 15u) << (4 * ((j >> 1) + 4 * (j & 1)));
                }
        *(u32x4 *)(p.out + b * 1024 + lane * 16) = v;
    }
}
template <typename T>
__global__ __launch_bounds__(256) void w4_pack_scales_kernel(PackParams p) {
    const int64_t n = (int64_t)((p.N + 15) / 16) * p.groups * 16;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int col = (int)(e / 16 / p.groups) * 16 + (int)(e & 15), grp = (int)(e / 16 % p.groups);
        const int64_t from = (int64_t)col * p.groups + grp;
        ((T *)p.out_scales)[e] = col < p.N ? ((const T *)p.scales)[from] : (T)0.f;
        if (p.zeros) ((uint8_t *)p.out_zeros)[e] = col < p.N ? p.zeros[from] & 15 : 0;
    }
}

struct Layout { size_t scales, zeros, bytes; };            // offsets behind the codes
Layout layout(const cascade_w4_weights *w) {
    const size_t col_blocks = ((size_t)w->n_out + 15) / 16, entries = col_blocks * (w->k / w->group) * 16;
    Layout l;
    l.scales = col_blocks * (((size_t)w->k + BLOCK - 1) / BLOCK) * 1024;
    l.zeros = l.scales + align_up(entries * (w->dtype == CASCADE_BF16 ? 2 : 4), 256);
    l.bytes = l.zeros + (w->zero_points ? align_up(entries, 256) : 0);
    return l;
}

int32_t check_weights(const cascade_w4_weights *w) {
    if (!w || w->n_out <= 0 || w->k <= 0 || w->group <= 0 || w->reserved || w->zero_points < 0 || w->zero_points > 1) return CASCADE_EINVAL;
    if (w->dtype != CASCADE_F32 && w->dtype != CASCADE_BF16) return CASCADE_EUNSUPPORTED;
    if (w->group != 32 && w->group != 64 && w->group != 128) return CASCADE_EUNSUPPORTED;
    if (w->k % w->group) return CASCADE_ESHAPE;
    if (w->k > 1 << 20 || w->n_out > 1 << 26) return CASCADE_EUNSUPPORTED;
    return CASCADE_OK;
}

int32_t check_gemm(const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    const int32_t st = check_weights(w);
    if (st != CASCADE_OK) return st;
    if (!d || d->rows < 0 || d->x_group < 0 || d->x_format < 0 || d->x_format > CASCADE_Q8_E4M3) return CASCADE_EINVAL;
    if (d->x_stride < 0 || d->residual_stride < 0 || d->y_stride < 0) return CASCADE_EINVAL;
    if (d->rows > 1 << 20) return CASCADE_EUNSUPPORTED;
    const int acts = CASCADE_EPI_GELU_ERF | CASCADE_EPI_GELU_TANH | CASCADE_EPI_SWIGLU;
    if (d->epilogue & ~(acts | CASCADE_EPI_BIAS | CASCADE_EPI_RESIDUAL)) return CASCADE_EUNSUPPORTED;
    if (__builtin_popcount(d->epilogue & acts) > 1) return CASCADE_EUNSUPPORTED;
    if ((d->epilogue & CASCADE_EPI_SWIGLU) && (d->epilogue & CASCADE_EPI_BIAS)) return CASCADE_EUNSUPPORTED;
    if (d->x_format && d->x_group) {
        if (d->x_group != 32 && d->x_group != 64 && d->x_group != 128 && d->x_group != 256) return CASCADE_EUNSUPPORTED;
        if (w->k % d->x_group) return CASCADE_ESHAPE;
    }
    return CASCADE_OK;
}

}  // namespace

extern "C" size_t cascade_w4_bytes(const cascade_w4_weights *w) { return check_weights(w) == CASCADE_OK ? layout(w).bytes : 0; }

extern "C" int32_t cascade_w4_pack(const cascade_w4_weights *w, const void *codes, const void *scales, const void *zeros, void *stream) {
    const int32_t st = check_weights(w);
    if (st != CASCADE_OK) return st;
    if (!w->packed || !codes || !scales || !zeros != !w->zero_points) return CASCADE_EINVAL;
    if ((uintptr_t)w->packed % 256) return CASCADE_EUNSUPPORTED;
    const Layout l = layout(w);
    PackParams p;
    p.codes = (const uint8_t *)codes; p.zeros = (const uint8_t *)zeros; p.scales = scales;
    p.out = (char *)w->packed; p.out_scales = p.out + l.scales; p.out_zeros = p.out + l.zeros;
    p.N = w->n_out; p.K = w->k; p.blocks = (w->k + BLOCK - 1) / BLOCK; p.groups = w->k / w->group;
    const int64_t blocks = (int64_t)((p.N + 15) / 16) * p.blocks, entries = (int64_t)((p.N + 15) / 16) * p.groups * 16;
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)std::min<int64_t>((blocks + 3) / 4, 1 << 16)), dim3(256), 0, s, p);
    const dim3 grid((unsigned)std::min<int64_t>((entries + 255) / 256, 1 << 16));
    if (w->dtype == CASCADE_BF16) hipLaunchKernelGGL(w4_pack_scales_kernel<bf16_t>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(w4_pack_scales_kernel<float>, grid, dim3(256), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

// Enough for fewer rows too: more of them are cut into fewer slices, so the largest of all counts up to this one.  Up to 64 rows each
// count has a cut of its own.  Behind them the slices only become fewer as the sums' share of the cost grows, from one 16 rows to
// the next as many blocks of sums: the first of each 16 has the most.  Reductions are cut up to 1024 workgroups, no more.
extern "C" size_t cascade_w4_gemm_workspace_bytes(const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    if (check_gemm(w, d) != CASCADE_OK) return 0;
    const int columns = 16 * 8 * (d->epilogue & CASCADE_EPI_SWIGLU ? 1 : 2), tiles = (int)(((int64_t)w->n_out + columns - 1) / columns);      // at least
    const int last = std::min(d->rows, 512 / std::min(tiles, 513) * 64);
    cascade_w4_gemm_desc fewer = *d;
    size_t most = 0;
    for (fewer.rows = 1; fewer.rows <= last; fewer.rows += fewer.rows < 65 ? 1 : 16) most = std::max(most, planes_bytes(cut_of(w, &fewer), w, &fewer));
    return most;
}

extern "C" int32_t cascade_w4_gemm(const cascade_w4_weights *w, const cascade_w4_weights *up, const cascade_w4_gemm_desc *d, const void *X,
                                   const float *x_scale, const void *bias, const void *residual, void *Y, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    const int32_t st = check_gemm(w, d);
    if (st != CASCADE_OK) return st;
    const bool swiglu = d->epilogue & CASCADE_EPI_SWIGLU;
    if (!w->packed || !up != !swiglu) return CASCADE_EINVAL;
    if (d->rows > 0 && (!X || !Y || X == Y || !x_scale != (d->x_format == CASCADE_Q8_NONE))) return CASCADE_EINVAL;
    if (d->rows > 0 && (!bias != !(d->epilogue & CASCADE_EPI_BIAS) || !residual != !(d->epilogue & CASCADE_EPI_RESIDUAL))) return CASCADE_EINVAL;
    if (swiglu) {
        if (!up->packed || up->reserved) return CASCADE_EINVAL;
        if (up->dtype != w->dtype || up->n_out != w->n_out || up->k != w->k || up->group != w->group || up->zero_points != w->zero_points)
            return CASCADE_ESHAPE;
    }
    W4Params p = {};
    p.M = d->rows; p.N = w->n_out; p.K = w->k;
    p.ldx = d->x_stride ? d->x_stride : p.K;
    p.ldres = d->residual_stride ? d->residual_stride : p.N;
    p.ldy = d->y_stride ? d->y_stride : p.N;
    if (p.ldx < p.K || p.ldres < p.N || p.ldy < p.N || (residual && residual == Y && p.ldres != p.ldy)) return CASCADE_ESHAPE;
    const bool f32 = w->dtype == CASCADE_F32;
    const int x_size = d->x_format ? 1 : f32 ? 4 : 2;
    if ((uintptr_t)X % 16 || p.ldx * x_size % 16 || (uintptr_t)w->packed % 256 || (swiglu && (uintptr_t)up->packed % 256)) return CASCADE_EUNSUPPORTED;
    if (p.ldx > (int64_t)1 << 22) return CASCADE_EUNSUPPORTED;               // 64 rows count their bytes in 31 bits
    if (p.M == 0) return CASCADE_OK;
    const Layout l = layout(w);
    for (int i = 0; i < (swiglu ? 2 : 1); ++i) {
        p.codes[i] = (const char *)(i ? up : w)->packed;
        p.scales[i] = p.codes[i] + l.scales;
        p.zeros[i] = p.codes[i] + (w->zero_points ? l.zeros : l.scales);       // (not used without zero points)
    }
    p.X = (const char *)X; p.x_scale = x_scale; p.bias = bias; p.residual = residual; p.Y = Y;
    p.blocks = (p.K + BLOCK - 1) / BLOCK; p.groups = p.K / w->group;
    p.row_blocks = (p.M + 15) / 16; p.col_blocks = (p.N + 15) / 16;
    const int x_group = d->x_format ? d->x_group : 0;
    p.group_shift = __builtin_ctz((unsigned)w->group);
    p.x_group_shift = x_group ? __builtin_ctz((unsigned)x_group) : 31;
    p.x_groups = x_group ? p.K / x_group : 1;
    p.has_zeros = w->zero_points; p.flags = d->epilogue;
    const Cut c = cut_of(w, d);
    if (c.slices > 1 && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < planes_bytes(c, w, d))) return CASCADE_EWORKSPACE;
    p.planes = (float *)workspace;
    p.cols_log2 = c.cols_log2; p.slices = c.slices; p.slice_blocks = c.slice_blocks; p.chunk = c.chunk; p.chunks_held = c.held;
    hipStream_t s = (hipStream_t)stream;
    if (d->x_format == CASCADE_Q8_E4M3) return f32 ? launch_x<X_E4M3, true>(p, c, s) : launch_x<X_E4M3, false>(p, c, s);
    if (d->x_format == CASCADE_Q8_INT8) return f32 ? launch_x<X_INT8, true>(p, c, s) : launch_x<X_INT8, false>(p, c, s);
    return f32 ? launch_x<X_F32, true>(p, c, s) : launch_x<X_BF16, false>(p, c, s);
}
