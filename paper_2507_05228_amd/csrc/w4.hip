// Products of few rows with 4-bit weights (cascade_w4_gemm), and the layout of the weights (cascade_w4_pack).
//
// What bounds it: every weight is used for a handful of rows, so a launch is as long as streaming the codes from HBM, half a byte
// each.  A workgroup owns 16 or 32 output columns, its 8 wavefronts split the reduction and read the codes straight into matrix
// operands, a ring of pieces ahead of their use; the partial sums meet in LDS in a fixed order.
//
// Packed layout.  Codes: blocks of 16 columns by 128 reduction elements, 1 KB each, blocks of a column side by side along the
// reduction.  In a block, lane (column l, quarter g) of a wavefront finds its 16 bytes at (16 g + l) * 16: word s holds elements
// 32 s + 8 g .. + 7, which is the operand of one 16x16x32 product, and in a word nibble p < 4 holds element 2p, nibble p + 4
// element 2p + 1.  So two nibbles 16 bits apart become a pair of bf16 numbers by a shift, a mask and an or: 0x4180 | code << 3 is
// 16 + code.  A second product with -(16 + zero) in every element takes that back, exactly but for the fp32 sums.  INT8 rows
// take codes as bytes (three operations for 8) and -zero, all in whole numbers.  Behind the codes: scales and zeros, [column
// blocks][groups][16].
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
    int64_t ldx, ldres, ldy;                               // elements
    int32_t M, N, K;
    int32_t blocks, groups;                                // of the reduction
    int32_t fold;                                          // 32-element steps that share all scales: 1, 2 or 4
    int32_t group_shift, x_group_shift, x_groups;          // log2 of the elements of a scale (x_group_shift 31: the row)
    int32_t has_zeros, flags;
};

// fp32 columns of a row as three bf16 numbers each, which add up to it exactly (8 bits of 24 each)
__device__ __forceinline__ void limbs(const f32x4 &a, const f32x4 &b, bf16x8 (&out)[3]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float v = e < 4 ? a[e] : b[e - 4];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            out[i][e] = (bf16_t)v;
            v -= (float)out[i][e];
        }
    }
}

template <int XT> struct XPiece;                           // what a lane holds of a row's 128 columns, as it came
template <> struct XPiece<X_BF16> { u32x4 v[4]; };
template <> struct XPiece<X_F32> { u32x4 v[8]; };
template <> struct XPiece<X_E4M3> { u32x2 v[4]; };
template <> struct XPiece<X_INT8> { u32x2 v[4]; };
template <int XT> constexpr int x_bytes() { return XT == X_BF16 ? 2 : XT == X_F32 ? 4 : 1; }

template <int XT>
__device__ __forceinline__ void request_x(XPiece<XT> &x, __amdgpu_buffer_rsrc_t r, uint32_t off, int left) {
    // columns 32 s + 8 g .. + 7 of the piece; `left`: columns from the lane's first one to the row's end
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t o = 32 * s < left ? off + 32 * s * x_bytes<XT>() : OUT_OF_RANGE;
        if constexpr (XT == X_BF16) x.v[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
        else if constexpr (XT == X_F32) {
            x.v[2 * s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
            x.v[2 * s + 1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o, 16, 0));
        } else x.v[s] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0));
    }
}

// The operand of step s: bf16 numbers (three sets of them for fp32), or bytes in the order of the codes' bytes
template <int XT> struct XOperand { bf16x8 v[XT == X_F32 ? 3 : 1]; };
template <> struct XOperand<X_INT8> { int64_t v; };
template <int XT>
__device__ __forceinline__ XOperand<XT> x_operand(const XPiece<XT> &x, int s) {
    XOperand<XT> o;
    if constexpr (XT == X_BF16) o.v[0] = __builtin_bit_cast(bf16x8, x.v[s]);
    else if constexpr (XT == X_F32) limbs(__builtin_bit_cast(f32x4, x.v[2 * s]), __builtin_bit_cast(f32x4, x.v[2 * s + 1]), o.v);
    else if constexpr (XT == X_E4M3) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(x.v[s][h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x.v[s][h], true);
            o.v[0][4 * h] = (bf16_t)a[0];
            o.v[0][4 * h + 1] = (bf16_t)a[1];
            o.v[0][4 * h + 2] = (bf16_t)b[0];
            o.v[0][4 * h + 3] = (bf16_t)b[1];
        }
    } else {
        const u32x2 b = {__builtin_amdgcn_perm(x.v[s][1], x.v[s][0], 0x05010400u), __builtin_amdgcn_perm(x.v[s][1], x.v[s][0], 0x07030602u)};
        o.v = __builtin_bit_cast(int64_t, b);
    }
    return o;
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
template <int XT>
__device__ __forceinline__ void step(Sum<XT> &acc, const XOperand<XT> &x, uint32_t w, uint32_t minus_zero) {
    if constexpr (XT == X_INT8) {
        const u32x2 z = {minus_zero, minus_zero};
        acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, codes_int8(w), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, __builtin_bit_cast(int64_t, z), acc, 0, 0, 0);
    } else {
        const u32x4 z = {minus_zero, minus_zero, minus_zero, minus_zero};
        const bf16x8 c = codes_bf16(w);
#pragma unroll
        for (int i = 0; i < (XT == X_F32 ? 3 : 1); ++i) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[i], c, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v[i], __builtin_bit_cast(bf16x8, z), acc, 0, 0, 0);
        }
    }
}

// One output from the formula, term by term.  The products above give NaN where a row holds an infinity (16 + code and
// 16 + zero meet it with opposite signs), and fp32 values next to the largest leave the range of the first of their parts.
template <int XT, bool F32>
__device__ __forceinline__ float plain_output(const W4Params &p, int which, int m, int n) {
    float sum = 0.f;
    for (int grp = 0; grp < p.groups; ++grp) {
        const int64_t at = ((int64_t)(n >> 4) * p.groups + grp) * 16 + (n & 15);
        const float scale = F32 ? ((const float *)p.scales[which])[at] : (float)((const bf16_t *)p.scales[which])[at];
        const float zero = p.has_zeros ? (float)(((const uint8_t *)p.zeros[which])[at]) : 8.f;
        for (int k = grp << p.group_shift; k < (grp + 1) << p.group_shift; ++k) {
            const int j = k & 7;
            const uint32_t *word = (const uint32_t *)(p.codes[which] + ((int64_t)(n >> 4) * p.blocks + k / BLOCK) * 1024 +
                                                      ((k >> 3 & 3) * 16 + (n & 15)) * 16) + (k >> 5 & 3);
            const float code = (float)((*word >> (4 * ((j >> 1) + 4 * (j & 1)))) & 15u);
            const int64_t e = m * p.ldx + k;
            float x;
            if constexpr (XT == X_BF16) x = (float)((const bf16_t *)p.X)[e];
            else if constexpr (XT == X_F32) x = ((const float *)p.X)[e];
            else if constexpr (XT == X_E4M3) x = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)p.X)[e], 0);
            else x = (float)((const int8_t *)p.X)[e];
            if constexpr (XT == X_E4M3 || XT == X_INT8) x *= p.x_scale[(int64_t)m * p.x_groups + (k >> p.x_group_shift)];
            sum = fmaf(x, scale * (code - zero), sum);
        }
        if (sum != sum) break;                             // stays NaN
    }
    return sum;
}

// TM: 16-row blocks.  TN: 16-column blocks (SWIGLU: gate and up of the same columns).  D: pieces in flight per wavefront.
// F32: scales, bias, residual and Y in fp32, else bf16.
template <int XT, bool F32, int TM, int TN, int D, bool SWIGLU>
__global__ __launch_bounds__(NW * 64) void w4_kernel(W4Params p) {
    static_assert(!SWIGLU || TN == 2, "gate and up");
    typedef typename std::conditional<F32, float, bf16_t>::type T;
    constexpr bool X8 = XT == X_E4M3 || XT == X_INT8;
    constexpr int TNO = SWIGLU ? 1 : TN, OUT = TNO * 256, PER = (OUT + NW * 64 - 1) / (NW * 64);
    __shared__ __attribute__((aligned(16))) float part[NW][TN][256];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row0 = blockIdx.y * (TM * 16), rows = min(p.M - row0, TM * 16);
    const int block0 = blockIdx.x * TNO, n_blocks = min((p.N + 15) / 16 - block0, TNO);

    __amdgpu_buffer_rsrc_t rw[SWIGLU ? 2 : 1], rs[SWIGLU ? 2 : 1], rz[SWIGLU ? 2 : 1];
#pragma unroll
    for (int i = 0; i < (SWIGLU ? 2 : 1); ++i) {
        const int64_t scales = (int64_t)block0 * p.groups * 16;
        rw[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.codes[i]) + (int64_t)block0 * p.blocks * 1024, 0,
                                                  (uint32_t)(n_blocks * p.blocks) * 1024u, 0x00020000);
        rs[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.scales[i]) + scales * sizeof(T), 0,
                                                  (uint32_t)(n_blocks * p.groups * 16 * sizeof(T)), 0x00020000);
        rz[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.zeros[i]) + scales, 0, p.has_zeros ? (uint32_t)(n_blocks * p.groups * 16) : 0u,
                                                  0x00020000);
    }
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(p.X) + row0 * p.ldx * x_bytes<XT>(), 0, (uint32_t)(((rows - 1) * p.ldx + p.K) * x_bytes<XT>()), 0x00020000);
    const __amdgpu_buffer_rsrc_t rxs = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(X8 ? p.x_scale + (int64_t)row0 * p.x_groups : nullptr), 0,
                                                                         X8 ? (uint32_t)(rows * p.x_groups * 4) : 0u, 0x00020000);
    uint32_t x_off[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) x_off[i] = 16 * i + l16 < rows ? (uint32_t)((16 * i + l16) * p.ldx + 8 * g) * x_bytes<XT>() : OUT_OF_RANGE;

    struct Piece {
        u32x4 w[TN];
        uint32_t scale[TN], zero[TN];                      // of the fold that this lane's quarter stands for
        XPiece<XT> x[TM];
        f32x4 xs[X8 ? TM : 1];
    } ring[D];
    const int folds_shift = 2 - __builtin_ctz(p.fold), folds = 1 << folds_shift;      // folds of a piece
    // Workgroups start 256 bytes of X apart and wrap around, as those of the bf16 kernel for few rows do (L2 channels)
    const int rot = (int)((blockIdx.x >> 3) % (uint32_t)p.blocks);
    auto request = [&](Piece &c, int piece) {
        const int at = piece + rot - (piece + rot >= p.blocks ? p.blocks : 0);
        const bool past = piece >= p.blocks;
        const int first = (at << 2) + (g & (folds - 1)) * p.fold;                // 32-element step at which the lane's fold begins
        const int group = (first << 5) >> p.group_shift;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int i = SWIGLU ? j : 0, b = SWIGLU ? 0 : j;
            const uint32_t o = past ? OUT_OF_RANGE : (uint32_t)(b * p.blocks + at) * 1024u + lane * 16;
            c.w[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw[i], o, 0, 0));
            const uint32_t so = past || group >= p.groups ? OUT_OF_RANGE : (uint32_t)((b * p.groups + group) * 16 + l16);
            if constexpr (F32) c.scale[j] = __builtin_amdgcn_raw_buffer_load_b32(rs[i], so * 4 | (so & OUT_OF_RANGE), 0, 0);
            else c.scale[j] = __builtin_amdgcn_raw_buffer_load_b16(rs[i], so * 2 | (so & OUT_OF_RANGE), 0, 0);
            c.zero[j] = __builtin_amdgcn_raw_buffer_load_b8(rz[i], so, 0, 0);
        }
        const int left = past ? 0 : p.K - at * BLOCK - 8 * g;
#pragma unroll
        for (int i = 0; i < TM; ++i) request_x<XT>(c.x[i], rx, x_off[i] + (past ? 0u : (uint32_t)at * BLOCK * x_bytes<XT>()), x_off[i] & OUT_OF_RANGE ? 0 : left);
    };

    f32x4 total[TM][TN];                                   // row 16 i + 4 g + r, column 16 j + l16
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto use = [&](const Piece &c, int piece) {
        const int at = piece + rot - (piece + rot >= p.blocks ? p.blocks : 0);
        Sum<XT> acc[TM][TN];
        uint32_t minus_zero[TN];
        float scale[TN];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if ((s & (p.fold - 1)) == 0) {                 // a fold begins
                const int from = folds == 1 ? lane : (s >> __builtin_ctz(p.fold)) * 16 + l16;
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    uint32_t sc = c.scale[j], z = c.zero[j];
                    if (folds > 1) {
                        sc = __shfl((int)sc, from, WAVE);
                        z = __shfl((int)z, from, WAVE);
                    }
                    scale[j] = F32 ? __builtin_bit_cast(float, sc) : __builtin_bit_cast(float, sc << 16);
                    if (!p.has_zeros) z = 8;
                    minus_zero[j] = XT == X_INT8 ? ((0u - z) & 255u) * 0x01010101u : (0xc180u | z << 3) * 0x00010001u;
                }
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = Sum<XT>{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const XOperand<XT> x = x_operand<XT>(c.x[i], s);
#pragma unroll
                for (int j = 0; j < TN; ++j) step<XT>(acc[i][j], x, c.w[j][s], minus_zero[j]);
            }
            if (((s + 1) & (p.fold - 1)) == 0) {           // and ends
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    f32x4 xs = {1.f, 1.f, 1.f, 1.f};
                    if (X8 && p.x_groups > 1) {
                        const int k = at * BLOCK + (s + 1 - p.fold) * 32;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int m = 16 * i + 4 * g + r;
                            const uint32_t o = m < rows && k < p.K ? (uint32_t)(m * p.x_groups + (k >> p.x_group_shift)) * 4u : OUT_OF_RANGE;
                            xs[r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rxs, o, 0, 0));
                        }
                    }
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[i][j][r] = fmaf((float)acc[i][j][r], X8 ? xs[r] * scale[j] : scale[j], total[i][j][r]);
                }
            }
        }
    };

#pragma unroll
    for (int d = 0; d < D; ++d) request(ring[d], wave + NW * d);
    for (int piece = wave; piece < p.blocks; piece += NW * D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (piece + NW * d < p.blocks) use(ring[d], piece + NW * d);
            request(ring[d], piece + NW * (D + d));
        }
    }

    const bool has_res = p.flags & CASCADE_EPI_RESIDUAL, has_bias = p.flags & CASCADE_EPI_BIAS;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (16 * i >= rows) break;
        if (i) __syncthreads();                            // the sums of the block before have been read
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][j][r * 64 + lane] = total[i][j][r];
        __syncthreads();
#pragma unroll
        for (int o = 0; o < PER; ++o) {
            const int at = tid + o * NW * 64, j = at >> 8, m = (at >> 4) & 15, c = at & 15, n = (block0 + j) * 16 + c;
            if (at >= OUT || 16 * i + m >= rows || n >= p.N) continue;
            const int64_t row = row0 + 16 * i + m;
            const int slot = (m & 3) * 64 + (m >> 2) * 16 + c;
            float v[2] = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                v[0] += part[w][j][slot];
                if (SWIGLU) v[1] += part[w][TN - 1][slot];
            }
#pragma unroll
            for (int u = 0; u < (SWIGLU ? 2 : 1); ++u) {
                if (X8 && p.x_groups == 1) v[u] *= p.x_scale[row];
                if (!(fabsf(v[u]) < __builtin_inff())) v[u] = plain_output<XT, F32>(p, u, (int)row, n);
            }
            float y = v[0];
            if (has_bias) y += (float)((const T *)p.bias)[n];
            if (SWIGLU) y = silu_f(y) * v[1];
            else y = F32 ? apply_act(y, p.flags) : apply_act_bf16(y, p.flags);
            if (has_res) y += (float)((const T *)p.residual)[row * p.ldres + n];
            ((T *)p.Y)[row * p.ldy + n] = (T)y;
        }
    }
}

template <int XT, bool F32, int TM, int TN, bool SWIGLU>
void launch(const W4Params &p, hipStream_t s) {
    constexpr int D = TM == 1 ? 4 : 2;
    const unsigned cols = ((p.N + 15) / 16 + (SWIGLU ? 1 : TN) - 1) / (SWIGLU ? 1 : TN), rows = (p.M + TM * 16 - 1) / (TM * 16);
    hipLaunchKernelGGL((w4_kernel<XT, F32, TM, TN, D, SWIGLU>), dim3(cols, rows), dim3(NW * 64), 0, s, p);
}
template <int XT, bool F32, int TM>
void launch_rows(const W4Params &p, hipStream_t s) {
    if (p.flags & CASCADE_EPI_SWIGLU) launch<XT, F32, TM, 2, true>(p, s);
    else if ((p.N + 15) / 16 >= 2 * 256) launch<XT, F32, TM, 2, false>(p, s);
    else launch<XT, F32, TM, 1, false>(p, s);
}
template <int XT, bool F32>
int32_t launch_x(const W4Params &p, hipStream_t s) {
    if (p.M <= 16) launch_rows<XT, F32, 1>(p, s);
    else if (p.M <= 32) launch_rows<XT, F32, 2>(p, s);
    else launch_rows<XT, F32, 4>(p, s);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
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
    if (w->k > 1 << 20 || w->n_out > INT32_MAX - 64) return CASCADE_EUNSUPPORTED;
    return CASCADE_OK;
}

int32_t check_gemm(const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    const int32_t st = check_weights(w);
    if (st != CASCADE_OK) return st;
    if (!d || d->rows < 0 || d->x_group < 0 || d->x_format < 0 || d->x_format > CASCADE_Q8_E4M3) return CASCADE_EINVAL;
    if (d->x_stride < 0 || d->residual_stride < 0 || d->y_stride < 0) return CASCADE_EINVAL;
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

extern "C" size_t cascade_w4_gemm_workspace_bytes(const cascade_w4_weights *w, const cascade_w4_gemm_desc *d) {
    if (check_gemm(w, d) != CASCADE_OK) return 0;
    return 0;
}

extern "C" int32_t cascade_w4_gemm(const cascade_w4_weights *w, const cascade_w4_weights *up, const cascade_w4_gemm_desc *d, const void *X,
                                   const float *x_scale, const void *bias, const void *residual, void *Y, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    (void)workspace; (void)workspace_bytes;
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
        p.zeros[i] = p.codes[i] + l.zeros;
    }
    p.X = (const char *)X; p.x_scale = x_scale; p.bias = bias; p.residual = residual; p.Y = Y;
    p.blocks = (p.K + BLOCK - 1) / BLOCK; p.groups = p.K / w->group;
    const int x_group = d->x_format ? d->x_group : 0;
    p.fold = std::min(w->group, x_group ? std::min(x_group, BLOCK) : BLOCK) / 32;
    p.group_shift = __builtin_ctz((unsigned)w->group);
    p.x_group_shift = x_group ? __builtin_ctz((unsigned)x_group) : 31;
    p.x_groups = x_group ? p.K / x_group : 1;
    p.has_zeros = w->zero_points; p.flags = d->epilogue;
    hipStream_t s = (hipStream_t)stream;
    if (d->x_format == CASCADE_Q8_E4M3) return f32 ? launch_x<X_E4M3, true>(p, s) : launch_x<X_E4M3, false>(p, s);
    if (d->x_format == CASCADE_Q8_INT8) return f32 ? launch_x<X_INT8, true>(p, s) : launch_x<X_INT8, false>(p, s);
    return f32 ? launch_x<X_F32, true>(p, s) : launch_x<X_BF16, false>(p, s);
}
