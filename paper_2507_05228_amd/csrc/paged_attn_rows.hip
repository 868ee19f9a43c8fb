// Attention over a paged cache, every type, head dimension and number of rows; built for few rows (generation), where it is
// bound by reading the cache.
//
// A workgroup takes up to 16 RB flattened rows of one kv head (paged_attn.h) and a stretch of their keys, its four
// wavefronts a quarter of the stretch each; nothing passes through LDS until the four states are merged at the end.  A
// wavefront walks over 32 keys at a time: scores are S^T = K Q^T (a matrix instruction takes 16 keys as rows, 16 query rows as
// columns), so that a lane holds scores of one query row, its key rows in global memory are read 16 bytes a lane straight into
// the operand, and the exponentials are, as they lie, the right operand of O^T = V^T P^T if the reduction index is counted
// 4 g .. 4 g + 3 of the first and of the second 16 keys for lane group g = lane / 16.  The left operand wants, per lane,
// one column of V for those 8 keys; the lane loads the 8 rows (16 lanes to a row, whole cache lines) for a run of columns
// and transposes the 8 x run block in registers (bf16: two byte permutations per pair of columns and keys; fp32: nothing).  The
// column of accumulator row i then is run * i + (number of the product), a permutation that the write-out undoes.
//
// Keys are requested again as soon as the scores of a step are formed, values behind its output product, one set of registers
// each: two or three wavefronts a SIMD keep 100 to 150 KB of a CU's requests under way, more than the 36 KB that 5 TB/s need at
// 1.5 us.  16 keys are one piece of a page, so that a descriptor of its own (scalar registers) holds their address and their end,
// and page numbers come through the scalar cache a step ahead: as vector loads they made every step wait for all that was under
// way.  32 sequences of 1650 to 8200 keys, 32 / 8 heads of 128 (0.64 GB): 121 us, 5.3 TB/s (copying reaches 5.1).
//
// The exponent offset of a row moves when a score exceeds it by more than 2^8 (in log2 units), so that nearly every step
// leaves the accumulators alone; sums of exponentials and products are fp32.  Over a bf16 cache an exponential enters the second
// product as two bf16 numbers (off by 2^-15 + 2^-18 at most): one rounding to bf16 would be as far off as that of the result, and the
// decode kernel for slabs has fp32 weights.  The matrix pipes have the time while the cache is read: with one number instead of two,
// 32 sequences of 1650 to 8200 keys 128.5 / 128.7 us, four of 333 to 2048 13.7 / 13.7, 64 rows over 4160 32.2 / 32.2; only long chunks of
// other head dimensions are bound by them, 1024 rows over 4024 keys, 32 / 8 heads of 96, 104 / 120.
#include "paged_attn.h"

namespace {

constexpr float RAISE = 8.0f;
// An exponential goes into the products as two bf16 numbers, its upper half (cut off) and what that leaves of OVER times it: more
// than nothing and of the same sign, so that a value that is infinite stays so in both products
constexpr float OVER = 1.0f + 0x1p-18f;
// Tiles up to which a merge has a workgroup for a row (0 / 8 / 32: one row over 32768 keys 37 / 30 / 30 us, nine over 3000 20 / 16 / 16;
// 100, 37 and 1 rows in fp32 19.5 / 19.5 / 21.5, sixteen rows of four sequences 30 / 30 / 27.5)
constexpr int FEW_TILES = 8;

template <typename T> struct Kind;
template <> struct Kind<bf16_t> {
    static constexpr int KD = 32;                          // head dimensions of a fragment of keys or queries
    typedef bf16x8 frag;
};
template <> struct Kind<float> {
    static constexpr int KD = 16;
    typedef f32x4 frag;
};

__device__ __forceinline__ f32x4 score_mfma(const bf16x8 &k, const bf16x8 &q, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 score_mfma(const f32x4 &k, const f32x4 &q, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[i], c, 0, 0, 0);
    return c;
}

// Sum or maximum over the four lanes that share a query row
__device__ __forceinline__ float rows_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, WAVE));
    return fmaxf(v, __shfl_xor(v, 32, WAVE));
}
__device__ __forceinline__ float rows_sum(float v) {
    v += __shfl_xor(v, 16, WAVE);
    return v + __shfl_xor(v, 32, WAVE);
}

// Wavefronts per SIMD that the registers allow, from below: keys and values of a step, queries and accumulators, and some 70 more
// (bf16 heads up to 64 and 65 to 128, 16 rows a tile, take 109 and 167 registers, room for one wavefront more than this counts)
constexpr int rows_occupancy(int size, int DM, int RB) {
    const int regs = DM / 4 * size + (DM / 16 * size + DM / 4) * RB + 70;
    return regs <= 168 ? 3 : regs <= 256 ? 2 : 1;
}

template <typename T, int DM, int RB>
__global__ __launch_bounds__(256, rows_occupancy(sizeof(T), DM, RB)) void paged_rows_kernel(PagedAttnParams p) {
    typedef typename Kind<T>::frag frag;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KD = Kind<T>::KD, KS = DM / KD, TILE = 16 * RB, KEYS = 32;
    constexpr int VW = DM / 16 * sizeof(T) / 4;            // 32-bit words of a V row in a lane
    constexpr int RUN = BF ? (DM / 16 < 8 ? DM / 16 : 8) : 4;      // neighbouring columns in a lane
    constexpr int NB = DM / 16;                            // products of 16 columns
    constexpr int RW = RUN * sizeof(T) / 4;

    extern __shared__ __attribute__((aligned(16))) float smem[];   // [4][TILE][DM] u, then [4][TILE][2]; before that the shards' steps
    const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedPlan<TILE, KEYS> plan;
    plan.make(p, p.few);
    const int piece = (int)(blockIdx.x / (uint32_t)p.Hkv), g = blockIdx.x - piece * p.Hkv;
    PagedWork wk;
    if (!plan.template pick<false>(p, p.few, piece, wk) || !wk.valid) return;

    // Keys that some row of the tile sees.  With one token those are all that the cache holds, as a rule, and a look at its limit
    // would only delay the first loads; several shards: first step of every shard, and its keys.
    int32_t *cum = (int32_t *)smem, *lens = cum + p.S + 1;
    const int64_t list0 = (int64_t)wk.b * p.S;
    const int tok0 = (int)((uint32_t)(wk.tile * TILE) / (uint32_t)p.rep);
    const int toks = (int)((uint32_t)(min((wk.tile + 1) * TILE, wk.n_rows) - 1) / (uint32_t)p.rep) - tok0 + 1;
    const int32_t *tile_limits = p.visible && toks > 1 ? p.visible + (int64_t)(wk.first_row + tok0) * p.S : nullptr;
    int only_len = 0;
    if (p.S > 1) {
        if (wave == 0) {
            int carry = 0;
            for (int s0 = 0; s0 < p.S; s0 += 64) {
                const int s = s0 + lane;
                int n = s < p.S ? paged_len(p, list0 + s) : 0;
                if (tile_limits && s < p.S) {
                    int most = 0;
                    for (int t0 = 0; t0 < toks; t0 += 4) {
                        int v[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = tile_limits[(int64_t)min(t0 + j, toks - 1) * p.S + s];
                        most = max(max(most, max(v[0], v[1])), max(v[2], v[3]));
                    }
                    n = min(n, most);
                }
                const int st = (n + KEYS - 1) / KEYS, incl = wave_inclusive(st);
                if (s < p.S) { lens[s] = n; cum[s] = carry + incl - st; }
                carry += __builtin_amdgcn_readlane(incl, 63);
            }
            if (lane == 0) cum[p.S] = carry;
        }
        __syncthreads();
    } else {
        only_len = paged_len(p, list0);
        if (tile_limits) {
            static_assert(TILE <= 64, "a lane for every token");
            int most = lane < toks ? tile_limits[lane] : 0;
#pragma unroll
            for (int o = 32; o; o >>= 1) most = max(most, __shfl_xor(most, o, WAVE));
            only_len = min(only_len, most);
        }
        only_len = __builtin_amdgcn_readfirstlane(max(only_len, 0));
    }
    int k0, k1;                                            // steps of this piece
    paged_cut(__builtin_amdgcn_readfirstlane(p.S > 1 ? cum[p.S] : (only_len + KEYS - 1) / KEYS), wk.piece, wk.n_pieces, k0, k1);

    // ---- query rows of this lane (column c16 of each block of 16)
    const T *qp = (const T *)p.q;
    frag Q[RB][KS];
    int token[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(wk.tile * TILE + rb * 16 + c16, wk.n_rows - 1), t = (int)((uint32_t)r / (uint32_t)p.rep);
        token[rb] = wk.first_row + t;
        const T *src = qp + (int64_t)token[rb] * p.q_stride + (int64_t)(g * p.rep + r - t * p.rep) * p.d;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = ks * KD + g4 * (KD / 4);
            Q[rb][ks] = frag{};
            if (c < p.d) Q[rb][ks] = *(const frag *)(src + c);
        }
    }

    f32x4 O[RB][NB];
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = -INFINITY;
        l[rb] = 0.f;
#pragma unroll
        for (int i = 0; i < NB; ++i) O[rb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    struct Step {
        int limit[RB];                                     // keys of the shard that a row may see
        int j0, rows, bad;                                 // first key; keys of the step that exist; bit kb: 16 keys whose list entry is no page
    };
    frag kf[2][KS];                                        // keys of a step; refilled as soon as its scores are formed
    float vf[8][VW];                                       // values, rows 4 g4 + j of the first, then of the second 16 keys; refilled behind the output product

    // Where step k lies: read a step before its loads are requested
    struct Place { int j0, shard, len, id[2]; };
    int shard = 0;
    auto locate = [&](int k) {
        Place x;
        int j0 = k * KEYS, len = only_len;
        if (p.S > 1) {
            while (k >= cum[shard + 1]) ++shard;           // (ends: k is below cum[S])
            j0 = (k - cum[shard]) * KEYS;
            len = lens[shard];
        }
        x.j0 = __builtin_amdgcn_readfirstlane(j0);
        x.len = __builtin_amdgcn_readfirstlane(len);
        x.shard = __builtin_amdgcn_readfirstlane(shard);
        const scalar_ints ids = (scalar_ints)p.table + (list0 + x.shard) * p.max_pages;
        x.id[0] = ids[x.j0 >> p.page_shift];
        x.id[1] = ids[min(x.j0 + 16, x.len - 1) >> p.page_shift];      // (a second 16 that does not exist: any entry that does)
        return x;
    };
    const uint32_t row_bytes = p.d * sizeof(T);
    const uint32_t k_off = c16 * row_bytes + g4 * 16, v_off = 4 * g4 * row_bytes + c16 * (RUN * sizeof(T));
    // (columns behind the head: outside every descriptor, which returns zeros)
    const auto k_at = [&](int ks) { return ks * KD + g4 * (KD / 4) < p.d ? k_off + ks * 64 : 0x40000000u; };
    // limits of the sequence's rows; without any, the descriptor is empty and its zeros are not looked at
    const __amdgpu_buffer_rsrc_t limits = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int32_t *>(p.visible ? p.visible + (int64_t)wk.first_row * p.S : nullptr), 0,
        p.visible ? (p.rows - wk.first_row) * p.S * 4 : 0, 0x00020000);
    uint32_t limit_off[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) limit_off[rb] = (uint32_t)(token[rb] - wk.first_row) * (uint32_t)(p.S * 4);
    auto seen_of = [&](const Step &x, int rb) {            // keys of a step that a row sees
        // (limits below 0 are 0: the lowest of the type would pass 2^31 in the difference)
        const int n = p.visible ? min(x.rows, max(x.limit[rb], 0) - x.j0) : x.rows;
        return min(max(n, 0), KEYS);
    };
    // The rows of 16 keys that exist: what lies behind them is outside the descriptor and arrives as zeros
    auto rows_of = [&](const void *pages, const Place &at, int kb) {
        const bool page = (uint32_t)at.id[kb] < (uint32_t)p.n_pages;
        const int exist = page ? min(max(at.len - at.j0 - 16 * kb, 0), 16) : 0;
        const int64_t first = exist ? ((((int64_t)at.id[kb] * p.Hkv + g) << p.page_shift) + ((at.j0 + 16 * kb) & ((1 << p.page_shift) - 1))) * p.d : 0;
        return __builtin_amdgcn_make_buffer_rsrc((T *)pages + first, 0, exist * row_bytes, 0x00020000);
    };
    auto load_keys = [&](const Place &at, Step &x) {
        const int rows = at.len - at.j0;                   // keys of the step that exist: at least 1
        x.j0 = at.j0;
        x.rows = rows;
        x.bad = ((uint32_t)at.id[0] >= (uint32_t)p.n_pages) | ((uint32_t)at.id[1] >= (uint32_t)p.n_pages && rows > 16) << 1;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)                    // (looked at a step later, so that nothing waits for it here)
            x.limit[rb] = (int)__builtin_amdgcn_raw_buffer_load_b32(limits, limit_off[rb], at.shard * 4, 0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const __amdgpu_buffer_rsrc_t r = rows_of(p.k_pages, at, kb);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                kf[kb][ks] = __builtin_bit_cast(frag, __builtin_amdgcn_raw_buffer_load_b128(r, p.d == DM ? k_off + ks * 64 : k_at(ks), 0, 0));
        }
    };
    auto load_values = [&](const Place &at) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const __amdgpu_buffer_rsrc_t r = rows_of(p.v_pages, at, kb);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < VW / RW; ++h) {
                    const uint32_t off = v_off + j * row_bytes + h * 16 * (RUN * sizeof(T));
                    if constexpr (RW == 4) {
                        const u32x4 t = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
#pragma unroll
                        for (int w = 0; w < 4; ++w) vf[kb * 4 + j][h * 4 + w] = __uint_as_float(t[w]);
                    } else {
                        const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
                        vf[kb * 4 + j][0] = __uint_as_float(t[0]);
                        vf[kb * 4 + j][1] = __uint_as_float(t[1]);
                    }
                }
        }
    };

    bool odd = false;
    // One step: scores, then the request of the next keys; exponentials and output product, then that of the next values
    auto step = [&](Step &x, const Place &next) {
        f32x4 s[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[rb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[rb][kb] = score_mfma(kf[kb][ks], Q[rb][ks], s[rb][kb]);
            }
        Step ahead;
        load_keys(next, ahead);
        int seen[RB];
        bool masked = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            seen[rb] = seen_of(x, rb);
            masked |= seen[rb] != KEYS;
        }
        masked = __any(masked) || x.bad;
        if (masked) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * kb + 4 * g4 + r >= seen[rb] || (x.bad >> kb & 1)) s[rb][kb][r] = -INFINITY;
        }
        bool raise = false;
        float top[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float t = fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3]));
            t = fmaxf(t, fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
            top[rb] = t * p.scale_log2;
            raise |= top[rb] > m[rb] + RAISE;
        }
        if (__any(raise)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const float m_new = fmaxf(m[rb], rows_max(top[rb]));
                const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[rb] - m_new);
                m[rb] = m_new;
                l[rb] *= f;
#pragma unroll
                for (int i = 0; i < NB; ++i) O[rb][i] *= f;
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float off = m[rb] == -INFINITY ? 0.f : m[rb];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[rb][kb][r] = __builtin_amdgcn_exp2f(fmaf(s[rb][kb][r], p.scale_log2, -off));
            l[rb] += ((s[rb][0][0] + s[rb][0][1]) + (s[rb][0][2] + s[rb][0][3])) + ((s[rb][1][0] + s[rb][1][1]) + (s[rb][1][2] + s[rb][1][3]));
        }
        // A value that is not finite must not meet the zero weight of a row that does not see it.  Steps in which every row
        // sees every key need no care; in the others such values leave the product, and what they do to the rows that see them
        // is made good behind the walk.
        if (masked) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    uint32_t u = __float_as_uint(vf[j][w]);
                    if (BF && (u & 0x7f80u) == 0x7f80u) { u &= 0xffff0000u; odd = true; }
                    if ((u & 0x7f800000u) == 0x7f800000u) { u = BF ? u & 0xffffu : 0u; odd = true; }
                    vf[j][w] = __uint_as_float(u);
                }
        }
        if constexpr (BF) {
            u32x4 P[2][RB];                                // [0] upper halves of the exponentials, [1] what they leave
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e0 = s[rb][j / 2][j % 2 * 2], e1 = s[rb][j / 2][j % 2 * 2 + 1];
                    const uint32_t b0 = __float_as_uint(e0), b1 = __float_as_uint(e1);
                    P[0][rb][j] = __builtin_amdgcn_perm(b1, b0, 0x07060302);
                    P[1][rb][j] = __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)fmaf(e0, OVER, -__uint_as_float(b0 & 0xffff0000u)),
                                                                      (bf16_t)fmaf(e1, OVER, -__uint_as_float(b1 & 0xffff0000u))});
                }
#pragma unroll
            for (int w = 0; w < VW; ++w) {                 // columns RUN c16 + 2 w and + 1 (mod RUN)
                u32x4 even, odd;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a = __builtin_bit_cast(uint32_t, vf[2 * j][w]), b = __builtin_bit_cast(uint32_t, vf[2 * j + 1][w]);
                    even[j] = __builtin_amdgcn_perm(b, a, 0x05040100);
                    odd[j] = __builtin_amdgcn_perm(b, a, 0x07060302);
                }
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const bf16x8 e = __builtin_bit_cast(bf16x8, P[half][rb]);
                        O[rb][2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), e, O[rb][2 * w], 0, 0, 0);
                        O[rb][2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), e, O[rb][2 * w + 1], 0, 0, 0);
                    }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        O[rb][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][i], s[rb][j / 4][j % 4], O[rb][i], 0, 0, 0);
        }
        load_values(next);
        x = ahead;
    };

    // this wavefront's quarter of the piece
    int a, b;
    paged_cut(k1 - k0, wave, 4, a, b);
    a += k0;
    b += k0;
    if (a < b) {
        // (the requests ahead are not conditional, behind the end they are of no rows: with a branch around them the compiler
        // cannot count the loads in flight and waits for all of them)
        Step x;
        Place at = locate(a);
        load_keys(at, x);
        load_values(at);
        const int first_shard = shard;
        for (int k = a; k < b; ++k) {
            at = locate(min(k + 1, b - 1));
            if (k + 1 == b) at.len = at.j0;                // (no rows: nothing is read)
            step(x, at);
        }
        if (__any(odd)) {
            // a weight times a value that is not finite is that value, whatever the weight
            shard = first_shard;
            for (int k = a; k < b; ++k) {
                const Place at = locate(k);
                int seen[RB];
                bool masked = false;
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    x.rows = at.len - at.j0;
                    x.j0 = at.j0;
                    x.limit[rb] = (int)__builtin_amdgcn_raw_buffer_load_b32(limits, limit_off[rb], at.shard * 4, 0);
                    seen[rb] = seen_of(x, rb);
                    masked |= seen[rb] != KEYS;
                }
                if (!__any(masked) && (uint32_t)at.id[0] < (uint32_t)p.n_pages && (uint32_t)at.id[1] < (uint32_t)p.n_pages) continue;
#pragma nounroll
                for (int key = 0; key < min(x.rows, KEYS); ++key) {
                    const int id = key < 16 ? at.id[0] : at.id[1];
                    if ((uint32_t)id >= (uint32_t)p.n_pages) continue;
                    const T *vr = (const T *)p.v_pages + ((((int64_t)id * p.Hkv + g) << p.page_shift) + ((at.j0 + key) & ((1 << p.page_shift) - 1))) * p.d;
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int c = i / RUN * 16 * RUN + RUN * (4 * g4 + r) + i % RUN;
                            const float v = (float)vr[c < p.d ? c : 0];
                            if ((__float_as_uint(v) & 0x7f800000u) != 0x7f800000u) continue;
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb)
                                if (key < seen[rb]) O[rb][i][r] += v;
                        }
                }
            }
        }
    }

    // ---- the four states meet in LDS
    if (p.S > 1) __syncthreads();                          // (the shards' steps lie there)
    float *su = smem, *sm = smem + 4 * TILE * DM;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float sum = rows_sum(l[rb]);
        if (g4 == 0) {
            sm[(wave * TILE + rb * 16 + c16) * 2] = m[rb];
            sm[(wave * TILE + rb * 16 + c16) * 2 + 1] = sum;
        }
        float *u = su + (wave * TILE + rb * 16 + c16) * DM;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) u[i / RUN * 16 * RUN + RUN * (4 * g4 + r) + i % RUN] = O[rb][i][r];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < TILE * (DM / 4); e += 256) {
        const int row = e / (DM / 4), c = e % (DM / 4) * 4, r = wk.tile * TILE + row;
        if (r >= wk.n_rows || c >= p.d) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[(w * TILE + row) * 2]);
        const float off = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm[(w * TILE + row) * 2] - off);
            sum += sm[(w * TILE + row) * 2 + 1] * f;
            u += *(const f32x4 *)(su + (w * TILE + row) * DM + c) * f;
        }
        if (wk.n_pieces > 1) {
            const int64_t at = ((int64_t)(wk.first_piece + wk.piece) * p.Hkv + g) * TILE + row;
            *(f32x4 *)(p.few.part_u + at * p.d + c) = u;
            if (c == 0) { p.few.part_ml[at * 2] = top; p.few.part_ml[at * 2 + 1] = sum; }
            continue;
        }
        const int t = (int)((uint32_t)r / (uint32_t)p.rep), h = g * p.rep + r - t * p.rep;
        const int64_t out = (int64_t)(wk.first_row + t) * p.o_stride + (int64_t)h * p.d + c;
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        u *= inv;
        if (!BF || p.o_f32) *(f32x4 *)((float *)p.o + out) = u;
        else *(bf16x4 *)((bf16_t *)p.o + out) = bf16x4{(bf16_t)u[0], (bf16_t)u[1], (bf16_t)u[2], (bf16_t)u[3]};
        if (c == 0 && p.lse) p.lse[(int64_t)h * p.rows + wk.first_row + t] = (top + __builtin_log2f(sum)) * LN2F;
    }
}

// Tiles whose walk was cut, of either kernel: their partials, weighted by exp2(m - largest m).  A wavefront takes a row at a
// time (four where there are few partials), DM / 4 lanes its columns; the lane groups that are left take every SUB-th partial, with a
// running maximum each, and meet at the end.
// ROWS rows at once, AT_ONCE partials of each requested at once.
template <typename T, int TILE, int DM, int ROWS, int AT_ONCE>
__device__ __forceinline__ void merge_rows(const PagedAttnParams &p, const PagedSet &set, const PagedWork &wk, int g, int row0) {
    constexpr int LPR = DM / 4, SUB = 64 / LPR;
    const int lane = threadIdx.x & 63, sub = lane / LPR, c = lane % LPR * 4, tile0 = wk.tile * TILE;
    const int64_t step = (int64_t)p.Hkv * TILE, at0 = ((int64_t)wk.first_piece * p.Hkv + g) * TILE;
    float top[ROWS], sum[ROWS];
    f32x4 u[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) { top[k] = -INFINITY; sum[k] = 0.f; u[k] = f32x4{0.f, 0.f, 0.f, 0.f}; }
    for (int i0 = sub; i0 < wk.n_pieces; i0 += SUB * AT_ONCE) {
        float2 a[ROWS][AT_ONCE];
        f32x4 x[ROWS][AT_ONCE];
#pragma unroll
        for (int k = 0; k < ROWS; ++k)
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                // (rows behind the last: that one again, not written)
                const int64_t at = at0 + min(row0 + 4 * k, wk.n_rows - 1 - tile0) + min(i0 + j * SUB, wk.n_pieces - 1) * step;
                a[k][j] = ((const float2 *)set.part_ml)[at];
                x[k][j] = *(const f32x4 *)(set.part_u + at * p.d + (c < p.d ? c : 0));
            }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            float most = top[k];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) most = fmaxf(most, a[k][j].x);   // (a repeated one changes nothing)
            const float off = most == -INFINITY ? 0.f : most, f = __builtin_amdgcn_exp2f(top[k] - off);
            top[k] = most;
            sum[k] *= f;
            u[k] *= f;
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                if (i0 + j * SUB >= wk.n_pieces) break;
                const float e = __builtin_amdgcn_exp2f(a[k][j].x - off);
                sum[k] += a[k][j].y * e;
                u[k] += x[k][j] * e;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {               // the lane groups' states
            const float other = __shfl_xor(top[k], o, WAVE), most = fmaxf(top[k], other), off = most == -INFINITY ? 0.f : most;
            const float f = __builtin_amdgcn_exp2f(top[k] - off), f1 = __builtin_amdgcn_exp2f(other - off);
            sum[k] = sum[k] * f + __shfl_xor(sum[k], o, WAVE) * f1;
#pragma unroll
            for (int j = 0; j < 4; ++j) u[k][j] = u[k][j] * f + __shfl_xor(u[k][j], o, WAVE) * f1;
            top[k] = most;
        }
        const int r = tile0 + row0 + 4 * k;
        if (sub || c >= p.d || r >= wk.n_rows) continue;
        const int t = (int)((uint32_t)r / (uint32_t)p.rep), h = g * p.rep + r - t * p.rep;
        const int64_t out = (int64_t)(wk.first_row + t) * p.o_stride + (int64_t)h * p.d + c;
        u[k] *= sum[k] == 0.f ? 0.f : 1.0f / sum[k];
        if (sizeof(T) == 4 || p.o_f32) *(f32x4 *)((float *)p.o + out) = u[k];
        else *(bf16x4 *)((bf16_t *)p.o + out) = bf16x4{(bf16_t)u[k][0], (bf16_t)u[k][1], (bf16_t)u[k][2], (bf16_t)u[k][3]};
        if (c == 0 && p.lse) p.lse[(int64_t)h * p.rows + wk.first_row + t] = (top[k] + __builtin_log2f(sum[k])) * LN2F;
    }
}
template <typename T, int TILE, int KEYS, int DM>
__device__ __forceinline__ void merge_set(const PagedAttnParams &p, const PagedSet &set, int first, int stride) {
    constexpr int SUB = 256 / DM, UNITS = TILE / 16;
    PagedPlan<TILE, KEYS> plan;
    plan.make(p, set);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // units: 16 rows of a tile and kv head, every fourth one a wavefront's; heads side by side as in the kernels that wrote the
    // partials, so that with 8 of them a die reads what its cache may still hold (512 rows over 2560 keys: 43.9 -> 41 us)
    for (int unit = first;; unit += stride) {
        const int rest = (int)((uint32_t)unit / (uint32_t)p.Hkv), g = unit - rest * p.Hkv, part = rest % UNITS, w = rest / UNITS;
        PagedWork wk;
        if (!plan.template pick<true>(p, set, w, wk)) return;
        const int left = wk.n_rows - wk.tile * TILE - part * 16;       // rows of the unit that exist
        if (!wk.valid || left <= wave) continue;
        const int row0 = part * 16 + wave;
        if (wk.n_pieces <= 2 * SUB && left > 4) merge_rows<T, TILE, DM, 4, 2>(p, set, wk, g, row0);
        else
            for (int k = 0; k < 16 && wave + k < left; k += 4) merge_rows<T, TILE, DM, 1, 8>(p, set, wk, g, row0 + k);
    }
}
// Few tiles, cut into many pieces: a workgroup to a row, its wavefronts a quarter of the partials each.
template <typename T, int TILE, int KEYS, int DM>
__device__ __forceinline__ void merge_set_by_workgroups(const PagedAttnParams &p, const PagedSet &set) {
    constexpr int LPR = DM / 4, SUB = 64 / LPR, AT_ONCE = 8, GROUPS = 4 * SUB;
    __shared__ float state[4][DM + 2];
    PagedPlan<TILE, KEYS> plan;
    plan.make(p, set);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane % LPR * 4;
    const int group = wave * SUB + lane / LPR;
    const int64_t step = (int64_t)p.Hkv * TILE;
    for (int unit = blockIdx.x;; unit += gridDim.x) {
        const int rest = (int)((uint32_t)unit / (uint32_t)p.Hkv), g = unit - rest * p.Hkv, row = rest % TILE, w = rest / TILE;
        PagedWork wk;
        if (!plan.template pick<true>(p, set, w, wk)) return;
        const int r = wk.tile * TILE + row;
        if (!wk.valid || r >= wk.n_rows) continue;         // (the same for the whole workgroup)
        const int64_t at0 = ((int64_t)wk.first_piece * p.Hkv + g) * TILE + row;
        float top = -INFINITY, sum = 0.f;
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = group; i0 < wk.n_pieces; i0 += GROUPS * AT_ONCE) {
            float2 a[AT_ONCE];
            f32x4 x[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int64_t at = at0 + min(i0 + j * GROUPS, wk.n_pieces - 1) * step;
                a[j] = ((const float2 *)set.part_ml)[at];
                x[j] = *(const f32x4 *)(set.part_u + at * p.d + (c < p.d ? c : 0));
            }
            float most = top;
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) most = fmaxf(most, a[j].x);
            const float off = most == -INFINITY ? 0.f : most, f = __builtin_amdgcn_exp2f(top - off);
            top = most;
            sum *= f;
            u *= f;
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                if (i0 + j * GROUPS >= wk.n_pieces) break;
                const float e = __builtin_amdgcn_exp2f(a[j].x - off);
                sum += a[j].y * e;
                u += x[j] * e;
            }
        }
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
            const float other = __shfl_xor(top, o, WAVE), most = fmaxf(top, other), off = most == -INFINITY ? 0.f : most;
            const float f = __builtin_amdgcn_exp2f(top - off), f1 = __builtin_amdgcn_exp2f(other - off);
            sum = sum * f + __shfl_xor(sum, o, WAVE) * f1;
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = u[j] * f + __shfl_xor(u[j], o, WAVE) * f1;
            top = most;
        }
        __syncthreads();                                   // (the last row's states have been read)
        if (lane < LPR) {
#pragma unroll
            for (int j = 0; j < 4; ++j) state[wave][c + j] = u[j];
            if (lane == 0) { state[wave][DM] = top; state[wave][DM + 1] = sum; }
        }
        __syncthreads();
        if (wave || lane >= LPR || c >= p.d) continue;
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) most = fmaxf(most, state[k][DM]);
        const float off = most == -INFINITY ? 0.f : most;
        sum = 0.f;
        u = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = __builtin_amdgcn_exp2f(state[k][DM] - off);
            sum += state[k][DM + 1] * f;
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] += state[k][c + j] * f;
        }
        const int t = (int)((uint32_t)r / (uint32_t)p.rep), h = g * p.rep + r - t * p.rep;
        const int64_t out = (int64_t)(wk.first_row + t) * p.o_stride + (int64_t)h * p.d + c;
        u *= sum == 0.f ? 0.f : 1.0f / sum;
        if (sizeof(T) == 4 || p.o_f32) *(f32x4 *)((float *)p.o + out) = u;
        else *(bf16x4 *)((bf16_t *)p.o + out) = bf16x4{(bf16_t)u[0], (bf16_t)u[1], (bf16_t)u[2], (bf16_t)u[3]};
        if (c == 0 && p.lse) p.lse[(int64_t)h * p.rows + wk.first_row + t] = (most + __builtin_log2f(sum)) * LN2F;
    }
}
template <typename T, int TILE, int DM>
__global__ __launch_bounds__(256) void paged_merge_few_kernel(PagedAttnParams p) {
    merge_set_by_workgroups<T, TILE, 32, DM>(p, p.few);
}

template <typename T, int TILE, int DM>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnParams p, int for_many) {
    if constexpr (sizeof(T) == 2 && DM <= 128) {
        if ((int)blockIdx.x < for_many) return merge_set<T, PAGED_TILE, PAGED_TILE_KEYS, DM>(p, p.many, blockIdx.x, for_many);
    }
    merge_set<T, TILE, 32, DM>(p, p.few, blockIdx.x - for_many, gridDim.x - for_many);
}

template <typename T, int DM, int RB>
int32_t launch_rows(const PagedAttnParams &p, hipStream_t s) {
    constexpr int TILE = 16 * RB;
    // (workgroups beyond those that are resident at once take turns)
    int64_t merge_many = 0, merge_few = 0;
    if (p.many.target) {
        const int32_t st = launch_paged_tile(p, s);
        if (st != CASCADE_OK) return st;
        merge_many = min((int64_t)1024, paged_grid(p, p.many, PAGED_TILE).split_tiles * p.Hkv * (PAGED_TILE / 16));
    }
    if (p.few.target) {
        const PagedGrid g = paged_grid(p, p.few, TILE);
        const int lds = max((int)sizeof(float) * 4 * TILE * (DM + 2), 4 * (2 * p.S + 1));
        auto kern = paged_rows_kernel<T, DM, RB>;
        static std::atomic<uint64_t> lds_ready{0};
        CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)kern, sizeof(float) * 4 * TILE * (DM + 2), lds_ready));
        hipLaunchKernelGGL(kern, dim3((unsigned)(g.pieces * p.Hkv)), dim3(256), lds, s, p);
        if (!p.many.target && g.split_tiles <= FEW_TILES) {
            hipLaunchKernelGGL((paged_merge_few_kernel<T, TILE, DM>), dim3((unsigned)min((int64_t)2048, g.split_tiles * p.Hkv * TILE)), dim3(256), 0, s, p);
            CASCADE_HIP_TRY(hipGetLastError());
            return CASCADE_OK;
        }
        merge_few = min((int64_t)1024, g.split_tiles * p.Hkv * (TILE / 16));
    }
    hipLaunchKernelGGL((paged_merge_kernel<T, TILE, DM>), dim3((unsigned)(merge_many + merge_few)), dim3(256), 0, s, p, (int)merge_many);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}
// 32 rows a tile where sequences have more than 16 on average, else 16.  Heads of more than 128 have no registers for 32, and fp32
// heads up to 64 are faster with 16 (12 heads of 64, 1024 rows over 4024 keys: 163 us against 176; 100, 37 and 1 rows over 1000, 448
// and 1: 23 against 28; 32 / 8 heads of 128, 256 rows over 2256 keys: 116 against 102).
int rows_tile(const PagedAttnParams &p, bool f32) {
    return (int64_t)p.rows * p.rep > (int64_t)16 * p.B && p.d <= 128 && !(f32 && p.d <= 64) ? 32 : 16;
}
template <typename T, int DM>
int32_t launch_dim(const PagedAttnParams &p, hipStream_t s) {
    if constexpr (DM == 128 || (DM == 64 && sizeof(T) == 2))
        if (rows_tile(p, sizeof(T) == 4) == 32) return launch_rows<T, DM, 2>(p, s);
    return launch_rows<T, DM, 1>(p, s);
}
// (fp32 heads of more than 128 need more than the 512 registers there are: 28 bytes a lane are spilled, written in front of the walk and
// read behind it and, 8 of them, in steps that move the exponent offset)
template <typename T>
int32_t launch_type(const PagedAttnParams &p, hipStream_t s) {
    return p.d <= 64 ? launch_dim<T, 64>(p, s) : p.d <= 128 ? launch_dim<T, 128>(p, s) : launch_dim<T, 256>(p, s);
}

// Sizes, and which sequences go to which kernel; as many pieces as workgroups are resident at once by rows_occupancy (32 / 8 heads of
// 128, five tokens of 8 sequences of 3000 keys, two workgroups a CU: 256, 512, 768, 1024 pieces 35.6, 36, 42.5, 45 us).  One token each
// would have room for three of them, but gains only where walks are very long, and loses where partials count, 512 / 768 pieces: 32
// sequences of 1650 to 8200 keys 128 / 128, 16 of 16000 217 / 209, 8 of 4096 34.9 / 34.8, 32 of 4000 with 64 / 8 heads 99 / 101, one of 32000
// 34.5 / 36.3, two tokens of 8 of 3000 28.3 / 29.3.  Beside sequences of many rows, where tiles hold
// 32 rows that a short sequence does not fill, 384 pieces instead of 512 leave fewer that start when others end (15 of one and
// four rows in 8 shards beside one of 509: 104 -> 98 us, 20 of one and three beside 300: 114 -> 109.5; without such a sequence 512
// are ahead, four of five rows 32 against 33, 64 rows over 4160 keys 28.5 against 30).  Kernels: bf16 with head dimensions of 64
// and 128 has paged_attn_tile.hip for the sequences of many rows, if the rows at hand can make one; with a single sequence it
// takes that with however many rows it has. With no more rows than sequences it is left out (one token each, most likely; its
// launch costs 4 us for nothing then, and a sequence that has several all the same is taken by the other kernel).  That holds for
// caches with many idle sequences too, although a chunk of fewer rows than there are sequences is guessed wrong: every workgroup looks at
// all sequences, so that the launch itself is dear there.  Without / with it, 32 / 8 heads of 128: one token of 100, 512 and 1024
// sequences of 64 keys 20.6 / 27.9, 117 / 149 and 334 / 394 us; in a cache of 1024 sequences one with 65, 512 and 1000 rows over 2000 and
// themselves 109 / 151, 355 / 369 and 458 / 418, and 70 through a descriptor of that sequence alone.
void set_sizes(PagedAttnParams &p, const cascade_paged_cache *c, const cascade_paged_attn_desc *d) {
    p.rows = d->rows; p.H = d->n_heads; p.Hkv = c->n_kv_heads; p.rep = p.H / p.Hkv; p.d = c->head_dim;
    p.S = c->n_shards; p.B = c->n_seqs; p.max_pages = c->max_pages; p.page_shift = page_shift(c); p.n_pages = c->n_pages;
    // (at least 8 steps of a piece, two a wavefront: with 4 / 8 / 16, 8 sequences in shards of 128 keys 22 / 22 / 24.5 us, nine rows over
    // 3000 keys 17 / 16 / 17, 24 over 3024 19 / 21 / 17.5)
    auto set = [&](PagedSet &x, int32_t above, int32_t upto, int target, int min_steps) {
        x.above = above; x.upto = upto;
        x.target = max(1, target / p.Hkv);
        x.inv_target = 1.0f / x.target;
        x.min_steps = min_steps;
    };
    const bool f32 = c->dtype == CASCADE_F32, tiles = !f32 && (p.d == 64 || p.d == 128) && (int64_t)p.rows * p.rep > PAGED_FEW && (p.B == 1 || p.rows > p.B);
    if (tiles) set(p.many, p.B == 1 ? 0 : PAGED_FEW, INT32_MAX, PAGED_TILE_TARGET, 4);
    const int tile = rows_tile(p, f32);
    if (!tiles || p.B > 1) set(p.few, 0, tiles ? PAGED_FEW : INT32_MAX, tiles && tile == 32 ? 384 : 256 * rows_occupancy(f32 ? 4 : 2, p.d, tile / 16), 8);
}
size_t set_parts(PagedAttnParams &p, bool f32, float *workspace) {
    size_t floats = 0;
    auto set = [&](PagedSet &x, int tile) {
        if (!x.target) return;
        const size_t parts = (size_t)paged_grid(p, x, tile).parts;
        x.max_parts = (int32_t)parts;
        x.part_u = workspace + floats;
        x.part_ml = x.part_u + parts * p.Hkv * tile * p.d;
        floats += align_up(parts * p.Hkv * tile * (p.d + 2), 4);
    };
    set(p.many, PAGED_TILE);
    set(p.few, rows_tile(p, f32));
    return floats;
}

int32_t check_attn(const cascade_paged_cache *c, const cascade_paged_attn_desc *d) {
    const int32_t st = check_paged_cache(c);
    if (st != CASCADE_OK) return st;
    if (!d || d->rows <= 0 || d->n_heads <= 0 || !(d->scale > 0.f) || d->q_stride < 0 || d->o_stride < 0) return CASCADE_EINVAL;
    if (d->n_heads % c->n_kv_heads) return CASCADE_ESHAPE;
    if (d->o_dtype != c->dtype && d->o_dtype != CASCADE_F32) return CASCADE_EUNSUPPORTED;
    const int64_t row = (int64_t)d->n_heads * c->head_dim;
    if (row > INT32_MAX || (int64_t)d->rows * (d->n_heads / c->n_kv_heads) > INT32_MAX ||
        (int64_t)d->rows * c->n_shards > INT32_MAX / 4)
        return CASCADE_EUNSUPPORTED;
    if ((d->q_stride && d->q_stride < row) || (d->o_stride && d->o_stride < row)) return CASCADE_ESHAPE;
    const int vec = c->dtype == CASCADE_BF16 ? 8 : 4, o_vec = d->o_dtype == CASCADE_BF16 ? 8 : 4;
    if (d->q_stride % vec || d->o_stride % o_vec) return CASCADE_EUNSUPPORTED;
    // a launch has less than 2^32 threads
    PagedAttnParams p = {};
    set_sizes(p, c, d);
    if (p.many.target && paged_grid(p, p.many, PAGED_TILE).pieces * p.Hkv >= 1 << 23) return CASCADE_EUNSUPPORTED;
    if (p.few.target && paged_grid(p, p.few, rows_tile(p, c->dtype == CASCADE_F32)).pieces * p.Hkv >= 1 << 24) return CASCADE_EUNSUPPORTED;
    return CASCADE_OK;
}

}   // namespace

extern "C" size_t cascade_paged_attn_workspace_bytes(const cascade_paged_cache *cache, const cascade_paged_attn_desc *desc) {
    if (check_attn(cache, desc) != CASCADE_OK) return 0;
    PagedAttnParams p = {};
    set_sizes(p, cache, desc);
    return align_up(set_parts(p, cache->dtype == CASCADE_F32, nullptr) * sizeof(float), 256);
}

extern "C" int32_t cascade_paged_attn(const cascade_paged_cache *cache, int32_t layer, const cascade_paged_attn_desc *desc,
                                      const int32_t *q_start_dev, const int32_t *visible_dev, const void *q, void *o, float *lse,
                                      void *workspace, size_t workspace_bytes, void *stream) {
    const int32_t st = check_attn(cache, desc);
    if (st != CASCADE_OK) return st;
    if (!q_start_dev || !q || !o) return CASCADE_EINVAL;
    if (layer < 0 || layer >= cache->n_layers) return CASCADE_ESHAPE;
    if (((uintptr_t)q | (uintptr_t)o) % 16) return CASCADE_EUNSUPPORTED;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < cascade_paged_attn_workspace_bytes(cache, desc)) return CASCADE_EWORKSPACE;
    const int es = cache->dtype == CASCADE_BF16 ? 2 : 4;
    const int64_t row = (int64_t)desc->n_heads * cache->head_dim;
    PagedAttnParams p = {};
    p.q = q; p.o = o; p.lse = lse;
    p.k_pages = (const char *)cache->k_pages + layer * layer_elems(cache) * es;
    p.v_pages = (const char *)cache->v_pages + layer * layer_elems(cache) * es;
    p.q_start = q_start_dev; p.visible = visible_dev; p.table = cache->page_table; p.len = cache->kv_len;
    p.q_stride = desc->q_stride ? desc->q_stride : row;
    p.o_stride = desc->o_stride ? desc->o_stride : row;
    set_sizes(p, cache, desc);
    set_parts(p, cache->dtype == CASCADE_F32, (float *)workspace);
    p.scale_log2 = desc->scale * 1.4426950408889634f;
    p.o_f32 = desc->o_dtype == CASCADE_F32;
    return cache->dtype == CASCADE_BF16 ? launch_type<bf16_t>(p, (hipStream_t)stream) : launch_type<float>(p, (hipStream_t)stream);
}
