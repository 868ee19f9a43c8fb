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
// The exponent offset of a row moves when a score exceeds it by more than 2^8 (in log2 units), so that nearly every step
// leaves the accumulators alone; sums of exponentials and products are fp32, the exponentials enter the second product in the
// cache's type (rounded to bf16: 2^-8 of a weight at most, as everywhere in this library).
#include "paged_attn.h"

namespace {

constexpr float RAISE = 8.0f;

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

__device__ __forceinline__ bool word_not_finite(float x, bool is_bf16_pair) {
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    return is_bf16_pair ? (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u : (w & 0x7f800000u) == 0x7f800000u;
}

template <typename T, int DM, int RB>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedAttnParams p) {
    typedef typename Kind<T>::frag frag;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KD = Kind<T>::KD, KS = DM / KD, TILE = 16 * RB, KEYS = 32;
    constexpr int VW = DM / 16 * sizeof(T) / 4;            // 32-bit words of a V row in a lane
    constexpr int RUN = BF ? (DM / 16 < 8 ? DM / 16 : 8) : 4;      // neighbouring columns in a lane
    constexpr int NB = DM / 16;                            // products of 16 columns
    constexpr int BUFS = (BF ? DM : 2 * DM) <= 256 ? 2 : 1;        // steps loaded ahead, where registers allow
    typedef __attribute__((ext_vector_type(RUN * sizeof(T) / 4))) uint32_t vload;

    extern __shared__ __attribute__((aligned(16))) float smem[];   // [4][TILE][DM] u, then [4][TILE][2]; before that the shards' steps
    const int lane = threadIdx.x & 63, c16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = blockIdx.y;
    PagedWork wk;
    if (!paged_find_work<TILE, KEYS, false>(p, blockIdx.x, wk)) return;

    // first step of every shard, and its length (several shards only)
    int32_t *cum = (int32_t *)smem, *lens = cum + p.S + 1;
    const int64_t list0 = (int64_t)wk.b * p.S;
    if (p.S > 1) {
        if (wave == 0) {
            int carry = 0;
            for (int s0 = 0; s0 < p.S; s0 += 64) {
                const int s = s0 + lane, n = s < p.S ? paged_len(p, list0 + s) : 0, st = (n + KEYS - 1) / KEYS;
                const int incl = wave_inclusive(st);
                if (s < p.S) { lens[s] = n; cum[s] = carry + incl - st; }
                carry += __shfl(incl, 63, WAVE);
            }
            if (lane == 0) cum[p.S] = carry;
        }
        __syncthreads();
    }

    // ---- query rows of this lane (column c16 of each block of 16)
    const T *qp = (const T *)p.q;
    frag Q[RB][KS];
    int token[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(wk.tile * TILE + rb * 16 + c16, wk.n_rows - 1), t = r / p.rep;
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
        frag k[2][KS];
        float v[8][VW];                                    // rows 4 g4 + j of the first, then of the second 16 keys
        int seen[RB];                                      // keys of the step that a row sees
        int64_t page[2];                                   // offset of the 16 keys' first row in the pools
    };
    Step st[BUFS];

    int shard = 0;
    const int only_len = p.S > 1 ? 0 : __builtin_amdgcn_readfirstlane(paged_len(p, list0));
    auto load = [&](int k, Step &x) {
        int j0 = k * KEYS, len;
        if (p.S > 1) {
            while (k >= cum[shard + 1]) ++shard;           // (ends: k is below cum[S])
            j0 = (k - cum[shard]) * KEYS;
            len = lens[shard];
        } else len = only_len;
        j0 = __builtin_amdgcn_readfirstlane(j0);
        len = __builtin_amdgcn_readfirstlane(len);
        const int s = __builtin_amdgcn_readfirstlane(shard);
        const int32_t *ids = p.table + (list0 + s) * p.max_pages;
        // the second 16 keys may begin behind the end: then the first ones stand in (and are not seen)
        int bad = 0;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int j = j0 + (kb == 1 && j0 + 16 < len ? 16 : 0);
            int id = ids[j >> p.page_shift];
            if ((uint32_t)id >= (uint32_t)p.n_pages) { bad |= 1 << kb; id = 0; }
            x.page[kb] = ((((int64_t)id * p.Hkv + g) << p.page_shift) + (j & ((1 << p.page_shift) - 1))) * p.d;
        }
        const int rows = len - j0;                         // keys of the step that exist: at least 1
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            int n = rows;
            if (p.visible) n = min(n, p.visible[(int64_t)token[rb] * p.S + s] - j0);
            // keys of a list entry that is no page do not exist: bit 30 for the first 16, 31 for the second
            x.seen[rb] = (min(max(n, 0), KEYS)) | bad << 30;
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int exist = min(rows - 16 * kb, 16) < 1 ? 16 : min(rows - 16 * kb, 16);    // (stand-in: the first 16, all there)
            const T *kr = (const T *)p.k_pages + x.page[kb] + (int64_t)min(c16, exist - 1) * p.d;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int c = ks * KD + g4 * (KD / 4);
                x.k[kb][ks] = *(const frag *)(kr + (c < p.d ? c : 0));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const T *vr = (const T *)p.v_pages + x.page[kb] + (int64_t)min(4 * g4 + j, exist - 1) * p.d;
#pragma unroll
                for (int h = 0; h < VW * 4 / (int)(RUN * sizeof(T)); ++h) {
                    const int c = h * 16 * RUN + RUN * c16;
                    const vload t = *(const vload *)(vr + (c < p.d ? c : 0));
#pragma unroll
                    for (int w = 0; w < (int)(RUN * sizeof(T) / 4); ++w)
                        x.v[kb * 4 + j][h * (RUN * sizeof(T) / 4) + w] = __builtin_bit_cast(float, (uint32_t)t[w]);
                }
            }
        }
    };

    auto step = [&](Step &x) {
        if (p.d < DM) {                                    // columns behind the head: zero on both sides
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    if (ks * KD + g4 * (KD / 4) >= p.d) x.k[kb][ks] = frag{};
        }
        f32x4 s[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[rb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[rb][kb] = score_mfma(x.k[kb][ks], Q[rb][ks], s[rb][kb]);
            }
        bool masked = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) masked |= x.seen[rb] != KEYS;
        masked = __any(masked);
        auto sees = [&](int rb, int kb, int r) {
            const int seen = x.seen[rb];
            return 16 * kb + 4 * g4 + r < (seen & 63) && !((uint32_t)seen >> (30 + kb) & 1);
        };
        if (masked) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!sees(rb, kb, r)) s[rb][kb][r] = -INFINITY;
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
        // sees every key need no care; in the others such values leave the product and are added row by row.
        if (masked) {
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) odd |= word_not_finite(x.v[j][w], BF);
            if (__any(odd)) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        uint32_t u = __builtin_bit_cast(uint32_t, x.v[j][w]);
                        if (BF) {
                            if ((u & 0x7f80u) == 0x7f80u) u &= 0xffff0000u;
                            if ((u & 0x7f800000u) == 0x7f800000u) u &= 0xffffu;
                        } else if ((u & 0x7f800000u) == 0x7f800000u) u = 0;
                        x.v[j][w] = __builtin_bit_cast(float, u);
                    }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma nounroll
                    for (int key = 0; key < KEYS; ++key) {
                        float w = s[rb][0][0];
#pragma unroll
                        for (int i = 1; i < 8; ++i)
                            if ((key >> 4) * 4 + (key & 3) == i) w = s[rb][i / 4][i % 4];
                        w = __shfl(w, (key >> 2 & 3) * 16 + c16, WAVE);
                        if (key >= (x.seen[rb] & 63) || ((uint32_t)x.seen[rb] >> (30 + (key >> 4)) & 1)) continue;
                        const T *vr = (const T *)p.v_pages + (key < 16 ? x.page[0] : x.page[1]) + (int64_t)(key & 15) * p.d;
#pragma unroll
                        for (int i = 0; i < NB; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int c = i / RUN * 16 * RUN + RUN * (4 * g4 + r) + i % RUN;
                                const float v = (float)vr[c < p.d ? c : 0];
                                if (word_not_finite(v, false)) O[rb][i][r] += w * v;
                            }
                    }
            }
        }
        if constexpr (BF) {
            bf16x8 P[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int j = 0; j < 8; ++j) P[rb][j] = (bf16_t)s[rb][j / 4][j % 4];
#pragma unroll
            for (int w = 0; w < VW; ++w) {                 // columns RUN c16 + 2 w and + 1 (mod RUN)
                u32x4 even, odd;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a = __builtin_bit_cast(uint32_t, x.v[2 * j][w]), b = __builtin_bit_cast(uint32_t, x.v[2 * j + 1][w]);
                    even[j] = __builtin_amdgcn_perm(b, a, 0x05040100);
                    odd[j] = __builtin_amdgcn_perm(b, a, 0x07060302);
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    O[rb][2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), P[rb], O[rb][2 * w], 0, 0, 0);
                    O[rb][2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), P[rb], O[rb][2 * w + 1], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        O[rb][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[j][i], s[rb][j / 4][j % 4], O[rb][i], 0, 0, 0);
        }
    };

    // this wavefront's quarter of the piece
    const int n = wk.k1 - wk.k0, a = wk.k0 + (int)((int64_t)n * wave / 4), b = wk.k0 + (int)((int64_t)n * (wave + 1) / 4);
    if (a < b) {
        if constexpr (BUFS == 2) {
            load(a, st[0]);
            // the request ahead is not conditional (behind the end it repeats the last step): with a branch around it the
            // compiler cannot count the loads in flight and waits for all of them
            for (int k = a;; k += 2) {
                load(min(k + 1, b - 1), st[1]);
                step(st[0]);
                if (k + 1 >= b) break;
                load(min(k + 2, b - 1), st[0]);
                step(st[1]);
                if (k + 2 >= b) break;
            }
        } else {
            for (int k = a; k < b; ++k) { load(k, st[0]); step(st[0]); }
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
    const int per_row = p.d / 4;
    for (int e = threadIdx.x; e < TILE * per_row; e += 256) {
        const int row = e / per_row, c = (e - row * per_row) * 4, r = wk.tile * TILE + row;
        if (r >= wk.n_rows) break;
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
            *(f32x4 *)(p.part_u + at * p.d + c) = u;
            if (c == 0) { p.part_ml[at * 2] = top; p.part_ml[at * 2 + 1] = sum; }
            continue;
        }
        const int t = r / p.rep, h = g * p.rep + r - t * p.rep;
        const int64_t out = (int64_t)(wk.first_row + t) * p.o_stride + (int64_t)h * p.d + c;
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        u *= inv;
        if (!BF || p.o_f32) *(f32x4 *)((float *)p.o + out) = u;
        else *(bf16x4 *)((bf16_t *)p.o + out) = bf16x4{(bf16_t)u[0], (bf16_t)u[1], (bf16_t)u[2], (bf16_t)u[3]};
        if (c == 0 && p.lse) p.lse[(int64_t)h * p.rows + wk.first_row + t] = (top + __builtin_log2f(sum)) * LN2F;
    }
}

template <typename T, int DM, int RB>
int32_t launch_rows(PagedAttnParams p, float *workspace, hipStream_t s) {
    constexpr int TILE = 16 * RB;
    p.target = max(1, PAGED_TARGET / p.Hkv);
    p.min_steps = 4;                                       // a step for each wavefront
    const PagedGrid g = paged_grid(p, TILE);
    p.max_parts = (int32_t)g.parts;
    p.part_ml = workspace;
    p.part_u = workspace + g.parts * p.Hkv * TILE * 2;
    const int lds = max((int)sizeof(float) * 4 * TILE * (DM + 2), 4 * (2 * p.S + 1));
    auto kern = paged_rows_kernel<T, DM, RB>;
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)kern, sizeof(float) * 4 * TILE * (DM + 2), lds_ready));
    hipLaunchKernelGGL(kern, dim3((unsigned)g.pieces, p.Hkv), dim3(256), lds, s, p);
    hipLaunchKernelGGL((paged_merge_kernel<T, TILE, 32>), dim3((unsigned)g.split_tiles, p.Hkv, RB), dim3(256), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}
template <typename T, int DM>
int32_t launch_dim(const PagedAttnParams &p, float *workspace, hipStream_t s) {
    // 32 rows a tile where sequences have more than 16 on average, else 16
    return (int64_t)p.rows * p.rep > (int64_t)16 * p.B ? launch_rows<T, DM, 2>(p, workspace, s) : launch_rows<T, DM, 1>(p, workspace, s);
}
template <typename T>
int32_t launch_type(const PagedAttnParams &p, float *workspace, hipStream_t s) {
    return p.d <= 64 ? launch_dim<T, 64>(p, workspace, s) : p.d <= 128 ? launch_dim<T, 128>(p, workspace, s) : launch_dim<T, 256>(p, workspace, s);
}

// bf16, head dimensions of 64 and 128: paged_attn_tile.hip takes the sequences of many rows
bool tiled(const cascade_paged_cache *c) { return c->dtype == CASCADE_BF16 && (c->head_dim == 64 || c->head_dim == 128); }

int32_t check_attn(const cascade_paged_cache *c, const cascade_paged_attn_desc *d) {
    const int32_t st = check_paged_cache(c);
    if (st != CASCADE_OK) return st;
    if (!d || d->rows <= 0 || d->n_heads <= 0 || !(d->scale > 0.f) || d->q_stride < 0 || d->o_stride < 0) return CASCADE_EINVAL;
    if (d->n_heads % c->n_kv_heads) return CASCADE_ESHAPE;
    if (d->o_dtype != c->dtype && d->o_dtype != CASCADE_F32) return CASCADE_EUNSUPPORTED;
    const int64_t row = (int64_t)d->n_heads * c->head_dim;
    if (row > INT32_MAX || (int64_t)d->rows * (d->n_heads / c->n_kv_heads) > INT32_MAX) return CASCADE_EUNSUPPORTED;
    if ((d->q_stride && d->q_stride < row) || (d->o_stride && d->o_stride < row)) return CASCADE_ESHAPE;
    const int vec = c->dtype == CASCADE_BF16 ? 8 : 4, o_vec = d->o_dtype == CASCADE_BF16 ? 8 : 4;
    if (d->q_stride % vec || d->o_stride % o_vec) return CASCADE_EUNSUPPORTED;
    return CASCADE_OK;
}

}   // namespace

extern "C" size_t cascade_paged_attn_workspace_bytes(const cascade_paged_cache *cache, const cascade_paged_attn_desc *desc) {
    if (check_attn(cache, desc) != CASCADE_OK) return 0;
    PagedAttnParams p = {};
    p.rows = desc->rows; p.rep = desc->n_heads / cache->n_kv_heads; p.B = cache->n_seqs;
    p.target = max(1, PAGED_TARGET / cache->n_kv_heads);
    size_t most = 0;
    for (int tile : {16, 32}) {
        const size_t floats = (size_t)paged_grid(p, tile).parts * cache->n_kv_heads * tile * (cache->head_dim + 2);
        most = floats > most ? floats : most;
    }
    if (tiled(cache) && (int64_t)p.rows * p.rep > PAGED_FEW) {
        p.target = max(1, PAGED_TILE_TARGET / cache->n_kv_heads);
        const size_t floats = (size_t)paged_grid(p, PAGED_TILE).parts * cache->n_kv_heads * PAGED_TILE * (cache->head_dim + 2);
        most = floats > most ? floats : most;
    }
    return align_up(most * sizeof(float), 256);
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
    p.rows = desc->rows; p.H = desc->n_heads; p.Hkv = cache->n_kv_heads; p.rep = p.H / p.Hkv; p.d = cache->head_dim;
    p.S = cache->n_shards; p.B = cache->n_seqs; p.max_pages = cache->max_pages; p.page_shift = page_shift(cache); p.n_pages = cache->n_pages;
    p.scale_log2 = desc->scale * 1.4426950408889634f;
    p.o_f32 = desc->o_dtype == CASCADE_F32;
    p.above = 0; p.upto = INT32_MAX;
    if (tiled(cache)) {
        // sequences of many rows, if the rows at hand can make one; then those of few, if there can be any (the launches follow
        // one another and may share the workspace)
        if ((int64_t)p.rows * p.rep > PAGED_FEW) {
            PagedAttnParams many = p;
            many.above = p.B == 1 ? 0 : PAGED_FEW;          // (a single one goes there with however many it has)
            const int32_t st = launch_paged_tile(many, (float *)workspace, (hipStream_t)stream);
            if (st != CASCADE_OK) return st;
            if (p.B == 1) return CASCADE_OK;
        }
        p.upto = PAGED_FEW;
    }
    return cache->dtype == CASCADE_BF16 ? launch_type<bf16_t>(p, (float *)workspace, (hipStream_t)stream)
                                        : launch_type<float>(p, (float *)workspace, (hipStream_t)stream);
}
