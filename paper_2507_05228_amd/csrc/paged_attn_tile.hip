// Attention over a paged cache, bf16, head dimensions 64 and 128, many rows: bound by the matrix pipes.
//
// A workgroup takes a tile of 32 NW flattened rows of one kv head (paged_attn.h; the query heads that share the kv head share
// its keys in LDS), 32 rows a wavefront, and walks over the keys that some row of the tile sees, 64 at a time, shard by shard.
// S^T = K Q^T and O^T = V^T P^T in 32x32x16 products: a lane holds scores of one query row, and the exponentials are, as they
// lie, the right operand of the second product, with its 16 keys counted 4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3 for lane half
// h = lane / 32.  K and V rows go from their pages straight into LDS (a page piece of 16 rows is a descriptor of its own, cut
// where the rows that the tile sees end: what lies behind arrives as zeros), two buffers each; the left operand of the
// second product, four keys of one column a lane, is what the transposing LDS read of gfx950 returns.  16-byte pieces of a row
// are permuted in LDS so that neither kind of read meets a bank twice.
//
// One barrier a step.  Behind it: scores of step t + 1 (matrix pipe) next to the exponentials of step t (vector pipe), then the
// output product of step t next to the maxima of step t + 1: one basic block, which the compiler interleaves.  K is requested two
// steps ahead of its use, V one.  Steps that some row of the tile does not see whole mask their scores before the maxima are
// taken, and look for values that are not finite (paged_attn_rows.hip has the reason).
#include "attn_bf16.h"
#include "paged_attn.h"

namespace {

constexpr float RAISE = 8.0f;
constexpr int KEYS = PAGED_TILE_KEYS;

__device__ __forceinline__ f32x16 mfma32(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
typedef __attribute__((ext_vector_type(4))) short i16x4;
__device__ __forceinline__ i16x4 read_transposed(const unsigned char *lds) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)lds);
}
__device__ __forceinline__ float halves_max(float v) {     // over the two lanes that share a query row
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ int wave_min_int(int v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o, WAVE));
    return v;
}
__device__ __forceinline__ int wave_max_int(int v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = max(v, __shfl_xor(v, o, WAVE));
    return v;
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, NW / 4) void paged_tile_kernel(PagedAttnParams p) {
    constexpr int TILE = 32 * NW, ROW = 2 * D, CPR = D / 8, KS = D / 16, DB = D / 32;
    constexpr int BUF = KEYS * ROW;                        // bytes of a tile of keys (or values)
    constexpr int RPI = 1024 / ROW;                        // rows that one instruction of a wavefront loads
    constexpr int NI = KEYS / RPI / NW;                    // instructions of a wavefront for a tile
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];   // three tiles of K, three of V, the shards' words
    int32_t *const cum = (int32_t *)(smem + 6 * BUF), *const limit = cum + p.S + 1, *const least = limit + p.S;
    int32_t *const odd_flag = least + p.S;

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.y;
    PagedWork wk;
    if (!paged_find_work<TILE, KEYS, false>(p, p.many, blockIdx.x, wk)) return;
    const int64_t list0 = (int64_t)wk.b * p.S;

    // ---- keys of every shard that some row of the tile sees, and those that all of them see
    {
        const int r0 = wk.tile * TILE, r1 = min(r0 + TILE, wk.n_rows) - 1;
        const int first = wk.first_row + r0 / p.rep, last = wk.first_row + r1 / p.rep;
        for (int s = wave; s < p.S; s += NW) {
            const int len = paged_len(p, list0 + s);
            int most = len, fewest = len;
            if (p.visible) {
                most = 0;
                for (int t = first + lane; t <= last; t += 64) {
                    const int v = min(max(p.visible[(int64_t)t * p.S + s], 0), len);
                    most = max(most, v);
                    fewest = min(fewest, v);
                }
                most = wave_max_int(most);
                fewest = wave_min_int(fewest);
            }
            if (lane == 0) { limit[s] = most; least[s] = fewest; }
        }
        if (tid == 0) *odd_flag = 0;
        __syncthreads();
        if (wave == 0) {
            int carry = 0;
            for (int s0 = 0; s0 < p.S; s0 += 64) {
                const int s = s0 + lane, st = s < p.S ? (limit[s] + KEYS - 1) / KEYS : 0, incl = wave_inclusive(st);
                if (s < p.S) cum[s] = carry + incl - st;
                carry += __builtin_amdgcn_readlane(incl, 63);
            }
            if (lane == 0) cum[p.S] = carry;
        }
        __syncthreads();
    }
    const int steps = __builtin_amdgcn_readfirstlane(cum[p.S]);
    int k0, k1;
    paged_cut(steps, wk.piece, wk.n_pieces, k0, k1);

    // ---- this lane's query row
    const int row = wk.tile * TILE + wave * 32 + l32, r = min(row, wk.n_rows - 1), tok = r / p.rep;
    const int token = wk.first_row + tok, head = g * p.rep + r - tok * p.rep;
    bf16x8 Q[KS];
    {
        const bf16_t *src = (const bf16_t *)p.q + (int64_t)token * p.q_stride + (int64_t)head * D + 8 * h;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) Q[ks] = *(const bf16x8 *)(src + 16 * ks);
    }
    f32x16 O[DB], S[2];
#pragma unroll
    for (int i = 0; i < DB; ++i) O[i] = f32x16{};
    float m = -INFINITY, l = 0.f;

    // ---- tiles
    struct Tile {
        int j0, shard, end, bad;                           // first key; keys of the shard that count; blocks of 16 without a page
        int64_t at;                                        // offset of the piece of a page that this wavefront loads
        int here;                                          // its rows that count
    };
    constexpr int ROWS_W = KEYS / NW;                      // rows that a wavefront loads: within 16
    auto tile_at = [&](int t, int &shard) {
        Tile x;
        if (p.S > 1)
            while (t >= cum[shard + 1]) ++shard;           // (ends: t is below cum[S])
        x.shard = __builtin_amdgcn_readfirstlane(shard);
        x.j0 = __builtin_amdgcn_readfirstlane((t - cum[shard]) * KEYS);
        x.end = __builtin_amdgcn_readfirstlane(limit[shard]);
        const int32_t *ids = p.table + (list0 + x.shard) * p.max_pages;
        x.bad = 0;
#pragma unroll
        for (int b = 0; b < KEYS / 16; ++b) {
            const int j = x.j0 + 16 * b;
            const int id = ids[min(j, x.end - 1) >> p.page_shift];
            if (j < x.end && (uint32_t)id >= (uint32_t)p.n_pages) x.bad |= 1 << b;
        }
        const int j = x.j0 + wave * ROWS_W;
        const int id = __builtin_amdgcn_readfirstlane(ids[min(j, x.end - 1) >> p.page_shift]);
        x.here = (uint32_t)id < (uint32_t)p.n_pages ? min(max(x.end - j, 0), ROWS_W) : 0;
        x.at = x.here ? ((((int64_t)id * p.Hkv + g) << p.page_shift) + (j & ((1 << p.page_shift) - 1))) * D : 0;
        return x;
    };
    const int ld_row = lane / CPR, ld_slot = lane % CPR;
    uint32_t k_off[NI], v_off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int rr = i * RPI + ld_row, tr = wave * ROWS_W + rr;
        k_off[i] = rr * ROW + (ld_slot ^ (D == 128 ? tr & 15 : (tr >> 1) & 7)) * 16;
        v_off[i] = rr * ROW + (ld_slot ^ (D == 128 ? (tr & 3) << 2 : (tr & 2) << 1)) * 16;
    }
    auto request = [&](const Tile &x, const void *pages, unsigned char *buf, const uint32_t (&off)[NI]) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((bf16_t *)pages + x.at, 0, x.here * ROW, 0x00020000);
#pragma unroll
        for (int i = 0; i < NI; ++i) load16_to_lds(rs, buf + (wave * ROWS_W + i * RPI) * ROW, off[i]);
    };
    unsigned char *const kbuf = smem, *const vbuf = smem + 3 * BUF;

    // ---- pieces of a step
    const int k_swz = D == 128 ? l32 & 15 : (l32 >> 1) & 7, k_row = l32 * ROW;
    auto scores = [&](const unsigned char *kb, f32x16 (&out)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            out[b] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                out[b] = mfma32(*(const bf16x8 *)(kb + b * 32 * ROW + k_row + (((2 * ks + h) ^ k_swz) * 16)), Q[ks], out[b]);
        }
    };
    auto top_of = [&](const f32x16 (&s)[2]) {
        float t = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) t = fmaxf(fmaxf(t, s[0][i]), s[1][i]);
        return t * p.scale_log2;
    };
    auto key_of = [&](int b, int i) { return 32 * b + 8 * (i >> 2) + 4 * h + (i & 3); };
    int seen_shard = -1, seen = 0, seen_least = 0;         // this row's limit in the shard of the tile in hand
    auto limits = [&](int shard) {
        if (shard == seen_shard) return;
        seen_shard = shard;
        seen = limit[shard];
        if (p.visible) seen = min(seen, p.visible[(int64_t)token * p.S + shard]);
        seen_least = __builtin_amdgcn_readfirstlane(wave_min_int(seen));
    };
    // masks what the rows do not see; the largest score that is left, in log2 units
    auto masked_top = [&](const Tile &x, f32x16 (&s)[2], float top) {
        limits(x.shard);
        if (x.j0 + KEYS > seen_least || x.bad) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (x.j0 + key_of(b, i) >= seen || (x.bad >> (2 * b + (i >> 3)) & 1)) s[b][i] = -INFINITY;
            top = top_of(s);
        }
        return top;
    };
    const int vr_row = (lane & 15) >> 2;                   // row of the four keys that this lane's address names
    const int v_col = 16 * (lane >> 4 & 1) + 4 * (lane & 3);       // and its first column of 32
    auto v_frag = [&](const unsigned char *vb, int kk, int db) {
        i16x4 v[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int tr = 16 * kk + 8 * half + 4 * h + vr_row, chunk = 4 * db + (v_col >> 3);
            const int swz = D == 128 ? (tr & 3) << 2 : (tr & 2) << 1;
            v[half] = read_transposed(vb + tr * ROW + (chunk ^ swz) * 16 + (v_col & 7) * 2);
        }
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };

    if (k0 < k1) {
        int shard_ahead = 0;
        Tile cur = tile_at(k0, shard_ahead), next, after;
        request(cur, p.k_pages, kbuf, k_off);
        // (behind the last step: nothing is requested, and scores of what the buffer holds are formed and not used)
        auto tile_or_none = [&](int t, const Tile &last) {
            if (t < k1) return tile_at(t, shard_ahead);
            Tile x = last;
            x.here = 0;
            return x;
        };
        next = tile_or_none(k0 + 1, cur);
        request(cur, p.v_pages, vbuf, v_off);
        request(next, p.k_pages, kbuf + BUF, k_off);
        after = tile_or_none(k0 + 2, next);
        request(next, p.v_pages, vbuf + BUF, v_off);
        request(after, p.k_pages, kbuf + 2 * BUF, k_off);
        phase_barrier<0, false>();
        scores(kbuf, S);
        float top = masked_top(cur, S, top_of(S));
        int b0 = 0, b1 = BUF, b2 = 2 * BUF;                // buffers of steps t, t + 1, t + 2 (mod 3)
        for (int t = k0; t < k1; ++t) {
            // K of step t + 1 and V of step t are there (each wavefront waited for its own in the step before); everyone is done
            // with K of t and V of t - 1
            phase_barrier<-1, false>();
            const Tile later = tile_or_none(t + 3, after); // (requested at the end of the step: its page numbers arrive meanwhile)
            const unsigned char *vb = vbuf + b0;
            const bool care = cur.j0 + KEYS > __builtin_amdgcn_readfirstlane(least[cur.shard]);
            bool not_finite = false;
            if (care) {                                    // (the same for all wavefronts)
                bool mine = false;
#pragma unroll
                for (int i = 0; i < BUF / (1024 * NW); ++i) {
                    const u32x4 w = *(const u32x4 *)(vb + (i * NW * 64 + tid) * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) mine |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
                }
                if (mine) *odd_flag = 1;
                phase_barrier<-1, true>();
                not_finite = __builtin_amdgcn_readfirstlane(*odd_flag) != 0;
                if (not_finite) {                          // out of the product; added below, row by row
#pragma unroll
                    for (int i = 0; i < BUF / (1024 * NW); ++i) {
                        u32x4 w = *(const u32x4 *)(vb + (i * NW * 64 + tid) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if ((w[j] & 0x7f80u) == 0x7f80u) w[j] &= 0xffff0000u;
                            if ((w[j] & 0x7f800000u) == 0x7f800000u) w[j] &= 0xffffu;
                        }
                        *(u32x4 *)(vb + (i * NW * 64 + tid) * 16) = w;
                    }
                    phase_barrier<-1, true>();
                    if (tid == 0) *odd_flag = 0;
                }
            }
            if (__any(top > m + RAISE)) {
                const float m_new = fmaxf(m, halves_max(top));
                const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= f;
#pragma unroll
                for (int i = 0; i < DB; ++i) O[i] *= f;
            }
            const float off = m == -INFINITY ? 0.f : m;
            f32x16 S_next[2];
            scores(kbuf + b1, S_next);                     // (behind the last step: unused)
            bf16x8 P[4];
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(S[kk >> 1][8 * (kk & 1) + j], p.scale_log2, -off));
                    sum[j & 3] += e;
                    P[kk][j] = (bf16_t)e;
                }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): K of step t + 2 and V of t + 1, requested a step ago
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int db = 0; db < DB; ++db) O[db] = mfma32(v_frag(vb, kk, db), P[kk], O[db]);
            float top_next = top_of(S_next);
            // The requests stand behind the reads of V: in front of a transposing read the compiler waits for every load into
            // LDS that is under way.
            __builtin_amdgcn_sched_barrier(0);
            request(later, p.k_pages, kbuf + b0, k_off);
            request(after, p.v_pages, vbuf + b2, v_off);
            if (not_finite) {
                // values of this tile from memory: keys that this row sees, columns that this lane holds
                const int32_t *ids = p.table + (list0 + cur.shard) * p.max_pages;
#pragma nounroll
                for (int key = 0; key < KEYS; ++key) {
                    float w = 0.f;
                    const int idx = (key >> 5) * 16 + (key >> 3 & 3) * 4 + (key & 3);      // register of the lane that holds it
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (idx == i) w = (float)P[i >> 3][i & 7];
                    w = __shfl(w, (key >> 2 & 1) * 32 + l32, WAVE);
                    const int j = cur.j0 + key;
                    if (j >= seen || (cur.bad >> (key >> 4) & 1)) continue;
                    const bf16_t *vr = (const bf16_t *)p.v_pages +
                        ((((int64_t)ids[j >> p.page_shift] * p.Hkv + g) << p.page_shift) + (j & ((1 << p.page_shift) - 1))) * D;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = (float)vr[32 * db + 8 * (i >> 2) + 4 * h + (i & 3)];
                            if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) O[db][i] += w * v;
                            if ((i & 3) == 3) __builtin_amdgcn_sched_barrier(0);       // (rare: few registers matter more than its time)
                        }
                }
            }
            if (t + 1 < k1) top_next = masked_top(next, S_next, top_next);
            top = top_next;
            S[0] = S_next[0];
            S[1] = S_next[1];
            cur = next;
            next = after;
            after = later;
            const int free = b0;
            b0 = b1; b1 = b2; b2 = free;
        }
    }
    {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false));
        l = __uint_as_float(x.x) + __uint_as_float(x.y);
    }
    if (row >= wk.n_rows) return;
    if (wk.n_pieces > 1) {
        const int64_t at = ((int64_t)(wk.first_piece + wk.piece) * p.Hkv + g) * TILE + wave * 32 + l32;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f32x4 *)(p.many.part_u + at * D + 32 * db + 8 * i + 4 * h) = f32x4{O[db][4 * i], O[db][4 * i + 1], O[db][4 * i + 2], O[db][4 * i + 3]};
        if (h == 0) { p.many.part_ml[at * 2] = m; p.many.part_ml[at * 2 + 1] = l; }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const int64_t out = (int64_t)token * p.o_stride + (int64_t)head * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 u = f32x4{O[db][4 * i], O[db][4 * i + 1], O[db][4 * i + 2], O[db][4 * i + 3]} * inv;
            const int c = 32 * db + 8 * i + 4 * h;
            if (p.o_f32) *(f32x4 *)((float *)p.o + out + c) = u;
            else *(bf16x4 *)((bf16_t *)p.o + out + c) = bf16x4{(bf16_t)u[0], (bf16_t)u[1], (bf16_t)u[2], (bf16_t)u[3]};
        }
    if (h == 0 && p.lse) p.lse[(int64_t)head * p.rows + token] = (m + __builtin_log2f(l)) * LN2F;
}

template <int D>
int32_t launch_dim(const PagedAttnParams &p, hipStream_t s) {
    constexpr int NW = PAGED_TILE / 32;
    auto kern = paged_tile_kernel<D, NW>;
    const int lds = 6 * KEYS * 2 * D + 4 * (3 * p.S + 2);
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)kern, 6 * KEYS * 2 * D + 4 * (3 * 1024 + 2), lds_ready));
    hipLaunchKernelGGL(kern, dim3((unsigned)paged_grid(p, p.many, PAGED_TILE).pieces, p.Hkv), dim3(64 * NW), lds, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

}   // namespace

int32_t launch_paged_tile(const PagedAttnParams &p, hipStream_t s) { return p.d == 64 ? launch_dim<64>(p, s) : launch_dim<128>(p, s); }
