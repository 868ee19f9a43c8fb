// Attention over a paged cache, bf16, head dimensions 64 and 128, many rows: bound by the matrix pipes.
//
// A workgroup takes a tile of 32 NW flattened rows of one kv head (paged_attn.h; the query heads that share the kv head share
// its keys in LDS), 32 rows a wavefront, and walks over the keys that some row of the tile sees, 64 at a time, shard by shard.
// S^T = K Q^T and O^T = V^T P^T in 32x32x16 products: a lane holds scores of one query row, and the exponentials are, as they
// lie, the right operand of the second product, with its 16 keys counted 4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3 for lane half
// h = lane / 32.  K and V rows go from their pages straight into LDS (a page piece of 16 rows is a descriptor of its own, cut
// where the rows that the tile sees end), three buffers each; the left operand of the second product, four keys of one column
// a lane, is what the transposing LDS read returns.  16-byte pieces of a row are permuted in LDS so that neither kind of read
// meets a bank twice (counted: no conflicts).
//
// A step has a vector half (the request of K two steps and of V one step ahead, the mask, maxima, exponentials of step t) and a
// matrix half (scores of step t + 1, output product of step t).  Wavefronts w and w + 4 share a SIMD; the second four run half a
// step behind the first, a barrier between the halves, so that a SIMD's matrix pipe works for one while the other takes
// exponentials.  In front of a transposing read the compiler waits for every load into LDS that is under way: the wait in the
// middle of the matrix half says so, and what it waits for was requested half a step before.  What the two halves of a
// workgroup read and write at a time: at slot 2 t the first four request into the buffers of K(t + 2) and V(t + 1), last read at
// slot 2 t - 2, while the others read K(t) and V(t - 1); every wavefront has waited for its own part of a tile at least one
// barrier before anyone reads it.
//
// The exponentials are rounded to bf16 in front of the second product (off by 2^-8 at most; their sum takes them in fp32), as in the
// attention of whole layers: a second product for what the rounding leaves, as paged_attn_rows.hip has it, would be half as much
// again for the matrix pipes, which bound this kernel.
//
// One sequence, 4096 rows over 16384 keys, 32 / 8 heads of 128 (0.96 TFLOP under the causal limit): 832 us, 1.16 PFLOP/s, where
// a large library product reaches 1.21; the matrix pipes are busy 58 % of the time at the 1.7 to 1.9 GHz that the device holds under
// this load, the LDS about as long.  Each of the following against what was the kernel then: all wavefronts in phase 1027 against 915;
// page numbers through vector loads 974 against 915 (their wait is one for all loads); operands of the products requested four to eight
// instructions ahead by hand 937 to 944 against 916; 16x16x32 products 1070 against 930; requests behind the reads of V 855 against
// 827; tiles of 128 rows 1526 against 893; priority for either half: no difference.
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

// LDS accesses of a wavefront's lanes on either side keep their order (the hardware keeps it; the compiler is told)
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, NW / 4) void paged_tile_kernel(PagedAttnParams p) {
    constexpr int TILE = 32 * NW, ROW = 2 * D, CPR = D / 8, KS = D / 16, DB = D / 32;
    constexpr int BUF = KEYS * ROW;                        // bytes of a tile of keys (or values)
    constexpr int RPI = 1024 / ROW;                        // rows that one instruction of a wavefront loads
    constexpr int NI = KEYS / RPI / NW;                    // instructions of a wavefront for a tile
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];   // three tiles of K, three of V, the shards' words
    int32_t *const cum = (int32_t *)(smem + 6 * BUF), *const limit = cum + p.S + 1, *const least = limit + p.S;
    int32_t *const any_bad = least + p.S, *const odd_flag = any_bad + 1;

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool second = wave >= NW / 2;                    // (the SIMD's other wavefront)
    const int piece = (int)(blockIdx.x / (uint32_t)p.Hkv), g = blockIdx.x - piece * p.Hkv;
    PagedWork wk;
    PagedPlan<TILE, KEYS> plan;
    plan.make(p, p.many);
    if (!plan.template pick<false>(p, p.many, piece, wk) || !wk.valid) return;
    const int64_t list0 = (int64_t)wk.b * p.S;

    // ---- keys of every shard that some row of the tile sees, and whether the lists name pages for them
    if (tid < 2) any_bad[tid] = 0;
    __syncthreads();
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
            const int pages = (most + (1 << p.page_shift) - 1) >> p.page_shift;
            bool bad = false;
            for (int i = lane; i < pages; i += 64) bad |= (uint32_t)p.table[(list0 + s) * p.max_pages + i] >= (uint32_t)p.n_pages;
            if (bad) *any_bad = 1;
        }
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
    const bool bad_pages = __builtin_amdgcn_readfirstlane(*any_bad) != 0;
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
        bool care;                                         // some row of the workgroup does not see all of it
    };
    constexpr int ROWS_W = KEYS / NW;                      // rows that a wavefront loads: within 16
    struct Walk { int shard, base, upto, end, least; };    // a shard: its first step, the next one's, its keys that count
    auto shard_at = [&](int s) {
        Walk w;
        w.shard = s;
        w.base = __builtin_amdgcn_readfirstlane(cum[s]);
        w.upto = __builtin_amdgcn_readfirstlane(cum[s + 1]);
        w.end = __builtin_amdgcn_readfirstlane(limit[s]);
        w.least = __builtin_amdgcn_readfirstlane(least[s]);
        return w;
    };
    auto tile_at = [&](int t, Walk &w) {
        while (t >= w.upto) w = shard_at(w.shard + 1);     // (ends: t is below cum[S])
        Tile x;
        x.shard = w.shard;
        x.j0 = (t - w.base) * KEYS;
        x.end = w.end;
        x.care = x.j0 + KEYS > w.least;
        const scalar_ints ids = (scalar_ints)p.table + (list0 + x.shard) * p.max_pages;
        x.bad = 0;
        if (bad_pages) {
#pragma unroll
            for (int b = 0; b < KEYS / 16; ++b) {
                const int j = x.j0 + 16 * b;
                if (j < x.end && (uint32_t)ids[j >> p.page_shift] >= (uint32_t)p.n_pages) x.bad |= 1 << b;
            }
        }
        const int j = x.j0 + wave * ROWS_W;
        const int id = ids[min(j, x.end - 1) >> p.page_shift];
        x.here = __builtin_amdgcn_readfirstlane((uint32_t)id < (uint32_t)p.n_pages ? min(max(x.end - j, 0), ROWS_W) : 0);
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
        for (int b = 0; b < 2; ++b) out[b] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                out[b] = mfma32(*(const bf16x8 *)(kb + b * 32 * ROW + k_row + (((2 * ks + h) ^ k_swz) * 16)), Q[ks], out[b]);
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
    // masks what the rows do not see
    auto mask = [&](const Tile &x, f32x16 (&s)[2]) {
        limits(x.shard);
        if (x.j0 + KEYS <= seen_least && !x.bad) return;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (x.j0 + key_of(b, i) >= seen || (x.bad >> (2 * b + (i >> 3)) & 1)) s[b][i] = -INFINITY;
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

    // Values that are not finite must not meet the zero weight of a row that does not see them.  In a tile that some row of the
    // workgroup does not see whole, a wavefront clears those among the rows that it loaded itself, once they have arrived; what
    // they do to the rows that see them is made good behind the walk.
    auto clear_odd = [&](unsigned char *vb) {
        unsigned char *const mine = vb + wave * ROWS_W * ROW + lane * 16;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            u32x4 w = *(const u32x4 *)(mine + i * 1024);
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((w[j] & 0x7f80u) == 0x7f80u) { w[j] &= 0xffff0000u; odd = true; }
                if ((w[j] & 0x7f800000u) == 0x7f800000u) { w[j] &= 0xffffu; odd = true; }
            }
            if (odd) { *(u32x4 *)(mine + i * 1024) = w; *odd_flag = 1; }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // (in front of the next barrier)
    };
    if (k0 < k1) {
        int s0 = 0;
        while (k0 >= cum[s0 + 1]) ++s0;
        Walk ahead = shard_at(__builtin_amdgcn_readfirstlane(s0));
        // (behind the last step: nothing is requested, and scores of what the buffer holds are formed and not used)
        auto tile_or_none = [&](int t, const Tile &last) {
            if (t < k1) return tile_at(t, ahead);
            Tile x = last;
            x.here = 0;
            x.care = false;
            return x;
        };
        Tile cur = tile_at(k0, ahead);
        request(cur, p.k_pages, kbuf, k_off);
        request(cur, p.v_pages, vbuf, v_off);
        Tile next = tile_or_none(k0 + 1, cur);
        request(next, p.k_pages, kbuf + BUF, k_off);
        Tile after = tile_or_none(k0 + 2, next);
        phase_barrier<0, false>();
        if (cur.care) clear_odd(vbuf);
        scores(kbuf, S);
        int b0 = 0, b1 = BUF, b2 = 2 * BUF;                // buffers of steps t, t + 1, t + 2 (mod 3)
        if (second) phase_barrier<-1, false>();            // half a step behind the first four wavefronts
        for (int t = k0; t < k1; ++t) {
            // ---- vector half
            request(after, p.k_pages, kbuf + b2, k_off);
            request(next, p.v_pages, vbuf + b1, v_off);
            const Tile later = tile_or_none(t + 3, after);
            mask(cur, S);
            const float top = top_of(S);
            if (__any(top > m + RAISE)) {
                const float m_new = fmaxf(m, halves_max(top));
                const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= f;
#pragma unroll
                for (int i = 0; i < DB; ++i) O[i] *= f;
            }
            const float off = m == -INFINITY ? 0.f : m;
            u32x4 P[4];
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(S[kk >> 1][8 * (kk & 1) + 2 * j], p.scale_log2, -off));
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(S[kk >> 1][8 * (kk & 1) + 2 * j + 1], p.scale_log2, -off));
                    sum[j] += e0 + e1;
                    P[kk][j] = __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)e0, (bf16_t)e1});
                }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            asm volatile("" : "+v"(l));                    // (here, not behind the products with 32 registers in tow)
            phase_barrier<-1, false>();
            // ---- matrix half
            const unsigned char *vb = vbuf + b0;
            scores(kbuf + b1, S);
            __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): what this wavefront requested half a step ago
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int db = 0; db < DB; ++db) O[db] = mfma32(v_frag(vb, kk, db), __builtin_bit_cast(bf16x8, P[kk]), O[db]);
            if (next.care) clear_odd(vbuf + b1);
            cur = next;
            next = after;
            after = later;
            const int free = b0;
            b0 = b1; b1 = b2; b2 = free;
            phase_barrier<-1, false>();
        }
        if (!second) phase_barrier<-1, false>();           // (as many for every wavefront)
        if (__builtin_amdgcn_readfirstlane(*odd_flag)) {
            // a weight times a value that is not finite is that value, whatever the weight
            Walk w = shard_at(__builtin_amdgcn_readfirstlane(s0));
            for (int t = k0; t < k1; ++t) {
                const Tile x = tile_at(t, w);
                if (!x.care) continue;
                limits(x.shard);
                const scalar_ints ids = (scalar_ints)p.table + (list0 + x.shard) * p.max_pages;
#pragma nounroll
                for (int key = 0; key < KEYS && x.j0 + key < x.end; ++key) {
                    const int j = x.j0 + key;
                    if (x.bad >> (key >> 4) & 1) continue;
                    const bf16_t *vr = (const bf16_t *)p.v_pages +
                        ((((int64_t)ids[j >> p.page_shift] * p.Hkv + g) << p.page_shift) + (j & ((1 << p.page_shift) - 1))) * D;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = (float)vr[32 * db + 8 * (i >> 2) + 4 * h + (i & 3)];
                            if (j < seen && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) O[db][i] += v;
                        }
                }
            }
        }
    }
    {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false));
        l = __uint_as_float(x.x) + __uint_as_float(x.y);
    }
    if (wk.n_pieces > 1) {
        // Through LDS, half of the columns at a time, so that a store writes whole lines (each wavefront its own rows: no barrier).
        // 512 rows over 2560 keys, 33 MB of partials: 41.5 us against 43.6 with stores from the accumulators.
        constexpr int COLS = D / 2, CHUNKS = COLS / 4, PER = 64 / CHUNKS;
        int tid_again = threadIdx.x;                       // (formed anew: the loop has no registers for more lane numbers)
        asm volatile("" : "+v"(tid_again));
        const int lane = tid_again & 63, l32 = lane & 31, h = lane >> 5;
        float *const mine = (float *)smem + wave * 32 * COLS;
        const int64_t at = ((int64_t)(wk.first_piece + wk.piece) * p.Hkv + g) * TILE + wave * 32;
        const int left = wk.n_rows - wk.tile * TILE - wave * 32;       // rows of this wavefront that exist
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int b = 0; b < DB / 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x16 &o = O[half * (DB / 2) + b];
                    *(f32x4 *)(mine + l32 * COLS + (((8 * b + 2 * i + h) ^ l32) & (CHUNKS - 1)) * 4) = f32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
                }
            wave_order();
#pragma unroll
            for (int i = 0; i < 32 / PER; ++i) {
                const int rr = i * PER + lane / CHUNKS, c = lane % CHUNKS;
                const f32x4 u = *(const f32x4 *)(mine + rr * COLS + ((c ^ rr) & (CHUNKS - 1)) * 4);
                if (rr < left) *(f32x4 *)(p.many.part_u + (at + rr) * D + half * COLS + c * 4) = u;
            }
            wave_order();
        }
        if (h == 0 && l32 < left) { p.many.part_ml[(at + l32) * 2] = m; p.many.part_ml[(at + l32) * 2 + 1] = l; }
        return;
    }
    if (row >= wk.n_rows) return;
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
    const int lds = 6 * KEYS * 2 * D + 4 * (3 * p.S + 3);
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)kern, 6 * KEYS * 2 * D + 4 * (3 * 1024 + 3), lds_ready));
    hipLaunchKernelGGL(kern, dim3((unsigned)(paged_grid(p, p.many, PAGED_TILE).pieces * p.Hkv)), dim3(64 * NW), lds, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

}   // namespace

int32_t launch_paged_tile(const PagedAttnParams &p, hipStream_t s) { return p.d == 64 ? launch_dim<64>(p, s) : launch_dim<128>(p, s); }
