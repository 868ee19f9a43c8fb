// Attention over a paged cache: parameters, and the division of the work among workgroups (host and device).
//
// Work: for every sequence b its new rows times the `rep` query heads of a kv head, flattened (row r is token r / rep, head
// r % rep of the group), in tiles of tile_rows; against every tile the keys of all shards, in steps of KEYS rows that begin
// anew with every shard.  How many rows and keys a sequence has is known on the device only, and lengths in a batch may
// differ by a factor of a thousand.  So a launch has as many workgroups as the work could need, and each one finds its piece
// from prefix sums over the sequences: the walks of a kernel's sequences (tiles times steps) are cut into about `target`
// pieces of equal length per kv head, none shorter than min_steps; a tile whose walk is cut leaves partials, which a second
// kernel merges.  64 sequences cost a wavefront one load each and two sums.
#pragma once
#include "device_utils.h"
#include "paged.h"

struct PagedAttnParams {
    const void *q, *k_pages, *v_pages;                     // the layer's pools
    void *o;
    float *lse;
    const int32_t *q_start, *visible, *table, *len;
    float *part_u, *part_ml;                               // [piece][kv head][tile_rows][d]; [piece][kv head][tile_rows][2]: m (log2 units), l
    int64_t q_stride, o_stride;
    int32_t rows, H, Hkv, rep, d, S, B, max_pages, page_shift, n_pages;
    float scale_log2;
    int32_t o_f32;
    int32_t above, upto;                                   // sequences of more than `above` and at most `upto` flattened rows
    int32_t min_steps, target;
    int32_t max_parts;                                     // partials that the workspace holds, per kv head
};

constexpr int PAGED_TARGET = 1024;                         // pieces of a launch, all kv heads together
constexpr int PAGED_TILE = 256, PAGED_TILE_TARGET = 256;   // paged_attn_tile.hip: rows of a tile; pieces
constexpr int PAGED_FEW = 32;                              // flattened rows of a sequence up to which it goes to paged_attn_rows.hip

struct PagedWork {
    int b, first_row, n_rows;                              // sequence, its first row in q, its flattened rows
    int tile, steps;                                       // steps: of the sequence's whole walk
    int piece, n_pieces, first_piece;                      // first_piece: number of this tile's first partial (n_pieces > 1)
    int k0, k1;                                            // steps of this piece
};

template <typename T> __device__ __forceinline__ T wave_inclusive(T v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T t = __shfl_up(v, o, WAVE);
        if ((int)(threadIdx.x & 63) >= o) v += t;
    }
    return v;
}

// Keys of a list that count
__device__ __forceinline__ int paged_len(const PagedAttnParams &p, int64_t list) {
    return min(max(p.len[list], 0), p.max_pages << p.page_shift);
}

// Piece number w of the launch (whole wavefronts call this, with the same w).  MERGE: tile number w among those with partials.
template <int TILE, int KEYS, bool MERGE>
__device__ __forceinline__ bool paged_find_work(const PagedAttnParams &p, int w, PagedWork &out) {
    const int lane = threadIdx.x & 63;
    int tiles = 0, steps = 0, lo = 0, n = 0;
    auto load = [&](int b) {
        tiles = steps = lo = n = 0;
        if (b >= p.B) return;
        lo = min(max(p.q_start[b], 0), p.rows);
        const int64_t flat = (int64_t)max(min(p.q_start[b + 1], p.rows) - lo, 0) * p.rep;
        if (flat <= p.above || flat > p.upto) return;
        n = (int)flat;
        tiles = (n + TILE - 1) / TILE;
        for (int s = 0; s < p.S; ++s) steps += (paged_len(p, (int64_t)b * p.S + s) + KEYS - 1) / KEYS;
    };
    unsigned long long total = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        load(b0 + lane);
        total += (unsigned long long)tiles * steps;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o, WAVE);
    const int per_piece = (int)max((unsigned long long)p.min_steps, (total + p.target - 1) / p.target);
    int before = 0, parts_before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (p.B > 64) load(b0 + lane);                     // (else they are those of the loop above)
        const int pieces = max(1, (int)(((int64_t)steps + per_piece - 1) / per_piece));
        const int parts = pieces > 1 ? tiles * pieces : 0;
        const int items = MERGE ? (pieces > 1 ? tiles : 0) : tiles * pieces;
        const int incl = wave_inclusive(items), parts_incl = wave_inclusive(parts);
        const uint64_t past = __ballot(before + incl > w);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            const int i = w - before - of(incl - items);
            out.n_pieces = of(pieces);
            // late tiles first: with a causal limit they are the long ones
            const int tile = MERGE ? i : i / out.n_pieces;
            out.b = b0 + at;
            out.first_row = of(lo);
            out.n_rows = of(n);
            out.steps = of(steps);
            out.piece = MERGE ? 0 : i - tile * out.n_pieces;
            out.first_piece = parts_before + of(parts_incl - parts) + tile * out.n_pieces;
            out.tile = of(tiles) - 1 - tile;
            out.k0 = (int)((int64_t)out.steps * out.piece / out.n_pieces);
            out.k1 = (int)((int64_t)out.steps * (out.piece + 1) / out.n_pieces);
            // (more partials than the launch has room for: only where sequences overlap, which they must not)
            return out.n_pieces == 1 || out.first_piece + out.n_pieces <= p.max_parts;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        parts_before += __builtin_amdgcn_readlane(parts_incl, 63);
    }
    return false;
}

// What a launch of tiles of `tile` rows may need: workgroups per kv head, and tiles with partials and partials among them
struct PagedGrid { int64_t pieces, split_tiles, parts; };
static inline PagedGrid paged_grid(const PagedAttnParams &p, int tile) {
    const int64_t tiles = (int64_t)p.rows * p.rep / tile + (p.B < p.rows ? p.B : p.rows);
    PagedGrid g;
    g.pieces = tiles + p.target;                           // sum of ceil(steps / per_piece) <= tiles + sum of steps / per_piece
    g.split_tiles = tiles < p.target ? tiles : p.target;   // a cut walk is longer than per_piece
    g.parts = g.pieces < 2 * p.target ? g.pieces : 2 * (int64_t)p.target;      // ceil(x) < 2 x above 1
    return g;
}

int32_t launch_paged_tile(PagedAttnParams p, float *workspace, hipStream_t s);

constexpr float LN2F = 0.6931471805599453f;

// Tiles whose walk was cut: their partials, weighted by exp2(m - largest m)
template <typename T, int TILE, int KEYS>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnParams p) {
    PagedWork wk;
    if (!paged_find_work<TILE, KEYS, true>(p, blockIdx.x, wk)) return;
    const int g = blockIdx.y, per_row = p.d / 4;
    const int64_t step = (int64_t)p.Hkv * TILE;
    for (int e = threadIdx.x + 256 * blockIdx.z; e < TILE * per_row; e += 256 * gridDim.z) {
        const int row = e / per_row, c = (e - row * per_row) * 4, r = wk.tile * TILE + row;
        if (r >= wk.n_rows) break;
        const int64_t at = ((int64_t)wk.first_piece * p.Hkv + g) * TILE + row;
        float top = -INFINITY;
        for (int i = 0; i < wk.n_pieces; ++i) top = fmaxf(top, p.part_ml[(at + i * step) * 2]);
        const float off = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < wk.n_pieces; ++i) {
            const float f = __builtin_amdgcn_exp2f(p.part_ml[(at + i * step) * 2] - off);
            sum += p.part_ml[(at + i * step) * 2 + 1] * f;
            u += *(const f32x4 *)(p.part_u + (at + i * step) * p.d + c) * f;
        }
        const int t = r / p.rep, h = g * p.rep + r - t * p.rep;
        const int64_t out = (int64_t)(wk.first_row + t) * p.o_stride + (int64_t)h * p.d + c;
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        u *= inv;
        if (sizeof(T) == 4 || p.o_f32) *(f32x4 *)((float *)p.o + out) = u;
        else *(bf16x4 *)((bf16_t *)p.o + out) = bf16x4{(bf16_t)u[0], (bf16_t)u[1], (bf16_t)u[2], (bf16_t)u[3]};
        if (c == 0 && p.lse) p.lse[(int64_t)h * p.rows + wk.first_row + t] = (top + __builtin_log2f(sum)) * LN2F;
    }
}

