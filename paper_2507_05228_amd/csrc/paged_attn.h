// Attention over a paged cache: parameters, and the division of the work among workgroups (host and device).
//
// Work: for every sequence b its new rows times the `rep` query heads of a kv head, flattened (row r is token r / rep, head
// r % rep of the group), in tiles of tile_rows; against every tile the keys of all shards, in steps of KEYS rows that begin
// anew with every shard.  How many rows and keys a sequence has is known on the device only, and lengths in a batch may
// differ by a factor of a thousand.  So a launch has as many workgroups as the work could need, and each one finds its piece
// from prefix sums over the sequences: the walks of a kernel's sequences (tiles times steps) are cut into about `target`
// pieces of equal length per kv head, none shorter than min_steps; a tile whose walk is cut leaves partials, which a second
// kernel merges.  64 sequences cost a wavefront one load each and two sums.
//
// Workgroup w of a launch has piece w / H_KV of kv head w % H_KV.  So those that find nothing to do start last (in front of others they
// held a CU for 2 us each), and with 8 kv heads, workgroups being dealt to the 8 dies in turn, a die's cache sees one head's keys: 4096
// rows over 16384 keys 908 -> 851 us against all pieces of one head after the other, 4096 rows of 64 heads over themselves 324 -> 287,
// one row of 64 sequences of 1024 54 -> 46, 32 of 1650 to 8200 130 -> 126.5, fp32 100, 37 and 1 rows 22 -> 19; 512 rows over 2560 42 -> 43.
#pragma once
#include "device_utils.h"
#include "paged.h"

// Lists and lengths do not change while a kernel runs: read through the scalar cache, beside the loads of keys and values
typedef const __attribute__((address_space(4))) int32_t *scalar_ints;

struct PagedSet {                                          // the sequences of one kernel
    int32_t above, upto;                                   // those of more than `above` and at most `upto` flattened rows
    int32_t min_steps, target;
    float inv_target;
    int32_t max_parts;                                     // partials that the workspace holds, per kv head
    float *part_u, *part_ml;                               // [piece][kv head][tile_rows][d]; [piece][kv head][tile_rows][2]: m (log2 units), l
};
struct PagedAttnParams {
    const void *q, *k_pages, *v_pages;                     // the layer's pools
    void *o;
    float *lse;
    const int32_t *q_start, *visible, *table, *len;
    int64_t q_stride, o_stride;
    int32_t rows, H, Hkv, rep, d, S, B, max_pages, page_shift, n_pages;
    float scale_log2;
    int32_t o_f32;
    PagedSet few, many;                                    // paged_attn_rows.hip, paged_attn_tile.hip
};

// paged_attn_tile.hip: rows of a tile, keys of a step, and pieces, a workgroup for every CU (128 / 256 / 512 pieces: 256 rows over 8448
// keys, 32 / 8 heads of 128, 70 / 61 / 77 us; 509 rows in 8 shards among short ones 117 / 99 / 111)
constexpr int PAGED_TILE = 256, PAGED_TILE_KEYS = 64, PAGED_TILE_TARGET = 256;
// Flattened rows of a sequence up to which it goes to paged_attn_rows.hip: up to one tile (64 / 256: 24 rows x 4 heads over 3024 keys 27 /
// 21 us, 64 x 4 over 4160 36 / 29; 256 / 512: 100 x 4 over 4196 37 / 43, four such over 3100 52 / 73)
constexpr int PAGED_FEW = 256;

struct PagedWork {
    int b, first_row, n_rows;                              // sequence, its first row in q, its flattened rows
    int tile, steps;                                       // steps: of the sequence's whole walk
    int piece, n_pieces, first_piece;                      // first_piece: number of this tile's first partial (n_pieces > 1)
    bool valid;
};

// Sum over the lanes up to this one.  Inside rows of 16 lanes by shifts, then the last lane of a row is handed to the rows
// behind it: data-parallel-primitive moves, no LDS traffic.
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_or_zero(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_inclusive(int v) {
    v += dpp_or_zero<0x111, 0xf>(v);                       // row_shr 1, 2, 4, 8
    v += dpp_or_zero<0x112, 0xf>(v);
    v += dpp_or_zero<0x114, 0xf>(v);
    v += dpp_or_zero<0x118, 0xf>(v);
    v += dpp_or_zero<0x142, 0xa>(v);                       // row_bcast 15 into rows 1 and 3
    return v + dpp_or_zero<0x143, 0xc>(v);                 // row_bcast 31 into rows 2 and 3
}

// Keys of a list that count
__device__ __forceinline__ int paged_len(const PagedAttnParams &p, int64_t list) {
    return min(max(p.len[list], 0), p.max_pages << p.page_shift);
}

// Part i of n nearly equal parts of [0, steps)
__device__ __forceinline__ void paged_cut(int steps, int i, int n, int &k0, int &k1) {
    const int each = n == 1 ? steps : (int)((uint32_t)steps / (uint32_t)n), more = n == 1 ? 0 : steps - each * n;
    k0 = i * each + min(i, more);
    k1 = k0 + each + (i < more);
}

// The division of a set's work, held by a wavefront: lane i has sequence b0 + i (of 64 at a time)
template <int TILE, int KEYS>
struct PagedPlan {
    int tiles, steps, lo, n;                               // of the lane's sequence
    int per_piece;

    __device__ __forceinline__ void load(const PagedAttnParams &p, const PagedSet &set, int b) {
        tiles = steps = lo = n = 0;
        if (b >= p.B) return;
        const int64_t list0 = (int64_t)b * p.S;
        lo = min(max(p.q_start[b], 0), p.rows);
        const int64_t flat = (int64_t)max(min(p.q_start[b + 1], p.rows) - lo, 0) * p.rep;
        for (int s0 = 0; s0 < p.S; s0 += 8) {              // eight loads in flight
            int n_s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) n_s[i] = paged_len(p, list0 + min(s0 + i, p.S - 1));
#pragma unroll
            for (int i = 0; i < 8; ++i) steps += s0 + i < p.S ? (n_s[i] + KEYS - 1) / KEYS : 0;
        }
        if (flat <= set.above || flat > set.upto) { steps = 0; return; }
        n = (int)flat;
        tiles = (n + TILE - 1) / TILE;
    }
    __device__ __forceinline__ void make(const PagedAttnParams &p, const PagedSet &set) {
        // (in fp32: every workgroup forms the same sum in the same order; the margin keeps the number of pieces inside its bound)
        float total = 0.f;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            load(p, set, b0 + (threadIdx.x & 63));
            total += (float)tiles * (float)steps;
        }
        total = wave_sum(total);
        per_piece = __builtin_amdgcn_readfirstlane(max(set.min_steps, (int)fminf(total * set.inv_target * 1.0001f + 1.f, 1e9f)));
    }
    // Piece number w; MERGE: tile number w among those with partials.  Whole wavefronts call this, with the same w.
    template <bool MERGE>
    __device__ __forceinline__ bool pick(const PagedAttnParams &p, const PagedSet &set, int w, PagedWork &out) {
        int before = 0, parts_before = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            if (p.B > 64) load(p, set, b0 + (threadIdx.x & 63));       // (else the lanes have them)
            const int pieces = steps <= per_piece ? 1 : (int)(((uint32_t)steps + (uint32_t)per_piece - 1) / (uint32_t)per_piece);
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
                const int tile = MERGE || out.n_pieces == 1 ? i : (int)((uint32_t)i / (uint32_t)out.n_pieces);
                out.b = b0 + at;
                out.first_row = of(lo);
                out.n_rows = of(n);
                out.steps = of(steps);
                out.piece = MERGE ? 0 : i - tile * out.n_pieces;
                out.first_piece = parts_before + of(parts_incl - parts) + tile * out.n_pieces;
                out.tile = of(tiles) - 1 - tile;
                // (more partials than the launch has room for: only where sequences overlap, which they must not)
                out.valid = out.n_pieces == 1 || out.first_piece + out.n_pieces <= set.max_parts;
                return true;
            }
            before += __builtin_amdgcn_readlane(incl, 63);
            parts_before += __builtin_amdgcn_readlane(parts_incl, 63);
        }
        return false;
    }
};

// What a set of tiles of `tile` rows may need: workgroups per kv head, and tiles with partials and partials among them
struct PagedGrid { int64_t pieces, split_tiles, parts; };
static inline PagedGrid paged_grid(const PagedAttnParams &p, const PagedSet &set, int tile) {
    const int64_t flat = (int64_t)p.rows * p.rep, seqs = flat / (set.above + 1);
    const int64_t n_seqs = p.B < seqs ? p.B : seqs, each = ((int64_t)set.upto + tile - 1) / tile;
    const int64_t tiles = flat / tile < n_seqs * (each - 1) ? flat / tile + n_seqs : n_seqs * each;
    PagedGrid g;
    g.pieces = tiles + set.target;                         // sum of ceil(steps / per_piece) <= tiles + sum of steps / per_piece
    g.split_tiles = tiles < set.target ? tiles : set.target;       // a cut walk is longer than per_piece
    g.parts = g.pieces < 2 * set.target ? g.pieces : 2 * (int64_t)set.target;     // ceil(x) < 2 x above 1
    return g;
}
int32_t launch_paged_tile(const PagedAttnParams &p, hipStream_t s);

constexpr float LN2F = 0.6931471805599453f;
