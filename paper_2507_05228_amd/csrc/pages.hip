// Pages of a paged cache: taking them for new rows, sharing, freeing, compacting and copying them.
//
// The state is plain arrays (lists, lengths, references) and a page is free if nothing refers to it: there is no list of free
// pages whose order could depend on timing.  Whoever needs pages gets the lowest free ones, list by list, so that the same
// calls give the same lists every time.  The index work is one workgroup with prefix sums, bound by latency: a scan of the
// references (32 KB for 8192 pages) and some ten barriers, 9 us for 8 sequences, 11 for 32 lists; forks of 16 sequences 8 us.  Not all
// of that must be: the eight references of a thread, and the lengths, the starts and the references, are waited for one after the
// other, and a pool of 100000 pages has thirteen such rounds (64 sequences, a row each: 45 us against 7 with 5000 pages).
// The rows' slots and limits go to as many wavefronts as there are 64 rows (4096 rows in 16 shards: 8 us, most of them for the
// shards' lengths, one load after the other; in the one workgroup, whose scattered stores held it up, 47); each of them counts
// the rows behind its own to the end of the sequence, which is quadratic in a sequence's rows.  Copies of pages are spread over the chip and bound by HBM: 0.27 GB read and written in
// 39 us, 6.9 TB/s (part of it stays in the last-level cache).
#include "device_utils.h"
#include "paged.h"

namespace {

constexpr int WG = 1024, WAVES = WG / 64;
constexpr int MAX_LISTS = 8192;                            // lists of one fork; of one round of an extension
constexpr int REFS_PER_THREAD = 8;

struct Lists {
    int32_t *table, *len, *refs;
    int32_t n_seqs, n_shards, max_pages, n_pages, page_shift;
};
Lists lists_of(const cascade_paged_cache *c) {
    return {c->page_table, c->kv_len, c->page_refs, c->n_seqs, c->n_shards, c->max_pages, c->n_pages, page_shift(c)};
}

__device__ __forceinline__ int32_t wave_scan(int32_t v) {  // inclusive
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t t = __shfl_up(v, o, WAVE);
        if ((int)(threadIdx.x & 63) >= o) v += t;
    }
    return v;
}
// Sum over the threads before this one, and over all; scratch holds 2 * WAVES words (the halves are used in turn, so one
// barrier a call is enough: `flip` alternates)
__device__ __forceinline__ int32_t block_scan(int32_t v, int32_t *scratch, int &flip, int32_t &total) {
    int32_t *part = scratch + flip * WAVES;
    flip ^= 1;
    const int32_t incl = wave_scan(v);
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = incl;
    __syncthreads();
    int32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += part[w];
        total += part[w];
    }
    return before + incl - v;
}

__device__ __forceinline__ int32_t list_len(const Lists &l, int64_t list) {
    return min(max(l.len[list], 0), l.max_pages << l.page_shift);
}
__device__ __forceinline__ int32_t pages_of(const Lists &l, int32_t rows) { return (rows + (1 << l.page_shift) - 1) >> l.page_shift; }

__device__ __forceinline__ int32_t block_max(int32_t v, int32_t *scratch, int &flip) {     // of values from 0 on
    int32_t *part = scratch + flip * WAVES, top = 0;
    flip ^= 1;
#pragma unroll
    for (int o = 32; o; o >>= 1) v = max(v, __shfl_xor(v, o, WAVE));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = max(top, part[w]);
    return top;
}
// The slot of a row of a list; -1 where the list has no page for it
__device__ __forceinline__ int32_t slot_of(const Lists &l, int64_t list, int32_t row) {
    if ((uint32_t)row >= (uint32_t)(l.max_pages << l.page_shift)) return -1;
    const int32_t page = l.table[list * l.max_pages + (row >> l.page_shift)];
    return (uint32_t)page < (uint32_t)l.n_pages ? (page << l.page_shift) + (row & ((1 << l.page_shift) - 1)) : -1;
}

// Bit i: page p0 + i is free
__device__ __forceinline__ uint32_t free_mask(const Lists &l, int64_t p0) {
    uint32_t free = 0;
#pragma unroll
    for (int i = 0; i < REFS_PER_THREAD; ++i)
        if (p0 + i < l.n_pages && l.refs[p0 + i] == 0) free |= 1u << i;
    return free;
}
// `head`: the mask of this thread's first pages, which take_free can have again (few pools have more than WG * REFS_PER_THREAD)
__device__ int32_t count_free(const Lists &l, uint32_t &head, int32_t *scratch, int &flip) {
    head = free_mask(l, (int64_t)threadIdx.x * REFS_PER_THREAD);
    int32_t mine = __popc(head), total;
    for (int64_t base = WG * REFS_PER_THREAD; base < l.n_pages; base += WG * REFS_PER_THREAD)
        mine += __popc(free_mask(l, base + (int64_t)threadIdx.x * REFS_PER_THREAD));
    block_scan(mine, scratch, flip, total);
    return total;
}

// take(page, rank) for the `wanted` lowest free pages (at least so many are free), whose references become 1.
// again: head is the mask of this thread's first pages as they are
template <typename F>
__device__ void take_free(const Lists &l, int32_t wanted, bool again, uint32_t head, int32_t *scratch, int &flip, F take) {
    int32_t rank0 = 0;
    for (int64_t base = 0; base < l.n_pages && rank0 < wanted; base += WG * REFS_PER_THREAD) {
        const int64_t p0 = base + (int64_t)threadIdx.x * REFS_PER_THREAD;
        const uint32_t free = base == 0 && again ? head : free_mask(l, p0);
        int32_t total, rank = rank0 + block_scan(__popc(free), scratch, flip, total);
#pragma unroll
        for (int i = 0; i < REFS_PER_THREAD; ++i) {
            if (!(free >> i & 1)) continue;
            if (rank < wanted) { l.refs[p0 + i] = 1; take((int32_t)(p0 + i), rank); }
            ++rank;
        }
        rank0 += total;
    }
}

// Index of the last of the n ascending values that is <= x (first[0] <= x)
__device__ __forceinline__ int32_t last_at_most(const int32_t *first, int32_t n, int32_t x) {
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Exclusive prefix sums of value(list) over n lists, into first[0 .. n) and total; value is called once per list
template <typename F>
__device__ int32_t scan_lists(int32_t n, int32_t *first, int32_t *scratch, int &flip, F value) {
    int32_t carry = 0, total;
    for (int32_t base = 0; base < n; base += WG) {
        const int32_t i = base + threadIdx.x, v = i < n ? value(i) : 0;
        const int32_t before = block_scan(v, scratch, flip, total);
        if (i < n) first[i] = carry + before;
        carry += total;
    }
    __syncthreads();
    return carry;
}

// ---------------------------------------------------------------------------- new rows
struct ExtendParams {
    Lists l;
    const int32_t *q_start, *row_shard;
    int32_t *slots, *visible, *accepted;
    int32_t rows, seqs_per_round;
    int32_t rows_here;                                     // the rows' slots and limits in this launch (one shard only)
};
__device__ __forceinline__ int32_t start_of(const ExtendParams &p, int b) { return min(max(p.q_start[b], 0), p.rows); }

// Pages, lists and lengths, by one workgroup; sequences in rounds of as many as LDS has words for.
__global__ __launch_bounds__(WG) void paged_extend_kernel(ExtendParams p) {
    extern __shared__ int32_t smem[];
    const Lists &l = p.l;
    const int S = l.n_shards, tid = threadIdx.x;
    const int round_lists = p.seqs_per_round * S;
    int32_t *count = smem, *first = count + round_lists;   // new rows of a list; rank of its first new page
    int32_t *len = first + round_lists, *ok = len + round_lists;   // its rows so far; per sequence
    int32_t *start = ok + p.seqs_per_round;                // first row of every sequence, and of the one behind
    __shared__ int32_t scratch[2 * WAVES];
    int flip = 0;
    uint32_t head;
    int32_t n_free = 0;
    bool exhausted = false;                                // (the same in every thread)
    for (int b0 = 0; b0 < l.n_seqs; b0 += p.seqs_per_round) {
        const int n_b = min(p.seqs_per_round, l.n_seqs - b0), n_l = n_b * S;
        const int64_t list0 = (int64_t)b0 * S;
        if (b0) __syncthreads();                           // the round before is done with the lists' words
        for (int i = tid; i < n_l; i += WG) { count[i] = 0; len[i] = list_len(l, list0 + i); }
        for (int i = tid; i <= n_b; i += WG) {
            start[i] = start_of(p, b0 + i);
            if (i < n_b) ok[i] = 1;
        }
        if (b0 == 0) n_free = count_free(l, head, scratch, flip);      // (a barrier for the words above too)
        else __syncthreads();
        const int t0 = start[0], t1 = max(start[n_b], t0);
        if (!p.row_shard) {                                // one shard
            for (int i = tid; i < n_b; i += WG) count[i] = max(start[i + 1] - start[i], 0);
        } else {
            for (int t = t0 + tid; t < t1; t += WG) {
                const uint32_t s = p.row_shard[t];
                if (s < (uint32_t)S) atomicAdd(&count[last_at_most(start, n_b, t) * S + s], 1);
            }
        }
        __syncthreads();
        auto need = [&](int i) {                           // pages; -1: more rows than a list has
            const int64_t n = (int64_t)len[i] + count[i];
            if (n > (int64_t)l.max_pages << l.page_shift) return -1;
            return pages_of(l, (int32_t)n) - pages_of(l, len[i]);
        };
        for (int i = tid; i < n_l; i += WG)
            if (need(i) < 0) ok[i / S] = 0;
        __syncthreads();
        const int32_t needed = scan_lists(n_l, first, scratch, flip, [&](int i) { return ok[i / S] ? need(i) : 0; });
        // A sequence is taken if all pages up to its own are there, or if it needs none.  Those that are taken and need some come
        // before all that find none, so that `first` needs no second pass.
        int32_t most = 0;
        for (int b = tid; b < n_b; b += WG) {
            const int32_t lo = first[b * S], hi = b + 1 < n_b ? first[(b + 1) * S] : needed;
            if (hi > lo) {
                if (exhausted || hi > n_free) ok[b] = 0;
                else most = hi;
            }
            p.accepted[b0 + b] = ok[b];
        }
        const int32_t granted = block_max(most, scratch, flip);    // the pages of all that are taken (`most` ascends with b)
        take_free(l, granted, b0 == 0, head, scratch, flip, [&](int32_t page, int32_t rank) {
            const int i = last_at_most(first, n_l, rank);
            l.table[(list0 + i) * l.max_pages + pages_of(l, len[i]) + rank - first[i]] = page;
        });
        n_free -= granted;
        exhausted |= needed > granted;
        for (int i = tid; i < n_l; i += WG)
            if (ok[i / S] && count[i]) l.len[list0 + i] = len[i] + count[i];
        if (p.rows_here) {
            __syncthreads();                               // the pages are in the lists
            for (int t = t0 + tid; t < t1; t += WG) {
                const int b = last_at_most(start, n_b, t), i = t - start[b], row = len[b] + i;
                const bool taken = ok[b] && (uint32_t)i < (uint32_t)count[b];
                p.slots[t] = taken ? slot_of(l, list0 + b, row) : -1;
                p.visible[t] = taken ? row + 1 : 0;
            }
        }
    }
    if (!p.rows_here) return;
    const int lo = start_of(p, 0), hi = max(start_of(p, l.n_seqs), lo);
    for (int t = tid; t < p.rows; t += WG)
        if (t < lo || t >= hi) { p.slots[t] = -1; p.visible[t] = 0; }       // rows of no sequence
}

// Slots and limits of 64 rows a wavefront, from the new lengths backwards: a row of shard s sees all rows of the shard but
// those behind it.  Behind it are those of the same sequence in the wavefront (population counts of ballots) and those beyond,
// which the wavefront counts into LDS for the sequence that its last row belongs to.
__global__ __launch_bounds__(256) void paged_rows_slots_kernel(ExtendParams p) {
    extern __shared__ int32_t smem[];                      // [4][S]
    const Lists &l = p.l;
    const int S = l.n_shards, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = (blockIdx.x * 4 + wave) * 64, t = t0 + lane;
    int32_t *beyond = smem + wave * S;
    for (int s = lane; s < S; s += 64) beyond[s] = 0;
    // the sequence of a row: the last that begins at or before it
    auto seq_of = [&](int row) {
        int lo = 0, hi = l.n_seqs;
        while (hi - lo > 1) {
            const int mid = lo + ((hi - lo) >> 1);
            if (p.q_start[mid] <= row) lo = mid; else hi = mid;
        }
        return lo;
    };
    const int b = seq_of(min(t, p.rows - 1)), begin = start_of(p, b), end = max(start_of(p, b + 1), begin);
    const bool inside = t < p.rows && t >= begin && t < end, taken = inside && p.accepted[b];
    const int shard = !inside ? -1 : p.row_shard ? p.row_shard[t] : 0;
    const int open = __shfl(b, 63, WAVE), open_end = __shfl(end, 63, WAVE);
    __builtin_amdgcn_wave_barrier();
    if (p.row_shard)
        for (int r0 = t0 + 64 + lane; r0 < open_end; r0 += 512) {      // eight loads in flight
            uint32_t s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = r0 + 64 * j < open_end ? p.row_shard[r0 + 64 * j] : ~0u;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (s[j] < (uint32_t)S) atomicAdd(&beyond[s[j]], 1);
        }
    else if (lane == 0) beyond[0] = max(open_end - t0 - 64, 0);
    __syncthreads();
    // rows behind this one in its sequence, within the wavefront
    const int last = min(end - t0, 64);                    // (lanes from here on belong to others)
    const uint64_t mine = last >= 64 ? ~0ull : (1ull << max(last, 0)) - 1;
    const uint64_t behind = lane == 63 ? 0 : mine & (~0ull << (lane + 1));
    int own_end = 0;
    for (int s0 = 0; s0 < S; s0 += 4) {
        int v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int s = s0 + j, n = __popcll(__ballot(shard == s) & behind) + (b == open && s < S ? beyond[s] : 0);
            v[j] = taken && s < S ? l.len[(int64_t)b * S + s] - n : 0;
            if (s == shard) own_end = v[j];
        }
        if (t >= p.rows) continue;
        int32_t *out = p.visible + (int64_t)t * S + s0;
        if (S % 4 == 0 && (uintptr_t)p.visible % 16 == 0) *(int4 *)out = make_int4(v[0], v[1], v[2], v[3]);
        else
            for (int j = 0; j < 4 && s0 + j < S; ++j) out[j] = v[j];
    }
    if (t < p.rows) p.slots[t] = taken && (uint32_t)shard < (uint32_t)S ? slot_of(l, (int64_t)b * S + shard, own_end - 1) : -1;
}

// ---------------------------------------------------------------------------- freed sequences
__global__ __launch_bounds__(256) void pages_free_kernel(Lists l, const int32_t *seqs, int32_t per_seq) {
    const int b = seqs[blockIdx.y];
    if ((uint32_t)b >= (uint32_t)l.n_seqs) return;
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e < l.n_shards) l.len[(int64_t)b * l.n_shards + e] = 0;
    if (e >= per_seq) return;
    // whoever takes the entry gives the reference back: a sequence named twice is freed once
    const int32_t page = atomicExch(&l.table[(int64_t)b * per_seq + e], -1);
    if ((uint32_t)page < (uint32_t)l.n_pages) atomicSub(&l.refs[page], 1);
}

// ---------------------------------------------------------------------------- forks
struct ForkParams {
    Lists l;
    const int32_t *src, *dst;
    int32_t *accepted;
    int32_t *list_len, *list_page;                         // workspace [n * S]: rows of the list; its new page, -1: none
    int32_t n;
    char *k_pages, *v_pages;
    int64_t layer_bytes;                                   // of a pool
    int32_t n_layers, Hkv, row_bytes;
};

__global__ __launch_bounds__(WG) void pages_fork_kernel(ForkParams p) {
    extern __shared__ int32_t smem[];
    const Lists &l = p.l;
    const int S = l.n_shards, n_l = p.n * S, tid = threadIdx.x;
    int32_t *first = smem, *ok = first + n_l, *rows = ok + p.n;     // per list, per pair, per list
    __shared__ int32_t scratch[2 * WAVES];
    int flip = 0;
    for (int i = tid; i < p.n; i += WG) rows[i] = p.dst[i];
    uint32_t head;
    const int32_t n_free = count_free(l, head, scratch, flip);     // (a barrier for the words above too)
    for (int i = tid; i < p.n; i += WG) {
        const int src = p.src[i], dst = rows[i];
        bool good = (uint32_t)src < (uint32_t)l.n_seqs && (uint32_t)dst < (uint32_t)l.n_seqs && src != dst;
        for (int s = 0; good && s < S; ++s) good = l.len[(int64_t)dst * S + s] <= 0;
        for (int j = 0; j < i; ++j) good &= rows[j] != dst;
        ok[i] = good;
    }
    __syncthreads();
    for (int i = tid; i < n_l; i += WG) rows[i] = ok[i / S] ? list_len(l, (int64_t)p.src[i / S] * S + i % S) : 0;
    const int32_t mask = (1 << l.page_shift) - 1;
    __syncthreads();
    const int32_t needed = scan_lists(n_l, first, scratch, flip, [&](int i) { return (int32_t)((rows[i] & mask) != 0); });
    // as in an extension: those that are taken and need pages come first
    int32_t most = 0;
    for (int i = tid; i < p.n; i += WG) {
        const int32_t lo = first[i * S], hi = i + 1 < p.n ? first[(i + 1) * S] : needed;
        if (hi > lo) {
            if (hi > n_free) ok[i] = 0;
            else most = hi;
        }
        p.accepted[i] = ok[i];
    }
    const int32_t granted = block_max(most, scratch, flip);
    for (int i = tid; i < n_l; i += WG) {
        p.list_len[i] = ok[i / S] ? rows[i] : 0;
        p.list_page[i] = -1;
    }
    __syncthreads();
    take_free(l, granted, true, head, scratch, flip, [&](int32_t page, int32_t rank) { p.list_page[last_at_most(first, n_l, rank)] = page; });
}

// Grid (lists, 2 * layers, kv heads): the used rows of a list's last page, which are contiguous per head.  The first
// workgroup of a list writes its entries too.
__global__ __launch_bounds__(256) void pages_fork_copy_kernel(ForkParams p) {
    const Lists &l = p.l;
    const int i = blockIdx.x, S = l.n_shards;
    const int32_t n = p.list_len[i];
    if (n == 0) return;
    const int pair = i / S, s = i - pair * S;
    const int64_t from = ((int64_t)p.src[pair] * S + s) * l.max_pages, to = ((int64_t)p.dst[pair] * S + s) * l.max_pages;
    const int full = n >> l.page_shift, part = n & ((1 << l.page_shift) - 1), page = p.list_page[i];
    if (blockIdx.y == 0 && blockIdx.z == 0) {
        for (int j = threadIdx.x; j < full; j += 256) {
            const int32_t id = l.table[from + j];
            l.table[to + j] = id;
            if ((uint32_t)id < (uint32_t)l.n_pages) atomicAdd(&l.refs[id], 1);
        }
        if (threadIdx.x == 0) {
            if (part) l.table[to + full] = page;
            l.len[(int64_t)p.dst[pair] * S + s] = n;
        }
    }
    if (!part) return;
    const int32_t old = l.table[from + full];
    if ((uint32_t)old >= (uint32_t)l.n_pages) return;
    char *pool = (blockIdx.y & 1 ? p.v_pages : p.k_pages) + (int64_t)(blockIdx.y >> 1) * p.layer_bytes;
    const int64_t head_bytes = (int64_t)p.row_bytes << l.page_shift;
    const u32x4 *a = (const u32x4 *)(pool + ((int64_t)old * p.Hkv + blockIdx.z) * head_bytes);
    u32x4 *b = (u32x4 *)(pool + ((int64_t)page * p.Hkv + blockIdx.z) * head_bytes);
    const int64_t vecs = (int64_t)part * p.row_bytes / 16;
    for (int64_t x = threadIdx.x; x < vecs; x += 256) b[x] = a[x];
}

// ---------------------------------------------------------------------------- whole pages
struct MoveParams {
    Lists l;
    const int32_t *src, *dst;
    const int32_t *n_dev; int32_t n;                       // number of pairs: on the device (not null) or n
    const int32_t *map, *first_moved;                      // compaction: new id of the pages from *first_moved on (else null)
    char *k_pages, *v_pages;
    int64_t layer_bytes;
    int32_t n_layers;
    int32_t page_vecs;                                     // 16-byte pieces of a page in one pool
};
constexpr int UNIT = 1024;                                 // 16-byte pieces that a workgroup copies at a time

// One workgroup at a time: which pages move where.  live[] of the pages behind the front, ascending, to the free ones in it.
__global__ __launch_bounds__(WG) void pages_compact_kernel(Lists l, int32_t *n_live_out, int32_t *src, int32_t *dst, int32_t *map,
                                                           int32_t *count) {
    __shared__ int32_t scratch[2 * WAVES];
    int flip = 0;
    uint32_t head;
    const int32_t n_live = l.n_pages - count_free(l, head, scratch, flip);
    int32_t moved = 0, holes = 0;
    for (int64_t base = 0; base < l.n_pages; base += WG * REFS_PER_THREAD) {
        const int64_t p0 = base + (int64_t)threadIdx.x * REFS_PER_THREAD;
        const uint32_t free = base ? free_mask(l, p0) : head;
        uint32_t hole = 0, mover = 0;
#pragma unroll
        for (int i = 0; i < REFS_PER_THREAD; ++i) {
            if (p0 + i >= l.n_pages) continue;
            if ((free >> i & 1) && p0 + i < n_live) hole |= 1u << i;
            if (!(free >> i & 1) && p0 + i >= n_live) mover |= 1u << i;
        }
        int32_t n_holes, n_moved;
        int32_t h = holes + block_scan(__popc(hole), scratch, flip, n_holes), m = moved + block_scan(__popc(mover), scratch, flip, n_moved);
#pragma unroll
        for (int i = 0; i < REFS_PER_THREAD; ++i) {
            if (hole >> i & 1) dst[h++] = (int32_t)(p0 + i);
            if (mover >> i & 1) src[m++] = (int32_t)(p0 + i);
            else if (p0 + i >= n_live && p0 + i < l.n_pages) map[p0 + i] = (int32_t)(p0 + i);
        }
        holes += n_holes;
        moved += n_moved;
    }
    __syncthreads();                                       // as many holes as movers: n_live pages in all
    for (int i = threadIdx.x; i < moved; i += WG) {
        map[src[i]] = dst[i];
        l.refs[dst[i]] = l.refs[src[i]];
        l.refs[src[i]] = 0;
    }
    if (threadIdx.x == 0) {
        count[0] = moved;
        count[1] = n_live;
        if (n_live_out) *n_live_out = n_live;
    }
}

__global__ __launch_bounds__(256) void pages_move_kernel(MoveParams p) {
    const Lists &l = p.l;
    const int32_t n = p.n_dev ? *p.n_dev : p.n;
    const int32_t units = (p.page_vecs + UNIT - 1) / UNIT, pools = 2 * p.n_layers;
    const int64_t total = (int64_t)n * pools * units;
    for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
        const int32_t u = (int32_t)(w % units);
        const int64_t rest = w / units;
        const int32_t pool_id = (int32_t)(rest % pools);
        const int64_t i = rest / pools;
        const int32_t a = p.src[i], b = p.dst[i];
        if ((uint32_t)a >= (uint32_t)l.n_pages || (uint32_t)b >= (uint32_t)l.n_pages || a == b) continue;
        char *pool = (pool_id & 1 ? p.v_pages : p.k_pages) + (int64_t)(pool_id >> 1) * p.layer_bytes;
        const u32x4 *from = (const u32x4 *)pool + (int64_t)a * p.page_vecs;
        u32x4 *to = (u32x4 *)pool + (int64_t)b * p.page_vecs;
        u32x4 v[UNIT / 256];
#pragma unroll
        for (int j = 0; j < UNIT / 256; ++j) {
            const int32_t x = u * UNIT + j * 256 + threadIdx.x;
            if (x < p.page_vecs) v[j] = from[x];
        }
#pragma unroll
        for (int j = 0; j < UNIT / 256; ++j) {
            const int32_t x = u * UNIT + j * 256 + threadIdx.x;
            if (x < p.page_vecs) to[x] = v[j];
        }
    }
    if (!p.map) return;
    const int32_t first = *p.first_moved;
    const int64_t entries = (int64_t)l.n_seqs * l.n_shards * l.max_pages;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) {
        const int32_t page = l.table[e];
        if (page >= first && page < l.n_pages) l.table[e] = p.map[page];
    }
}

MoveParams move_params(const cascade_paged_cache *c) {
    const int es = c->dtype == CASCADE_BF16 ? 2 : 4;
    MoveParams p = {};
    p.l = lists_of(c);
    p.k_pages = (char *)c->k_pages; p.v_pages = (char *)c->v_pages;
    p.layer_bytes = layer_elems(c) * es;
    p.n_layers = c->n_layers;
    p.page_vecs = (int32_t)((int64_t)c->n_kv_heads * c->page_size * c->head_dim * es / 16);
    return p;
}
int32_t launch_move(const MoveParams &p, int64_t most, hipStream_t s) {
    const int64_t units = most * 2 * p.n_layers * ((p.page_vecs + UNIT - 1) / UNIT);
    hipLaunchKernelGGL(pages_move_kernel, dim3((unsigned)(units < 4096 ? (units < 1 ? 1 : units) : 4096)), dim3(256), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}
// A page of one pool in 16-byte pieces counts in 32 bits
bool page_fits(const cascade_paged_cache *c) {
    return (int64_t)c->n_kv_heads * c->page_size * c->head_dim * 4 <= INT32_MAX;
}

}   // namespace

extern "C" int32_t cascade_paged_extend(const cascade_paged_cache *cache, int32_t rows, const int32_t *q_start_dev,
                                        const int32_t *row_shard_dev, int32_t *slots, int32_t *visible, int32_t *accepted,
                                        void *stream) {
    const int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (rows <= 0 || !q_start_dev || !slots || !visible || !accepted || (cache->n_shards > 1 && !row_shard_dev)) return CASCADE_EINVAL;
    if (rows > INT32_MAX - 1024) return CASCADE_EUNSUPPORTED;      // (rows are walked over 1024 at a time, counted in 32 bits)
    ExtendParams p = {};
    p.l = lists_of(cache);
    p.q_start = q_start_dev; p.row_shard = row_shard_dev; p.slots = slots; p.visible = visible; p.accepted = accepted;
    p.rows = rows;
    const int S = cache->n_shards;
    p.seqs_per_round = min(cache->n_seqs, max(1, 4096 / S));
    // one launch for a few rows of one shard, else the rows' part by as many wavefronts as it has 64 rows
    p.rows_here = !row_shard_dev && rows <= 2 * WG;
    const int bytes = 4 * (p.seqs_per_round * (3 * S + 2) + 1);
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)paged_extend_kernel, 4 * (4096 * 5 + 1), lds_ready));
    hipLaunchKernelGGL(paged_extend_kernel, dim3(1), dim3(WG), bytes, (hipStream_t)stream, p);
    if (!p.rows_here) hipLaunchKernelGGL(paged_rows_slots_kernel, dim3((rows + 255) / 256), dim3(256), 16 * S, (hipStream_t)stream, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

extern "C" int32_t cascade_pages_free(const cascade_paged_cache *cache, int32_t n, const int32_t *seqs_dev, void *stream) {
    const int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (n <= 0 || !seqs_dev) return CASCADE_EINVAL;
    if (n > 65535) return CASCADE_EUNSUPPORTED;
    const int32_t per_seq = cache->n_shards * cache->max_pages;
    hipLaunchKernelGGL(pages_free_kernel, dim3((per_seq + 255) / 256, n), dim3(256), 0, (hipStream_t)stream, lists_of(cache), seqs_dev, per_seq);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

// Compaction: pairs (as many as half the pages, each), the map of new ids, their number and the number of pages in use; a
// fork: rows and new page of every list.
extern "C" size_t cascade_pages_workspace_bytes(const cascade_paged_cache *cache) {
    if (check_paged_cache(cache) != CASCADE_OK) return 0;
    const size_t compact = 2 + 2 * ((size_t)cache->n_pages / 2 + 1) + cache->n_pages, fork = 2 * MAX_LISTS;
    return align_up(4 * (compact > fork ? compact : fork), 256);
}

extern "C" int32_t cascade_pages_fork(const cascade_paged_cache *cache, int32_t n, const int32_t *src_dev, const int32_t *dst_dev,
                                      int32_t *accepted, void *workspace, size_t workspace_bytes, void *stream) {
    const int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (n <= 0 || !src_dev || !dst_dev || !accepted) return CASCADE_EINVAL;
    if ((int64_t)n * cache->n_shards > MAX_LISTS || 2 * (int64_t)cache->n_layers > 65535 || !page_fits(cache)) return CASCADE_EUNSUPPORTED;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < cascade_pages_workspace_bytes(cache)) return CASCADE_EWORKSPACE;
    const int es = cache->dtype == CASCADE_BF16 ? 2 : 4, n_l = n * cache->n_shards;
    ForkParams p = {};
    p.l = lists_of(cache);
    p.src = src_dev; p.dst = dst_dev; p.accepted = accepted; p.n = n;
    p.list_len = (int32_t *)workspace; p.list_page = p.list_len + n_l;
    p.k_pages = (char *)cache->k_pages; p.v_pages = (char *)cache->v_pages;
    p.layer_bytes = layer_elems(cache) * es;
    p.n_layers = cache->n_layers; p.Hkv = cache->n_kv_heads; p.row_bytes = cache->head_dim * es;
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)pages_fork_kernel, 4 * 3 * MAX_LISTS, lds_ready));
    hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(WG), 4 * (2 * n_l + n), (hipStream_t)stream, p);
    hipLaunchKernelGGL(pages_fork_copy_kernel, dim3(n_l, 2 * p.n_layers, p.Hkv), dim3(256), 0, (hipStream_t)stream, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

extern "C" int32_t cascade_pages_compact(const cascade_paged_cache *cache, int32_t *n_live, void *workspace, size_t workspace_bytes,
                                         void *stream) {
    const int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (!page_fits(cache)) return CASCADE_EUNSUPPORTED;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < cascade_pages_workspace_bytes(cache)) return CASCADE_EWORKSPACE;
    int32_t *count = (int32_t *)workspace, *src = count + 2, *dst = src + cache->n_pages / 2 + 1, *map = dst + cache->n_pages / 2 + 1;
    MoveParams p = move_params(cache);
    p.src = src; p.dst = dst; p.n_dev = count; p.first_moved = count + 1; p.map = map;
    hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(WG), 0, (hipStream_t)stream, p.l, n_live, src, dst, map, count);
    return launch_move(p, cache->n_pages / 2 + 1, (hipStream_t)stream);
}

extern "C" int32_t cascade_pages_copy(const cascade_paged_cache *cache, int32_t n, const int32_t *src_dev, const int32_t *dst_dev,
                                      void *stream) {
    const int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (n <= 0 || !src_dev || !dst_dev) return CASCADE_EINVAL;
    if (!page_fits(cache)) return CASCADE_EUNSUPPORTED;
    MoveParams p = move_params(cache);
    p.src = src_dev; p.dst = dst_dev; p.n = n;
    return launch_move(p, n, (hipStream_t)stream);
}
