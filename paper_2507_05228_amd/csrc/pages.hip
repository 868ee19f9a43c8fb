// Pages of a paged cache: taking them for new rows, sharing, freeing, compacting and copying them.
//
// The state is plain arrays (lists, lengths, references) and a page is free if nothing refers to it: there is no list of free
// pages whose order could depend on timing.  Whoever needs pages gets the lowest free ones, list by list, so that the same
// calls give the same lists every time.  The index work is one workgroup with prefix sums (it is bound by latency: a scan
// of the references, 32 KB for 8192 pages, and a few barriers); copies of pages are spread over the chip and bound by HBM.
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

__device__ int32_t count_free(const Lists &l, int32_t *scratch, int &flip) {
    int32_t mine = 0, total;
    for (int p = threadIdx.x; p < l.n_pages; p += WG) mine += l.refs[p] == 0;
    block_scan(mine, scratch, flip, total);
    return total;
}

// take(page, rank) for the `wanted` lowest free pages (at least so many are free), whose references become 1
template <typename F>
__device__ void take_free(const Lists &l, int32_t wanted, int32_t *scratch, int &flip, F take) {
    int32_t rank0 = 0;
    for (int64_t base = 0; base < l.n_pages && rank0 < wanted; base += WG * REFS_PER_THREAD) {
        const int64_t p0 = base + (int64_t)threadIdx.x * REFS_PER_THREAD;
        uint32_t free = 0;
#pragma unroll
        for (int i = 0; i < REFS_PER_THREAD; ++i)
            if (p0 + i < l.n_pages && l.refs[p0 + i] == 0) free |= 1u << i;
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
};

__global__ __launch_bounds__(WG) void paged_extend_kernel(ExtendParams p) {
    extern __shared__ int32_t smem[];
    const Lists &l = p.l;
    const int S = l.n_shards, tid = threadIdx.x;
    const int round_lists = p.seqs_per_round * S;
    int32_t *count = smem, *first = count + round_lists;   // new rows of a list; rank of its first new page
    int32_t *before = first + round_lists;                 // rows of the list's shard in the round before its sequence
    int32_t *ok = before + round_lists;                    // per sequence
    int32_t *part = ok + p.seqs_per_round;                 // [WAVES][S] rows of each shard in a wavefront's 64
    __shared__ int32_t scratch[2 * WAVES];
    int flip = 0;
    auto start_of = [&](int b) { return min(max(p.q_start[b], 0), p.rows); };

    int32_t n_free = count_free(l, scratch, flip);
    bool exhausted = false;                                // (the same in every thread)
    for (int b0 = 0; b0 < l.n_seqs; b0 += p.seqs_per_round) {
        const int n_b = min(p.seqs_per_round, l.n_seqs - b0), n_l = n_b * S;
        const int t0 = start_of(b0), t1 = max(start_of(b0 + n_b), t0);
        // the round's sequence of a row (t0 <= t < t1)
        auto seq_of = [&](int t) {
            int lo = 0, hi = n_b;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.q_start[b0 + mid] <= t) lo = mid; else hi = mid;
            }
            return lo;
        };
        __syncthreads();                                   // the round before is done with the lists' words
        for (int i = tid; i < n_l; i += WG) count[i] = 0;
        for (int i = tid; i < n_b; i += WG) ok[i] = 1;
        __syncthreads();
        if (!p.row_shard) {                                // one shard
            for (int i = tid; i < n_b; i += WG) count[i] = max(start_of(b0 + i + 1) - start_of(b0 + i), 0);
        } else {
            for (int t = t0 + tid; t < t1; t += WG) {
                const uint32_t s = p.row_shard[t];
                if (s < (uint32_t)S) atomicAdd(&count[seq_of(t) * S + s], 1);
            }
        }
        __syncthreads();
        const int64_t list0 = (int64_t)b0 * S;
        auto need = [&](int i) {                           // pages; -1: more rows than a list has
            const int64_t n = (int64_t)list_len(l, list0 + i) + count[i];
            if (n > (int64_t)l.max_pages << l.page_shift) return -1;
            return pages_of(l, (int32_t)n) - pages_of(l, (int32_t)n - count[i]);
        };
        for (int i = tid; i < n_l; i += WG)
            if (need(i) < 0) ok[i / S] = 0;
        __syncthreads();
        const int32_t needed = scan_lists(n_l, first, scratch, flip, [&](int i) { return ok[i / S] ? need(i) : 0; });
        // A sequence is taken if all pages up to its own are there, or if it needs none.  Those that are taken and need some come
        // before all that find none, so that `first` needs no second pass.
        auto pages_end = [&](int b) { return b + 1 < n_b ? first[(b + 1) * S] : needed; };
        int32_t most = 0;
        for (int b = tid; b < n_b; b += WG) {
            const int32_t lo = first[b * S], hi = pages_end(b);
            if (hi > lo) {
                if (exhausted || hi > n_free) ok[b] = 0;
                else most = hi;
            }
            p.accepted[b0 + b] = ok[b];
        }
        // the pages of all that are taken: the largest `most` (they ascend with b)
        int32_t granted = 0;
        {
            int32_t *top = scratch + flip * WAVES;
            flip ^= 1;
            int32_t m = most;
#pragma unroll
            for (int o = 32; o; o >>= 1) m = max(m, __shfl_xor(m, o, WAVE));
            if ((tid & 63) == 0) top[tid >> 6] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) granted = max(granted, top[w]);
        }
        take_free(l, granted, scratch, flip, [&](int32_t page, int32_t rank) {
            const int i = last_at_most(first, n_l, rank);
            const int32_t at = pages_of(l, list_len(l, list0 + i)) + rank - first[i];
            l.table[(list0 + i) * l.max_pages + at] = page;
        });
        n_free -= granted;
        exhausted |= needed > granted;

        if (p.row_shard) {                                 // rows of a shard in the round before each sequence
            for (int s = tid; s < S; s += WG) {
                int32_t sum = 0;
                for (int b = 0; b < n_b; ++b) { before[b * S + s] = sum; sum += count[b * S + s]; }
            }
        }
        __syncthreads();                                   // pages, lengths as they were, and counts are there
        auto slot_of = [&](int64_t list, int32_t row) {
            const int32_t page = l.table[list * l.max_pages + (row >> l.page_shift)];
            return (uint32_t)page < (uint32_t)l.n_pages ? (page << l.page_shift) + (row & ((1 << l.page_shift) - 1)) : -1;
        };
        if (!p.row_shard) {
            for (int t = t0 + tid; t < t1; t += WG) {
                const int b = seq_of(t), i = t - start_of(b0 + b);
                const bool taken = ok[b] && (uint32_t)i < (uint32_t)count[b];
                const int32_t row = list_len(l, list0 + b) + i;
                p.slots[t] = taken ? slot_of(list0 + b, row) : -1;
                p.visible[t] = taken ? row + 1 : 0;
            }
        } else {
            // 64 rows a wavefront: a row's rank in its shard is a population count of a ballot, plus the rows of the
            // wavefronts before, plus those of earlier passes (held by the thread of that shard)
            const int wave = tid >> 6, lane = tid & 63;
            const uint64_t up_to = ~0ull >> (63 - lane);
            int32_t *seen = part + WAVES * S;              // [S] rows of earlier passes
            for (int s = tid; s < S; s += WG) seen[s] = 0;
            for (int base = t0; base < t1; base += WG) {
                const int t = base + tid;
                const int shard = t < t1 ? p.row_shard[t] : -1;
                for (int s = 0; s < S; ++s) {
                    const int n = __popcll(__ballot(shard == s));
                    if (lane == 0) part[wave * S + s] = n;
                }
                __syncthreads();
                for (int s = tid; s < S; s += WG) {        // exclusive sums over the wavefronts
                    int32_t sum = seen[s];
                    for (int w = 0; w < WAVES; ++w) {
                        const int32_t n = part[w * S + s];
                        part[w * S + s] = sum;
                        sum += n;
                    }
                    seen[s] = sum;
                }
                __syncthreads();
                const int b = t < t1 ? seq_of(t) : 0;
                const bool taken = ok[b] != 0;
                int32_t mine = -1;
                for (int s = 0; s < S; ++s) {
                    const int32_t rank = part[wave * S + s] + __popcll(__ballot(shard == s) & up_to) - before[b * S + s];
                    if (t >= t1) continue;
                    const int32_t end = list_len(l, list0 + b * S + s) + rank;
                    p.visible[(int64_t)t * S + s] = taken ? end : 0;
                    if (s == shard) mine = end - 1;
                }
                if (t < t1) p.slots[t] = taken && (uint32_t)shard < (uint32_t)S ? slot_of(list0 + b * S + shard, mine) : -1;
                __syncthreads();                           // the next pass writes `part`
            }
        }
        __syncthreads();                                   // every length has been read
        for (int i = tid; i < n_l; i += WG)
            if (ok[i / S] && count[i]) l.len[list0 + i] = list_len(l, list0 + i) + count[i];
    }
    // rows of no sequence
    const int lo = start_of(0), hi = max(start_of(l.n_seqs), lo);
    for (int t = tid; t < p.rows; t += WG) {
        if (t >= lo && t < hi) continue;
        p.slots[t] = -1;
        for (int s = 0; s < S; ++s) p.visible[(int64_t)t * S + s] = 0;
    }
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
    for (int i = tid; i < p.n; i += WG) {
        const int src = p.src[i], dst = p.dst[i];
        bool good = (uint32_t)src < (uint32_t)l.n_seqs && (uint32_t)dst < (uint32_t)l.n_seqs && src != dst;
        for (int j = 0; good && j < i; ++j) good = p.dst[j] != dst;
        for (int s = 0; good && s < S; ++s) good = l.len[(int64_t)dst * S + s] <= 0;
        ok[i] = good;
    }
    __syncthreads();
    for (int i = tid; i < n_l; i += WG) rows[i] = ok[i / S] ? list_len(l, (int64_t)p.src[i / S] * S + i % S) : 0;
    const int32_t mask = (1 << l.page_shift) - 1;
    const int32_t n_free = count_free(l, scratch, flip);
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
    int32_t granted = 0;
    {
        int32_t *top = scratch + flip * WAVES;
        flip ^= 1;
#pragma unroll
        for (int o = 32; o; o >>= 1) most = max(most, __shfl_xor(most, o, WAVE));
        if ((tid & 63) == 0) top[tid >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) granted = max(granted, top[w]);
    }
    for (int i = tid; i < n_l; i += WG) {
        p.list_len[i] = ok[i / S] ? rows[i] : 0;
        p.list_page[i] = -1;
    }
    __syncthreads();
    take_free(l, granted, scratch, flip, [&](int32_t page, int32_t rank) { p.list_page[last_at_most(first, n_l, rank)] = page; });
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
    const int32_t n_live = l.n_pages - count_free(l, scratch, flip);
    int32_t moved = 0, holes = 0;
    for (int64_t base = 0; base < l.n_pages; base += WG * REFS_PER_THREAD) {
        const int64_t p0 = base + (int64_t)threadIdx.x * REFS_PER_THREAD;
        uint32_t hole = 0, mover = 0;
#pragma unroll
        for (int i = 0; i < REFS_PER_THREAD; ++i) {
            if (p0 + i >= l.n_pages) continue;
            const bool free = l.refs[p0 + i] == 0;
            if (free && p0 + i < n_live) hole |= 1u << i;
            if (!free && p0 + i >= n_live) mover |= 1u << i;
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
    ExtendParams p = {};
    p.l = lists_of(cache);
    p.q_start = q_start_dev; p.row_shard = row_shard_dev; p.slots = slots; p.visible = visible; p.accepted = accepted;
    p.rows = rows;
    const int S = cache->n_shards;
    p.seqs_per_round = min(cache->n_seqs, max(1, 4096 / S));
    const int bytes = 4 * (p.seqs_per_round * (3 * S + 1) + (WAVES + 1) * S);
    static std::atomic<uint64_t> lds_ready{0};
    CASCADE_HIP_TRY(ensure_dynamic_lds((const void *)paged_extend_kernel, 144 * 1024, lds_ready));
    hipLaunchKernelGGL(paged_extend_kernel, dim3(1), dim3(WG), bytes, (hipStream_t)stream, p);
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
