// Next tokens from logits (cascade_sample): temperature, top-k, top-p, min-p, one given random number a row.
//
// No row is sorted.  All three filters keep a prefix of the row in descending order, and the token is the place where the running
// sum of the weights passes a target, so everything asked of a row is "at which place does the running count, or the running sum,
// reach this".  Pass 1 (a workgroup per chunk of a row) puts every logit into one of 1024 bins of 1/24 in the exponent, on a grid
// that does not depend on the row's maximum, so that the chunks' bins add up; a bin holds how many and the sum of their weights
// relative to the bin's middle.  Pass 2 (a workgroup per row) adds the chunks, scans the bins, and looks closer where a border falls
// inside a bin: the bin's elements are gathered from the row and sorted (up to 1024), or counted again in 1024 finer bins of the
// numbers' own bit patterns until they are few or all alike.  Where all that can be kept has at most 1024 elements, one
// gathering answers everything; the chunks keep their largest elements (64, or a bin's end more) beside their bins, which
// usually hold all that is to be gathered, because a second look at a row takes one CU 6 us for a quarter of a megabyte.
//
// One token is the latency of a chain of short steps that each run once: the second pass is written for little code (rolled loops,
// lane moves, one copy of a step), which its wavefronts fetch from cold caches.
//
// Measured (us, bf16): one row of 128256 7.4 + 13; 256 rows with mixed settings 37 (1.8 TB/s: some 45 instructions and an LDS atomic
// a logit) + 55 to 65 (the rows whose borders lie deep, by their settings); 32 fp32 rows of 50257 without filters 7.3 + 30 (a second
// look at each row).  The second pass spills: 1024 threads leave 128 registers, eight pieces under way and what lives across the
// look at a row want more (bf16 340 bytes of scratch memory a lane, fp32 176).
//
// Weights are exp(z / 24), z = 24 l / temperature in 64 bits; relative to the middle of the bin, at most a 48th away, they are whole
// numbers of 2^-29, so that sums within a bin are exact and do not depend on any order; the rounding (2^-30 of a weight, either
// way) is what the result is exact to, up to |z| = 2^26; z's own rounding, 2^-52 |l| / temperature of a weight, is what counts further
// out, where neighbouring fp32 numbers are four bins apart or more.  Elements behind the last bin, of weight below e^-42.6 of the largest, count as
// none: 2^20 of them are 3e-13 of the sum.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "common.h"
#include "device_utils.h"

// Pass 1 and pass 2 have to place an element alike: products are rounded before anything is added, fma() where one is meant
#pragma clang fp contract(off)

namespace {

constexpr int BINS = 1024, SCALE = 24;                     // 42.7 in the exponent; one to a thread of the second pass
constexpr int COUNT_SHIFT = 46;                            // of a bin's word: sum below (2^13 .. 2^15 elements of less than 2^30)
constexpr int LIST = 1024;                                 // elements that are sorted, and threads of the second pass
constexpr double UNIT = 0x1p-29;                           // of a weight within its bin

// What the first pass leaves of a chunk, in words of 8 bytes: where its bins begin; its maximum, and where that is (greedy rows);
// the last bin whose elements it kept all (-1: none) and how many it kept; the bins; the elements kept (~key, index)
enum { HEAD_BASE, HEAD_MOST, HEAD_KEPT, HEADS };
constexpr int KEEP = 64, ROOM = 128;                       // largest elements kept, and up to so many where a bin ends later
constexpr int CHUNK_WORDS = HEADS + BINS + ROOM;

struct SampleParams {
    const void *logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
    uint64_t *chunks;                                      // [rows][n_chunks][CHUNK_WORDS]
    int64_t stride;
    int32_t vocab, n_chunks;
};

// order of the values as whole numbers (no NaN, no -0)
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __builtin_bit_cast(float, k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}
// Largest value of a window of keys that ends at k: -0, which no element has, would let 0 in
__device__ __forceinline__ float end_of(uint32_t k) { return value_of(k == 0x7fffffffu ? k - 1 : k); }
constexpr uint32_t KEY_MIN = 0x00800000u, KEY_INF = 0xff800000u;                 // smallest finite value's key, +inf's

// Where a value lies on the grid; c = 24 / temperature.  Its bin is the nearest whole number.  Beside an infinite maximum, or one so
// far out on the grid that fp32 numbers are more than all bins apart, nothing else counts: then the maximum lies at 0.
__device__ __forceinline__ bool stands_alone(float most, double c) { return most == INFINITY || fabs((double)most * c) >= 0x1p40; }
__device__ __forceinline__ double grid(float v, double c, bool alone, float most) { return alone ? (v >= most ? 0.0 : -0x1p1000) : (double)v * c; }
// exp(d / 24) in units of 2^-29, |d| <= 1/2: power series (remainder 3.3e-11 at the ends, a 50th of a unit); the last step adds
// 1.5 * 2^52, which leaves the rounded whole number in the low word
constexpr double TO_WHOLE = 0x1.8p52;
__device__ __forceinline__ uint32_t low_word(double x) { return (uint32_t)__builtin_bit_cast(uint64_t, x); }
__device__ __forceinline__ uint32_t weight(double d) {
    constexpr double U = 1.0 / UNIT;
    constexpr double S = SCALE;
    double e = fma(d, U / (24 * S * S * S * S), U / (6 * S * S * S));
    e = fma(e, d, U / (2 * S * S));
    e = fma(e, d, U / S);
    return low_word(fma(e, d, U + TO_WHOLE));
}
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Piece { uint32_t w[4]; };
template <typename T> constexpr int PER = 16 / (int)sizeof(T);                   // logits of a request

template <typename T> __device__ __forceinline__ float logit(const Piece<T> &p, int e) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, p.w[e]);
    else return __builtin_bit_cast(float, e & 1 ? p.w[e >> 1] & 0xffff0000u : p.w[e >> 1] << 16);
}
// Logits i .. i + PER - 1 of a row of V; past its end -inf.  Whole pieces are requested without a branch.
template <typename T>
__device__ __forceinline__ Piece<T> request(const T *row, int64_t i, int V) {
    Piece<T> p;
    if (V >= PER<T>) p = *(const Piece<T> *)(row + (V - i >= PER<T> ? i : 0));
    return p;
}
template <typename T>
__device__ __forceinline__ void mend(const T *row, int64_t i, int V, Piece<T> &p) {
    if (V - i >= PER<T>) return;
    typedef typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type bits;
    for (int e = PER<T> - 1; e >= 0; --e) {                // each behind those before it
        const uint32_t x = i + e < V ? (uint32_t)__builtin_bit_cast(bits, row[i + e]) : sizeof(T) == 4 ? 0xff800000u : 0xff80u;
        if constexpr (sizeof(T) == 4) {
            p.w[3] = p.w[2]; p.w[2] = p.w[1]; p.w[1] = p.w[0]; p.w[0] = x;
        } else {
            p.w[3] = p.w[3] << 16 | p.w[2] >> 16; p.w[2] = p.w[2] << 16 | p.w[1] >> 16; p.w[1] = p.w[1] << 16 | p.w[0] >> 16;
            p.w[0] = p.w[0] << 16 | x;
        }
    }
}

__device__ __forceinline__ double grid_scale(const SampleParams &p, int row, bool &greedy) {
    const float t = p.temperature ? p.temperature[row] : 1.f;
    greedy = !(t > 0.f);
    return greedy ? 0.0 : SCALE / (double)t;
}

// Running sums over a wavefront by lane moves: inside rows of 16, then the rows' sums
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V moved(V v) {                  // 0 where no lane gives
    if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    else {
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        const u32x2 r = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, ROWS, 0xf, false), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, ROWS, 0xf, false)};
        return __builtin_bit_cast(V, r);
    }
}
template <typename V>
__device__ __forceinline__ V row_running_sum(V v) {
    v += moved<0x111, 0xf>(v);                             // from 1, 2, 4 and 8 lanes before
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    return v + moved<0x118, 0xf>(v);
}
template <typename V>
__device__ __forceinline__ V wave_running_sum(V v) {
    v = row_running_sum(v);
    v += moved<0x142, 0xa>(v);                             // the last lane of a row to the next one, of the first two to the others
    return v + moved<0x143, 0xc>(v);
}
template <typename V>
__device__ __forceinline__ V of_lane(V v, int lane) {      // the same for all lanes
    if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    else {
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        return __builtin_bit_cast(V, u32x2{(uint32_t)__builtin_amdgcn_readlane((int)w[0], lane), (uint32_t)__builtin_amdgcn_readlane((int)w[1], lane)});
    }
}

// ---------------------------------------------------------------------------- pass 1: the bins of a chunk
constexpr int chunk_of(int threads) { return threads * 32; }

template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_bins_kernel(SampleParams p) {
    constexpr int N = 32 / PER<T>, WAVES = NT / 64, MINE = (BINS + NT - 1) / NT;
    __shared__ unsigned long long bins[MINE * NT];
    __shared__ float wave_most[WAVES];
    __shared__ int wave_first[WAVES];
    __shared__ uint32_t wave_count[WAVES], kept;
    __shared__ int last_kept;
    const int row = blockIdx.x / p.n_chunks, chunk = blockIdx.x - row * p.n_chunks, tid = threadIdx.x, wave = tid >> 6;
    const T *logits = (const T *)p.logits + row * p.stride;
    const int64_t i0 = (int64_t)chunk * chunk_of(NT) + tid * PER<T>;
    Piece<T> v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = request(logits, i0 + j * NT * PER<T>, p.vocab);
    bool greedy;
    const double c = grid_scale(p, row, greedy);
#pragma unroll
    for (int b = 0; b < MINE; ++b) bins[tid + b * NT] = 0;
    if (tid == 0) {
        kept = 0;
        last_kept = BINS - 1;
    }
    // f(logit, index) for all of the thread's, one copy of the code for its pieces, which move up
    auto each = [&](auto f) {
#pragma unroll 1
        for (int j = 0; j < N; ++j) {
            const Piece<T> now = v[0];
#pragma unroll
            for (int k = 0; k + 1 < N; ++k) v[k] = v[k + 1];
            v[N - 1] = now;
#pragma unroll
            for (int e = 0; e < PER<T>; ++e) f(logit(now, e), (int)(i0 + j * NT * PER<T> + e));
        }
    };
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        mend(logits, i0 + j * NT * PER<T>, p.vocab, v[j]);
#pragma unroll
        for (int e = 0; e < PER<T>; ++e) most = fmaxf(most, logit(v[j], e));
    }
    most = wave_max(most);
    if ((tid & 63) == 0) wave_most[wave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wave_most[w]);
    uint64_t *out = p.chunks + (int64_t)blockIdx.x * CHUNK_WORDS;
    const bool alone = most > -INFINITY && stands_alone(most, c);
    const double base = most == -INFINITY || most == INFINITY ? 0.0 : rint((double)most * c);
    // Values below `least` are out of the bins' reach; the few others that are, too, are kept back by the bin's number
    const float least = alone ? most : fmaxf((float)((base - BINS - 2 - fabs(base) * 0x1p-20) / c), -0x1.fffffep127f);
    const uint32_t zero = low_word(base + TO_WHOLE);
    if (greedy) {
        int first = INT32_MAX;
        each([&](float l, int i) { first = l == most ? min(first, i) : first; });
        for (int o = 32; o; o >>= 1) first = min(first, __shfl_xor(first, o, WAVE));
        if ((tid & 63) == 0) wave_first[wave] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < WAVES; ++w) first = min(first, wave_first[w]);
            out[HEAD_MOST] = (uint64_t)__builtin_bit_cast(uint32_t, most) << 32 | (uint32_t)first;
        }
        return;
    }
    if (alone) each([&](float l, int) { if (l >= least) atomicAdd(&bins[0], (1ull << COUNT_SHIFT) | weight(0.0)); });
    else each([&](float l, int) {
        const double z = (double)l * c, t = z + TO_WHOLE;
        const uint32_t b = zero - low_word(t);
        if (l >= least && b < (uint32_t)BINS) atomicAdd(&bins[b], (1ull << COUNT_SHIFT) | weight(z - (t - TO_WHOLE)));     // (no NaN)
    });
    __syncthreads();

    // the bin down to which elements are kept: the first ones that hold KEEP, without the last if they are more than there is room for
    uint32_t mine[MINE], sum = 0;
#pragma unroll
    for (int b = 0; b < MINE; ++b) {
        const uint64_t w = bins[tid * MINE + b];
        mine[b] = (uint32_t)(w >> COUNT_SHIFT);
        sum += mine[b];
    }
    const uint32_t upto = wave_running_sum(sum);
    if ((tid & 63) == 63) wave_count[wave] = upto;
    __syncthreads();
    uint32_t run = upto - sum;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) run += w < wave ? wave_count[w] : 0u;
#pragma unroll
    for (int b = 0; b < MINE; ++b) {
        if (run < (uint32_t)KEEP && run + mine[b] >= (uint32_t)KEEP) last_kept = run + mine[b] <= (uint32_t)ROOM ? tid * MINE + b : tid * MINE + b - 1;
        run += mine[b];
    }
    for (int b = tid; b < BINS; b += NT) out[HEADS + b] = bins[b];
    __syncthreads();
    // (rows that no filter cuts are not asked for their largest)
    const bool cut = (p.top_k && p.top_k[row] > 0) || (p.top_p && p.top_p[row] < 1.f) || (p.min_p && p.min_p[row] > 0.f);
    const int last = cut ? last_kept : -1;
    if (cut) {
        const float lowest = alone ? least : fmaxf((float)((base - last - 2 - fabs(base) * 0x1p-20) / c), least);
        uint32_t candidates = 0;                           // few of the 32, which are then read again
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < PER<T>; ++e) candidates |= logit(v[j], e) >= lowest ? 1u << (j * PER<T> + e) : 0u;
        for (; candidates; candidates &= candidates - 1) {
            const int which = __builtin_ctz(candidates), i = (int)i0 + which / PER<T> * (NT * PER<T>) + which % PER<T>;
            const float l = (float)logits[i];
            if (!alone && (int)(zero - low_word((double)l * c + TO_WHOLE)) > last) continue;
            const uint32_t at = atomicAdd(&kept, 1u);
            if (at < (uint32_t)ROOM) out[HEADS + BINS + at] = (uint64_t)~key_of(l + 0.f) << 32 | (uint32_t)i;
        }
    }
    __syncthreads();
    if (tid == 0) {
        out[HEAD_BASE] = __builtin_bit_cast(uint64_t, base);
        out[HEAD_MOST] = (uint64_t)__builtin_bit_cast(uint32_t, most) << 32;
        out[HEAD_KEPT] = (uint64_t)(uint32_t)last << 32 | min(kept, (uint32_t)ROOM);
    }
}

// ---------------------------------------------------------------------------- pass 2: the row
// Steps of the whole workgroup (LIST threads) in which each wavefront leaves a value and reads all of them behind one barrier.  Two
// sets of places in turn: whoever writes a set has passed the barrier of the other one, behind which nobody reads it any more.
constexpr int WAVES = LIST / 64;
struct Meet {
    uint64_t at[2][WAVES];
};
struct Steps {
    Meet &meet;
    int turn;

    template <typename V> __device__ __forceinline__ V *places() {
        turn ^= 1;
        return (V *)meet.at[turn];
    }
    template <typename V> __device__ __forceinline__ V running_sum(V v) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        V *waves = places<V>();
        v = wave_running_sum(v);
        if (lane == 63) waves[wave] = v;
        __syncthreads();
        const V before = row_running_sum(lane < wave ? waves[lane & (WAVES - 1)] : (V)0);
        return of_lane(before, 15) + v;
    }
    // first thread for which `is` holds; LIST: none
    __device__ __forceinline__ int first_thread(bool is) {
        const uint64_t b = __ballot(is);
        uint32_t *waves = places<uint32_t>();
        const int lane = threadIdx.x & 63;
        if (lane == 0) waves[threadIdx.x >> 6] = b ? (threadIdx.x & ~63u) + __builtin_ctzll(b) : LIST;
        __syncthreads();
        const uint32_t first = waves[lane & (WAVES - 1)];
        const uint64_t any = __ballot(first < (uint32_t)LIST);
        return any ? of_lane((int)first, __builtin_ctzll(any) & 63) : LIST;
    }
    __device__ __forceinline__ uint32_t total(uint32_t v) { return of_last(running_sum(v)); }
    template <typename V> __device__ __forceinline__ V of_last(V v) {            // the last thread's
        V *waves = places<V>();
        if (threadIdx.x == LIST - 1) waves[0] = v;
        __syncthreads();
        return waves[0];
    }
};

enum { AT_PLACE, AT_BIN, ABOVE_BIN };
struct Run {
    float lo, hi;
};
template <typename T>
struct Row {
    const T *logits;
    int32_t V;
    double c;
    bool alone;
    float most;

    __device__ __forceinline__ double place(float v) const { return grid(v, c, alone, most); }

    // The thread's pieces, eight requested at a time: f(pieces, index of the first logit, indices from one piece to the next)
    template <typename F> __device__ __forceinline__ void each_batch(F f) const {
        constexpr int STEP = LIST * PER<T>, N = 8;
        for (int64_t i0 = (int64_t)threadIdx.x * PER<T>; i0 < V; i0 += N * STEP) {
            Piece<T> v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = request(logits, i0 + j * STEP, V);
#pragma unroll
            for (int j = 0; j < N; ++j) mend(logits, i0 + j * STEP, V, v[j]);
            f(v, (int)i0, STEP);
        }
    }
    // f(value, index) for the logits in any of n runs, which are few: a bit for each one that is, those are then read again
    template <typename F> __device__ __forceinline__ void each_in(const Run *runs, int n, F f) const {
        each_batch([&](const Piece<T> (&v)[8], int i0, int step) {
            uint32_t in[8 * PER<T> / 32] = {};
#pragma unroll 1
            for (int r = 0; r < n; ++r) {
                const float lo = runs[r].lo, hi = runs[r].hi;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < PER<T>; ++e) {
                        const float l = logit(v[j], e);
                        const int bit = j * PER<T> + e;
                        in[bit >> 5] |= l >= lo && l <= hi ? 1u << (bit & 31) : 0u;
                    }
            }
#pragma unroll
            for (int w = 0; w < 8 * PER<T> / 32; ++w)
#pragma unroll 1
                for (; in[w]; in[w] &= in[w] - 1) {
                    const int bit = 32 * w + __builtin_ctz(in[w]), i = i0 + bit / PER<T> * step + bit % PER<T>;
                    f((float)logits[i], i);
                }
        });
    }
    // f(value, index) for every logit
    template <typename F> __device__ __forceinline__ void each(F f) const {
        each_batch([&](const Piece<T> (&v)[8], int i0, int step) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < PER<T>; ++e) f(logit(v[j], e), i0 + j * step + e);
        });
    }
    template <int WHAT> __device__ __forceinline__ bool reaches(uint32_t key, double z) const {
        const double at = place(value_of(key));
        return WHAT == ABOVE_BIN ? rint(at) > z : WHAT == AT_BIN ? rint(at) >= z : at >= z;
    }
    // smallest key whose place on the grid is at least z (AT_BIN: whose bin is at least z, ABOVE_BIN: above z; KEY_INF + 1: none),
    // found by every wavefront for itself
    template <int WHAT>
    __device__ __forceinline__ uint32_t first_key(double z) const {
        uint32_t lo = KEY_MIN, n = KEY_INF + 1 - KEY_MIN;  // the answer is lo .. lo + n
        const float near = (float)((WHAT == AT_PLACE ? z : WHAT == AT_BIN ? z - 0.5 : z + 0.5) / c);
        const uint32_t guess = key_of(near);               // usually within a few keys of it: one question instead of six
        if (!alone && guess > KEY_MIN + 32 && guess < KEY_INF - 32) {
            const uint64_t b = __ballot(reaches<WHAT>(guess - 32 + (threadIdx.x & 63), z));
            if (b && !(b & 1)) return guess - 32 + __builtin_ctzll(b);
        }
        while (n) {
            const uint32_t step = (n + 63) >> 6, at = (threadIdx.x & 63) * step;
            const bool is = at >= n || reaches<WHAT>(lo + (at < n ? at : 0), z);
            const uint64_t b = __ballot(is);
            if (!b) {                                      // behind the last one asked
                lo += 63 * step + 1;
                n -= 63 * step + 1;
                continue;
            }
            const uint32_t hit = (uint32_t)__builtin_ctzll(b);
            if (hit == 0) return lo;
            const uint32_t next = min(hit * step, n);
            lo += (hit - 1) * step + 1;
            n = next - (hit - 1) * step - 1;
        }
        return lo;
    }
};

constexpr int MOST_RUNS = 4;
constexpr int MOST_CHUNKS = 128;                           // 2^20 logits in chunks of 8192

struct Shared {
    int32_t down[MOST_CHUNKS];                             // bins by which a chunk's begin below the row's; BINS: none of it counts
    uint32_t kept[MOST_CHUNKS];                            // elements that the chunk kept
    double mass[BINS];                                     // running sums of the bins
    uint32_t count[BINS];
    uint64_t list[LIST];                                   // sorted elements (~key, index), or the sums of finer bins
    uint32_t fine[LIST];                                   // their counts
    // elements of whole bins, gathered together because borders are expected in them: element, bin, and the running count and sum
    uint32_t known;                                        // how many
    bool wanted[BINS];                                     // whose
    uint64_t known_element[LIST];
    int32_t known_bin[LIST];
    uint32_t known_count[LIST];
    double known_mass[LIST];
    uint64_t before_sum[BINS];                             // sum and number of the known elements in front of a bin's
    uint32_t before_count[BINS];
    Run runs[MOST_RUNS];
    uint32_t n;
    int32_t at;
    double found[2];
    uint64_t sum;
    Meet meet;
};

// One exchange of a bitonic sort between lanes O apart
template <int O>
__device__ __forceinline__ void exchange(uint64_t &mine, bool keep_low) {
    uint64_t other;
    if constexpr (O == 1) other = moved<0xB1, 0xf>(mine);
    else if constexpr (O == 2) other = moved<0x4E, 0xf>(mine);
    else if constexpr (O == 4) other = moved<0x1B, 0xf>(moved<0x141, 0xf>(mine));          // 7 - i, then 3 - i
    else if constexpr (O == 8) other = moved<0x128, 0xf>(mine);
    else if constexpr (O == 16) {
        const u32x2 w = __builtin_bit_cast(u32x2, mine);
        other = __builtin_bit_cast(uint64_t, u32x2{(uint32_t)__builtin_amdgcn_ds_swizzle((int)w[0], 0x401f), (uint32_t)__builtin_amdgcn_ds_swizzle((int)w[1], 0x401f)});
    } else other = __shfl_xor((unsigned long long)mine, O, WAVE);
    mine = (mine < other) == keep_low ? mine : other;
}
// Exchanges between lanes O, O / 2, .. 1 apart; up: the sequence is to ascend
template <int O>
__device__ __forceinline__ void exchanges(uint64_t &mine, bool up) {
    exchange<O>(mine, ((threadIdx.x & O) == 0) == up);
    if constexpr (O > 1) exchanges<O / 2>(mine, up);
}
// Sorts the n <= LIST elements of the list (the others ~0) and returns the caller's
__device__ __attribute__((noinline)) uint64_t sorted(uint32_t n, Shared &sh) {
    const int tid = threadIdx.x;
    __syncthreads();
    uint64_t mine = sh.list[tid];
    uint32_t width = 64;
    while (width < n) width <<= 1;
    const bool in = (uint32_t)tid < width;                 // of whole wavefronts
    if (in) {
        exchanges<1>(mine, !(tid & 2));
        exchanges<2>(mine, !(tid & 4));
        exchanges<4>(mine, !(tid & 8));
        exchanges<8>(mine, !(tid & 16));
        exchanges<16>(mine, !(tid & 32));
        exchanges<32>(mine, !(tid & 64));
    }
#pragma unroll 1
    for (uint32_t k = 128; k <= width; k <<= 1) {
#pragma unroll 1
        for (uint32_t o = k >> 1; o >= 64; o >>= 1) {
            __syncthreads();
            sh.list[tid] = mine;
            __syncthreads();
            const uint64_t other = sh.list[tid ^ o];
            mine = (mine < other) == (((tid & o) == 0) == ((tid & k) == 0)) ? mine : other;
        }
        if (in) exchanges<32>(mine, !(tid & k));
    }
    __syncthreads();
    return mine;
}
__device__ __forceinline__ void start_list(Shared &sh) {
    if (threadIdx.x == 0) sh.n = 0;
    sh.list[threadIdx.x] = ~0ull;
    __syncthreads();
}
__device__ __forceinline__ void put(uint64_t element, Shared &sh) {
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < LIST) sh.list[at] = element;
}
// Gathers the row's elements of keys klo .. khi (at most LIST) into the list
template <typename T>
__device__ __attribute__((noinline)) void gather(const Row<T> &row, uint32_t klo, uint32_t khi, Shared &sh) {
    if (threadIdx.x == 0) sh.runs[0] = {value_of(klo), end_of(khi)};
    start_list(sh);
    row.each_in(sh.runs, 1, [&](float v, int i) { put((uint64_t)~key_of(v + 0.f) << 32 | (uint32_t)i, sh); });
}
// exp(-b / 24), b >= 0 a whole number: 2 to the whole and the rest, the rest by its power series (1e-15)
__device__ __forceinline__ double bin_weight(double b) {
    const double y = b * (-1.4426950408889634074 / SCALE), i = rint(y), f = (y - i) * 0.693147180559945309417;
    double e = 1.0;
#pragma unroll
    for (int k = 13; k; --k) e = fma(e * f, 1.0 / k, 1.0);
    return ldexp(e, (int)i);
}

struct Place {
    uint32_t count;                                        // elements up to and with this one
    double mass, own;                                      // their sum, and its weight
    int32_t index;
};

// The first place in descending order at which the running count reaches k (by_count), or the running sum reaches t
// (over: exceeds it).  One that does not exist is the last place.  `index`: whether the element itself is wanted.
template <typename T>
__device__ __attribute__((noinline)) Place search(const Row<T> &row, double base, Shared &sh, Steps &steps, bool by_count, uint32_t k, double t, bool over, bool index) {
    const int tid = threadIdx.x;
    auto reached = [&](uint32_t n, double m) { return by_count ? n >= k : over ? m > t : m >= t; };
    const int bin = min(tid, BINS - 1);
    const bool holds = tid < BINS && sh.count[bin] > (bin ? sh.count[bin - 1] : 0);
    int b = steps.first_thread(holds && reached(sh.count[bin], sh.mass[bin]));
    if (b >= BINS) {                                       // the last place
        by_count = true;
        k = sh.count[BINS - 1];
        b = steps.first_thread(holds && sh.count[bin] >= k);
    }
    uint32_t before = b ? sh.count[b - 1] : 0, n = sh.count[b] - before;
    if (by_count && !index && sh.count[b] == k) return Place{k, sh.mass[b], 0.0, -1};
    const double below = b ? sh.mass[b - 1] : 0.0, unit = bin_weight(b) * UNIT;
    if (sh.known && sh.wanted[b]) {
        const bool mine = (uint32_t)tid < sh.known && sh.known_bin[tid] == b;
        int f = steps.first_thread(mine && reached(sh.known_count[tid], sh.known_mass[tid]));
        if (f >= LIST) f = steps.first_thread(mine && sh.known_count[tid] == before + n);
        const uint64_t e = sh.known_element[f];
        const double z = row.place(value_of(~(uint32_t)(e >> 32)));
        return Place{sh.known_count[f], sh.known_mass[f], unit * weight(z - rint(z)), (int32_t)(uint32_t)e};
    }
    uint32_t klo = row.template first_key<AT_BIN>(base - b), khi = row.template first_key<ABOVE_BIN>(base - b) - 1;
    uint64_t sum = 0;                                      // of the bin's elements in front of klo .. khi
    while (n > LIST && klo < khi) {
        const uint32_t span = khi - klo, shift = max(0, 22 - (int)__builtin_clz(span)), fine = (span >> shift) + 1;
        const float lo = value_of(klo), hi = end_of(khi);
        sh.list[tid] = 0;
        sh.fine[tid] = 0;
        if (tid == 0) sh.runs[0] = {lo, hi};
        __syncthreads();
        auto add = [&](float v, int) {
            const uint32_t at = fine - 1 - ((key_of(v + 0.f) - klo) >> shift);
            const double z = row.place(v);
            atomicAdd(&sh.fine[at], 1u);
            atomicAdd((unsigned long long *)&sh.list[at], (unsigned long long)weight(z - rint(z)));
        };
        if (n < (uint32_t)row.V / 16) row.each_in(sh.runs, 1, add);
        else row.each([&](float v, int i) { if (v >= lo && v <= hi) add(v, i); });
        __syncthreads();
        const uint32_t c = sh.fine[tid];
        const uint64_t m = sh.list[tid];
        const uint32_t cs = before + steps.running_sum(c);
        const uint64_t ms = sum + steps.running_sum(m);
        int f = steps.first_thread(c && reached(cs, below + unit * (double)ms));
        if (f >= LIST) {                                   // sums of the bins and of their parts differ in the last bits
            by_count = true;
            k = before + n;
            f = steps.first_thread(c && cs >= k);
        }
        if (tid == f) {
            sh.n = c;
            sh.at = (int32_t)(cs - c);
            sh.sum = ms - m;
        }
        __syncthreads();
        n = sh.n;
        before = (uint32_t)sh.at;
        sum = sh.sum;
        __syncthreads();
        const uint32_t from = klo + ((fine - 1 - (uint32_t)f) << shift);
        khi = min(khi, from + ((1u << shift) - 1));
        klo = from;
    }
    if (n <= LIST) {
        gather(row, klo, khi, sh);
        const uint64_t mine = sorted(n, sh);
        const bool is = (uint32_t)tid < n;
        const double z = is ? row.place(value_of(~(uint32_t)(mine >> 32))) : 0.0;
        const uint32_t w = is ? weight(z - rint(z)) : 0;
        const double mass = below + unit * (double)(sum + steps.running_sum((uint64_t)w));
        int f = steps.first_thread(is && reached(before + tid + 1, mass));
        f = f < LIST ? f : (int)n - 1;
        if (tid == f) {
            sh.found[0] = mass;
            sh.found[1] = unit * w;
            sh.at = (int32_t)(uint32_t)mine;
        }
        __syncthreads();
        const Place r = {before + (uint32_t)f + 1, sh.found[0], sh.found[1], sh.at};
        __syncthreads();
        return r;
    }
    // all alike: the place by arithmetic, its index by counting in the order of the row
    const double z = row.place(value_of(klo));
    const uint32_t w = weight(z - rint(z));
    auto mass_at = [&](uint32_t i) { return below + unit * (double)(sum + (uint64_t)w * i); };
    uint32_t lo = 1, hi = n;                               // first i <= n that reaches it, or n
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (reached(before + mid, mass_at(mid))) hi = mid;
        else lo = mid + 1;
    }
    Place r = {before + lo, mass_at(lo), unit * w, -1};
    if (!index) return r;
    const float value = value_of(klo);
    uint32_t passed = 0;
    for (int64_t i0 = 0; i0 < row.V; i0 += LIST * PER<T>) {
        const int64_t i = i0 + tid * PER<T>;
        Piece<T> v = request(row.logits, i, row.V);
        mend(row.logits, i, row.V, v);
        uint32_t mine = 0;
#pragma unroll
        for (int e = 0; e < PER<T>; ++e) mine += logit(v, e) == value;
        const uint32_t upto = passed + steps.running_sum(mine);
        if (upto >= lo && upto - mine < lo) {
            uint32_t left = lo - (upto - mine);
#pragma unroll
            for (int e = 0; e < PER<T>; ++e)
                if (logit(v, e) == value && --left == 0) sh.at = (int)(i + e);
        }
        if (tid == LIST - 1) sh.n = upto;
        __syncthreads();
        passed = sh.n;
        __syncthreads();
        if (passed >= lo) break;
    }
    r.index = sh.at;
    __syncthreads();
    return r;
}

// Gathers the elements of the bins that are wanted (n of them, at most LIST) in one look at the row
template <typename T>
__device__ __attribute__((noinline)) void gather_wanted(const Row<T> &row, double base, uint32_t n, Shared &sh, Steps &steps) {
    const int tid = threadIdx.x;
    // runs of wanted bins, each found by the wavefront of its number; what is left of them beyond four belongs to the last run
    const bool is_wanted = tid < BINS && sh.wanted[min(tid, BINS - 1)];
    const bool begins = is_wanted && (tid == 0 || !sh.wanted[tid - 1]), ends = is_wanted && (tid == BINS - 1 || !sh.wanted[tid + 1]);
    const uint32_t run = steps.running_sum((uint32_t)begins), n_runs = min(steps.of_last(run), (uint32_t)MOST_RUNS);
    if (begins && run <= (uint32_t)MOST_RUNS) sh.fine[run - 1] = tid;
    if (ends) atomicMax(&sh.fine[MOST_RUNS + min(run, (uint32_t)MOST_RUNS) - 1], (uint32_t)tid);
    __syncthreads();
    if (const uint32_t w = tid >> 6; w < n_runs) {
        const float hi = end_of(row.template first_key<ABOVE_BIN>(base - (double)sh.fine[w]) - 1);
        const float lo = value_of(row.template first_key<AT_BIN>(base - (double)sh.fine[MOST_RUNS + w]));
        if ((tid & 63) == 0) sh.runs[w] = {lo, hi};
    }
    start_list(sh);
    row.each_in(sh.runs, (int)n_runs, [&](float v, int i) {
        if (sh.wanted[(int)(base - rint(row.place(v)))]) put((uint64_t)~key_of(v + 0.f) << 32 | (uint32_t)i, sh);
    });
    const uint64_t e = sorted(n, sh);
    const bool is = (uint32_t)tid < n;
    const double z = is ? row.place(value_of(~(uint32_t)(e >> 32))) : base;
    const int b = is ? (int)(base - rint(z)) : BINS;
    const uint64_t w = is ? weight(z - rint(z)) : 0, sum = steps.running_sum(w);
    sh.known_element[tid] = e;
    sh.known_bin[tid] = b;
    __syncthreads();
    if (is && (tid == 0 || sh.known_bin[tid - 1] != b)) {
        sh.before_sum[b] = sum - w;
        sh.before_count[b] = tid;
    }
    __syncthreads();
    if (is) {
        sh.known_count[tid] = (b ? sh.count[b - 1] : 0) + tid - sh.before_count[b] + 1;
        sh.known_mass[tid] = (b ? sh.mass[b - 1] : 0.0) + bin_weight(b) * UNIT * (double)(sum - sh.before_sum[b]);
    }
    if (tid == 0) sh.known = n;
    __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(LIST) void sample_row_kernel(SampleParams p) {
    __shared__ Shared sh;
    Steps steps{sh.meet, 0};
    const int r = blockIdx.x, tid = threadIdx.x;
    bool greedy;
    Row<T> row = {(const T *)p.logits + r * p.stride, p.vocab, grid_scale(p, r, greedy), false, 0.f};
    const uint64_t *chunks = p.chunks + (int64_t)r * p.n_chunks * CHUNK_WORDS;
    // every wavefront looks at all chunks: the row's maximum, the first chunk that has it, where its bins begin
    const int lane = tid & 63;
    uint64_t heads[MOST_CHUNKS / 64][HEADS];
    float most = -INFINITY, mosts[MOST_CHUNKS / 64];
#pragma unroll
    for (int h = 0; h < MOST_CHUNKS / 64; ++h) {
        const int c = lane + 64 * h;
        mosts[h] = -INFINITY;
        for (int k = 0; k < HEADS; ++k) heads[h][k] = 0;
        if (c < p.n_chunks) {
            for (int k = 0; k < HEADS; ++k) heads[h][k] = chunks[(int64_t)c * CHUNK_WORDS + k];
            mosts[h] = __builtin_bit_cast(float, (uint32_t)(heads[h][HEAD_MOST] >> 32));
        }
        most = fmaxf(most, mosts[h]);
    }
    most = wave_max(most);
    double base = 0.0;
    int first = 0;
#pragma unroll
    for (int h = MOST_CHUNKS / 64 - 1; h >= 0; --h) {
        const uint64_t b = __ballot(mosts[h] == most);
        if (b) {
            const int from = __builtin_ctzll(b);
            first = of_lane((int)(uint32_t)heads[h][HEAD_MOST], from);
            base = of_lane(__builtin_bit_cast(double, heads[h][HEAD_BASE]), from);
        }
    }
    if (greedy || most == -INFINITY) {
        if (tid == 0) {
            p.token[r] = most == -INFINITY ? 0 : first;
            if (p.prob) p.prob[r] = most == -INFINITY ? 0.f : 1.f;
        }
        return;
    }
    row.alone = stands_alone(most, row.c);
    row.most = most;
    if (row.alone) base = 0.0;

    // the chunks' bins, each from its own place on the grid on
    int downs[MOST_CHUNKS / 64];
#pragma unroll
    for (int h = 0; h < MOST_CHUNKS / 64; ++h) {
        const double down = row.alone ? 0.0 : base - __builtin_bit_cast(double, heads[h][HEAD_BASE]);
        downs[h] = mosts[h] == -INFINITY || (row.alone && mosts[h] < most) || !(down < (double)BINS) ? BINS : (int)down;
        if (tid < 64) {
            sh.down[lane + 64 * h] = downs[h];
            sh.kept[lane + 64 * h] = downs[h] < BINS ? (uint32_t)heads[h][HEAD_KEPT] : 0u;
        }
    }
    __syncthreads();
    uint32_t count = 0;
    uint64_t mass = 0;
    if (tid < BINS) {
#pragma unroll 1
        for (int c0 = 0; c0 < p.n_chunks; c0 += 16) {      // sixteen requests at a time, those that count nothing to a place that exists
            uint64_t bin[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int at = tid - sh.down[min(c0 + j, MOST_CHUNKS - 1)];
                const bool is = c0 + j < p.n_chunks && at >= 0;
                bin[j] = is ? chunks[(c0 + j) * CHUNK_WORDS + HEADS + at] : 0;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                count += (uint32_t)(bin[j] >> COUNT_SHIFT);
                mass += bin[j] & ((1ull << COUNT_SHIFT) - 1);
            }
        }
    }
    const double unit = bin_weight(tid) * UNIT;
    const uint32_t counts = steps.running_sum(count);
    const double masses = steps.running_sum((double)mass * unit);
    if (tid < BINS) {
        sh.count[tid] = counts;
        sh.mass[tid] = masses;
    }
    __syncthreads();
    const uint32_t all = sh.count[BINS - 1];

    const int32_t top_k = p.top_k ? p.top_k[r] : 0;
    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f, u = p.uniform[r];
    const uint32_t k = top_k > 0 ? min((uint32_t)top_k, all) : all;
    const double least = min_p > 0.f ? row.place(most) + SCALE * log((double)min_p) : -INFINITY;
    const double uniform = u >= 0.f ? (double)u : 0.0;

    if (tid == 0) sh.known = 0;
    const int bin = min(tid, BINS - 1);
    const uint32_t own_count = tid < BINS ? sh.count[bin] - (bin ? sh.count[bin - 1] : 0) : 0;
    auto bin_with = [&](bool is) { return min(steps.first_thread(own_count && is), BINS - 1); };     // the first one
    auto mass_to = [&](int b) { return b ? sh.mass[b - 1] : 0.0; };                                  // of the bins in front
    uint32_t kept = k;
    double left = k < all ? -1.0 : sh.mass[BINS - 1];      // mass of what top_k leaves, as soon as it is known
    // the bin in which the kept ones end at the latest; as long as the mass that top_k leaves is wanted, all of that
    const int k_bin = bin_with(sh.count[bin] >= kept);
    const int least_bin = least > -INFINITY ? (int)fmin(fmax(base - rint(least), 0.0), (double)BINS) : BINS;
    int b = k_bin;
    if (left >= 0.0 && top_p < 1.f) b = min(b, bin_with(sh.mass[bin] >= (double)top_p * left));
    if (left >= 0.0 || !(top_p < 1.f)) b = min(b, least_bin);
    if (sh.count[b] > LIST) {
        // The borders that will be looked for, as far as the bins tell: where top_k cuts, where top_p does, where min_p does, where the
        // token is.  Each cut lies within one bin, so that the masses behind it are known up to that bin's.
        bool wanted = false;
        double lo = k < all ? mass_to(k_bin) : left, hi = k < all ? sh.mass[k_bin] : left;
        int end = k_bin;
        if (top_p < 1.f) {
            const int from = bin_with(sh.mass[bin] >= (double)top_p * lo), to = bin_with(sh.mass[bin] >= (double)top_p * hi);
            wanted |= tid >= from && tid <= to;
            lo = fmin(lo, mass_to(from));
            hi = fmin(hi, sh.mass[to]);
            end = min(end, to);
        }
        if (least_bin < BINS) {
            wanted |= tid == least_bin;
            lo = fmin(lo, mass_to(least_bin));
            hi = fmin(hi, sh.mass[least_bin]);
            end = min(end, least_bin);
        }
        const int from = bin_with(sh.mass[bin] > uniform * lo), to = bin_with(sh.mass[bin] > uniform * hi);
        wanted = (wanted || (tid >= from && tid <= to)) && tid <= end && own_count;
        wanted |= k < all && sh.count[k_bin] != k && tid == k_bin && (top_p < 1.f || k_bin <= end);
        if (tid < BINS) sh.wanted[bin] = wanted;
        if (tid < 2 * MOST_RUNS) sh.fine[tid] = 0;
        const uint32_t n = steps.total(wanted ? own_count : 0u);
        if (n && n <= LIST) gather_wanted(row, base, n, sh, steps);
        if (left < 0.0 && top_p < 1.f) {
            left = search(row, base, sh, steps, true, k, 0.0, false, false).mass;
            b = min(min(k_bin, least_bin), bin_with(sh.mass[bin] >= (double)top_p * left));
        }
    }
    const uint32_t n = sh.count[b];
    if (n <= LIST && !sh.known) {
        bool have = true;                                  // whether the chunks kept all of bins 0 .. b
#pragma unroll
        for (int h = 0; h < MOST_CHUNKS / 64; ++h) have &= b - downs[h] <= (int32_t)(heads[h][HEAD_KEPT] >> 32) || b < downs[h];
        if (__all(have)) {
            start_list(sh);
#pragma unroll 1
            for (int c = tid >> 6; c < p.n_chunks; c += WAVES)
#pragma unroll 1
                for (uint32_t e = lane; e < sh.kept[c]; e += 64) {
                    const uint64_t element = chunks[c * CHUNK_WORDS + HEADS + BINS + e];
                    if (base - rint(row.place(value_of(~(uint32_t)(element >> 32)))) <= (double)b) put(element, sh);
                }
        } else gather(row, row.template first_key<AT_BIN>(base - b), KEY_INF, sh);
        const uint64_t mine = sorted(n, sh);
        const bool is = (uint32_t)tid < n;
        const double z = is ? row.place(value_of(~(uint32_t)(mine >> 32))) : 0.0, f = rint(z);
        const double own = is ? bin_weight(base - f) * UNIT * weight(z - f) : 0.0;
        const double upto = steps.running_sum(own);
        double *sums = (double *)sh.list;                  // (the list is in registers now)
        sums[tid] = upto;
        __syncthreads();
        kept = min(kept, n);
        if (top_p < 1.f) {
            if (left < 0.0) left = sums[kept - 1];
            kept = min(kept, (uint32_t)steps.first_thread(is && upto >= (double)top_p * left) + 1u);
        }
        kept = min(kept, max(1u, steps.total(is && z >= least)));
        const double mass_kept = sums[kept - 1];
        // (1 and more take the last place: sums in a fixed tree are not monotone, an earlier one may be a last bit above the last)
        const double target = uniform * mass_kept;
        const uint32_t at = min((uint32_t)steps.first_thread(is && target < mass_kept && upto > target), kept - 1);
        if ((uint32_t)tid == at) {
            p.token[r] = (int32_t)(uint32_t)mine;
            if (p.prob) p.prob[r] = (float)(own / mass_kept);
        }
        return;
    }
    double mass_kept = left;
    if (left < 0.0) mass_kept = search(row, base, sh, steps, true, k, 0.0, false, false).mass;
    if (top_p < 1.f) {
        const Place q = search(row, base, sh, steps, false, 0, (double)top_p * left, false, false);
        if (q.count < kept) {
            kept = q.count;
            mass_kept = q.mass;
        }
    }
    if (least_bin < BINS) {
        uint32_t mine = 0;
        if (sh.known && sh.wanted[least_bin]) {
            mine = (uint32_t)tid < sh.known && sh.known_bin[tid] == least_bin && row.place(value_of(~(uint32_t)(sh.known_element[tid] >> 32))) >= least;
            if (tid == 0 && least_bin) mine += sh.count[least_bin - 1];
        } else if (least <= row.place(most)) {
            const float lowest = value_of(min(row.template first_key<AT_PLACE>(least), KEY_INF));
            row.each([&](float v, int) { mine += v >= lowest; });
        }
        const uint32_t q = max(1u, steps.total(mine));
        if (q < kept) {
            kept = q;
            mass_kept = search(row, base, sh, steps, true, kept, 0.0, false, false).mass;
        }
    }
    const double target = uniform * mass_kept;
    Place q = search(row, base, sh, steps, !(target < mass_kept), kept, target, true, true);
    if (q.count > kept) q = search(row, base, sh, steps, true, kept, 0.0, false, true);
    if (tid == 0) {
        p.token[r] = q.index;
        if (p.prob) p.prob[r] = (float)(q.own / mass_kept);
    }
}

// Threads of a workgroup of the first pass: small chunks while they are few (latency), larger ones where the bins they write would
// otherwise weigh as much as the logits
int bins_threads(int32_t rows, int32_t vocab) { return (int64_t)rows * ((vocab + 8191) / 8192) <= 1024 ? 256 : 512; }
int32_t most_rows_of_small_chunks(int32_t vocab) { return 1024 / ((vocab + 8191) / 8192); }
int chunks_of(int threads, int32_t vocab) { return (vocab + chunk_of(threads) - 1) / chunk_of(threads); }
size_t chunk_bytes(int32_t rows, int32_t vocab) { return (size_t)rows * chunks_of(bins_threads(rows, vocab), vocab) * CHUNK_WORDS * 8; }

int32_t check(const cascade_sample_desc *d) {
    if (!d || d->rows < 0 || d->vocab <= 0 || d->stride < 0 || d->reserved) return CASCADE_EINVAL;
    if (d->dtype != CASCADE_F32 && d->dtype != CASCADE_BF16) return CASCADE_EUNSUPPORTED;
    if (d->vocab > 1 << 20 || d->rows > 1 << 16) return CASCADE_EUNSUPPORTED;
    if (d->stride && d->stride < d->vocab) return CASCADE_ESHAPE;
    return CASCADE_OK;
}

template <typename T>
int32_t launch(const SampleParams &p, int32_t rows, int threads, hipStream_t s) {
    const dim3 grid((unsigned)(rows * p.n_chunks));
    if (threads == 256) hipLaunchKernelGGL((sample_bins_kernel<T, 256>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((sample_bins_kernel<T, 512>), grid, dim3(512), 0, s, p);
    hipLaunchKernelGGL(sample_row_kernel<T>, dim3(rows), dim3(LIST), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

}  // namespace

// Enough for fewer rows too: the last ones that take small chunks need more than those after them
extern "C" size_t cascade_sample_workspace_bytes(const cascade_sample_desc *d) {
    if (check(d) != CASCADE_OK) return 0;
    return std::max(chunk_bytes(d->rows, d->vocab), chunk_bytes(std::min(d->rows, most_rows_of_small_chunks(d->vocab)), d->vocab));
}

extern "C" int32_t cascade_sample(const cascade_sample_desc *d, const void *logits, const float *temperature, const int32_t *top_k,
                                  const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *prob,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    const int32_t st = check(d);
    if (st != CASCADE_OK) return st;
    if (d->rows == 0) return CASCADE_OK;
    if (!logits || !uniform || !token) return CASCADE_EINVAL;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < chunk_bytes(d->rows, d->vocab)) return CASCADE_EWORKSPACE;
    SampleParams p;
    p.logits = logits; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.uniform = uniform;
    p.token = token; p.prob = prob; p.chunks = (uint64_t *)workspace;
    p.stride = d->stride ? d->stride : d->vocab;
    const int threads = bins_threads(d->rows, d->vocab);
    p.vocab = d->vocab; p.n_chunks = chunks_of(threads, d->vocab);
    return d->dtype == CASCADE_BF16 ? launch<bf16_t>(p, d->rows, threads, (hipStream_t)stream)
                                    : launch<float>(p, d->rows, threads, (hipStream_t)stream);
}
