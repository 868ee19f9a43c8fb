// Next tokens from logits (cascade_sample): temperature, top-k, top-p, min-p, one given random number a row.
//
// No row is sorted.  All three filters keep a prefix of the row in descending order, and the token is the place where the running
// sum of the weights passes a target, so everything asked of a row is "at which place does the running count, or the running sum,
// reach this".  Pass 1 (a workgroup per chunk of a row) puts every logit into one of 704 bins of 1/16 in the exponent, on a grid
// that does not depend on the row's maximum, so that the chunks' bins add up; a bin holds how many and the sum of their weights
// relative to the bin's edge.  Pass 2 (a workgroup per row) adds the chunks, scans the bins, and looks closer where a border falls
// inside a bin: the bin's elements are gathered from the row and sorted (up to 1024), or counted again in 1024 finer bins of the
// numbers' own bit patterns until they are few or all alike.  Where all that can be kept has at most 1024 elements, one
// gathering answers everything.
//
// Weights are exp(z / 16), z = 16 l / temperature in 64 bits; relative to the bin's edge, which lies within a sixteenth, they are whole
// numbers of 2^-29, so that sums within a bin are exact and do not depend on any order; the rounding (2^-30 of a weight, either
// way) is what the result is exact to.  Elements of weight below e^-43 of the largest are left out: 2^20 of them are 2e-13 of the sum.
#include <algorithm>
#include <cmath>
#include "common.h"
#include "device_utils.h"

namespace {

constexpr int BINS = 704;                                  // 44 in the exponent
constexpr int COUNT_SHIFT = 46;                            // of a bin's word: sum below (2^13 .. 2^15 elements of less than 2^30)
constexpr int CHUNK_WORDS = BINS + 2;                      // of 8 bytes: grid place of the maximum; maximum and where; bins
constexpr int LIST = 1024;                                 // elements that are sorted, and threads of the second pass
constexpr double UNIT = 0x1p-29;                           // of a weight within its bin

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
constexpr uint32_t KEY_MIN = 0x00800000u, KEY_INF = 0xff800000u;                 // smallest finite value's key, +inf's

// Where a value lies on the grid; c = 16 / temperature.  With an infinity in the row, only infinities count, at 0.
__device__ __forceinline__ double grid(float v, double c, bool inf) { return inf ? (v == INFINITY ? 0.0 : -0x1p1000) : (double)v * c; }
// exp(d / 16) in units of 2^-29, 0 <= d < 1: power series around the middle, remainder 1.3e-12
__device__ __forceinline__ uint32_t weight(double d) {
    const double x = fma(d, 0.0625, -0.03125);
    double e = fma(x, 1.0 / 120, 1.0 / 24);
    e = fma(e, x, 1.0 / 6);
    e = fma(e, x, 0.5);
    e = fma(e, x, 1.0);
    e = fma(e, x, 1.0);
    return (uint32_t)fma(e, 1.0317434074991026710 / UNIT, 0.5);                  // e^(1/32)
}

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Piece { uint32_t w[4]; };
template <typename T> constexpr int PER = 16 / (int)sizeof(T);                   // logits of a request

// NaN to -inf, -0 to 0
__device__ __forceinline__ float clean(float v) { return fmaxf(v, -INFINITY) + 0.f; }
template <typename T> __device__ __forceinline__ float logit(const Piece<T> &p, int e) {
    if constexpr (sizeof(T) == 4) return clean(__builtin_bit_cast(float, p.w[e]));
    else return clean(__builtin_bit_cast(float, e & 1 ? p.w[e >> 1] & 0xffff0000u : p.w[e >> 1] << 16));
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
#pragma unroll
    for (int j = 0; j < 4; ++j) p.w[j] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int e = 0; e < PER<T>; ++e)
        if (i + e < V) {
            if constexpr (sizeof(T) == 4) p.w[e] = __builtin_bit_cast(uint32_t, row[i + e]);
            else p.w[e >> 1] = (p.w[e >> 1] & (e & 1 ? 0xffffu : 0xffff0000u)) | (uint32_t)__builtin_bit_cast(uint16_t, row[i + e]) << (e & 1 ? 16 : 0);
        }
}

__device__ __forceinline__ double grid_scale(const SampleParams &p, int row, bool &greedy) {
    const float t = p.temperature ? p.temperature[row] : 1.f;
    greedy = !(t > 0.f);
    return greedy ? 0.0 : 16.0 / (double)t;
}

// ---------------------------------------------------------------------------- pass 1: the bins of a chunk
constexpr int chunk_of(int threads) { return threads * 32; }

template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_bins_kernel(SampleParams p) {
    constexpr int N = 32 / PER<T>, WAVES = NT / 64;        // pieces of a thread
    __shared__ unsigned long long bins[BINS];
    __shared__ float wave_most[WAVES];
    __shared__ int wave_first[WAVES];
    const int row = blockIdx.x / p.n_chunks, chunk = blockIdx.x - row * p.n_chunks, tid = threadIdx.x;
    const T *logits = (const T *)p.logits + row * p.stride;
    const int64_t i0 = (int64_t)chunk * chunk_of(NT) + tid * PER<T>;
    Piece<T> v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = request(logits, i0 + j * NT * PER<T>, p.vocab);
    bool greedy;
    const double c = grid_scale(p, row, greedy);
    for (int b = tid; b < BINS; b += NT) bins[b] = 0;
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        mend(logits, i0 + j * NT * PER<T>, p.vocab, v[j]);
#pragma unroll
        for (int e = 0; e < PER<T>; ++e) most = fmaxf(most, logit(v[j], e));
    }
    most = wave_max(most);
    if ((tid & 63) == 0) wave_most[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wave_most[w]);
    uint64_t *out = p.chunks + (int64_t)blockIdx.x * CHUNK_WORDS;
    const bool inf = most == INFINITY;
    const double top = most == -INFINITY ? 0.0 : floor(grid(most, c, inf));
    int first = INT32_MAX;
    if (greedy) {
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
#pragma unroll
            for (int e = PER<T> - 1; e >= 0; --e)
                if (logit(v[j], e) == most) first = (int)(i0 + j * NT * PER<T> + e);
        for (int o = 32; o; o >>= 1) first = min(first, __shfl_xor(first, o, WAVE));
        if ((tid & 63) == 0) wave_first[tid >> 6] = first;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) first = min(first, wave_first[w]);
    } else if (most > -INFINITY) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < PER<T>; ++e) {
                const float l = logit(v[j], e);
                const double z = grid(l, c, inf), f = floor(z), down = top - f;  // (-inf: down is infinite, or NaN where c is 0)
                if (l > -INFINITY && down < (double)BINS)
                    atomicAdd(&bins[(int)down], (1ull << COUNT_SHIFT) | weight(z - f));
            }
    }
    if (tid == 0) {
        out[0] = __builtin_bit_cast(uint64_t, top);
        out[1] = (uint64_t)__builtin_bit_cast(uint32_t, most) << 32 | (uint32_t)first;
    }
    if (greedy) return;
    __syncthreads();
    for (int b = tid; b < BINS; b += NT) out[2 + b] = bins[b];
}

// ---------------------------------------------------------------------------- pass 2: the row
// Whole-workgroup steps, LIST threads; every one ends behind a barrier, so that they follow each other freely.
struct Scratch {
    double d[LIST / 64];
    uint64_t u[LIST / 64];
    uint32_t n[LIST / 64];
};
template <typename V>
__device__ __forceinline__ V running_sum(V v, V *waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const V up = __shfl_up(v, o, WAVE);
        if (lane >= o) v += up;
    }
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    V before = 0;
    for (int w = 0; w < wave; ++w) before += waves[w];
    __syncthreads();
    return before + v;
}
// first thread for which `is` holds; LIST: none
__device__ __forceinline__ int first_thread(bool is, uint32_t *waves) {
    const uint64_t b = __ballot(is);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = b ? (threadIdx.x & ~63u) + __builtin_ctzll(b) : LIST;
    __syncthreads();
    uint32_t m = LIST;
    for (int w = 0; w < LIST / 64; ++w) m = min(m, waves[w]);
    __syncthreads();
    return (int)m;
}
__device__ __forceinline__ uint32_t total_count(uint32_t v, uint32_t *waves) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor((int)v, o, WAVE);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t s = 0;
    for (int w = 0; w < LIST / 64; ++w) s += waves[w];
    __syncthreads();
    return s;
}

template <typename T>
struct Row {
    const T *logits;
    int32_t V;
    double c;
    bool inf;

    // f(value, index) for every logit, pieces of a thread requested four at a time
    template <typename F> __device__ __forceinline__ void each(F f) const {
        constexpr int STEP = LIST * PER<T>;
        for (int64_t i0 = (int64_t)threadIdx.x * PER<T>; i0 < V; i0 += 4 * STEP) {
            Piece<T> v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = request(logits, i0 + j * STEP, V);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mend(logits, i0 + j * STEP, V, v[j]);
#pragma unroll
                for (int e = 0; e < PER<T>; ++e) f(logit(v[j], e), (int)(i0 + j * STEP + e));
            }
        }
    }
    // smallest key whose place on the grid is at least z (ABOVE: beyond the bin that begins at z; KEY_INF + 1: none), found by
    // every wavefront for itself
    template <bool ABOVE = false>
    __device__ __forceinline__ uint32_t first_key(double z) const {
        uint32_t lo = KEY_MIN, n = KEY_INF + 1 - KEY_MIN;  // the answer is lo .. lo + n
        while (n) {
            const uint32_t step = (n + 63) >> 6, at = (threadIdx.x & 63) * step;
            const double place = grid(value_of(lo + (at < n ? at : 0)), c, inf);
            const bool is = at >= n || (ABOVE ? floor(place) > z : place >= z);
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

struct Shared {
    double mass[BINS];                                     // running sums of the bins
    uint32_t count[BINS];
    uint64_t list[LIST];                                   // sorted elements (~key, index), or the sums of finer bins
    uint32_t fine[LIST];                                   // their counts
    uint32_t n;
    int32_t at;
    Scratch s;
};

// Gathers the elements of keys klo .. khi (n of them, at most LIST), sorts them and returns the caller's, or ~0
template <typename T>
__device__ uint64_t gather(const Row<T> &row, uint32_t klo, uint32_t khi, uint32_t n, Shared &sh) {
    const float lo = value_of(klo), hi = value_of(khi);
    const int tid = threadIdx.x;
    if (tid == 0) sh.n = 0;
    sh.list[tid] = ~0ull;
    __syncthreads();
    row.each([&](float v, int i) {
        if (v >= lo && v <= hi) {
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < LIST) sh.list[at] = (uint64_t)~key_of(v) << 32 | (uint32_t)i;
        }
    });
    __syncthreads();
    uint64_t mine = sh.list[tid];
    uint32_t width = 64;
    while (width < n) width <<= 1;
    for (uint32_t k = 2; k <= width; k <<= 1)              // bitonic; exchanges inside a wavefront by lane
        for (uint32_t o = k >> 1; o; o >>= 1) {
            uint64_t other;
            if (o < 64) other = __shfl_xor((unsigned long long)mine, (int)o, WAVE);
            else {
                __syncthreads();
                sh.list[tid] = mine;
                __syncthreads();
                other = sh.list[tid ^ o];
            }
            const bool keep_low = ((tid & o) == 0) == ((tid & k) == 0);
            mine = (mine < other) == keep_low ? mine : other;
        }
    __syncthreads();
    return mine;
}

struct Place {
    uint32_t count;                                        // elements up to and with this one
    double mass, own;                                      // their sum, and its weight
    int32_t index;
};

// The first place in descending order at which the running count reaches k (by_count), or the running sum reaches t
// (over: exceeds it).  One that does not exist is the last place.  `index`: whether the element itself is wanted.
template <typename T>
__device__ Place search(const Row<T> &row, double top, Shared &sh, bool by_count, uint32_t k, double t, bool over, bool index) {
    const int tid = threadIdx.x;
    auto reached = [&](uint32_t n, double m) { return by_count ? n >= k : over ? m > t : m >= t; };
    const int bin = min(tid, BINS - 1);
    const bool holds = tid < BINS && sh.count[bin] > (bin ? sh.count[bin - 1] : 0);
    int b = first_thread(holds && reached(sh.count[bin], sh.mass[bin]), sh.s.n);
    if (b >= BINS) {                                       // the last place
        by_count = true;
        k = sh.count[BINS - 1];
        b = first_thread(holds && sh.count[bin] >= k, sh.s.n);
    }
    uint32_t before = b ? sh.count[b - 1] : 0, n = sh.count[b] - before;
    if (by_count && !index && sh.count[b] == k) return Place{k, sh.mass[b], 0.0, -1};
    const double base = b ? sh.mass[b - 1] : 0.0, unit = exp(-0.0625 * b) * UNIT;
    uint32_t klo = row.first_key(top - b), khi = row.template first_key<true>(top - b) - 1;
    uint64_t sum = 0;                                      // of the bin's elements in front of klo .. khi
    while (n > LIST && klo < khi) {
        const uint32_t span = khi - klo, shift = max(0, 22 - (int)__builtin_clz(span)), fine = (span >> shift) + 1;
        const float lo = value_of(klo), hi = value_of(khi);
        sh.list[tid] = 0;
        sh.fine[tid] = 0;
        __syncthreads();
        row.each([&](float v, int) {
            if (v >= lo && v <= hi) {
                const uint32_t at = fine - 1 - ((key_of(v) - klo) >> shift);
                const double z = grid(v, row.c, row.inf);
                atomicAdd(&sh.fine[at], 1u);
                atomicAdd((unsigned long long *)&sh.list[at], (unsigned long long)weight(z - floor(z)));
            }
        });
        __syncthreads();
        const uint32_t c = sh.fine[tid];
        const uint64_t m = sh.list[tid];
        const uint32_t cs = before + running_sum(c, sh.s.n);
        const uint64_t ms = sum + running_sum(m, sh.s.u);
        int f = first_thread(c && reached(cs, base + unit * (double)ms), sh.s.n);
        if (f >= LIST) {                                   // sums of the bins and of their parts differ in the last bits
            by_count = true;
            k = before + n;
            f = first_thread(c && cs >= k, sh.s.n);
        }
        if (tid == f) {
            sh.n = c;
            sh.s.n[0] = cs - c;
            sh.s.u[0] = ms - m;
        }
        __syncthreads();
        n = sh.n;
        before = sh.s.n[0];
        sum = sh.s.u[0];
        __syncthreads();
        const uint32_t from = klo + ((fine - 1 - (uint32_t)f) << shift);
        khi = min(khi, from + ((1u << shift) - 1));
        klo = from;
    }
    if (n <= LIST) {
        const uint64_t mine = gather(row, klo, khi, n, sh);
        const bool is = (uint32_t)tid < n;
        const double z = is ? grid(value_of(~(uint32_t)(mine >> 32)), row.c, row.inf) : 0.0;
        const uint32_t w = is ? weight(z - floor(z)) : 0;
        const double mass = base + unit * (double)(sum + running_sum((uint64_t)w, sh.s.u));
        int f = first_thread(is && reached(before + tid + 1, mass), sh.s.n);
        f = f < LIST ? f : (int)n - 1;
        if (tid == f) {
            sh.s.d[0] = mass;
            sh.s.d[1] = unit * w;
            sh.at = (int32_t)(uint32_t)mine;
        }
        __syncthreads();
        const Place r = {before + (uint32_t)f + 1, sh.s.d[0], sh.s.d[1], sh.at};
        __syncthreads();
        return r;
    }
    // all alike: the place by arithmetic, its index by counting in the order of the row
    const double z = grid(value_of(klo), row.c, row.inf);
    const uint32_t w = weight(z - floor(z));
    auto mass_at = [&](uint32_t i) { return base + unit * (double)(sum + (uint64_t)w * i); };
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
        const uint32_t upto = passed + running_sum(mine, sh.s.n);
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

template <typename T>
__global__ __launch_bounds__(LIST) void sample_row_kernel(SampleParams p) {
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = threadIdx.x;
    bool greedy;
    Row<T> row = {(const T *)p.logits + r * p.stride, p.vocab, grid_scale(p, r, greedy), false};
    const uint64_t *chunks = p.chunks + (int64_t)r * p.n_chunks * CHUNK_WORDS;
    float most = -INFINITY;
    double top = 0.0;
    int first = 0;
    for (int c = 0; c < p.n_chunks; ++c) {                 // the first chunk that has the maximum
        const uint64_t w = chunks[(int64_t)c * CHUNK_WORDS + 1];
        const float m = __builtin_bit_cast(float, (uint32_t)(w >> 32));
        if (m > most) {
            most = m;
            first = (int)(uint32_t)w;
            top = __builtin_bit_cast(double, chunks[(int64_t)c * CHUNK_WORDS]);
        }
    }
    if (greedy || most == -INFINITY) {
        if (tid == 0) {
            p.token[r] = most == -INFINITY ? 0 : first;
            if (p.prob) p.prob[r] = most == -INFINITY ? 0.f : 1.f;
        }
        return;
    }
    row.inf = most == INFINITY;

    // the chunks' bins, each from its own place on the grid on
    uint32_t count = 0;
    uint64_t mass = 0;
    if (tid < BINS)
        for (int c = 0; c < p.n_chunks; ++c) {
            const uint64_t *w = chunks + (int64_t)c * CHUNK_WORDS;
            const float m = __builtin_bit_cast(float, (uint32_t)(w[1] >> 32));
            if (m == -INFINITY || (row.inf && m < INFINITY)) continue;
            const double down = top - __builtin_bit_cast(double, w[0]);
            if (!(down <= (double)tid)) continue;
            const uint64_t bin = w[2 + tid - (int)down];
            count += (uint32_t)(bin >> COUNT_SHIFT);
            mass += bin & ((1ull << COUNT_SHIFT) - 1);
        }
    const double unit = exp(-0.0625 * tid) * UNIT;
    const uint32_t counts = running_sum(count, sh.s.n);
    const double masses = running_sum((double)mass * unit, sh.s.d);
    if (tid < BINS) {
        sh.count[tid] = counts;
        sh.mass[tid] = masses;
    }
    __syncthreads();
    const uint32_t all = sh.count[BINS - 1];

    const int32_t top_k = p.top_k ? p.top_k[r] : 0;
    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f, u = p.uniform[r];
    const uint32_t k = top_k > 0 ? min((uint32_t)top_k, all) : all;
    const double least = min_p > 0.f ? grid(most, row.c, row.inf) + 16.0 * log((double)min_p) : -INFINITY;
    const double uniform = u >= 0.f ? (double)u : 0.0;

    uint32_t kept = k;
    double left = k < all ? -1.0 : sh.mass[BINS - 1];      // mass of what top_k leaves, as soon as it is known
    auto last_bin = [&]() {                                // the bin in which the kept ones end at the latest
        const uint32_t n = tid < BINS ? sh.count[tid] : all;
        const double m = tid < BINS ? sh.mass[tid] : 0.0;
        const bool known = left >= 0.0 || !(top_p < 1.f);  // else all that top_k leaves is needed, for its mass
        return min(first_thread(n >= kept || (known && ((top_p < 1.f && n && m >= (double)top_p * left) || top - tid <= least)), sh.s.n), BINS - 1);
    };
    int b = last_bin();
    if (sh.count[b] > LIST && left < 0.0 && top_p < 1.f) {
        left = search(row, top, sh, true, k, 0.0, false, false).mass;
        b = last_bin();
    }
    const uint32_t n = sh.count[b];
    if (n <= LIST) {
        const uint64_t mine = gather(row, row.first_key(top - b), KEY_INF, n, sh);
        const bool is = (uint32_t)tid < n;
        const double z = is ? grid(value_of(~(uint32_t)(mine >> 32)), row.c, row.inf) : 0.0, f = floor(z);
        const double own = is ? exp(-0.0625 * (top - f)) * UNIT * weight(z - f) : 0.0;
        const double upto = running_sum(own, sh.s.d);
        double *sums = (double *)sh.list;                  // (the list is in registers now)
        sums[tid] = upto;
        __syncthreads();
        kept = min(kept, n);
        if (top_p < 1.f) {
            if (left < 0.0) left = sums[kept - 1];
            kept = min(kept, (uint32_t)first_thread(is && upto >= (double)top_p * left, sh.s.n) + 1u);
        }
        kept = min(kept, max(1u, total_count(is && z >= least, sh.s.n)));
        const double mass_kept = sums[kept - 1];
        const uint32_t at = min((uint32_t)first_thread(is && upto > uniform * mass_kept, sh.s.n), kept - 1);
        if ((uint32_t)tid == at) {
            p.token[r] = (int32_t)(uint32_t)mine;
            if (p.prob) p.prob[r] = (float)(own / mass_kept);
        }
        return;
    }
    double mass_kept = left;
    if (k < all && top_p >= 1.f) mass_kept = search(row, top, sh, true, k, 0.0, false, false).mass;
    if (top_p < 1.f) {
        const Place q = search(row, top, sh, false, 0, (double)top_p * left, false, false);
        if (q.count < kept) {
            kept = q.count;
            mass_kept = q.mass;
        }
    }
    if (min_p > 0.f) {
        const float lowest = value_of(min(row.first_key(least), KEY_INF));
        uint32_t mine = 0;
        if (least <= grid(most, row.c, row.inf)) row.each([&](float v, int) { mine += v >= lowest; });
        const uint32_t q = max(1u, total_count(mine, sh.s.n));
        if (q < kept) {
            kept = q;
            mass_kept = search(row, top, sh, true, kept, 0.0, false, false).mass;
        }
    }
    const double target = uniform * mass_kept;
    Place q = search(row, top, sh, !(target < mass_kept), kept, target, true, true);
    if (q.count > kept) q = search(row, top, sh, true, kept, 0.0, false, true);
    if (tid == 0) {
        p.token[r] = q.index;
        if (p.prob) p.prob[r] = (float)(q.own / mass_kept);
    }
}

// Threads of a workgroup of the first pass: small chunks while they are few (latency), larger ones where the bins they write would
// otherwise weigh as much as the logits
int bins_threads(int32_t rows, int32_t vocab) { return (int64_t)rows * ((vocab + 8191) / 8192) <= 1024 ? 256 : 1024; }
int chunks_of(const cascade_sample_desc *d) {
    const int chunk = chunk_of(bins_threads(d->rows, d->vocab));
    return (d->vocab + chunk - 1) / chunk;
}

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
    else hipLaunchKernelGGL((sample_bins_kernel<T, 1024>), grid, dim3(1024), 0, s, p);
    hipLaunchKernelGGL(sample_row_kernel<T>, dim3(rows), dim3(LIST), 0, s, p);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

}  // namespace

extern "C" size_t cascade_sample_workspace_bytes(const cascade_sample_desc *d) {
    if (check(d) != CASCADE_OK) return 0;
    return (size_t)d->rows * chunks_of(d) * CHUNK_WORDS * 8;
}

extern "C" int32_t cascade_sample(const cascade_sample_desc *d, const void *logits, const float *temperature, const int32_t *top_k,
                                  const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *prob,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    const int32_t st = check(d);
    if (st != CASCADE_OK) return st;
    if (d->rows == 0) return CASCADE_OK;
    if (!logits || !uniform || !token) return CASCADE_EINVAL;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < cascade_sample_workspace_bytes(d)) return CASCADE_EWORKSPACE;
    SampleParams p;
    p.logits = logits; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.uniform = uniform;
    p.token = token; p.prob = prob; p.chunks = (uint64_t *)workspace;
    p.stride = d->stride ? d->stride : d->vocab;
    p.vocab = d->vocab; p.n_chunks = chunks_of(d);
    const int threads = bins_threads(d->rows, d->vocab);
    return d->dtype == CASCADE_BF16 ? launch<bf16_t>(p, d->rows, threads, (hipStream_t)stream)
                                    : launch<float>(p, d->rows, threads, (hipStream_t)stream);
}
