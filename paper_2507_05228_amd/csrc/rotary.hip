// Rotary positions (cascade_rope), and the same on the way into a paged cache (cascade_paged_append).
//
// Bound by HBM: every element is read and written once.  A workgroup takes a few rows; its threads first form cosine and
// sine of every (row, pair) once, into LDS, so that the angle costs one evaluation for all heads of a row, then walk over
// (row, head) in 16-byte vectors.  The angle is position * f_i in turns, in double precision (32 bits of position times
// 53 bits of frequency leave the fraction of a turn exact to 2^-23 at the largest position); the fraction is reduced to an
// eighth of a turn either way before it is rounded to fp32, where the two power series below are exact to fp32.
// 8192 rows of 40 heads of 128, bf16 (0.168 GB): 27 us in a row, 35 with other inputs in between (4.8 TB/s); rows and keys of
// 4096 tokens on their way into a cache (0.1 GB): 17 us; four rows 3 us, nearly all of it launch and one load after another.
#include <type_traits>
#include "device_utils.h"
#include "paged.h"

namespace {

struct RotaryParams {
    const void *q; void *q_out;
    const void *k, *v; void *k_pages, *v_pages;            // the layer's pools
    const int32_t *positions, *slots;
    int64_t q_stride, q_out_stride, kv_stride;
    double log2_theta, inv_factor, low, inv_span, turns;   // turns: original_len / (2 pi)
    int32_t rows, H, Hkv, d, rot, ramp;
    int32_t page_shift;
    uint32_t n_slots;
    float amplitude;
    int32_t rows_per_wg;
};

constexpr int MAX_PAIRS = 256;
constexpr int MAX_ROWS = 8;                                // of a workgroup

// cos and sin of 2 pi x, x in turns
__device__ __forceinline__ void cos_sin_turns(double x, float &c, float &s) {
    const double quarter = rint(x * 4.0);
    const float y = (float)(x * 4.0 - quarter) * 1.57079632679489662f;     // |y| <= pi / 4 (x * 4 is exact)
    const float z = y * y;
    // Taylor series; the first terms left out are 2e-9 (sine) and 1e-10 (cosine) of the largest argument's value
    const float sn = fmaf(y * z, fmaf(z, fmaf(z, fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), y);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
    const double turn = quarter - 4.0 * floor(quarter * 0.25);
    const bool odd = turn == 1.0 || turn == 3.0, c_neg = turn == 1.0 || turn == 2.0, s_neg = turn >= 2.0;
    c = odd ? sn : cs;
    s = odd ? cs : sn;
    if (c_neg) c = -c;
    if (s_neg) s = -s;
}

template <typename T, int VEC> struct Vec { typedef T type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct Vec<T, 1> { typedef T type; };
template <typename V> __device__ __forceinline__ float elem(const V &v, int i) {
    if constexpr (std::is_same<V, float>::value || std::is_same<V, bf16_t>::value) return (float)v;
    else return (float)v[i];
}
template <typename V> __device__ __forceinline__ void set_elem(V &v, int i, float x) {
    if constexpr (std::is_same<V, float>::value || std::is_same<V, bf16_t>::value) v = (V)x;
    else v[i] = x;
}

// VEC: elements per access (16 bytes, or one where rows, heads or the rotated part are not made of such vectors)
template <typename T, int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
    typedef typename Vec<T, VEC>::type vec;
    __shared__ float cs[MAX_PAIRS], sn[MAX_PAIRS];         // of every (row, pair)
    __shared__ int32_t row_slot[MAX_ROWS];
    const int half = p.rot / 2;
    const int row0 = blockIdx.x * p.rows_per_wg, n_rows = min(p.rows_per_wg, p.rows - row0);
    for (int e = threadIdx.x; e < n_rows * half; e += 256) {
        const int r = e / half, i = e - r * half;
        double f = exp2(-2.0 * i / p.rot * p.log2_theta);
        if (p.ramp) {
            const double g = fmin(fmax((p.turns * f - p.low) * p.inv_span, 0.0), 1.0);
            f *= (1.0 - g) * p.inv_factor + g;
        } else f *= p.inv_factor;
        float c, s;
        cos_sin_turns((double)p.positions[row0 + r] * (f * 0.15915494309189533577), c, s);
        cs[e] = c * p.amplitude;
        sn[e] = s * p.amplitude;
    }
    if (p.slots)
        if ((int)threadIdx.x < n_rows) row_slot[threadIdx.x] = p.slots[row0 + threadIdx.x];
    __syncthreads();

    // element offset of a row's head in the pools; the slot is checked before
    auto page_offset = [&](int slot, int g) {
        const int page = slot >> p.page_shift, r = slot & ((1 << p.page_shift) - 1);
        return ((((int64_t)page * p.Hkv + g) << p.page_shift) + r) * p.d;
    };
    const int n_q = p.q ? p.H : 0, n_heads = n_q + p.Hkv;
    // Where head h of local row r is read and written; false: it is not stored
    auto at = [&](int r, int h, const T *&src, T *&dst) {
        const int64_t row = row0 + r;
        if (h < n_q) {
            src = (const T *)p.q + row * p.q_stride + (int64_t)h * p.d;
            dst = (T *)p.q_out + row * p.q_out_stride + (int64_t)h * p.d;
            return true;
        }
        const int slot = row_slot[r];
        if ((uint32_t)slot >= p.n_slots) return false;
        src = (const T *)p.k + row * p.kv_stride + (int64_t)(h - n_q) * p.d;
        dst = (T *)p.k_pages + page_offset(slot, h - n_q);
        return true;
    };
    // f(local row, head, unit) for every unit < n_units of every head, units of a head on neighbouring threads
    auto for_units = [&](int heads, int n_units, auto f) {
        if (heads <= 0 || n_units <= 0) return;
        const int lanes = min(n_units, 256), per = 256 / lanes, mine = threadIdx.x / lanes, u0 = threadIdx.x - mine * lanes;
        if (mine >= per) return;
        int r = mine / heads, h = mine - r * heads;
        const int dr = per / heads, dh = per - dr * heads;
        while (r < n_rows) {
            for (int u = u0; u < n_units; u += lanes) f(r, h, u);
            r += dr;
            h += dh;
            if (h >= heads) { h -= heads; ++r; }
        }
    };
    // rotated pairs
    if constexpr (!INTERLEAVED) {
        for_units(n_heads, half / VEC, [&](int r, int h, int u) {
            const T *src; T *dst;
            if (!at(r, h, src, dst)) return;
            const vec a = *(const vec *)(src + u * VEC), b = *(const vec *)(src + half + u * VEC);
            const float *c = cs + r * half + u * VEC, *s = sn + r * half + u * VEC;
            vec x, y;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                set_elem(x, i, elem(a, i) * c[i] - elem(b, i) * s[i]);
                set_elem(y, i, elem(a, i) * s[i] + elem(b, i) * c[i]);
            }
            *(vec *)(dst + u * VEC) = x;
            *(vec *)(dst + half + u * VEC) = y;
        });
    } else if constexpr (VEC > 1) {
        for_units(n_heads, p.rot / VEC, [&](int r, int h, int u) {
            const T *src; T *dst;
            if (!at(r, h, src, dst)) return;
            const vec a = *(const vec *)(src + u * VEC);
            const float *c = cs + r * half + u * (VEC / 2), *s = sn + r * half + u * (VEC / 2);
            vec x;
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
                x[2 * i] = (float)a[2 * i] * c[i] - (float)a[2 * i + 1] * s[i];
                x[2 * i + 1] = (float)a[2 * i] * s[i] + (float)a[2 * i + 1] * c[i];
            }
            *(vec *)(dst + u * VEC) = x;
        });
    } else {
        for_units(n_heads, half, [&](int r, int h, int u) {
            const T *src; T *dst;
            if (!at(r, h, src, dst)) return;
            const float a = (float)src[2 * u], b = (float)src[2 * u + 1], c = cs[r * half + u], s = sn[r * half + u];
            dst[2 * u] = (T)(a * c - b * s);
            dst[2 * u + 1] = (T)(a * s + b * c);
        });
    }
    // columns behind the rotated ones (queries in place have theirs already)
    const int skip = p.q == p.q_out ? n_q : 0;
    for_units(n_heads - skip, (p.d - p.rot) / VEC, [&](int r, int h, int u) {
        const T *src; T *dst;
        if (!at(r, h + skip, src, dst)) return;
        *(vec *)(dst + p.rot + u * VEC) = *(const vec *)(src + p.rot + u * VEC);
    });
    if (!p.slots) return;
    for_units(p.Hkv, p.d / VEC, [&](int r, int h, int u) {
        const int slot = row_slot[r];
        if ((uint32_t)slot >= p.n_slots) return;
        *(vec *)((T *)p.v_pages + page_offset(slot, h) + u * VEC) =
            *(const vec *)((const T *)p.v + (int64_t)(row0 + r) * p.kv_stride + (int64_t)h * p.d + u * VEC);
    });
}

int32_t set_rope(RotaryParams &p, const cascade_rope_desc *r, int32_t head_dim) {
    if (r->layout != CASCADE_ROPE_HALF && r->layout != CASCADE_ROPE_INTERLEAVED) return CASCADE_EINVAL;
    if (r->scaling != CASCADE_ROPE_UNSCALED && r->scaling != CASCADE_ROPE_LINEAR && r->scaling != CASCADE_ROPE_RAMP) return CASCADE_EINVAL;
    const auto above0 = [](double x) { return x > 0.0 && x <= 1e300; };    // (false for NaN)
    if (r->rot_dim <= 0 || !above0(r->theta) || !(r->amplitude >= -1e30 && r->amplitude <= 1e30)) return CASCADE_EINVAL;
    if (r->scaling != CASCADE_ROPE_UNSCALED && !above0(r->factor)) return CASCADE_EINVAL;
    if (r->scaling == CASCADE_ROPE_RAMP && !(r->original_len > 0 && r->low < r->high && r->low >= -1e30 && r->high <= 1e30)) return CASCADE_EINVAL;
    if (r->rot_dim % 2 || r->rot_dim > 2 * MAX_PAIRS) return CASCADE_EUNSUPPORTED;
    if (r->rot_dim > head_dim) return CASCADE_ESHAPE;
    p.rot = r->rot_dim;
    p.log2_theta = __builtin_log2(r->theta);
    p.inv_factor = r->scaling == CASCADE_ROPE_UNSCALED ? 1.0 : 1.0 / r->factor;
    p.ramp = r->scaling == CASCADE_ROPE_RAMP;
    p.low = r->low;
    p.inv_span = p.ramp ? 1.0 / (r->high - r->low) : 0.0;
    p.turns = p.ramp ? r->original_len * 0.15915494309189533577 : 0.0;
    p.amplitude = (float)r->amplitude;
    return CASCADE_OK;
}

template <typename T>
int32_t launch_rotary(RotaryParams p, bool interleaved, uintptr_t alignment, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(T);
    // Vectors of 16 bytes where every row, head and rotated part begins and ends on one
    const bool wide = alignment % 16 == 0 && p.q_stride % VEC == 0 && p.q_out_stride % VEC == 0 && p.kv_stride % VEC == 0 &&
                      p.d % VEC == 0 && (interleaved ? p.rot % VEC == 0 : (p.rot / 2) % VEC == 0);
    // Rows of a workgroup: enough workgroups for the 256 CUs first, then as many rows as share one evaluation of the angles
    const int most = p.rot ? max(1, min(MAX_ROWS, 2 * MAX_PAIRS / p.rot)) : MAX_ROWS;
    p.rows_per_wg = max(1, min(most, p.rows / 1024));
    // A launch has less than 2^32 threads: 2^23 workgroups' rows at a time
    const auto moved = [](auto *x, int64_t elems) { return x ? (decltype(x))((const T *)x + elems) : x; };
    const int64_t at_once = (int64_t)p.rows_per_wg << 23;
    for (int64_t first = 0; first < p.rows; first += at_once) {
        RotaryParams c = p;
        c.rows = (int32_t)min(at_once, p.rows - first);
        c.q = moved(p.q, first * p.q_stride);
        c.q_out = moved(p.q_out, first * p.q_out_stride);
        c.k = moved(p.k, first * p.kv_stride);
        c.v = moved(p.v, first * p.kv_stride);
        if (p.positions) c.positions = p.positions + first;
        if (p.slots) c.slots = p.slots + first;
        const dim3 grid((unsigned)(((int64_t)c.rows + p.rows_per_wg - 1) / p.rows_per_wg));
        if (wide && interleaved) hipLaunchKernelGGL((rotary_kernel<T, VEC, true>), grid, dim3(256), 0, s, c);
        else if (wide) hipLaunchKernelGGL((rotary_kernel<T, VEC, false>), grid, dim3(256), 0, s, c);
        else if (interleaved) hipLaunchKernelGGL((rotary_kernel<T, 1, true>), grid, dim3(256), 0, s, c);
        else hipLaunchKernelGGL((rotary_kernel<T, 1, false>), grid, dim3(256), 0, s, c);
        CASCADE_HIP_TRY(hipGetLastError());
    }
    return CASCADE_OK;
}

}   // namespace

extern "C" int32_t cascade_rope(const cascade_rope_desc *desc, int32_t dtype, int32_t rows, int32_t n_heads, int32_t head_dim,
                                const int32_t *positions_dev, const void *x, int64_t x_stride, void *y, int64_t y_stride,
                                void *stream) {
    if (!desc || !positions_dev || !x || !y || rows <= 0 || n_heads <= 0 || head_dim <= 0 || x_stride < 0 || y_stride < 0) return CASCADE_EINVAL;
    if (dtype != CASCADE_F32 && dtype != CASCADE_BF16) return CASCADE_EUNSUPPORTED;
    RotaryParams p = {};
    const int32_t st = set_rope(p, desc, head_dim);
    if (st != CASCADE_OK) return st;
    const int64_t row = (int64_t)n_heads * head_dim;
    if (row > INT32_MAX) return CASCADE_EUNSUPPORTED;
    p.q = x; p.q_out = y;
    p.q_stride = x_stride ? x_stride : row;
    p.q_out_stride = y_stride ? y_stride : row;
    if (p.q_stride < row || p.q_out_stride < row || (x == y && p.q_stride != p.q_out_stride)) return CASCADE_ESHAPE;
    p.positions = positions_dev;
    p.rows = rows; p.H = n_heads; p.d = head_dim;
    const uintptr_t alignment = (uintptr_t)x | (uintptr_t)y;
    const bool interleaved = desc->layout == CASCADE_ROPE_INTERLEAVED;
    return dtype == CASCADE_BF16 ? launch_rotary<bf16_t>(p, interleaved, alignment, (hipStream_t)stream)
                                 : launch_rotary<float>(p, interleaved, alignment, (hipStream_t)stream);
}

extern "C" int32_t cascade_paged_append(const cascade_paged_cache *cache, int32_t layer, int32_t rows, const int32_t *slots_dev,
                                        const void *k, const void *v, int64_t kv_stride, const cascade_rope_desc *rope,
                                        const int32_t *positions_dev, int32_t n_heads, const void *q, int64_t q_stride,
                                        void *q_out, int64_t q_out_stride, void *stream) {
    int32_t st = check_paged_cache(cache);
    if (st != CASCADE_OK) return st;
    if (!slots_dev || !k || !v || rows <= 0 || kv_stride < 0 || q_stride < 0 || q_out_stride < 0 || n_heads < 0) return CASCADE_EINVAL;
    if (!rope != !positions_dev || !q != !q_out || (q && (!rope || n_heads == 0))) return CASCADE_EINVAL;
    if (layer < 0 || layer >= cache->n_layers) return CASCADE_ESHAPE;
    RotaryParams p = {};
    if (rope && (st = set_rope(p, rope, cache->head_dim)) != CASCADE_OK) return st;
    const int es = cache->dtype == CASCADE_BF16 ? 2 : 4;
    const int64_t kv_row = (int64_t)cache->n_kv_heads * cache->head_dim, q_row = (int64_t)n_heads * cache->head_dim;
    if (kv_row > INT32_MAX || q_row > INT32_MAX) return CASCADE_EUNSUPPORTED;
    p.k = k; p.v = v;
    p.kv_stride = kv_stride ? kv_stride : kv_row;
    if (p.kv_stride < kv_row) return CASCADE_ESHAPE;
    if (q) {
        p.q = q; p.q_out = q_out;
        p.q_stride = q_stride ? q_stride : q_row;
        p.q_out_stride = q_out_stride ? q_out_stride : q_row;
        if (p.q_stride < q_row || p.q_out_stride < q_row || (q == q_out && p.q_stride != p.q_out_stride)) return CASCADE_ESHAPE;
    }
    p.k_pages = (char *)cache->k_pages + layer * layer_elems(cache) * es;
    p.v_pages = (char *)cache->v_pages + layer * layer_elems(cache) * es;
    p.positions = positions_dev; p.slots = slots_dev;
    p.rows = rows; p.H = q ? n_heads : 0; p.Hkv = cache->n_kv_heads; p.d = cache->head_dim;
    p.page_shift = page_shift(cache);
    p.n_slots = (uint32_t)cache->n_pages << p.page_shift;
    const uintptr_t alignment = (uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out;
    const bool interleaved = rope && rope->layout == CASCADE_ROPE_INTERLEAVED;
    return cache->dtype == CASCADE_BF16 ? launch_rotary<bf16_t>(p, interleaved, alignment, (hipStream_t)stream)
                                        : launch_rotary<float>(p, interleaved, alignment, (hipStream_t)stream);
}
