// The residual's addition, the norm behind it and the norm's result in 8 bits, in one pass (cascade_add_norm).
//
// Bound by HBM: every element is read once, every result written once.  A workgroup holds a row in registers, 8 neighbouring
// columns a thread and step (16-byte requests in bf16), so that the statistics, the largest magnitude of a group and the
// quantisation need no second read; the columns' scales of a group lie in neighbouring lanes of one wavefront and meet by lane
// exchanges, the sums of a row in LDS.  The layer norm takes the mean first and the squares of the distances from it then.
// Measured: 8192 rows of 4096 with delta, sum and int8 in bf16 50 us (4.6 TB/s; a large copy 5.1), 64 rows of 8192 5.3, one row 3.4.
#include <algorithm>
#include <type_traits>
#include "common.h"
#include "device_utils.h"

namespace {

struct AddNormParams {
    const void *x, *delta, *gain, *bias;
    void *sum, *y;
    uint8_t *q;
    float *q_scale;
    int64_t x_stride, delta_stride, sum_stride, y_stride, q_stride;
    int32_t rows, D;
    int32_t group_lanes;                                   // lanes of a scale; 0: the row
    int32_t n_scales;                                      // of a row
    float eps, inv_D;
};

constexpr int PER = 8;                                     // neighbouring columns of a thread
constexpr int MAX_WAVES = 16;

// 8 columns with no alignment but the element's (the memory unit takes 16-byte requests at any address), as the words they came in
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Columns {
    uint32_t w[PER * sizeof(T) / 4];
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[e]);
        else return __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
};

// Columns c .. c + 7 of a row of D; past the row's end zeros.  Whole pieces are requested without a branch (lanes that have
// none ask for the row's first columns), so that the requests of a thread go out together.
template <typename T>
__device__ __forceinline__ Columns<T> load_columns(const T *row, int c, int D) {
    Columns<T> r;
    if (D >= PER) r = *(const Columns<T> *)(row + (D - c >= PER ? c : 0));
    return r;
}
// ... and what a piece that ends inside has to be mended by
template <typename T>
__device__ __forceinline__ void mend_columns(const T *row, int c, int D, Columns<T> &r) {
    if (D - c < PER) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(r.w) / 4; ++i) r.w[i] = 0;
        constexpr int BITS = 8 * sizeof(T);
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (c + e < D) {
                if constexpr (sizeof(T) == 4) r.w[e] = __builtin_bit_cast(uint32_t, row[c + e]);
                else r.w[e >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, row[c + e]) << (e & 1 ? BITS : 0);
            }
    }
}
template <typename T>
__device__ __forceinline__ void store_columns(T *p, int n, const float (&v)[PER]) {
    if (n >= PER) {
        Columns<T> c;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < PER; ++e) c.w[e] = __builtin_bit_cast(uint32_t, v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < PER; e += 2) c.w[e >> 1] = __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)v[e], (bf16_t)v[e + 1]});
        }
        *(Columns<T> *)p = c;
    } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (e < n) p[e] = (T)v[e];
    }
}

// Sums and maxima over the workgroup.  `slot` must differ from that of the exchange before.
__device__ __forceinline__ float group_sum(float v, float (*slots)[MAX_WAVES], int slot) {
    v = wave_sum(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[slot][threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += slots[slot][w];
    return s;
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
    for (int o = 1; o < lanes; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, WAVE));
    return v;
}
__device__ __forceinline__ uint32_t group_max(uint32_t v, float (*slots)[MAX_WAVES], int slot) {
    v = lanes_max(v, WAVE);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[slot][threadIdx.x >> 6] = __builtin_bit_cast(float, v);
    __syncthreads();
    uint32_t s = 0;
    for (int w = 0; w < waves; ++w) s = max(s, __builtin_bit_cast(uint32_t, slots[slot][w]));
    return s;
}

// NV: steps of blockDim.x * 8 columns that a row takes
template <typename T, int NV, bool LAYER, int FORMAT>
__global__ __launch_bounds__(1024) void add_norm_kernel(AddNormParams p) {
    __shared__ float slots[4][MAX_WAVES];
    int slot = 0;
    const int step = blockDim.x * PER;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        int c0 = threadIdx.x * PER;
        // Places in the row anew for each one: kept for all of them, they take registers that spill (2048 rows of 32768, sum and
        // int8: bf16 142 -> 114 us, fp32, with fewer steps requested together, 363 -> 198)
        if constexpr (NV == 4) asm volatile("" : "+v"(c0));
        const T *x = (const T *)p.x + row * p.x_stride, *delta = (const T *)p.delta + row * p.delta_stride;
        constexpr int AT_ONCE = NV == 4 && sizeof(T) == 4 ? 2 : NV;              // steps requested together: what registers hold
        Columns<T> xs[AT_ONCE], ds[AT_ONCE], gs[NV], bs[NV];
        auto request = [&](int from) {
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                xs[j] = load_columns(x, c0 + (from + j) * step, p.D);
                if (p.delta) ds[j] = load_columns(delta, c0 + (from + j) * step, p.D);
            }
        };
        request(0);
        if constexpr (NV == 1) {                           // early where registers allow: one wait less for short launches
            gs[0] = load_columns((const T *)p.gain, c0, p.D);
            if (p.bias) bs[0] = load_columns((const T *)p.bias, c0, p.D);
        }
        float s[NV][PER];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = j % AT_ONCE;
            if (j && k == 0) {
                __builtin_amdgcn_sched_barrier(0);
                request(j);
            }
            mend_columns(x, c0 + j * step, p.D, xs[k]);
            if (p.delta) mend_columns(delta, c0 + j * step, p.D, ds[k]);
#pragma unroll
            for (int e = 0; e < PER; ++e) s[j][e] = xs[k][e] + (p.delta ? ds[k][e] : 0.f);
        }
        if (p.sum) {
#pragma unroll
            for (int j = 0; j < NV; ++j) store_columns((T *)p.sum + row * p.sum_stride + c0 + j * step, p.D - c0 - j * step, s[j]);
        }
        if constexpr (LAYER) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < PER; ++e) t += s[j][e];
            const float mean = group_sum(t, slots, slot++ & 3) * p.inv_D;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < PER; ++e) s[j][e] = c0 + j * step + e < p.D ? s[j][e] - mean : 0.f;
        }
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < PER; ++e) t = fmaf(s[j][e], s[j][e], t);
        const float r = 1.0f / sqrtf(group_sum(t, slots, slot++ & 3) * p.inv_D + p.eps);
        uint32_t largest[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = c0 + j * step, n = p.D - c;
            if constexpr (NV > 1) {
                gs[j] = load_columns((const T *)p.gain, c, p.D);
                if (p.bias) bs[j] = load_columns((const T *)p.bias, c, p.D);
            }
            mend_columns((const T *)p.gain, c, p.D, gs[j]);
            if (p.bias) mend_columns((const T *)p.bias, c, p.D, bs[j]);
            largest[j] = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                s[j][e] = fmaf(s[j][e] * r, gs[j][e], p.bias ? bs[j][e] : 0.f);
                // magnitudes order as whole numbers, infinities and then NaN above them all
                largest[j] = max(largest[j], __builtin_bit_cast(uint32_t, s[j][e]) & 0x7fffffffu);
            }
            if (p.y) store_columns((T *)p.y + row * p.y_stride + c, n, s[j]);
        }
        if constexpr (FORMAT != CASCADE_Q8_NONE) {
            if (p.group_lanes) {
#pragma unroll
                for (int j = 0; j < NV; ++j) largest[j] = lanes_max(largest[j], p.group_lanes);
            } else {
#pragma unroll
                for (int j = 1; j < NV; ++j) largest[0] = max(largest[0], largest[j]);
                largest[0] = group_max(largest[0], slots, slot++ & 3);
#pragma unroll
                for (int j = 1; j < NV; ++j) largest[j] = largest[0];
            }
            constexpr float MOST = FORMAT == CASCADE_Q8_INT8 ? 127.f : 448.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = c0 + j * step, n = p.D - c;
                const bool finite = largest[j] < 0x7f800000u;
                const float scale = finite ? fmaxf(__builtin_bit_cast(float, largest[j]) / MOST, 0x1p-100f) : __builtin_nanf("");
                const float inv = finite ? 1.0f / scale : 0.f;
                if (p.group_lanes) {
                    if (n > 0 && (threadIdx.x & (p.group_lanes - 1)) == 0) p.q_scale[row * p.n_scales + c / (p.group_lanes * PER)] = scale;
                } else if (c == 0) p.q_scale[row] = scale;
                uint32_t w[2] = {0, 0};
                if (finite) {
                    if constexpr (FORMAT == CASCADE_Q8_INT8) {
#pragma unroll
                        for (int e = 0; e < PER; ++e)
                            w[e >> 2] |= ((uint32_t)(int)rintf(fminf(fmaxf(s[j][e] * inv, -MOST), MOST)) & 255u) << (8 * (e & 3));
                    } else {
                        float v[PER];
#pragma unroll
                        for (int e = 0; e < PER; ++e) v[e] = fminf(fmaxf(s[j][e] * inv, -MOST), MOST);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
                            w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w[h], true);
                        }
                    }
                }
                uint8_t *q = p.q + row * p.q_stride + c;
                if (n >= PER) {
                    Columns<uint8_t> out;
                    out.w[0] = w[0];
                    out.w[1] = w[1];
                    *(Columns<uint8_t> *)q = out;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (e < n) q[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        }
    }
}

template <typename T, int NV, bool LAYER>
void launch(const AddNormParams &p, int format, int threads, int groups, hipStream_t s) {
    if (format == CASCADE_Q8_INT8)
        hipLaunchKernelGGL((add_norm_kernel<T, NV, LAYER, CASCADE_Q8_INT8>), dim3(groups), dim3(threads), 0, s, p);
    else if (format == CASCADE_Q8_E4M3)
        hipLaunchKernelGGL((add_norm_kernel<T, NV, LAYER, CASCADE_Q8_E4M3>), dim3(groups), dim3(threads), 0, s, p);
    else
        hipLaunchKernelGGL((add_norm_kernel<T, NV, LAYER, CASCADE_Q8_NONE>), dim3(groups), dim3(threads), 0, s, p);
}

template <typename T, bool LAYER>
int32_t launch_rows(const AddNormParams &p, int format, hipStream_t s) {
    const int chunks = (p.D + PER - 1) / PER, threads = std::min(1024, (chunks + 63) / 64 * 64);
    const int steps = (chunks + threads - 1) / threads;
    const int groups = std::min(p.rows, 1 << 20);          // a launch counts its threads in 32 bits
    if (steps == 1) launch<T, 1, LAYER>(p, format, threads, groups, s);
    else if (steps == 2) launch<T, 2, LAYER>(p, format, threads, groups, s);
    else launch<T, 4, LAYER>(p, format, threads, groups, s);
    CASCADE_HIP_TRY(hipGetLastError());
    return CASCADE_OK;
}

}  // namespace

extern "C" int32_t cascade_add_norm(const cascade_add_norm_desc *d, const void *x, const void *delta, const void *gain, const void *bias,
                                    void *sum, void *y, void *q, float *q_scale, void *stream) {
    if (!d) return CASCADE_EINVAL;
    if (d->rows > 0 && (!x || !gain || (!sum && !y && !q) || !q != !q_scale || !q != (d->q_format == CASCADE_Q8_NONE))) return CASCADE_EINVAL;
    if (d->rows < 0 || d->d_model <= 0 || d->q_group < 0 || d->q_format < 0 || d->q_format > CASCADE_Q8_E4M3) return CASCADE_EINVAL;
    if (d->norm_kind != CASCADE_NORM_LAYERNORM && d->norm_kind != CASCADE_NORM_RMSNORM) return CASCADE_EINVAL;
    if (d->x_stride < 0 || d->delta_stride < 0 || d->sum_stride < 0 || d->y_stride < 0 || d->q_stride < 0) return CASCADE_EINVAL;
    if (sum && sum == y) return CASCADE_EINVAL;
    if (q && (q == x || q == delta || q == sum || q == y)) return CASCADE_EINVAL;
    if (d->dtype != CASCADE_F32 && d->dtype != CASCADE_BF16) return CASCADE_EUNSUPPORTED;
    if (d->d_model > PER * 4 * 1024) return CASCADE_EUNSUPPORTED;
    const int group = d->q_format ? d->q_group : 0;
    if (group && group != 32 && group != 64 && group != 128 && group != 256) return CASCADE_EUNSUPPORTED;
    if (group && d->d_model % group) return CASCADE_ESHAPE;
    AddNormParams p = {};
    p.x = x; p.delta = delta; p.gain = gain; p.bias = bias; p.sum = sum; p.y = y; p.q = (uint8_t *)q; p.q_scale = q_scale;
    p.D = d->d_model; p.rows = d->rows; p.eps = d->eps; p.inv_D = (float)(1.0 / d->d_model);
    p.x_stride = d->x_stride ? d->x_stride : p.D;
    p.delta_stride = d->delta_stride ? d->delta_stride : p.D;
    p.sum_stride = d->sum_stride ? d->sum_stride : p.D;
    p.y_stride = d->y_stride ? d->y_stride : p.D;
    p.q_stride = d->q_stride ? d->q_stride : p.D;
    if (std::min({p.x_stride, p.delta_stride, p.sum_stride, p.y_stride, p.q_stride}) < p.D) return CASCADE_ESHAPE;
    for (const auto &o : {std::pair<void *, int64_t>(sum, p.sum_stride), std::pair<void *, int64_t>(y, p.y_stride)})
        if (o.first && ((o.first == x && o.second != p.x_stride) || (o.first == delta && o.second != p.delta_stride))) return CASCADE_ESHAPE;
    p.group_lanes = group / PER;
    p.n_scales = group ? p.D / group : 1;
    if (p.rows == 0) return CASCADE_OK;
    const bool layer = d->norm_kind == CASCADE_NORM_LAYERNORM;
    hipStream_t s = (hipStream_t)stream;
    if (d->dtype == CASCADE_BF16) return layer ? launch_rows<bf16_t, true>(p, d->q_format, s) : launch_rows<bf16_t, false>(p, d->q_format, s);
    return layer ? launch_rows<float, true>(p, d->q_format, s) : launch_rows<float, false>(p, d->q_format, s);
}
