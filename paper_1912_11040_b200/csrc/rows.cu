// Operators on the rows of a padded batch that feed a model's matrix products: root-mean-square norm with the addition
// of the residual stream and its gradient, and conversion to and from microscaled numbers (mx.cuh).
//
// All of them are passes over the data: a row is read once, kept in registers, and what leaves is written once.
#include <float.h>

#include <algorithm>

#include "mx.cuh"

namespace {

constexpr int MAX_WIDTH = AUG_MAX_NORM_WIDTH;     // 512 threads with 32 values each

// ---------------------------------------------------------------- who holds which values of a row
// TPR threads share a row, E values each.  VEC: eight neighbours at a time (128- or 256-bit accesses; four threads hold
// a block), for rows whose width is a multiple of 8 and that start on 16-byte boundaries.  Otherwise value e of
// thread l is column e TPR + l: a warp reads 32 neighbours, whatever the row's alignment, and its lanes hold a block.
template <int TPR, int E, bool VEC>
struct RowPart {
    static constexpr int THREADS = TPR > 32 ? TPR : 256;
    static constexpr int ROWS = THREADS / TPR;           // rows a CTA works on at a time
    static __device__ __forceinline__ int column(int l, int e) { return VEC ? ((e >> 3) * TPR + l) * 8 + (e & 7) : e * TPR + l; }
    template <typename T>
    static __device__ __forceinline__ void load(const T *row, int l, int D, bool valid, float *v) {
        if constexpr (VEC) {
#pragma unroll
            for (int c = 0; c < E / 8; ++c) {
                const int col = (c * TPR + l) * 8;
                if (valid && col < D)
                    mx::load8(row + col, v + 8 * c);
                else
                    for (int i = 0; i < 8; ++i) v[8 * c + i] = 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = valid && e * TPR + l < D ? mx::load1(row + e * TPR + l) : 0.f;
        }
    }
    template <typename T>
    static __device__ __forceinline__ void store(T *row, int l, int D, const float *v) {
        if constexpr (VEC) {
#pragma unroll
            for (int c = 0; c < E / 8; ++c) {
                const int col = (c * TPR + l) * 8;
                if (col < D) mx::store8(row + col, v + 8 * c);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e * TPR + l < D) mx::store1(row + e * TPR + l, v[e]);
        }
    }
    // Sum over the threads of a row, the same value in all of them.  `red`: TPR / 32 floats of shared memory.
    static __device__ __forceinline__ float sum(float s, float *red) {
#pragma unroll
        for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        if constexpr (TPR > 32) {
            __syncthreads();                             // the last sum has been read
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
            __syncthreads();
            s = 0.f;
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w) s += red[w];
        }
        return s;
    }
};

// A row of values as microscaled codes and scales, up to the padded width 128 G.
template <int TPR, int E, bool VEC>
__device__ __forceinline__ void store_mx(const float *v, int l, int G, bool four, uint8_t *codes, uint8_t *scales) {
    const int emax = four ? mx::EMAX_E2M1 : mx::EMAX_E4M3;
    if constexpr (VEC) {
#pragma unroll
        for (int c = 0; c < E / 8; ++c) {
            const int chunk = c * TPR + l;               // eight values; 16 chunks to a group
            const float *u = v + 8 * c;
            unsigned a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) a = max(a, mx::abs_bits(u[i]));
            a = max(a, __shfl_xor_sync(~0u, a, 1));
            a = max(a, __shfl_xor_sync(~0u, a, 2));
            const unsigned byte = mx::scale_byte(a, emax);
            const float inv = mx::inverse_scale(byte);
            float q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = byte == 255u ? 0.f : u[i] * inv;
            // the four scales of a group in its first thread
            unsigned s = byte;
            s |= __shfl_down_sync(~0u, s, 4) << 8;
            s |= __shfl_down_sync(~0u, s, 8) << 16;
            if (chunk < 16 * G) {
                if (four)
                    reinterpret_cast<unsigned *>(codes)[chunk] = mx::pack8_e2m1(q);
                else
                    reinterpret_cast<uint2 *>(codes)[chunk] =
                        make_uint2(mx::pack4_e4m3(q[0], q[1], q[2], q[3]), mx::pack4_e4m3(q[4], q[5], q[6], q[7]));
                if ((chunk & 15) == 0) reinterpret_cast<unsigned *>(scales)[chunk >> 4] = s;
            }
        }
    } else {
        const int lane = l & 31;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int block = (e * TPR + l) >> 5;        // a warp's
            const unsigned byte = mx::scale_byte(__reduce_max_sync(~0u, mx::abs_bits(v[e])), emax);
            const float q = byte == 255u ? 0.f : v[e] * mx::inverse_scale(byte);
            const float q1 = __shfl_down_sync(~0u, q, 1), q2 = __shfl_down_sync(~0u, q, 2), q3 = __shfl_down_sync(~0u, q, 3);
            if (block < 4 * G && (lane & 3) == 0) {
                if (four) {
                    const float u[8] = {q, q1, q2, q3, 0.f, 0.f, 0.f, 0.f};
                    reinterpret_cast<unsigned short *>(codes)[8 * block + (lane >> 2)] = (unsigned short)mx::pack8_e2m1(u);
                } else {
                    reinterpret_cast<unsigned *>(codes)[8 * block + (lane >> 2)] = mx::pack4_e4m3(q, q1, q2, q3);
                }
                if (lane == 0) scales[block] = (uint8_t)byte;
            }
        }
    }
    // groups that the threads' columns do not reach: a narrow row's padding
    const int words = four ? 16 : 32;                    // 32-bit words of a group
    for (int i = (TPR * E / mx::GROUP) * words + l; i < G * words; i += TPR) reinterpret_cast<unsigned *>(codes)[i] = 0;
    for (int g = TPR * E / mx::GROUP + l; g < G; g += TPR) reinterpret_cast<unsigned *>(scales)[g] = 0;
}

// ---------------------------------------------------------------- y = h / sqrt(mean(h^2) + eps) w, h = x + r
struct NormArgs {
    const void *x, *r;
    const float *w;
    void *sum, *y;
    uint8_t *scales;
    int D, G, y_type;
    float eps, pad, inv_D;
};

// Bound by memory: every value read once, its row held in registers between the sum of squares and the product.  The
// norm is that of x + r in fp32, before the sum is rounded to be stored.
template <typename T, int TPR, int E, bool VEC>
__global__ void __launch_bounds__(RowPart<TPR, E, VEC>::THREADS)
rms_norm_kernel(NormArgs a, RowBatch batch) {
    using P = RowPart<TPR, E, VEC>;
    __shared__ float red[TPR > 32 ? TPR / 32 : 1];
    const int l = threadIdx.x % TPR, D = a.D;
    for (int base = blockIdx.x * P::ROWS; base < batch.rows; base += gridDim.x * P::ROWS) {
        const int row = base + (int)threadIdx.x / TPR;
        const bool valid = batch.holds(row);
        const int64_t at = (int64_t)row * D;
        float v[E];
        P::load(static_cast<const T *>(a.x) + at, l, D, valid, v);
        if (a.r) {
            float u[E];
            P::load(static_cast<const T *>(a.r) + at, l, D, valid, u);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += u[e];
        }
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss = fmaf(v[e], v[e], ss);
        ss = P::sum(ss, red);
        float rs = rsqrtf(fmaf(ss, a.inv_D, a.eps));
        // squares beyond fp32 (or values that are not finite): once more, scaled down
        const bool big = !(ss <= FLT_MAX);
        if (TPR <= 32 ? __any_sync(~0u, big) : big) {
            constexpr float DOWN = 0x1p-96f;
            float s2 = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) s2 = fmaf(v[e] * DOWN, v[e] * DOWN, s2);
            s2 = P::sum(s2, red);
            if (big) rs = rsqrtf(s2 * a.inv_D) * DOWN;
        }
        if (a.sum && row < batch.rows) {
            if (valid) {
                P::store(static_cast<T *>(a.sum) + at, l, D, v);
            } else {
                float p[E];
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = a.pad;
                P::store(static_cast<T *>(a.sum) + at, l, D, p);
            }
        }
        const bool mxo = a.y_type >= AUG_ELEM_MX8;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int col = P::column(l, e);
            v[e] = valid ? v[e] * rs * (a.w && col < D ? __ldg(a.w + col) : 1.f) : mxo ? 0.f : a.pad;
        }
        if (mxo) {
            // rows beyond the batch take part in the shuffles, with nothing to write
            const bool four = a.y_type == AUG_ELEM_MX4, in = row < batch.rows;
            store_mx<TPR, E, VEC>(v, l, in ? a.G : 0, four,
                                  static_cast<uint8_t *>(a.y) + (int64_t)row * a.G * (four ? 64 : 128),
                                  a.scales + (int64_t)row * a.G * 4);
        } else if (row < batch.rows) {
            if (a.y_type == AUG_ELEM_F32)
                P::store(static_cast<float *>(a.y) + at, l, D, v);
            else
                P::store(static_cast<__nv_bfloat16 *>(a.y) + at, l, D, v);
        }
    }
}

// ---------------------------------------------------------------- its gradients
// With n = h rs, rs = 1 / sqrt(mean(h^2) + eps), and the gradient dy of y = n w:
//   dh = rs (w dy - n mean(w dy n)) (+ the gradient that reaches h from elsewhere),   dw = sum over rows of dy n.
// One pass: a row's h and dy stay in registers between the two sums and the product, and every thread carries its
// columns' share of dw over all rows of its CTA.  The CTAs' shares go to `partial`, and a second kernel adds them
// in a fixed order: no atomics, the same result every time.
struct GradArgs {
    const void *h, *dy, *dsum;
    const float *w;
    void *dx;
    float *partial;
    int D;
    float eps, inv_D;
};
constexpr int GRAD_CTAS = 296;            // most CTAs, and rows of `partial`

template <typename T, int TPR, int E, bool VEC>
__global__ void __launch_bounds__(RowPart<TPR, E, VEC>::THREADS)
rms_norm_grad_kernel(GradArgs a, RowBatch batch) {
    using P = RowPart<TPR, E, VEC>;
    __shared__ float red[TPR > 32 ? TPR / 32 : 1];
    extern __shared__ float share[];                     // [D], where a CTA has several rows at a time
    const int l = threadIdx.x % TPR, D = a.D;
    float dw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = 0.f;
    for (int base = blockIdx.x * P::ROWS; base < batch.rows; base += gridDim.x * P::ROWS) {
        const int row = base + (int)threadIdx.x / TPR;
        const bool valid = batch.holds(row);
        const int64_t at = (int64_t)row * D;
        float h[E], g[E];
        P::load(static_cast<const T *>(a.h) + at, l, D, valid, h);
        P::load(static_cast<const T *>(a.dy) + at, l, D, valid, g);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss = fmaf(h[e], h[e], ss);
        const float rs = rsqrtf(fmaf(P::sum(ss, red), a.inv_D, a.eps));
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int col = P::column(l, e);
            const float n = h[e] * rs;
            dw[e] = fmaf(g[e], n, dw[e]);
            g[e] *= a.w && col < D ? __ldg(a.w + col) : 1.f;
            dot = fmaf(g[e], n, dot);
            h[e] = n;
        }
        dot = P::sum(dot, red) * a.inv_D;
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = rs * fmaf(-dot, h[e], g[e]);
        if (a.dsum) {
            P::load(static_cast<const T *>(a.dsum) + at, l, D, valid, h);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] += h[e];
        }
        if (row < batch.rows) P::store(static_cast<T *>(a.dx) + at, l, D, g);
    }
    float *mine = a.partial + (int64_t)blockIdx.x * D;
    if constexpr (P::ROWS == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (P::column(l, e) < D) mine[P::column(l, e)] = dw[e];
    } else {
        for (int s = 0; s < P::ROWS; ++s) {              // one row's threads after the other
            if ((int)threadIdx.x / TPR == s) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int col = P::column(l, e);
                    if (col < D) share[col] = s ? share[col] + dw[e] : dw[e];
                }
            }
            __syncthreads();
        }
        for (int col = threadIdx.x; col < D; col += P::THREADS) mine[col] = share[col];
    }
}

// dw[c] = sum of n shares: 32 columns and 8 parts of the shares a CTA
constexpr int ADD_PARTS = 8;
__global__ void __launch_bounds__(32 * ADD_PARTS)
add_shares_kernel(const float *partial, int n, int D, float *dw) {
    __shared__ float s[ADD_PARTS][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float a = 0.f;
    if (col < D)
#pragma unroll 8
        for (int i = part; i < n; i += ADD_PARTS) a += partial[(int64_t)i * D + col];
    s[part][lane] = a;
    __syncthreads();
    if (part == 0 && col < D) {
#pragma unroll
        for (int p = 1; p < ADD_PARTS; ++p) a += s[p][lane];
        dw[col] = a;
    }
}

// ---------------------------------------------------------------- microscaled numbers
// Sixteen threads convert a group of 128 values.  VEC: eight neighbours a thread; else column 32 j + lane.
constexpr int MX_THREADS = 256;
__device__ __forceinline__ int row_of(int64_t unit, int64_t units, const Divisor &by_G) {
    return units <= INT32_MAX ? by_G.of((int)unit) : (int)(unit / by_G.by);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(MX_THREADS)
mx_quantize_kernel(const T *x, uint8_t *codes, uint8_t *scales, int D, int G, bool four, Divisor by_G, RowBatch batch) {
    // units: groups of a row.  VEC: half a warp each, else a warp each
    constexpr int LANES = VEC ? 16 : 32, E = mx::GROUP / LANES;
    const int64_t units = (int64_t)batch.rows * G, step = (int64_t)gridDim.x * (MX_THREADS / LANES);
    const int l = threadIdx.x % LANES;
    for (int64_t base = (int64_t)blockIdx.x * (MX_THREADS / LANES); base < units; base += step) {
        const int64_t unit = base + threadIdx.x / LANES;
        const bool in = unit < units;
        const int row = in ? row_of(unit, units, by_G) : 0, g = in ? (int)(unit - (int64_t)row * G) : 0;
        const bool valid = in && batch.holds(row);
        float v[E];
        RowPart<LANES, E, VEC>::load(x + (int64_t)row * D + g * mx::GROUP, l, D - g * mx::GROUP, valid, v);
        store_mx<LANES, E, VEC>(v, l, in ? 1 : 0, four, codes + unit * (four ? 64 : 128), scales + unit * 4);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(MX_THREADS)
mx_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, T *x, int D, int G, bool four, float pad,
                     Divisor by_G, RowBatch batch) {
    constexpr int LANES = VEC ? 16 : 32, E = mx::GROUP / LANES;
    const int64_t units = (int64_t)batch.rows * G, step = (int64_t)gridDim.x * (MX_THREADS / LANES);
    const int l = threadIdx.x % LANES;
    for (int64_t unit = (int64_t)blockIdx.x * (MX_THREADS / LANES) + threadIdx.x / LANES; unit < units; unit += step) {
        const int row = row_of(unit, units, by_G), g = (int)(unit - (int64_t)row * G);
        float v[E];
        if (batch.holds(row)) {
            const uint8_t *c = codes + unit * (four ? 64 : 128);
            if constexpr (VEC) {
                if (four) {
                    mx::unpack8_e2m1(reinterpret_cast<const unsigned *>(c)[l], v);
                } else {
                    const uint2 q = reinterpret_cast<const uint2 *>(c)[l];
                    const unsigned w[4] = {q.x & 0xffffu, q.x >> 16, q.y & 0xffffu, q.y >> 16};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = mx::unpack2_e4m3((unsigned short)w[i]);
                        v[2 * i] = f.x;
                        v[2 * i + 1] = f.y;
                    }
                }
                const float s = mx::scale_value(scales[unit * 4 + (l >> 2)]);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= s;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = 32 * e + l;
                    float u[8];
                    if (four) {
                        mx::unpack8_e2m1((unsigned)c[i >> 1] >> (4 * (i & 1)), u);
                    } else {
                        u[0] = mx::unpack2_e4m3(c[i]).x;
                    }
                    v[e] = u[0] * mx::scale_value(scales[unit * 4 + e]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = pad;
        }
        RowPart<LANES, E, VEC>::store(x + (int64_t)row * D + g * mx::GROUP, l, D - g * mx::GROUP, v);
    }
}

// Threads that share a row, by its width: as few as hold it with 32 values each, so that most rows are read, summed
// and written by one warp, without a barrier.
template <typename T, bool VEC, typename F>
int by_width(int D, F f) {
    if constexpr (VEC) {
        if (D <= 128) return f.template operator()<T, 16, 8, true>();
        if (D <= 256) return f.template operator()<T, 32, 8, true>();
        if (D <= 512) return f.template operator()<T, 32, 16, true>();
        if (D <= 1024) return f.template operator()<T, 32, 32, true>();
        if (D <= 4096) return f.template operator()<T, 128, 32, true>();
        return f.template operator()<T, 512, 32, true>();
    } else {
        if (D <= 128) return f.template operator()<T, 32, 4, false>();
        if (D <= 256) return f.template operator()<T, 32, 8, false>();
        if (D <= 512) return f.template operator()<T, 32, 16, false>();
        if (D <= 1024) return f.template operator()<T, 32, 32, false>();
        if (D <= 4096) return f.template operator()<T, 128, 32, false>();
        return f.template operator()<T, 512, 32, false>();
    }
}
template <typename F>
int by_type_and_width(int type, bool vec, int D, F f) {
    if (type == AUG_ELEM_F32) return vec ? by_width<float, true>(D, f) : by_width<float, false>(D, f);
    return vec ? by_width<__nv_bfloat16, true>(D, f) : by_width<__nv_bfloat16, false>(D, f);
}

struct LaunchNorm {
    AugCtx *ctx;
    NormArgs a;
    RowBatch batch;
    template <typename T, int TPR, int E, bool VEC>
    int operator()() const {
        using P = RowPart<TPR, E, VEC>;
        const int ctas = (batch.rows + P::ROWS - 1) / P::ROWS;
        rms_norm_kernel<T, TPR, E, VEC><<<ctas, P::THREADS, 0, ctx->stream>>>(a, batch);
        return cudaGetLastError() == cudaSuccess ? AUG_OK : AUG_ECUDA;
    }
};

struct LaunchGrad {
    AugCtx *ctx;
    GradArgs a;
    RowBatch batch;
    int *ctas;
    template <typename T, int TPR, int E, bool VEC>
    int operator()() const {
        using P = RowPart<TPR, E, VEC>;
        *ctas = std::min((batch.rows + P::ROWS - 1) / P::ROWS, GRAD_CTAS);
        rms_norm_grad_kernel<T, TPR, E, VEC>
            <<<*ctas, P::THREADS, P::ROWS > 1 ? sizeof(float) * a.D : 0, ctx->stream>>>(a, batch);
        return cudaGetLastError() == cudaSuccess ? AUG_OK : AUG_ECUDA;
    }
};

// CTAs for `units` of work, `per` of them a CTA: enough to fill the device several times over
int mx_ctas(const AugCtx *ctx, int64_t units, int per) {
    return (int)std::min<int64_t>((units + per - 1) / per, (int64_t)ctx->sm_count * 8);
}

}  // namespace

extern "C" {

int64_t feat_mx_code_bytes(int mx_type, int D) {
    if (!is_mx_type(mx_type) || D < 1) return AUG_EINVAL;
    return (int64_t)mx::groups(D) * (mx_type == AUG_ELEM_MX4 ? 64 : 128);
}

int64_t feat_mx_scale_bytes(int D) { return D < 1 ? (int64_t)AUG_EINVAL : (int64_t)mx::groups(D) * 4; }

int64_t feat_rms_norm_partial_floats(int D) {
    return D < 1 || D > MAX_WIDTH ? (int64_t)AUG_EINVAL : (int64_t)GRAD_CTAS * D;
}

int feat_rms_norm(AugCtx *ctx, const void *x_dev, const void *residual_dev, int in_type, const float *weight_dev,
                  const int *frame_counts_dev, int B, int T_max, int D, float eps, void *sum_dev, void *y_dev, int y_type,
                  uint8_t *scales_dev) {
    bool none;
    const int rc = check_rows(ctx, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !y_dev || !is_row_type(in_type) || !(is_row_type(y_type) || is_mx_type(y_type))) return AUG_EINVAL;
    if (!(eps > 0.f) || !(eps <= FLT_MAX)) return AUG_EINVAL;
    if (is_mx_type(y_type) != (scales_dev != nullptr)) return AUG_EINVAL;
    if (D > MAX_WIDTH) return AUG_ECAP;
    const uintptr_t rows_at = (uintptr_t)x_dev | (uintptr_t)residual_dev | (uintptr_t)sum_dev;
    if (rows_at & (elem_bytes(in_type) - 1) || (uintptr_t)weight_dev & 3) return AUG_EINVAL;
    if (is_mx_type(y_type) ? !on16(y_dev) || !on16(scales_dev) : ((uintptr_t)y_dev & (elem_bytes(y_type) - 1)) != 0)
        return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && ((rows_at | (uintptr_t)y_dev) & 15) == 0;
    const NormArgs a = {x_dev, residual_dev, weight_dev, sum_dev, y_dev, scales_dev, D, mx::groups(D), y_type, eps,
                        ctx->cfg.pad_value, 1.f / (float)D};
    const RowBatch batch(frame_counts_dev, T_max, B);
    if (by_type_and_width(in_type, vec, D, LaunchNorm{ctx, a, batch}) != AUG_OK) return AUG_ECUDA;
    ctx->launches++;
    return AUG_OK;
}

int feat_rms_norm_grad(AugCtx *ctx, const void *h_dev, const void *dy_dev, const void *dsum_dev, int type,
                       const float *weight_dev, const int *frame_counts_dev, int B, int T_max, int D, float eps,
                       void *dx_dev, float *dweight_dev, float *partial_dev) {
    bool none;
    const int rc = check_rows(ctx, B, T_max, D, &none);
    if (rc != AUG_OK) return rc;
    if (D > MAX_WIDTH) return AUG_ECAP;
    if (!dweight_dev || (uintptr_t)dweight_dev & 3) return AUG_EINVAL;
    if (none) return cudaMemsetAsync(dweight_dev, 0, sizeof(float) * D, ctx->stream) == cudaSuccess ? AUG_OK : AUG_ECUDA;
    if (!h_dev || !dy_dev || !dx_dev || !partial_dev || !is_row_type(type)) return AUG_EINVAL;
    if (!(eps > 0.f) || !(eps <= FLT_MAX)) return AUG_EINVAL;
    const uintptr_t rows_at = (uintptr_t)h_dev | (uintptr_t)dy_dev | (uintptr_t)dsum_dev | (uintptr_t)dx_dev;
    if (rows_at & (elem_bytes(type) - 1) || ((uintptr_t)weight_dev | (uintptr_t)partial_dev) & 3) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && (rows_at & 15) == 0;
    const GradArgs a = {h_dev, dy_dev, dsum_dev, weight_dev, dx_dev, partial_dev, D, eps, 1.f / (float)D};
    const RowBatch batch(frame_counts_dev, T_max, B);
    int ctas = 0;
    if (by_type_and_width(type, vec, D, LaunchGrad{ctx, a, batch, &ctas}) != AUG_OK) return AUG_ECUDA;
    add_shares_kernel<<<(D + 31) / 32, 32 * ADD_PARTS, 0, ctx->stream>>>(partial_dev, ctas, D, dweight_dev);
    AUG_CUDA_OK(cudaGetLastError());
    ctx->launches += 2;
    return AUG_OK;
}

int feat_mx_quantize(AugCtx *ctx, const void *x_dev, int in_type, const int *frame_counts_dev, int B, int T_max, int D,
                     uint8_t *codes_dev, int mx_type, uint8_t *scales_dev) {
    bool none;
    const int rc = check_rows(ctx, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !codes_dev || !scales_dev || !is_row_type(in_type) || !is_mx_type(mx_type)) return AUG_EINVAL;
    if ((uintptr_t)x_dev & (elem_bytes(in_type) - 1) || !on16(codes_dev) || !on16(scales_dev)) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && on16(x_dev), four = mx_type == AUG_ELEM_MX4;
    const RowBatch batch(frame_counts_dev, T_max, B);
    const int G = mx::groups(D), per = MX_THREADS / (vec ? 16 : 32), ctas = mx_ctas(ctx, (int64_t)batch.rows * G, per);
    auto go = [&](auto kern, auto *x) {
        kern<<<ctas, MX_THREADS, 0, ctx->stream>>>(x, codes_dev, scales_dev, D, G, four, Divisor(G), batch);
    };
    if (in_type == AUG_ELEM_F32)
        go(vec ? mx_quantize_kernel<float, true> : mx_quantize_kernel<float, false>, static_cast<const float *>(x_dev));
    else
        go(vec ? mx_quantize_kernel<__nv_bfloat16, true> : mx_quantize_kernel<__nv_bfloat16, false>,
           static_cast<const __nv_bfloat16 *>(x_dev));
    AUG_CUDA_OK(cudaGetLastError());
    ctx->launches++;
    return AUG_OK;
}

int feat_mx_dequantize(AugCtx *ctx, const uint8_t *codes_dev, int mx_type, const uint8_t *scales_dev,
                       const int *frame_counts_dev, int B, int T_max, int D, void *x_dev, int out_type) {
    bool none;
    const int rc = check_rows(ctx, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !codes_dev || !scales_dev || !is_row_type(out_type) || !is_mx_type(mx_type)) return AUG_EINVAL;
    if ((uintptr_t)x_dev & (elem_bytes(out_type) - 1) || !on16(codes_dev) || !on16(scales_dev)) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && on16(x_dev), four = mx_type == AUG_ELEM_MX4;
    const RowBatch batch(frame_counts_dev, T_max, B);
    const int G = mx::groups(D), per = MX_THREADS / (vec ? 16 : 32), ctas = mx_ctas(ctx, (int64_t)batch.rows * G, per);
    auto go = [&](auto kern, auto *x) {
        kern<<<ctas, MX_THREADS, 0, ctx->stream>>>(codes_dev, scales_dev, x, D, G, four, ctx->cfg.pad_value, Divisor(G), batch);
    };
    if (out_type == AUG_ELEM_F32)
        go(vec ? mx_dequantize_kernel<float, true> : mx_dequantize_kernel<float, false>, static_cast<float *>(x_dev));
    else
        go(vec ? mx_dequantize_kernel<__nv_bfloat16, true> : mx_dequantize_kernel<__nv_bfloat16, false>,
           static_cast<__nv_bfloat16 *>(x_dev));
    AUG_CUDA_OK(cudaGetLastError());
    ctx->launches++;
    return AUG_OK;
}

}  // extern "C"
