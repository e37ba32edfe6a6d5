// Operators on the rows of a padded batch that feed a model's matrix products: root-mean-square norm with the addition
// of the residual stream and its gradient, and conversion to and from microscaled numbers (mx.cuh).
//
// All of them are passes over the data: a row is read once, kept in registers, and what leaves is written once.  Their
// kernels are chained to the ones before (chain_wait), but none lets a caller's next one start early: that may read
// through the non-coherent path what they write, as the features' kernels do.  Calls back to back: norm of
// 64 x 1998 x 80 14.3 -> 12.4 us, gradient of 64 x 998 x 1024 75 -> 73, 128 x 375 x 640 quantised and back 39.5 -> 34.8.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "mx.cuh"

namespace {

constexpr int MAX_WIDTH = AUG_MAX_NORM_WIDTH;     // 512 threads with 32 values each

// A gain, which an earlier kernel may have written: read behind chain_wait, and not through the non-coherent path.  (As a
// plain load, which the compiler keeps in order with the row's stores, it costs registers: norm of 64 x 1998 x 1024 to 8
// bits 141 us for 137.)
__device__ __forceinline__ float load_gain(const float *w) {
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(w));
    return v;
}

// ---------------------------------------------------------------- who holds which values of a row
// TPR threads share a row, E values each.  VEC: eight neighbours at a time (128-bit accesses), for rows whose width is
// a multiple of 8 and that start on 16-byte boundaries.  Otherwise value e of thread l is column e TPR + l: a warp
// reads 32 neighbours, whatever the row's alignment.
template <typename T, int TPR, int E, bool VEC>
struct RowPart {
    static constexpr int THREADS = TPR <= 256 ? 256 : TPR;
    static constexpr int ROWS = THREADS / TPR;           // rows a CTA works on at a time
    static constexpr int STEP = VEC ? 8 : 1, STEPS = E / STEP;       // values that are accessed together
    // CTAs a multiprocessor of the norm and of its gradient, by the registers that they take
    static constexpr int norm_ctas() {
        return TPR > 256 ? 1 : E <= 4 ? 4 : E <= 8 ? (!VEC ? 3 : sizeof(T) == 4 ? 4 : 5) : (VEC && E <= 16 && (sizeof(T) == 2 || TPR == 8)) || (!VEC && E <= 12) ? 3 : 2;
    }
    static constexpr int grad_ctas() { return TPR > 256 || E > 16 ? 1 : E <= 4 || (VEC && E <= 8 && TPR <= 32) || (!VEC && E == 12 && sizeof(T) == 4) ? 3 : 2; }
    static __device__ __forceinline__ int column(int l, int step) { return (step * TPR + l) * STEP; }

    // Values as they were read, so that the next row's can be on their way in few registers.  What lies beyond the row's
    // width is zero from the start, and nothing but a row that holds values is read into the rest.
    struct Raw {
        uint4 q[VEC ? E * sizeof(T) / 16 : 1];
        unsigned s[VEC ? 1 : E];                         // (the bits of one value each)
        __device__ __forceinline__ Raw() {
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < E * (int)sizeof(T) / 16; ++i) q[i] = make_uint4(0, 0, 0, 0);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] = 0;
            }
        }
        __device__ __forceinline__ void read(const void *base, int64_t at, int l, int D, bool on) {
            const T *row = static_cast<const T *>(base) + at;
#pragma unroll
            for (int c = 0; c < STEPS; ++c) {
                const int col = column(l, c);
                if (on && col < D) {
                    if constexpr (VEC) {
                        constexpr int W = 8 * sizeof(T) / 16;
#pragma unroll
                        for (int i = 0; i < W; ++i) q[c * W + i] = reinterpret_cast<const uint4 *>(row + col)[i];
                    } else {
                        s[c] = mx::bits1(row + col);
                    }
                }
            }
        }
        __device__ __forceinline__ float value(int e) const {
            if constexpr (!VEC) {
                return __uint_as_float(sizeof(T) == 4 ? s[e] : s[e] << 16);
            } else if constexpr (sizeof(T) == 4) {
                const uint4 &w = q[e >> 2];
                return __uint_as_float((e & 3) == 0 ? w.x : (e & 3) == 1 ? w.y : (e & 3) == 2 ? w.z : w.w);
            } else {
                const uint4 &v = q[e >> 3];
                const unsigned w = (e & 7) < 2 ? v.x : (e & 7) < 4 ? v.y : (e & 7) < 6 ? v.z : v.w;
                return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
            }
        }
    };
    template <typename U>
    static __device__ __forceinline__ void store(U *row, int l, int D, const float *v) {
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int col = column(l, c);
            if (col < D) {
                if constexpr (VEC)
                    mx::store8(row + col, v + 8 * c);
                else
                    mx::store1(row + col, v[c]);
            }
        }
    }
    template <typename U>
    static __device__ __forceinline__ void fill(U *row, int l, int D, float v) {
        float u[8] = {v, v, v, v, v, v, v, v};
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int col = column(l, c);
            if (col < D) {
                if constexpr (VEC)
                    mx::store8(row + col, u);
                else
                    mx::store1(row + col, v);
            }
        }
    }
    // The gains of this thread's columns, times v: from shared memory, where they are padded to the threads' columns,
    // or from memory.
    static __device__ __forceinline__ void scale(float *v, const float *shared, const float *w, int l, int D) {
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int col = column(l, c);
            if (shared) {
                if constexpr (VEC) {
                    float g[8];
                    mx::load8(shared + col, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[8 * c + i] *= g[i];
                } else {
                    v[c] *= shared[col];
                }
            } else if (col < D) {
#pragma unroll
                for (int i = 0; i < STEP; ++i) v[STEP * c + i] *= load_gain(w + col + i);
            }
        }
    }
    // The threads of a row wait for each other (they are a warp or less, some warps, or the CTA).
    static __device__ __forceinline__ void meet() {
        if constexpr (TPR <= 32)
            __syncwarp();
        else if constexpr (ROWS == 1)
            __syncthreads();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
    }
    // Two sums over the threads of a row, the same in all of them.  `red` is used in turns, so that one meeting a sum
    // is enough: what is read after it is written again only after the next one.
    struct Scratch {
        float2 part[TPR > 32 ? 2 : 1][TPR > 32 ? THREADS / 32 : 1];
    };
    static __device__ __forceinline__ float2 sum(float a, float b, Scratch &red, int &turn) {
#pragma unroll
        for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) {
            a += __shfl_xor_sync(~0u, a, o);
            b += __shfl_xor_sync(~0u, b, o);
        }
        if constexpr (TPR > 32) {
            if ((threadIdx.x & 31) == 0) red.part[turn][threadIdx.x >> 5] = make_float2(a, b);
            meet();
            const float2 *p = red.part[turn] + (threadIdx.x / TPR) * (TPR / 32);
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w) {
                a += p[w].x;
                b += p[w].y;
            }
            turn ^= 1;
        }
        return make_float2(a, b);
    }
};

// 1 / sqrt(x) to its last bit but one: a step of Newton's on the approximation (two units), so that values beside a border of
// 8 bits fall to the side where they belong as often as the other roundings allow.  0 for infinity.
__device__ __forceinline__ float reciprocal_sqrt(float x) {
    const float r = rsqrtf(x), e = fmaf(-x * r, r, 1.f);
    return x <= FLT_MAX ? fmaf(0.5f * r, e, r) : r;
}
// Sums of squares and of products in four parts
template <int E>
__device__ __forceinline__ float squares(const float *v, float scale) {
    float s[4] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) s[e & 3] = fmaf(v[e] * scale, v[e] * scale, s[e & 3]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}
template <int E>
__device__ __forceinline__ float products(const float *u, const float *v) {
    float s[4] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) s[e & 3] = fmaf(u[e], v[e], s[e & 3]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Gains that are kept in shared memory, padded with zeros to the columns that a row's threads have
constexpr int GAINS_SHARED = 4096;
template <int THREADS>
__device__ __forceinline__ void share_gains(float *to, const float *w, int D, int padded) {
    for (int i = threadIdx.x; i < padded; i += THREADS) to[i] = i < D ? load_gain(w + i) : 0.f;
    __syncthreads();
}

// Eight neighbours u of a row as codes: `codes` and `scales` are those of its first chunk of eight, and `chunk` this
// one's number; four neighbouring threads hold a block and sixteen a group, whose scales the first of them writes.
// A block wholly beyond the width D is zeros, although a norm that is not finite leaves NaN there (0 times it).  (No width, INT32_MAX,
// for rows that have nothing but zeros there.)
// All lanes of a warp take part, those without `on` for the shuffles alone.
template <bool FOUR>
__device__ __forceinline__ void store_chunk(const float *u, bool on, int chunk, int D, uint8_t *codes, uint8_t *scales) {
    float a = fabsf(u[0]);
#pragma unroll
    for (int i = 1; i < 7; i += 2) a = mx::max_abs(a, u[i], u[i + 1]);
    a = mx::max_abs(a, u[7], __shfl_xor_sync(~0u, mx::max_nan(a, fabsf(u[7])), 1));
    a = mx::max_nan(a, __shfl_xor_sync(~0u, a, 2));
    unsigned byte = mx::scale_byte(a, FOUR ? mx::EMAX_E2M1 : mx::EMAX_E4M3);
    const float inv = mx::inverse_scale(byte);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = u[i] * inv;
    if (__any_sync(~0u, byte == 255u)) {                 // blocks that are not finite: codes of zero
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = byte == 255u ? 0.f : q[i];
        if (8 * (chunk & ~3) >= D) byte = 0;
    }
    unsigned s = byte;
    s |= __shfl_down_sync(~0u, s, 4) << 8;
    s |= __shfl_down_sync(~0u, s, 8) << 16;
    if (on) {
        if (FOUR)
            reinterpret_cast<unsigned *>(codes)[chunk] = mx::pack8_e2m1(q);
        else
            reinterpret_cast<uint2 *>(codes)[chunk] =
                make_uint2(mx::pack4_e4m3(q[0], q[1], q[2], q[3]), mx::pack4_e4m3(q[4], q[5], q[6], q[7]));
        if ((chunk & 15) == 0) reinterpret_cast<unsigned *>(scales)[chunk >> 4] = s;
    }
}

// ---------------------------------------------------------------- y = h / sqrt(mean(h^2) + eps) w, h = x + r
struct NormArgs {
    const void *x, *r;
    const float *w;
    void *sum, *y;
    uint8_t *scales;
    int D, G;
    float eps, pad, inv_D;
};
template <int Y>
constexpr bool IS_CODES = Y == AUG_ELEM_MX8 || Y == AUG_ELEM_MX4;

// A row without values: pad_value, or codes and scales of zeros.
template <typename P, typename T, int TPR, int Y>
__device__ __forceinline__ void pad_row(const NormArgs &a, int row, int l) {
    const int64_t at = (int64_t)row * a.D;
    if (a.sum) P::fill(static_cast<T *>(a.sum) + at, l, a.D, a.pad);
    if constexpr (IS_CODES<Y>) {
        constexpr int WORDS = Y == AUG_ELEM_MX4 ? 4 : 8;             // 16-byte words of a group
        uint4 *codes = static_cast<uint4 *>(a.y) + (int64_t)row * a.G * WORDS;
        for (int i = l; i < a.G * WORDS; i += TPR) codes[i] = make_uint4(0, 0, 0, 0);
        unsigned *scales = reinterpret_cast<unsigned *>(a.scales) + (int64_t)row * a.G;
        for (int g = l; g < a.G; g += TPR) scales[g] = 0;
    } else if constexpr (Y == AUG_ELEM_F32) {
        P::fill(static_cast<float *>(a.y) + at, l, a.D, a.pad);
    } else {
        P::fill(static_cast<__nv_bfloat16 *>(a.y) + at, l, a.D, a.pad);
    }
}

// Bound by memory: every value is read once and its row held in registers between the sum of squares and the product.
// CTAs stay, and the next row (and whether the one after it holds values) is on its way while one is worked on.  The norm is
// that of x + r in fp32, before the sum is rounded to be stored.
//
// 64 x 1998 rows of 1024 in 16 bits (two thirds of them hold values), residual and sum, to 8 bits: 137 us, the bytes take 116;
// 64 x 998 in fp32 140 of 136.  What kept it from that were instructions: with a branch for every value's column, rows that hold
// nothing worked on like the others and the gains read a value at a time it was 177 (44 M warp instructions for 52 M values).
template <typename T, int TPR, int E, bool VEC, int Y>
__global__ void __launch_bounds__(RowPart<T, TPR, E, VEC>::THREADS, RowPart<T, TPR, E, VEC>::norm_ctas())
rms_norm_kernel(const NormArgs a, const RowBatch batch) {
    using P = RowPart<T, TPR, E, VEC>;
    constexpr bool AHEAD = VEC ? E * sizeof(T) <= 96 : E <= 24;
    __shared__ typename P::Scratch red;
    extern __shared__ __align__(16) float sm[];
    const int l = threadIdx.x % TPR, D = a.D, step = gridDim.x * P::ROWS;
    constexpr int TURNED = !VEC && IS_CODES<Y> ? P::ROWS * TPR * E : 0;
    float *turned = sm + (threadIdx.x / TPR) * (TPR * E);      // a row in order, where its threads hold it otherwise
    const float *gains = a.w && D <= GAINS_SHARED ? sm + TURNED : nullptr;
    int row = blockIdx.x * P::ROWS + (int)threadIdx.x / TPR, turn = 0;
    // the first row is read before it is known whether it holds values
    typename P::Raw x, r;
    chain_wait();
    x.read(a.x, (int64_t)row * D, l, D, row < batch.rows);
    if (a.r) r.read(a.r, (int64_t)row * D, l, D, row < batch.rows);
    bool valid = batch.holds(row), next = batch.holds(row + step);
    if (gains) share_gains<P::THREADS>(sm + TURNED, a.w, D, TPR * E);
    for (int base = blockIdx.x * P::ROWS; base < batch.rows; base += step, row += step) {
        const int64_t at = (int64_t)row * D;
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = x.value(e);
        if (a.r) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += r.value(e);
        }
        if (AHEAD) {
            x.read(a.x, at + (int64_t)step * D, l, D, next);
            if (a.r) r.read(a.r, at + (int64_t)step * D, l, D, next);
        }
        const bool later = batch.holds(row + 2 * step);
        // threads of rows that share a warp stay together
        if (TPR < 32 || valid) {
            const float ss = P::sum(squares<E>(v, 1.f), 0.f, red, turn).x;
            const float mean = fmaf(ss, a.inv_D, a.eps);
            float rs = reciprocal_sqrt(mean);
            // squares beyond fp32, alone or with eps (or values that are not finite): once more, scaled down, eps with them
            const bool big = !(mean <= FLT_MAX);
            if (TPR <= 32 ? __any_sync(~0u, big) : big) {
                constexpr float DOWN = 0x1p-96f;
                const float s2 = P::sum(squares<E>(v, DOWN), 0.f, red, turn).x;
                if (big) rs = reciprocal_sqrt(fmaf(s2, a.inv_D, a.eps * DOWN * DOWN)) * DOWN;
            }
            if (a.sum && valid) P::store(static_cast<T *>(a.sum) + at, l, D, v);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] *= rs;
            if (a.w) P::scale(v, gains, a.w, l, D);
            if constexpr (IS_CODES<Y>) {
                uint8_t *codes = static_cast<uint8_t *>(a.y) + (int64_t)row * a.G * (Y == AUG_ELEM_MX4 ? 64 : 128);
                uint8_t *scales = a.scales + (int64_t)row * a.G * 4;
                if constexpr (VEC) {
#pragma unroll
                    for (int c = 0; c < E / 8; ++c) {
                        const int chunk = c * TPR + l;
                        if (c * TPR < 16 * a.G)
                            store_chunk<Y == AUG_ELEM_MX4>(v + 8 * c, valid && chunk < 16 * a.G, chunk, D, codes, scales);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) turned[e * TPR + l] = v[e];
                    P::meet();
                    for (int c = 0; c < 16 * a.G; c += TPR) {
                        const bool on = c + l < 16 * a.G;
                        float u[8] = {};
                        if (on) mx::load8(turned + 8 * (c + l), u);
                        store_chunk<Y == AUG_ELEM_MX4>(u, on, c + l, D, codes, scales);
                    }
                    P::meet();
                }
            } else if (valid) {
                if constexpr (Y == AUG_ELEM_F32)
                    P::store(static_cast<float *>(a.y) + at, l, D, v);
                else
                    P::store(static_cast<__nv_bfloat16 *>(a.y) + at, l, D, v);
            }
        }
        if (!valid && row < batch.rows) pad_row<P, T, TPR, Y>(a, row, l);
        if (!AHEAD) {
            x.read(a.x, at + (int64_t)step * D, l, D, next);
            if (a.r) r.read(a.r, at + (int64_t)step * D, l, D, next);
        }
        valid = next;
        next = later;
    }
}

// ---------------------------------------------------------------- its gradients
// With n = h rs, rs = 1 / sqrt(mean(h^2) + eps), and the gradient dy of y = n w:
//   dh = rs (w dy - n rs mean(w dy h)) (+ the gradient that reaches h from elsewhere),   dw = sum over rows of dy n.
// One pass: both sums of a row are taken at once, its values stay in registers until dh is written, the next row's are
// on their way meanwhile, and every thread carries its columns' share of dw over all rows of its CTA.  The CTAs'
// shares go to `partial`, and a second kernel adds them in a fixed order: no atomics, the same result every time.
//
// 64 x 998 rows of 1024 in 16 bits with dsum: 72 us, the bytes take 62.  With a row to a warp, 32 values a thread and nothing
// on its way it was 195: 206 registers left room for eight warps a multiprocessor, which waited for memory.
struct GradArgs {
    const void *h, *dy, *dsum;
    const float *w;
    void *dx;
    float *partial;
    int D;
    float eps, inv_D;
};
constexpr int MOST_SHARES = 444;          // most CTAs of the gradient, and rows of `partial`: three a multiprocessor

template <typename T, int TPR, int E, bool VEC>
__global__ void __launch_bounds__(RowPart<T, TPR, E, VEC>::THREADS, RowPart<T, TPR, E, VEC>::grad_ctas())
rms_norm_grad_kernel(const GradArgs a, const RowBatch batch) {
    using P = RowPart<T, TPR, E, VEC>;
    constexpr bool AHEAD = VEC ? E <= 16 : E <= 8;
    __shared__ typename P::Scratch red;
    extern __shared__ __align__(16) float sm[];
    const int l = threadIdx.x % TPR, D = a.D, step = gridDim.x * P::ROWS;
    const float *gains = a.w && D <= GAINS_SHARED ? sm : nullptr;
    float dw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = 0.f;
    int row = blockIdx.x * P::ROWS + (int)threadIdx.x / TPR, turn = 0;
    typename P::Raw rh, rdy, rds;
    auto read = [&](int64_t at, bool on) {
        rh.read(a.h, at, l, D, on);
        rdy.read(a.dy, at, l, D, on);
        if (a.dsum) rds.read(a.dsum, at, l, D, on);
    };
    chain_wait();
    bool valid = batch.holds(row), next = batch.holds(row + step);
    read((int64_t)row * D, row < batch.rows);
    if (gains) share_gains<P::THREADS>(sm, a.w, D, TPR * E);
    for (int base = blockIdx.x * P::ROWS; base < batch.rows; base += step, row += step) {
        const int64_t at = (int64_t)row * D;
        float h[E], dy[E], g[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            h[e] = rh.value(e);
            dy[e] = rdy.value(e);
        }
        if (TPR < 32 && !valid) {                        // rows that share a warp stay together
#pragma unroll
            for (int e = 0; e < E; ++e) h[e] = dy[e] = 0.f;
        }
        typename P::Raw ds = rds;
        if (AHEAD) read(at + (int64_t)step * D, next);
        const bool later = batch.holds(row + 2 * step);
        if (TPR < 32 || valid) {
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = dy[e];
            if (a.w) P::scale(g, gains, a.w, l, D);
            const float2 both = P::sum(products<E>(h, h), products<E>(g, h), red, turn);
            const float rs = reciprocal_sqrt(fmaf(both.x, a.inv_D, a.eps)), c = rs * rs * (both.y * a.inv_D);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                dw[e] = fmaf(dy[e], h[e] * rs, dw[e]);
                g[e] = rs * fmaf(-c, h[e], g[e]);
            }
            if (a.dsum) {
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] += ds.value(e);
            }
            if (valid) P::store(static_cast<T *>(a.dx) + at, l, D, g);
        }
        if (!valid && row < batch.rows) P::fill(static_cast<T *>(a.dx) + at, l, D, 0.f);
        if (!AHEAD) read(at + (int64_t)step * D, next);
        valid = next;
        next = later;
    }
    chain_next();
    float *mine = a.partial + (int64_t)blockIdx.x * D;
    // rows that share a warp are added there; then one warp's, or one row's threads after the other
#pragma unroll
    for (int o = TPR; o < 32; o <<= 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) dw[e] += __shfl_xor_sync(~0u, dw[e], o);
    }
    constexpr int UNIT = TPR < 32 ? 32 : TPR, UNITS = P::THREADS / UNIT;
    if constexpr (UNITS > 1) __syncthreads();            // the gains make room for the CTA's shares
    for (int s = 0; s < UNITS; ++s) {
        if ((int)threadIdx.x / UNIT == s && (int)threadIdx.x % UNIT < TPR) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int col = P::column(l, e / P::STEP) + e % P::STEP;
                if (col < D) {
                    if constexpr (UNITS > 1)
                        sm[col] = s ? sm[col] + dw[e] : dw[e];
                    else
                        mine[col] = dw[e];
                }
            }
        }
        if constexpr (UNITS > 1) __syncthreads();
    }
    if constexpr (UNITS > 1)
        for (int col = threadIdx.x; col < D; col += P::THREADS) mine[col] = sm[col];
}

// dw[c] = sum of n shares: 32 columns and 32 parts of the shares a CTA
constexpr int ADD_PARTS = 32;
__global__ void __launch_bounds__(32 * ADD_PARTS)
add_shares_kernel(const float *partial, int n, int D, float *dw) {
    __shared__ float s[ADD_PARTS][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float a = 0.f;
    chain_wait();
    if (col < D) {
#pragma unroll 8
        for (int i = part; i < n; i += ADD_PARTS) a += partial[(int64_t)i * D + col];
    }
    s[part][lane] = a;
    __syncthreads();
    a = s[lane][part];                                   // column `part`, lane by lane
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
    if (lane == 0 && blockIdx.x * 32 + part < D) dw[blockIdx.x * 32 + part] = a;
}

// ---------------------------------------------------------------- microscaled numbers
// A chunk, eight neighbours of a row, is a thread's; LPR threads share a row, or a part of it of STEPS LPR chunks, and
// look at ROWS of them one after the other, so that every thread has ROWS x STEPS chunks on their way before the first is converted.
// Rows that cannot be read or written eight values at a time pass through shared memory (LPR = 32), 32 neighbours an
// access.  What bounds this is how many instructions a value takes, so that whose row it is is asked once a row.
// 64 x 1998 rows of 1024 in 16 bits: to 4 bits 50 us (bytes 38), back from 8 bits 55 (55); with one chunk a thread and a 64-bit
// division for each of them 109 and 95.
template <int LPR, int STEPS, int ROWS, bool VEC>
struct ChunkPart {
    static constexpr int THREADS = 256, PER_CTA = THREADS / LPR * ROWS;    // parts
    static constexpr int SPAN = LPR * STEPS;                               // chunks of a part
    static constexpr int TURNED = VEC ? 1 : 256;                           // floats of a warp
    int row[ROWS], first[ROWS];      // row, and this thread's first chunk of it
    bool in[ROWS], valid[ROWS];
    __device__ __forceinline__ ChunkPart(int parts, int per_row, const RowBatch &batch) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int part = (int)blockIdx.x * PER_CTA + r * (THREADS / LPR) + (int)threadIdx.x / LPR;
            in[r] = part < parts;
            row[r] = per_row == 1 ? part : part / per_row;
            first[r] = (per_row == 1 ? 0 : part % per_row * SPAN) + (int)threadIdx.x % LPR;
            valid[r] = in[r] && batch.holds(row[r]);
        }
    }
};

template <int L, int S, int R, bool V>
struct PartShape {                       // the numbers of a ChunkPart, to choose a kernel by
    static constexpr int LPR = L, STEPS = S, ROWS = R, SPAN = L * S, PER_CTA = 256 / L * R;
    static constexpr bool VEC = V;
};

template <typename T, int LPR, int STEPS, int ROWS, bool VEC, bool FOUR>
__global__ void __launch_bounds__(256)
mx_quantize_kernel(const T *x, uint8_t *codes, uint8_t *scales, int D, int G, int parts, int per_row, const RowBatch batch) {
    using P = ChunkPart<LPR, STEPS, ROWS, VEC>;
    __shared__ __align__(16) float turned[8][P::TURNED];
    chain_wait();
    const P p(parts, per_row, batch);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float v[ROWS][STEPS][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const T *from = x + (int64_t)p.row[r] * D;
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int col = 8 * (p.first[r] + c * LPR);
            if constexpr (VEC) {
                if (p.valid[r] && col < D) {
                    mx::load8(from + col, v[r][c]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[r][c][e] = 0.f;
                }
            } else {                                     // 256 neighbours of the row
                const int col0 = col - 7 * lane;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[r][c][e] = p.valid[r] && col0 + 32 * e < D ? mx::load1(from + col0 + 32 * e) : 0.f;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int chunk = p.first[r] + c * LPR;
            if (chunk - (int)threadIdx.x % LPR >= 16 * G) break;
            if constexpr (!VEC) {
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 8; ++e) turned[warp][32 * e + lane] = v[r][c][e];
                __syncwarp();
                mx::load8(turned[warp] + 8 * lane, v[r][c]);
            }
            store_chunk<FOUR>(v[r][c], p.in[r] && chunk < 16 * G, chunk, INT32_MAX, codes + (int64_t)p.row[r] * G * (FOUR ? 64 : 128),
                              scales + (int64_t)p.row[r] * G * 4);
        }
}

template <typename T, int LPR, int STEPS, int ROWS, bool VEC, bool FOUR>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, T *x, int D, int G, int parts, int per_row, float pad,
                     const RowBatch batch) {
    using P = ChunkPart<LPR, STEPS, ROWS, VEC>;
    __shared__ __align__(16) float turned[8][P::TURNED];
    chain_wait();
    const P p(parts, per_row, batch);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint2 q[ROWS][STEPS];
    unsigned byte[ROWS][STEPS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int chunk = p.first[r] + c * LPR;
            q[r][c] = make_uint2(0, 0);
            byte[r][c] = 0;
            if (p.valid[r] && 8 * chunk < D) {
                byte[r][c] = scales[(int64_t)p.row[r] * G * 4 + (chunk >> 2)];
                if (FOUR)
                    q[r][c].x = reinterpret_cast<const unsigned *>(codes + (int64_t)p.row[r] * G * 64)[chunk];
                else
                    q[r][c] = reinterpret_cast<const uint2 *>(codes + (int64_t)p.row[r] * G * 128)[chunk];
            }
        }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        T *to = x + (int64_t)p.row[r] * D;
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int col = 8 * (p.first[r] + c * LPR);
            if (col - 8 * ((int)threadIdx.x % LPR) >= D) break;
            float v[8];
            if (FOUR) {
                mx::unpack8_e2m1(q[r][c].x, v);
            } else {
                mx::unpack4_e4m3(q[r][c].x, v);
                mx::unpack4_e4m3(q[r][c].y, v + 4);
            }
            const float s = mx::scale_value(byte[r][c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= s;
            if (!p.valid[r]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = pad;
            }
            if constexpr (VEC) {
                if (p.in[r] && col < D) mx::store8(to + col, v);
            } else {
                __syncwarp();
                mx::store8(turned[warp] + 8 * lane, v);
                __syncwarp();
                const int col0 = col - 7 * lane;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (p.in[r] && col0 + 32 * e < D) mx::store1(to + col0 + 32 * e, turned[warp][32 * e + lane]);
            }
        }
    }
}

// Threads that share a row, by its width: as few as hold it with so many bytes of values a thread that the next row fits
// into registers beside it, one warp or less where that will do, without a barrier then.  Measured both ways: 64 x 1998 rows of
// 40 fp32 by eight threads 10.1 us, by sixteen 14.4; 64 x 998 of 640 by a warp 37, by two 71; 64 x 998 of 1536 bf16 by two warps
// 88, by four 370 (32 values a thread, most of them beyond the row); 64 x 798 of 513 by a warp 38, by two 62.
template <typename T, bool VEC, bool CODES, typename F>
int norm_by_width(int D, F f) {
    constexpr bool WIDE = VEC && sizeof(T) == 2;         // 32 values in 64 bytes
    if constexpr (VEC && !CODES) {                       // (a group of codes takes sixteen threads)
        if (D <= 64) return f.template operator()<T, 8, 8, VEC>();
        if (D <= 128) return f.template operator()<T, 8, 16, VEC>();
    }
    if constexpr (VEC && CODES)
        if (D <= 128) return f.template operator()<T, 16, 8, VEC>();
    if constexpr (!VEC)
        if (D <= 128) return f.template operator()<T, 32, 4, VEC>();
    if (D <= 256) return f.template operator()<T, 32, 8, VEC>();
    if constexpr (!VEC)
        if (D <= 384) return f.template operator()<T, 32, 12, VEC>();
    if (D <= 512) return f.template operator()<T, 32, 16, VEC>();
    if constexpr (WIDE) {
        if (D <= 768) return f.template operator()<T, 32, 24, VEC>();
        if (D <= 1024) return f.template operator()<T, 32, 32, VEC>();
        if (D <= 1536) return f.template operator()<T, 64, 24, VEC>();
        if (D <= 2048) return f.template operator()<T, 64, 32, VEC>();
        if (D <= 4096) return f.template operator()<T, 128, 32, VEC>();
        if (D <= 8192) return f.template operator()<T, 256, 32, VEC>();
    } else {
        if constexpr (!VEC)
            if (D <= 640) return f.template operator()<T, 32, 20, VEC>();
        if (D <= 768) return f.template operator()<T, 32, 24, VEC>();
        if (D <= 1024) return f.template operator()<T, 64, 16, VEC>();
        if (D <= 1536) return f.template operator()<T, 64, 24, VEC>();
        if (D <= 2048) return f.template operator()<T, 128, 16, VEC>();
        if (D <= 4096) return f.template operator()<T, 256, 16, VEC>();
        if (D <= 8192) return f.template operator()<T, 512, 16, VEC>();
    }
    return f.template operator()<T, 512, 32, VEC>();
}
// The gradient holds three rows and their successors, and the shares of dw: 64 x 1998 rows of 80 fp32 by sixteen threads 26 us,
// and with the sixteen rows' shares of a CTA added one after the other 32.  The last kind, for rows above 4096 (in 16 bits on 16-byte
// boundaries 8192), does not fit into the registers that 512 threads leave: 64 x 64 x 16384 with dsum 154 us in 16 bits (bytes 59) and
// 233 in fp32 (118), 64 x 64 x 10001 without it 595 (28) and 272 (56).
template <typename T, bool VEC, typename F>
int grad_by_width(int D, F f) {
    constexpr bool WIDE = VEC && sizeof(T) == 2;
    if constexpr (VEC) {
        if (D <= 64) return f.template operator()<T, 8, 8, VEC>();
        if (D <= 128) return f.template operator()<T, 16, 8, VEC>();
    } else {
        if (D <= 128) return f.template operator()<T, 32, 4, VEC>();
    }
    if (D <= 256) return f.template operator()<T, 32, 8, VEC>();
    if constexpr (!VEC)
        if (D <= 384) return f.template operator()<T, 32, 12, VEC>();
    if constexpr (WIDE) {
        if (D <= 512) return f.template operator()<T, 32, 16, VEC>();
        if (D <= 1024) return f.template operator()<T, 64, 16, VEC>();
        if (D <= 2048) return f.template operator()<T, 128, 16, VEC>();
        if (D <= 4096) return f.template operator()<T, 256, 16, VEC>();
        if (D <= 8192) return f.template operator()<T, 512, 16, VEC>();
    } else {
        if (D <= 512) return f.template operator()<T, 64, 8, VEC>();
        if constexpr (!VEC)
            if (D <= 768) return f.template operator()<T, 64, 12, VEC>();
        if (D <= 1024) return f.template operator()<T, 128, 8, VEC>();
        if (D <= 2048) return f.template operator()<T, 256, 8, VEC>();
        if (D <= 4096) return f.template operator()<T, 512, 8, VEC>();
    }
    return f.template operator()<T, 512, 32, VEC>();
}

template <int Y>
struct LaunchNorm {
    AugCtx *ctx;
    NormArgs a;
    RowBatch batch;
    template <typename T, int TPR, int E, bool VEC>
    int operator()() const {
        using P = RowPart<T, TPR, E, VEC>;
        const size_t smem = sizeof(float) * ((!VEC && IS_CODES<Y> ? P::ROWS * TPR * E : 0) +
                                             (a.w && a.D <= GAINS_SHARED ? TPR * E : 0));
        if (smem > (40 << 10) && smem_opt_in<rms_norm_kernel<T, TPR, E, VEC, Y>>(ctx->device) != AUG_OK) return AUG_ECUDA;
        const int ctas = std::min((batch.rows + P::ROWS - 1) / P::ROWS, ctx->sm_count * P::norm_ctas());
        return launch_chained(rms_norm_kernel<T, TPR, E, VEC, Y>, dim3(ctas), P::THREADS, smem, ctx->stream, a, batch);
    }
    template <typename T, bool VEC>
    int by_width() const { return norm_by_width<T, VEC, IS_CODES<Y>>(a.D, *this); }
};

struct LaunchGrad {
    AugCtx *ctx;
    GradArgs a;
    RowBatch batch;
    float *dw;
    template <typename T, int TPR, int E, bool VEC>
    int operator()() const {
        using P = RowPart<T, TPR, E, VEC>;
        // gains, and later the CTA's shares where it has several rows at a time
        const size_t smem = a.w && a.D <= GAINS_SHARED ? sizeof(float) * TPR * E : P::ROWS > 1 ? sizeof(float) * a.D : 0;
        const int most = std::min(MOST_SHARES, ctx->sm_count * P::grad_ctas());
        const int ctas = std::min((batch.rows + P::ROWS - 1) / P::ROWS, most);
        if (launch_chained(rms_norm_grad_kernel<T, TPR, E, VEC>, dim3(ctas), P::THREADS, smem, ctx->stream, a, batch) != AUG_OK)
            return AUG_ECUDA;
        return launch_chained(add_shares_kernel, dim3((a.D + 31) / 32), 32 * ADD_PARTS, 0, ctx->stream, a.partial, ctas, a.D, dw);
    }
    template <typename T, bool VEC>
    int by_width() const { return grad_by_width<T, VEC>(a.D, *this); }
};

// Below the smallest normal number squares that underflow would count beside eps, and 1 / (mean + eps) would overflow in the
// gradient of a row of zeros (0 times it is NaN).
bool is_eps(float eps) { return eps >= FLT_MIN && eps <= FLT_MAX; }

template <typename F>
int by_type(int type, bool vec, const F &f) {
    if (type == AUG_ELEM_F32) return vec ? f.template by_width<float, true>() : f.template by_width<float, false>();
    return vec ? f.template by_width<__nv_bfloat16, true>() : f.template by_width<__nv_bfloat16, false>();
}

// go(rows as what they are, whether the codes have 4 bits)
template <typename V, typename F>
int with_types(V *rows, int type, int mx_type, F go) {
    using F32 = std::conditional_t<std::is_const_v<V>, const float, float>;
    using BF16 = std::conditional_t<std::is_const_v<V>, const __nv_bfloat16, __nv_bfloat16>;
    auto go2 = [&](auto *x) { return mx_type == AUG_ELEM_MX4 ? go(x, std::true_type()) : go(x, std::false_type()); };
    return type == AUG_ELEM_F32 ? go2(static_cast<F32 *>(rows)) : go2(static_cast<BF16 *>(rows));
}

// Conversions: four chunks a thread, of as many rows as are narrow enough for that; two where they pass through shared
// memory, eight accesses each.  Fails where the row parts are more than an int counts.
template <typename F>
int by_chunks(int rows, int G, bool vec, F go) {
    auto launch = [&](auto part) {
        using P = decltype(part);
        const int per_row = (16 * G + P::SPAN - 1) / P::SPAN;
        const int64_t parts = (int64_t)rows * per_row;
        if (parts > INT32_MAX - P::PER_CTA) return (int)AUG_ECAP;
        return go(part, (int)((parts + P::PER_CTA - 1) / P::PER_CTA), (int)parts, per_row);
    };
    if (!vec) return G <= 2 ? launch(PartShape<32, 1, 2, false>{}) : launch(PartShape<32, 2, 1, false>{});
    if (G == 1) return launch(PartShape<16, 1, 4, true>{});
    if (G == 2) return launch(PartShape<32, 1, 4, true>{});
    if (G <= 4) return launch(PartShape<32, 2, 2, true>{});
    return launch(PartShape<32, 4, 1, true>{});
}

}  // namespace

extern "C" {

int64_t feat_mx_code_bytes(int mx_type, int D) {
    if (!is_mx_type(mx_type) || D < 1) return AUG_EINVAL;
    return (int64_t)mx::groups(D) * (mx_type == AUG_ELEM_MX4 ? 64 : 128);
}

int64_t feat_mx_scale_bytes(int D) { return D < 1 ? (int64_t)AUG_EINVAL : (int64_t)mx::groups(D) * 4; }

int64_t feat_rms_norm_partial_floats(int D) {
    return D < 1 || D > MAX_WIDTH ? (int64_t)AUG_EINVAL : (int64_t)MOST_SHARES * D;
}

int feat_rms_norm(AugCtx *ctx, const void *x_dev, const void *residual_dev, int in_type, const float *weight_dev,
                  const int *frame_counts_dev, int B, int T_max, int D, float eps, void *sum_dev, void *y_dev, int y_type,
                  uint8_t *scales_dev) {
    bool none;
    const int rc = check_rows(ctx, frame_counts_dev, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !y_dev || !is_row_type(in_type) || !(is_row_type(y_type) || is_mx_type(y_type))) return AUG_EINVAL;
    if (!is_eps(eps)) return AUG_EINVAL;
    if (is_mx_type(y_type) != (scales_dev != nullptr)) return AUG_EINVAL;
    if (D > MAX_WIDTH) return AUG_ECAP;
    // an output over an input of another width, or two outputs in one place, would be written while rows are still read
    if (y_dev == sum_dev || (y_type != in_type && (y_dev == x_dev || y_dev == residual_dev))) return AUG_EINVAL;
    const uintptr_t rows_at = (uintptr_t)x_dev | (uintptr_t)residual_dev | (uintptr_t)sum_dev;
    if (rows_at & (elem_bytes(in_type) - 1) || (uintptr_t)weight_dev & 3) return AUG_EINVAL;
    if (is_mx_type(y_type) ? !on16(y_dev) || !on16(scales_dev) : ((uintptr_t)y_dev & (elem_bytes(y_type) - 1)) != 0)
        return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && ((rows_at | (uintptr_t)y_dev) & 15) == 0;
    const NormArgs a = {x_dev, residual_dev, weight_dev, sum_dev, y_dev, scales_dev, D, mx::groups(D), eps,
                        ctx->cfg.pad_value, 1.f / (float)D};
    const RowBatch batch(frame_counts_dev, T_max, B);
    const int failed = y_type == AUG_ELEM_F32    ? by_type(in_type, vec, LaunchNorm<AUG_ELEM_F32>{ctx, a, batch})
                       : y_type == AUG_ELEM_BF16 ? by_type(in_type, vec, LaunchNorm<AUG_ELEM_BF16>{ctx, a, batch})
                       : y_type == AUG_ELEM_MX8  ? by_type(in_type, vec, LaunchNorm<AUG_ELEM_MX8>{ctx, a, batch})
                                                 : by_type(in_type, vec, LaunchNorm<AUG_ELEM_MX4>{ctx, a, batch});
    if (failed != AUG_OK) return AUG_ECUDA;
    ctx->launches++;
    return AUG_OK;
}

int feat_rms_norm_grad(AugCtx *ctx, const void *h_dev, const void *dy_dev, const void *dsum_dev, int type,
                       const float *weight_dev, const int *frame_counts_dev, int B, int T_max, int D, float eps,
                       void *dx_dev, float *dweight_dev, float *partial_dev) {
    bool none;
    const int rc = check_rows(ctx, frame_counts_dev, B, T_max, D, &none);
    if (rc != AUG_OK) return rc;
    if (D > MAX_WIDTH) return AUG_ECAP;
    if (!dweight_dev || (uintptr_t)dweight_dev & 3) return AUG_EINVAL;
    if (none) return cudaMemsetAsync(dweight_dev, 0, sizeof(float) * D, ctx->stream) == cudaSuccess ? AUG_OK : AUG_ECUDA;
    if (!h_dev || !dy_dev || !dx_dev || !partial_dev || !is_row_type(type)) return AUG_EINVAL;
    if (!is_eps(eps)) return AUG_EINVAL;
    const uintptr_t rows_at = (uintptr_t)h_dev | (uintptr_t)dy_dev | (uintptr_t)dsum_dev | (uintptr_t)dx_dev;
    if (rows_at & (elem_bytes(type) - 1) || ((uintptr_t)weight_dev | (uintptr_t)partial_dev) & 3) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && (rows_at & 15) == 0;
    const GradArgs a = {h_dev, dy_dev, dsum_dev, weight_dev, dx_dev, partial_dev, D, eps, 1.f / (float)D};
    const RowBatch batch(frame_counts_dev, T_max, B);
    if (by_type(type, vec, LaunchGrad{ctx, a, batch, dweight_dev}) != AUG_OK) return AUG_ECUDA;
    ctx->launches += 2;
    return AUG_OK;
}

int feat_mx_quantize(AugCtx *ctx, const void *x_dev, int in_type, const int *frame_counts_dev, int B, int T_max, int D,
                     uint8_t *codes_dev, int mx_type, uint8_t *scales_dev) {
    bool none;
    const int rc = check_rows(ctx, frame_counts_dev, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !codes_dev || !scales_dev || !is_row_type(in_type) || !is_mx_type(mx_type)) return AUG_EINVAL;
    if ((uintptr_t)x_dev & (elem_bytes(in_type) - 1) || !on16(codes_dev) || !on16(scales_dev)) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && on16(x_dev);
    const RowBatch batch(frame_counts_dev, T_max, B);
    const int G = mx::groups(D);
    const int failed = by_chunks(batch.rows, G, vec, [&](auto shape, int ctas, int parts, int per_row) {
        using P = decltype(shape);
        auto go = [&](auto *x, auto four) {
            using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
            return launch_chained(mx_quantize_kernel<T, P::LPR, P::STEPS, P::ROWS, P::VEC, decltype(four)::value>, dim3(ctas), 256, 0,
                                  ctx->stream, x, codes_dev, scales_dev, D, G, parts, per_row, batch);
        };
        return with_types(x_dev, in_type, mx_type, go);
    });
    if (failed != AUG_OK) return failed;
    ctx->launches++;
    return AUG_OK;
}

int feat_mx_dequantize(AugCtx *ctx, const uint8_t *codes_dev, int mx_type, const uint8_t *scales_dev,
                       const int *frame_counts_dev, int B, int T_max, int D, void *x_dev, int out_type) {
    bool none;
    const int rc = check_rows(ctx, frame_counts_dev, B, T_max, D, &none);
    if (rc != AUG_OK || none) return rc;
    if (!x_dev || !codes_dev || !scales_dev || !is_row_type(out_type) || !is_mx_type(mx_type)) return AUG_EINVAL;
    if ((uintptr_t)x_dev & (elem_bytes(out_type) - 1) || !on16(codes_dev) || !on16(scales_dev)) return AUG_EINVAL;
    const bool vec = (D & 7) == 0 && on16(x_dev);
    const RowBatch batch(frame_counts_dev, T_max, B);
    const int G = mx::groups(D);
    const int failed = by_chunks(batch.rows, G, vec, [&](auto shape, int ctas, int parts, int per_row) {
        using P = decltype(shape);
        auto go = [&](auto *x, auto four) {
            using T = std::remove_pointer_t<decltype(x)>;
            return launch_chained(mx_dequantize_kernel<T, P::LPR, P::STEPS, P::ROWS, P::VEC, decltype(four)::value>, dim3(ctas), 256, 0,
                                  ctx->stream, codes_dev, scales_dev, x, D, G, parts, per_row, ctx->cfg.pad_value, batch);
        };
        return with_types(x_dev, out_type, mx_type, go);
    });
    if (failed != AUG_OK) return failed;
    ctx->launches++;
    return AUG_OK;
}

}  // extern "C"
