// Rows of a batch times a layer's weights, both microscaled (mx.cuh): out = A W^T + bias, A in 8 or 4 bits, W in 4.
#include <algorithm>

#include "mx.cuh"

namespace {

struct ProductArgs {
    const uint8_t *a, *a_scales, *w, *w_scales;
    const float *bias;
    void *out;
    int K, G, N;           // G: groups of 128 along K
    bool bf16_out;
    float pad;
};

// 2^(a + w - 254 - down) v, without overflow or underflow on the way; NaN where either byte says so
__device__ __forceinline__ float scaled(float v, unsigned a, unsigned w, int down) {
    const int e = (int)(a + w) - 254 - down, h = e >> 1;          // -257 .. 254
    const float p = ldexpf(ldexpf(v, h), e - h);
    return a == 255u || w == 255u ? __uint_as_float(0x7fffffffu) : p;
}

// Eight e2m1 codes as signed bytes of twice their value (0 1 2 3 4 6 8 12)
__device__ __forceinline__ uint2 twice_e2m1(unsigned c) {
    const unsigned i = c & 0x77777777u;
    unsigned neg_lo, neg_hi;
    asm("prmt.b32 %0, %1, %2, 0xD9C8;" : "=r"(neg_lo) : "r"(c << 4), "r"(c));      // signs of codes 0-3 over whole bytes
    asm("prmt.b32 %0, %1, %2, 0xFBEA;" : "=r"(neg_hi) : "r"(c << 4), "r"(c));
    const unsigned p_lo = __byte_perm(0x03020100u, 0x0C080604u, i), p_hi = __byte_perm(0x03020100u, 0x0C080604u, i >> 16);
    const unsigned n_lo = __byte_perm(0xFDFEFF00u, 0xF4F8FAFCu, i), n_hi = __byte_perm(0xFDFEFF00u, 0xF4F8FAFCu, i >> 16);
    return make_uint2((p_lo & ~neg_lo) | (n_lo & neg_lo), (p_hi & ~neg_hi) | (n_hi & neg_hi));
}

// ---------------------------------------------------------------- few rows
// A frame (or a few) of a stream: bound by reading the weights, half a byte each.  A lane holds a block of 32 of a
// row's values and of each of COLS columns' weights; P lanes, a power of two, share a column.  4-bit products are
// sums of whole numbers, four at a time (both operands doubled), exact until the block's scale is applied.
constexpr int FEW_THREADS = 256, FEW_COLS = 4;

template <bool A4>
__global__ void __launch_bounds__(FEW_THREADS)
few_rows_kernel(ProductArgs p, RowBatch batch, int P) {
    const int lane = threadIdx.x & 31, part = lane & (P - 1), per_warp = 32 / P;
    const int warp = (blockIdx.x * FEW_THREADS + threadIdx.x) >> 5;
    const int n0 = (warp * per_warp + lane / P) * FEW_COLS, blocks = 4 * p.G;
    for (int row = blockIdx.y; row < batch.rows; row += gridDim.y) {
        float acc[FEW_COLS] = {};
        const bool valid = batch.holds(row);
        const uint8_t *a = p.a + (int64_t)row * p.G * (A4 ? 64 : 128);
        for (int b = part; valid && b < blocks; b += P) {
            const unsigned sa = p.a_scales[(int64_t)row * blocks + b];
            uint4 w[FEW_COLS];
            unsigned sw[FEW_COLS];
#pragma unroll
            for (int c = 0; c < FEW_COLS; ++c) {
                const int n = min(n0 + c, p.N - 1);
                w[c] = __ldg(reinterpret_cast<const uint4 *>(p.w + (int64_t)n * p.G * 64) + b);
                sw[c] = __ldg(p.w_scales + (int64_t)n * blocks + b);
            }
            if constexpr (A4) {
                const uint4 q = reinterpret_cast<const uint4 *>(a)[b];
                const unsigned aw[4] = {q.x, q.y, q.z, q.w};
                uint2 av[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) av[i] = twice_e2m1(aw[i]);
#pragma unroll
                for (int c = 0; c < FEW_COLS; ++c) {
                    const unsigned ww[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
                    int dot = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint2 wv = twice_e2m1(ww[i]);
                        dot = __dp4a((int)av[i].x, (int)wv.x, dot);
                        dot = __dp4a((int)av[i].y, (int)wv.y, dot);
                    }
                    acc[c] += scaled((float)dot, sa, sw[c], 2);
                }
            } else {
                const uint4 q[2] = {reinterpret_cast<const uint4 *>(a)[2 * b], reinterpret_cast<const uint4 *>(a)[2 * b + 1]};
                const unsigned aw[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[1].x, q[1].y, q[1].z, q[1].w};
                float dot[FEW_COLS] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float av[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = mx::unpack2_e4m3((unsigned short)(aw[2 * i + (j >> 1)] >> (16 * (j & 1))));
                        av[2 * j] = f.x;
                        av[2 * j + 1] = f.y;
                    }
#pragma unroll
                    for (int c = 0; c < FEW_COLS; ++c) {
                        float wv[8];
                        mx::unpack8_e2m1(i == 0 ? w[c].x : i == 1 ? w[c].y : i == 2 ? w[c].z : w[c].w, wv);
#pragma unroll
                        for (int j = 0; j < 8; ++j) dot[c] = fmaf(av[j], wv[j], dot[c]);
                    }
                }
#pragma unroll
                for (int c = 0; c < FEW_COLS; ++c) acc[c] += scaled(dot[c], sa, sw[c], 0);
            }
        }
        for (int o = P >> 1; o; o >>= 1)
#pragma unroll
            for (int c = 0; c < FEW_COLS; ++c) acc[c] += __shfl_xor_sync(~0u, acc[c], o);
        if (part == 0) {
#pragma unroll
            for (int c = 0; c < FEW_COLS; ++c) {
                const int n = n0 + c;
                if (n >= p.N) break;
                const float v = valid ? acc[c] + (p.bias ? __ldg(p.bias + n) : 0.f) : p.pad;
                const int64_t at = (int64_t)row * p.N + n;
                if (p.bf16_out)
                    static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(v);
                else
                    static_cast<float *>(p.out)[at] = v;
            }
        }
    }
}

int launch_few_rows(AugCtx *ctx, const ProductArgs &p, const RowBatch &batch, bool a4) {
    int P = 4;
    while (P < 32 && P < 4 * p.G) P *= 2;
    const int cols = FEW_THREADS / P * FEW_COLS;                  // of a CTA
    const dim3 grid((p.N + cols - 1) / cols, std::min(batch.rows, 65535));
    if (a4)
        few_rows_kernel<true><<<grid, FEW_THREADS, 0, ctx->stream>>>(p, batch, P);
    else
        few_rows_kernel<false><<<grid, FEW_THREADS, 0, ctx->stream>>>(p, batch, P);
    AUG_CUDA_OK(cudaGetLastError());
    ctx->launches++;
    return AUG_OK;
}

}  // namespace

extern "C" int feat_mx_product(AugCtx *ctx, const uint8_t *a_codes_dev, int a_type, const uint8_t *a_scales_dev,
                               const uint8_t *w_codes_dev, const uint8_t *w_scales_dev, const float *bias_dev,
                               const int *frame_counts_dev, int B, int T_max, int K, int N, void *out_dev, int out_type) {
    bool none;
    const int rc = check_rows(ctx, B, T_max, K, &none);
    if (rc != AUG_OK || none) return rc;
    if (N < 1 || !is_mx_type(a_type) || !is_row_type(out_type)) return AUG_EINVAL;
    if (!a_codes_dev || !a_scales_dev || !w_codes_dev || !w_scales_dev || !out_dev) return AUG_EINVAL;
    if (!on16(a_codes_dev) || !on16(a_scales_dev) || !on16(w_codes_dev) || !on16(w_scales_dev)) return AUG_EINVAL;
    if ((uintptr_t)bias_dev & 3 || (uintptr_t)out_dev & (elem_bytes(out_type) - 1)) return AUG_EINVAL;
    if (K > AUG_MAX_PRODUCT_WIDTH || N > AUG_MAX_PRODUCT_WIDTH) return AUG_ECAP;
    const ProductArgs p = {a_codes_dev, a_scales_dev, w_codes_dev, w_scales_dev, bias_dev, out_dev, K, mx::groups(K), N,
                           out_type == AUG_ELEM_BF16, ctx->cfg.pad_value};
    const RowBatch batch(frame_counts_dev, T_max, B);
    return launch_few_rows(ctx, p, batch, a_type == AUG_ELEM_MX4);
}
