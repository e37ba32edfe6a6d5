// Rows of a batch times a layer's weights, both microscaled (mx.cuh): out = A W^T + bias, A in 8 or 4 bits, W in 4.
#include <cuda.h>

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
constexpr int FEW_ROWS = 8;

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

// ---------------------------------------------------------------- tiles on the tensor cores
// Rows by the hundred: block-scaled tcgen05.mma, 128 rows by NT columns a tile, accumulated in tensor memory.
//
// A layer has far more rows than columns, so a CTA keeps NT columns of W with all of K in shared memory (for
// 1024 x 208 columns 104 KB) and lets the rows stream past: what is read per tile is its 128 rows alone.  One CTA a
// multiprocessor works through a contiguous part of the tiles, ordered by columns first, so that it loads weights once
// or twice and all CTAs pass the same rows at about the same time (they come from L2 after the first).
//
//   warp 0      fetches 128 rows x 128 bytes a stage with TMA, swizzled as the tensor cores read them, and the weights
//               when the columns change
//   warp 1      issues: scales of a stage from shared to tensor memory, then its multiplications
//   warps 2-5   fetch the scales: the rows' stage by stage, the weights' when the columns change
//   warps 6-13  take finished tiles out of tensor memory (two accumulators: one fills while the other empties), add the
//               bias, round, and send 32 rows of 128 bytes at a time off by TMA, or write them where a row's stride
//               or a tile's end does not allow that
//
// 4-bit rows multiply in 4 bits (64 of K an instruction, 256 a stage); 8-bit rows multiply in 8 bits (32 and 128), for
// which warps 2-5 unpack the weights to e4m3, of which e2m1 is a part, when they put them into shared memory.
constexpr int TILE_M = 128, MAX_NT = 224, TILE_THREADS = 448;
constexpr int STAGE_A = TILE_M * 128, STAGE_SCALES = 1024;
constexpr int ACC_COLUMNS = MAX_NT, SCALE_COLUMNS = 2 * MAX_NT, TMEM_COLUMNS = 512;
constexpr int LIVE_UNITS = 4096;         // tiles of a CTA that are checked for rows with values; later ones count as such
constexpr int MAX_STAGES = 8, MAX_KS = 64;
constexpr int LOADERS = 128, SCALE_LAG = 2, WRITERS = 8, WRITER_BYTES = 4096;

struct TilePlan {
    int NT, KS, stages;                  // columns of a tile, stages along K, depth of the ring
    int MT, units;                       // row tiles, tiles
    int sfb_group;                       // bytes of a group's weight scales: 512 for up to 128 columns, else 1024
    int off_sfb, off_a, off_sfa, off_out, off_misc, smem;
    bool by_tma;                         // the output's rows can be written by TMA
};

struct TileBars {
    unsigned long long a_full[MAX_STAGES], s_full[MAX_STAGES], empty[MAX_STAGES];
    unsigned long long b_full[MAX_KS], bs_full, b_free, acc_full[2], acc_free[2], drained;
    unsigned tmem;
    int dead;                            // a wait ran out: every role ends
    float bias[WRITERS][MAX_NT];         // a copy a warp
    unsigned live[LIVE_UNITS / 32];
};

__device__ __forceinline__ unsigned smem_at(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned long long *b, unsigned n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned long long *b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_at(b)) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned long long *b, unsigned parity) {
    unsigned ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_at(b)), "r"(parity) : "memory");
    return ok;
}
constexpr long long WAIT_CLOCKS = 4000000000ll;
// Waits for a phase, for at most about two seconds; false, in all lanes, once it or another wait of the
// CTA has run out.
__device__ __noinline__ bool bar_wait_long(unsigned long long *b, unsigned parity, int *dead) {
    const long long t0 = clock64();
    for (;;) {
        if (bar_try(b, parity)) return true;
        if (*reinterpret_cast<volatile int *>(dead)) return false;
        if (clock64() - t0 > WAIT_CLOCKS) {
            *reinterpret_cast<volatile int *>(dead) = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(unsigned long long *b, unsigned parity, int *dead) {
    const bool ok = bar_try(b, parity) || bar_wait_long(b, parity, dead);
    return __all_sync(~0u, ok);
}

// Shared memory descriptor of rows of 128 bytes, swizzled in groups of eight (K-major operand)
__device__ __forceinline__ unsigned long long operand_desc(unsigned at) {
    return (unsigned long long)((at & 0x3ffff) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61;
}
// of 32 x 16 bytes of scales, one behind the other
__device__ __forceinline__ unsigned long long scales_desc(unsigned at) {
    return (unsigned long long)((at & 0x3ffff) >> 4) | 8ull << 32 | 1ull << 46;
}
__device__ __forceinline__ void copy_scales(unsigned column, unsigned long long desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
}
template <bool A4>
__device__ __forceinline__ void multiply(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sfa,
                                         unsigned sfb, bool add) {
    if constexpr (A4)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"((unsigned)add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void commit(unsigned long long *b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of the warp's 32 lanes; there once tmem_loaded() has returned
__device__ __forceinline__ void tmem_load32(unsigned at, unsigned *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at) : "memory");
}
// (the registers pass through, so that nothing reads them before)
__device__ __forceinline__ void tmem_loaded(unsigned *r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tma_load(void *to, const CUtensorMap *map, int x, int y, unsigned long long *bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                     smem_at(to)), "l"(map), "r"(x), "r"(y), "r"(smem_at(bar)) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, const void *from) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];\n"
                 "cp.async.bulk.commit_group;" ::"l"(map), "r"(x), "r"(y), "r"(smem_at(from)) : "memory");
}
__device__ __forceinline__ void bar_expect(unsigned long long *b, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(b)), "r"(bytes) : "memory");
}

// 16 bytes of e2m1 codes (32 of them) as e4m3: the same numbers by a table of eight, and the signs
__device__ __forceinline__ void e2m1_to_e4m3(unsigned c, unsigned &lo, unsigned &hi) {
    const unsigned i = c & 0x77777777u;
    unsigned s_lo, s_hi;
    asm("prmt.b32 %0, %1, %2, 0x5140;" : "=r"(s_lo) : "r"(c << 4), "r"(c));       // code's sign in the byte's top bit
    asm("prmt.b32 %0, %1, %2, 0x7362;" : "=r"(s_hi) : "r"(c << 4), "r"(c));
    lo = __byte_perm(0x3C383000u, 0x4C484440u, i) | (s_lo & 0x80808080u);
    hi = __byte_perm(0x3C383000u, 0x4C484440u, i >> 16) | (s_hi & 0x80808080u);
}

// Scales of NT columns of W, all of K, by the loaders: eight groups of two columns a thread at a time
__device__ __forceinline__ void load_weight_scales(const ProductArgs &p, const TilePlan &t, char *smem, int n0, int lt) {
    for (int g0 = 0; g0 < p.G; g0 += 8) {
        unsigned s[2][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = lt + LOADERS * h, n = n0 + r;
            const unsigned *from = reinterpret_cast<const unsigned *>(p.w_scales) + (int64_t)n * p.G + g0;
#pragma unroll
            for (int g = 0; g < 8; ++g) s[h][g] = r < t.NT && n < p.N && g0 + g < p.G ? __ldg(from + g) : 0u;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < 8; ++g)
                if (g0 + g < p.G && 512 * h < t.sfb_group)
                    *reinterpret_cast<unsigned *>(smem + t.off_sfb + (g0 + g) * t.sfb_group + 512 * h + (lt & 31) * 16 +
                                                  (lt >> 5) * 4) = s[h][g];
    }
}
// One group of 128 of K of NT columns of W, unpacked to e4m3: read, and put into shared memory
constexpr int UNPACKED = MAX_NT * 4 / LOADERS;           // pieces of 16 bytes a thread, four to a column
__device__ __forceinline__ void read_weights(const ProductArgs &p, const TilePlan &t, int n0, int g, int lt, uint4 *q) {
#pragma unroll
    for (int i = 0; i < UNPACKED; ++i) {
        const int r = (lt + LOADERS * i) >> 2, n = n0 + r;
        q[i] = r < t.NT && n < p.N && g < p.G ? __ldg(reinterpret_cast<const uint4 *>(p.w + ((int64_t)n * p.G + g) * 64) + (lt & 3))
                                              : make_uint4(0, 0, 0, 0);
    }
}
__device__ __forceinline__ void put_weights(const TilePlan &t, char *to, int lt, const uint4 *q) {
#pragma unroll
    for (int i = 0; i < UNPACKED; ++i) {
        const int r = (lt + LOADERS * i) >> 2, j = 2 * (lt & 3);
        if (r >= t.NT) break;
        uint4 a, b;
        e2m1_to_e4m3(q[i].x, a.x, a.y);
        e2m1_to_e4m3(q[i].y, a.z, a.w);
        e2m1_to_e4m3(q[i].z, b.x, b.y);
        e2m1_to_e4m3(q[i].w, b.z, b.w);
        *reinterpret_cast<uint4 *>(to + r * 128 + ((j ^ (r & 7)) << 4)) = a;
        *reinterpret_cast<uint4 *>(to + r * 128 + (((j + 1) ^ (r & 7)) << 4)) = b;
    }
}

// Whether any of the 128 rows from m0 on holds values
__device__ bool tile_holds(const RowBatch &batch, int m0) {
    if (!batch.counts) return true;
    const int end = min(m0 + TILE_M, batch.rows);
    int b = batch.utterance(m0), t = m0 - b * batch.T_max;
    for (int at = m0; at < end; at = (++b) * batch.T_max, t = 0)
        if (t < batch.counts[b]) return true;
    return false;
}

template <bool A4>
__global__ void __launch_bounds__(TILE_THREADS, 1)
tile_product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap w_map,
                    const __grid_constant__ CUtensorMap out_map, const ProductArgs p, const RowBatch batch, const TilePlan t,
                    int *status) {
    extern __shared__ __align__(1024) char smem_raw[];
    char *smem = smem_raw + ((1024 - (smem_at(smem_raw) & 1023)) & 1023);
    TileBars *bars = reinterpret_cast<TileBars *>(smem + t.off_misc);
    int *dead = &bars->dead;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int u0 = (int)((int64_t)t.units * blockIdx.x / gridDim.x), u1 = (int)((int64_t)t.units * (blockIdx.x + 1) / gridDim.x);
    if (tid == 0) {
        for (int s = 0; s < t.stages; ++s) {
            bar_init(&bars->a_full[s], 1);
            bar_init(&bars->s_full[s], LOADERS / 32);
            bar_init(&bars->empty[s], 1);
        }
        for (int s = 0; s < t.KS; ++s) bar_init(&bars->b_full[s], A4 ? 1 : LOADERS / 32);
        bar_init(&bars->bs_full, LOADERS / 32);
        bar_init(&bars->b_free, 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(&bars->acc_full[i], 1);
            bar_init(&bars->acc_free[i], WRITERS);
        }
        bar_init(&bars->drained, 1);
        bars->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&bars->tmem)),
                     "r"(TMEM_COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // which tiles have rows with values, a bit each, the same for every role
    for (int w = warp; w < LIVE_UNITS / 32 && 32 * w < u1 - u0; w += TILE_THREADS / 32) {
        const int u = u0 + 32 * w + lane;
        const unsigned bits = __ballot_sync(~0u, u < u1 && tile_holds(batch, u % t.MT * TILE_M));
        if (lane == 0) bars->live[w] = bits;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = bars->tmem;
    auto live = [&](int u) { return u - u0 >= LIVE_UNITS || (bars->live[(u - u0) >> 5] >> ((u - u0) & 31) & 1); };
    const int S = t.stages;
    constexpr int GROUPS = A4 ? 2 : 1;                   // groups of a stage
    bool ok = true;
    // Every role goes through the CTA's tiles in the same order.  Weights are loaded for the first tile with values of
    // each run of the same columns, `runs` counts these.
    int n = -1, runs = 0;

    if (warp == 0) {
        int slot = 0, phase = 0, issued = 0, weights = 0;
        for (int u = u0; u < u1 && ok; ++u) {
            if (!live(u)) continue;
            const int m0 = u % t.MT * TILE_M;
            const bool fresh = u / t.MT != n;
            if (fresh) {
                n = u / t.MT;
                if (A4 && runs && !(ok = bar_wait(&bars->b_free, (runs - 1) & 1, dead))) break;
                ++runs;
                weights = 0;
            }
            for (int ks = 0; ks < t.KS; ++ks) {
                if (A4 && fresh) {
                    if (lane == 0) {
                        bar_expect(&bars->b_full[ks], t.NT * 128);
                        tma_load(smem + ks * t.NT * 128, &w_map, ks * 128, n * t.NT, &bars->b_full[ks]);
                    }
                    ++weights;
                }
                if (!(ok = bar_wait(&bars->empty[slot], phase ^ 1, dead))) break;
                if (lane == 0) {
                    bar_expect(&bars->a_full[slot], STAGE_A);
                    tma_load(smem + t.off_a + slot * STAGE_A, &a_map, ks * 128, m0, &bars->a_full[slot]);
                }
                ++issued;
                if (++slot == S) slot = 0, phase ^= 1;
            }
        }
        if (!ok) {                                       // copies in flight end before the CTA does
            const long long start = clock64();
            for (int i = 0; i < weights; ++i)
                while (!bar_try(&bars->b_full[i], (runs - 1) & 1) && clock64() - start < WAIT_CLOCKS) {}
            for (int i = 0; i < S && i < issued; ++i) {
                if (--slot < 0) slot = S - 1, phase ^= 1;
                while (!bar_try(&bars->a_full[slot], phase) && clock64() - start < WAIT_CLOCKS) {}
            }
        }
    } else if (warp == 1) {
        const unsigned idesc = (A4 ? 1u << 7 | 1u << 10 : 0u) | (unsigned)(t.NT >> 3) << 17 | 1u << 23 | 1u << 27;
        int slot = 0, phase = 0, it = 0, j = 0;
        for (int u = u0; u < u1 && ok; ++u) {
            if (!live(u)) continue;
            const bool fresh = u / t.MT != n;
            if (fresh) {
                n = u / t.MT;
                if (runs && lane == 0) commit(&bars->b_free);
                if (!(ok = bar_wait(&bars->bs_full, runs++ & 1, dead))) break;
            }
            const unsigned acc = tmem + (j & 1) * ACC_COLUMNS;
            if (!(ok = bar_wait(&bars->acc_free[j & 1], ((j >> 1) & 1) ^ 1, dead))) break;
            for (int ks = 0; ks < t.KS; ++ks, ++it) {
                if (fresh && !(ok = bar_wait(&bars->b_full[ks], (runs - 1) & 1, dead))) break;
                if (!(ok = bar_wait(&bars->a_full[slot], phase, dead) && bar_wait(&bars->s_full[slot], phase, dead))) break;
                tmem_fence_after();
                if (lane == 0) {
                    const unsigned a = smem_at(smem + t.off_a + slot * STAGE_A), b = smem_at(smem + ks * t.NT * 128);
                    const unsigned sfa = smem_at(smem + t.off_sfa + slot * STAGE_SCALES);
                    const unsigned column = tmem + SCALE_COLUMNS + (it & 1) * 32;
                    const int groups = min(GROUPS, p.G - ks * GROUPS);
                    for (int g = 0; g < groups; ++g) {
                        const unsigned sfb = smem_at(smem + t.off_sfb + (ks * GROUPS + g) * t.sfb_group);
                        copy_scales(column + 4 * g, scales_desc(sfa + 512 * g));
                        copy_scales(column + 8 + 8 * g, scales_desc(sfb));
                        if (t.sfb_group > 512) copy_scales(column + 12 + 8 * g, scales_desc(sfb + 512));
                    }
                    const unsigned long long da = operand_desc(a), db = operand_desc(b);
                    const int steps = A4 ? 2 * groups : 4;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= steps) break;
                        const int g = A4 ? k >> 1 : 0;
                        const unsigned id = A4 ? 2 * (k & 1) : k;      // which of the column's four scales to begin with
                        multiply<A4>(acc, da + 2 * k, db + 2 * k, idesc | id << 4 | id << 29, column + 4 * g, column + 8 + 8 * g,
                                     ks > 0 || k > 0);
                    }
                    commit(&bars->empty[slot]);
                }
                __syncwarp();
                if (++slot == S) slot = 0, phase ^= 1;
            }
            if (ok && lane == 0) commit(&bars->acc_full[j & 1]);
            ++j;
        }
        // nothing of this CTA's is under way when the tensor memory is given back
        if (lane == 0) {
            commit(&bars->drained);
            const long long start = clock64();
            while (!bar_try(&bars->drained, 0) && clock64() - start < WAIT_CLOCKS) {}
        }
        __syncwarp();
        tmem_fence_before();
    } else if (warp < 6) {
        const int lt = tid - 64;
        int slot = 0, phase = 0;
        int pending = 0, done = 0;                       // stages whose scales are on their way, slot of the first of them
        auto deliver = [&](unsigned long long *bar) {
            fence_async();
            __syncwarp();
            if (lane == 0) bar_arrive(bar);
        };
        auto deliver_scales = [&]() {
            deliver(&bars->s_full[done]);
            if (++done == S) done = 0;
            --pending;
        };
        for (int u = u0; u < u1 && ok; ++u) {
            if (!live(u)) continue;
            const bool fresh = u / t.MT != n;
            uint4 w[UNPACKED];
            if (fresh) {
                // the tiles before need their scales before they are done with their weights
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                while (pending) deliver_scales();
                n = u / t.MT;
                if (runs && !(ok = bar_wait(&bars->b_free, (runs - 1) & 1, dead))) break;
                ++runs;
                if (!A4) read_weights(p, t, n * t.NT, 0, lt, w);
                load_weight_scales(p, t, smem, n * t.NT, lt);
                deliver(&bars->bs_full);
            }
            const int m = u % t.MT * TILE_M + lt;
            const uint8_t *from = p.a_scales + (int64_t)min(m, batch.rows - 1) * p.G * 4;
            const unsigned bytes = m < batch.rows ? 4 : 0;
            for (int ks = 0; ks < t.KS; ++ks) {
                if (!(ok = bar_wait(&bars->empty[slot], phase ^ 1, dead))) break;
                const unsigned to = smem_at(smem + t.off_sfa + slot * STAGE_SCALES + (lt & 31) * 16 + (lt >> 5) * 4);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
                    if (ks * GROUPS + g < p.G)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 512 * g),
                                     "l"(from + 4 * (ks * GROUPS + g)), "r"(bytes) : "memory");
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (!A4 && fresh) {                      // a group of weights behind the next one's reads
                    uint4 next[UNPACKED];
                    read_weights(p, t, n * t.NT, ks + 1, lt, next);
                    put_weights(t, smem + ks * t.NT * 128, lt, w);
                    deliver(&bars->b_full[ks]);
#pragma unroll
                    for (int i = 0; i < UNPACKED; ++i) w[i] = next[i];
                }
                if (++pending > SCALE_LAG) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(SCALE_LAG) : "memory");
                    deliver_scales();
                }
                if (++slot == S) slot = 0, phase ^= 1;
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        while (pending) deliver_scales();
    } else {
        const int q = warp & 3, half = (warp - 6) >> 2;  // the lanes of tensor memory that this warp may read; every other piece
        char *stage = smem + t.off_out + (warp - 6) * WRITER_BYTES;
        float *bias = bars->bias[warp - 6];
        int j = 0;
        const int size = p.bf16_out ? 2 : 4, unit = 16 / size, wide = 128 / size;      // a piece: 32 rows of 128 bytes
        const bool vec = (p.N & (unit - 1)) == 0 && (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
        for (int u = u0; u < u1 && ok; ++u) {
            const int n0 = u / t.MT * t.NT, row0 = u % t.MT * TILE_M + 32 * q, cols = min(t.NT, p.N - n0);
            const int rows = min(32, batch.rows - row0);     // may be negative
            const bool alive = live(u), valid = alive && batch.holds(row0 + lane);
            const bool some = __any_sync(~0u, valid);
            if (u / t.MT != n) {
                n = u / t.MT;
                __syncwarp();
                for (int c = lane; c < MAX_NT; c += 32) bias[c] = p.bias && c < cols ? __ldg(p.bias + n0 + c) : 0.f;
                __syncwarp();
            }
            char *out = static_cast<char *>(p.out) + ((int64_t)row0 * p.N + n0) * size;
            if (alive) {
                if (!(ok = bar_wait(&bars->acc_full[j & 1], (j >> 1) & 1, dead))) break;
                tmem_fence_after();
            }
            const unsigned acc = tmem + (j & 1) * ACC_COLUMNS + ((unsigned)q << 21);
            for (int c0 = half * wide; c0 < cols; c0 += 2 * wide) {
                unsigned r[2][32];
                const bool both = p.bf16_out && c0 + 32 < cols;      // 64 columns of 16 bits, 32 of 32
                if (some) {
                    tmem_load32(acc + c0, r[0]);
                    if (both) tmem_load32(acc + c0 + 32, r[1]);
                    tmem_loaded(r[0]);
                    if (both) tmem_loaded(r[1]);
                }
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();                            // the piece before has left
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h && !both) break;
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = valid ? __uint_as_float(r[h][i]) + bias[c0 + 32 * h + i] : p.pad;
                    if (p.bf16_out) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            mx::store8(reinterpret_cast<__nv_bfloat16 *>(stage + lane * 128 + (((4 * h + i) ^ (lane & 7)) << 4)),
                                       v + 8 * i);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<float4 *>(stage + lane * 128 + ((i ^ (lane & 7)) << 4)) =
                                make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    }
                }
                if (t.by_tma && (c0 + wide <= cols || n0 + cols == p.N)) {
                    fence_async();
                    __syncwarp();
                    if (lane == 0 && rows > 0) tma_store(&out_map, n0 + c0, row0, stage);
                } else if (vec) {
                    __syncwarp();
                    const int i = lane & 7, c = c0 + i * unit;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int y = 4 * k + (lane >> 3);
                        if (y < rows && c < cols)
                            *reinterpret_cast<uint4 *>(out + ((int64_t)y * p.N + c) * size) =
                                *reinterpret_cast<const uint4 *>(stage + y * 128 + ((i ^ (y & 7)) << 4));
                    }
                } else {
                    __syncwarp();
                    for (int y = 0; y < rows; ++y)
                        for (int c = lane; c < wide && c0 + c < cols; c += 32) {
                            const char *from = stage + y * 128 + (((c / unit) ^ (y & 7)) << 4) + c % unit * size;
                            char *to = out + ((int64_t)y * p.N + c0 + c) * size;
                            if (p.bf16_out)
                                *reinterpret_cast<unsigned short *>(to) = *reinterpret_cast<const unsigned short *>(from);
                            else
                                *reinterpret_cast<float *>(to) = *reinterpret_cast<const float *>(from);
                        }
                }
            }
            if (alive) {                                 // all of it has been taken
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&bars->acc_free[j & 1]);
                ++j;
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
        tmem_fence_before();
    }
    __syncthreads();
    if (tid == 0 && bars->dead && atomicCAS(&status[0], -1, 0) == -1) status[1] = aug::R_WAIT;
    if (warp == 1) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLUMNS) : "memory");
    }
}

// Columns of a tile and what shared memory holds; false where K is too long for 16 columns.
bool plan_tiles(const AugCtx *ctx, int rows, const ProductArgs &p, bool a4, TilePlan *best) {
    const int groups = a4 ? 2 : 1, KS = (p.G + groups - 1) / groups, MT = (rows + TILE_M - 1) / TILE_M;
    double least = 0;
    bool found = false;
    int last = 0;
    if (KS > MAX_KS) return false;
    for (int tiles = (p.N + MAX_NT - 1) / MAX_NT; tiles <= (p.N + 15) / 16; ++tiles) {
        TilePlan t;
        t.NT = ((p.N + tiles - 1) / tiles + 15) / 16 * 16;
        if (t.NT == last) continue;
        last = t.NT;
        t.KS = KS;
        t.by_tma = (int64_t)p.N * (p.bf16_out ? 2 : 4) % 16 == 0 && on16(p.out);
        t.MT = MT;
        const int64_t units = (int64_t)MT * ((p.N + t.NT - 1) / t.NT);
        if (units > INT32_MAX / 2) break;
        t.units = (int)units;
        t.sfb_group = t.NT > 128 ? 1024 : 512;
        t.off_sfb = KS * t.NT * 128;
        t.off_a = (t.off_sfb + p.G * t.sfb_group + 1023) & ~1023;
        const int fixed = WRITERS * WRITER_BYTES + (int)sizeof(TileBars) + 1024;
        t.stages = std::min(MAX_STAGES, (ctx->smem_per_sm - 1024 - fixed - t.off_a) / (STAGE_A + STAGE_SCALES));
        if (t.stages < SCALE_LAG + 1) continue;
        t.off_sfa = t.off_a + t.stages * STAGE_A;
        t.off_out = t.off_sfa + t.stages * STAGE_SCALES;
        t.off_misc = t.off_out + WRITERS * WRITER_BYTES;
        t.smem = t.off_misc + (int)sizeof(TileBars) + 1024;
        // rounds of tiles on the busiest multiprocessor, their columns and what every tile costs besides
        const double cost = (double)((t.units + ctx->sm_count - 1) / ctx->sm_count) * (t.NT + 32);
        if (!found || cost < least) {
            least = cost;
            *best = t;
            found = true;
        }
    }
    return found;
}

// The driver's function that describes a tensor to the TMA unit
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return (EncodeTiled) nullptr;
        return reinterpret_cast<EncodeTiled>(fn);
    }();
    return f;
}

template <bool A4>
int launch_tiles(AugCtx *ctx, const ProductArgs &p, const RowBatch &batch, const TilePlan &t) {
    const EncodeTiled encode = encode_tiled();
    if (!encode || smem_opt_in<tile_product_kernel<A4>>(ctx->device) != AUG_OK) return AUG_ECUDA;
    auto describe = [&](CUtensorMap *map, CUtensorMapDataType type, void *base, uint64_t width, uint64_t rows, uint64_t bytes,
                        int box_x, int box_y) {
        const cuuint64_t dims[2] = {width, rows}, strides[1] = {bytes};
        const cuuint32_t box[2] = {(cuuint32_t)box_x, (cuuint32_t)box_y}, steps[2] = {1, 1};
        return encode(map, type, 2, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    CUtensorMap a, w, out;
    const uint64_t a_bytes = (uint64_t)p.G * (A4 ? 64 : 128), w_bytes = (uint64_t)p.G * 64, size = p.bf16_out ? 2 : 4;
    if (!describe(&a, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<uint8_t *>(p.a), a_bytes, batch.rows, a_bytes, 128, TILE_M))
        return AUG_ECUDA;
    w = out = a;                                         // (those that are not used)
    if (A4 && !describe(&w, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<uint8_t *>(p.w), w_bytes, p.N, w_bytes, 128, t.NT))
        return AUG_ECUDA;
    if (t.by_tma && !describe(&out, p.bf16_out ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, p.out, p.N,
                              batch.rows, p.N * size, 128 / (int)size, 32))
        return AUG_ECUDA;
    tile_product_kernel<A4><<<std::min(t.units, ctx->sm_count), TILE_THREADS, t.smem, ctx->stream>>>(a, w, out, p, batch, t,
                                                                                                     ctx->status);
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
    const bool a4 = a_type == AUG_ELEM_MX4;
    TilePlan t;
    if (batch.rows <= FEW_ROWS || !plan_tiles(ctx, batch.rows, p, a4, &t)) return launch_few_rows(ctx, p, batch, a4);
    return a4 ? launch_tiles<true>(ctx, p, batch, t) : launch_tiles<false>(ctx, p, batch, t);
}
