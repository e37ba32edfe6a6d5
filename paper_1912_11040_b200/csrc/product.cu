// Rows of a batch times a layer's weights, both microscaled (mx.cuh): out = A W^T + bias, A in 8 or 4 bits, W in 4.
#include <cuda.h>

#include <algorithm>

#include "mx.cuh"

namespace {

struct ProductArgs {
    const uint8_t *a, *a_scales, *w, *w_scales;
    const float *bias;
    void *out;
    int G, N;              // groups of 128 along K, columns
    bool bf16_out;
    float pad;
};

// 2^(a + w - 254 - down) v in two steps, neither of which overflows or underflows unless the result does; NaN where either
// byte says so
__device__ __forceinline__ float scaled(float v, unsigned a, unsigned w, int down) {
    const int e = (int)(a + w) - 254 - down, h = max(e >> 1, -126), k = max(e - h, -126);
    const float p = v * __int_as_float((h + 127) << 23) * __int_as_float((k + 127) << 23);
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
// A frame (or a few) of a stream: bound by reading the weights, half a byte each.  A lane holds a block of 32 of each
// of COLS columns' weights and goes through R rows with them; P lanes, a power of two, share a column.  4-bit products
// are sums of whole numbers, four at a time (both operands doubled), exact until the block's scale is applied.
//
// 1024 x 4096 weights (2.2 MB, 0.35 us of bytes): one row 3.1 us, about two of which any launch takes; four 3.9; eight 5.2
// (8-bit rows 6.2).  The tiles below take 5.8 (9) for nine rows, which is why this ends at eight.
constexpr int FEW_THREADS = 256, FEW_COLS = 4, FEW_ROWS = 8;

template <bool A4, int R>
__global__ void __launch_bounds__(FEW_THREADS)
few_rows_kernel(ProductArgs p, RowBatch batch, int P) {
    const int lane = threadIdx.x & 31, part = lane & (P - 1), per_warp = 32 / P;
    const int warp = (blockIdx.x * FEW_THREADS + threadIdx.x) >> 5;
    const int n0 = (warp * per_warp + lane / P) * FEW_COLS, blocks = 4 * p.G;
    chain_wait();
    for (int row0 = blockIdx.y * R; row0 < batch.rows; row0 += gridDim.y * R) {
        float acc[R][FEW_COLS] = {};
        for (int b = part; b < blocks; b += P) {
            uint4 w[FEW_COLS];
            unsigned sw[FEW_COLS];
#pragma unroll
            for (int c = 0; c < FEW_COLS; ++c) {
                const int n = min(n0 + c, p.N - 1);
                w[c] = reinterpret_cast<const uint4 *>(p.w + (int64_t)n * p.G * 64)[b];
                sw[c] = p.w_scales[(int64_t)n * blocks + b];
            }
            unsigned as[R];                              // (the last row again beyond it)
            uint4 a[R][A4 ? 1 : 2];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int row = min(row0 + r, batch.rows - 1);
                as[r] = p.a_scales[(int64_t)row * blocks + b];
                const uint4 *from = reinterpret_cast<const uint4 *>(p.a + (int64_t)row * p.G * (A4 ? 64 : 128));
#pragma unroll
                for (int h = 0; h < (A4 ? 1 : 2); ++h) a[r][h] = from[(A4 ? 1 : 2) * b + h];
            }
            if constexpr (A4) {
                uint2 wv[FEW_COLS][4];
#pragma unroll
                for (int c = 0; c < FEW_COLS; ++c) {
                    const unsigned ww[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) wv[c][i] = twice_e2m1(ww[i]);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const unsigned sa = as[r], aw[4] = {a[r][0].x, a[r][0].y, a[r][0].z, a[r][0].w};
                    int dot[FEW_COLS] = {};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint2 av = twice_e2m1(aw[i]);
#pragma unroll
                        for (int c = 0; c < FEW_COLS; ++c)
                            dot[c] = __dp4a((int)av.y, (int)wv[c][i].y, __dp4a((int)av.x, (int)wv[c][i].x, dot[c]));
                    }
#pragma unroll
                    for (int c = 0; c < FEW_COLS; ++c) acc[r][c] += scaled((float)dot[c], sa, sw[c], 2);
                }
            } else {
                float dot[R][FEW_COLS] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) {            // eight values at a time
                    float wv[FEW_COLS][8];
#pragma unroll
                    for (int c = 0; c < FEW_COLS; ++c)
                        mx::unpack8_e2m1(i == 0 ? w[c].x : i == 1 ? w[c].y : i == 2 ? w[c].z : w[c].w, wv[c]);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const uint4 q = a[r][i >> 1];
                        float av[8];
                        mx::unpack4_e4m3(i & 1 ? q.z : q.x, av);
                        mx::unpack4_e4m3(i & 1 ? q.w : q.y, av + 4);
#pragma unroll
                        for (int c = 0; c < FEW_COLS; ++c)
#pragma unroll
                            for (int j = 0; j < 8; ++j) dot[r][c] = fmaf(av[j], wv[c][j], dot[r][c]);
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int c = 0; c < FEW_COLS; ++c) acc[r][c] += scaled(dot[r][c], as[r], sw[c], 0);
            }
        }
        for (int o = P >> 1; o; o >>= 1)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < FEW_COLS; ++c) acc[r][c] += __shfl_xor_sync(~0u, acc[r][c], o);
        // every lane has all sums of its columns: each writes some of them
        for (int k = part; k < R * FEW_COLS; k += P) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < R * FEW_COLS; ++i) v = i == k ? acc[i / FEW_COLS][i % FEW_COLS] : v;
            const int row = row0 + k / FEW_COLS, n = n0 + k % FEW_COLS;
            if (row >= batch.rows || n >= p.N) continue;
            v = batch.holds(row) ? v + (p.bias ? p.bias[n] : 0.f) : p.pad;
            const int64_t at = (int64_t)row * p.N + n;
            if (p.bf16_out)
                static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(v);
            else
                static_cast<float *>(p.out)[at] = v;
        }
    }
}

template <bool A4>
int launch_few_rows(AugCtx *ctx, const ProductArgs &p, const RowBatch &batch) {
    int P = 4;
    while (P < 32 && P < 4 * p.G) P *= 2;
    const int cols = FEW_THREADS / P * FEW_COLS;                  // of a CTA
    auto go = [&](auto kern, int R) {
        const dim3 grid((p.N + cols - 1) / cols, std::min((batch.rows + R - 1) / R, 65535));
        return launch_chained(kern, grid, FEW_THREADS, 0, ctx->stream, p, batch, P);
    };
    const int rc = batch.rows == 1   ? go(few_rows_kernel<A4, 1>, 1)
                   : batch.rows <= 4 ? go(few_rows_kernel<A4, 4>, 4)
                                     : go(few_rows_kernel<A4, FEW_ROWS>, FEW_ROWS);
    if (rc != AUG_OK) return rc;
    ctx->launches++;
    return AUG_OK;
}

// ---------------------------------------------------------------- tiles on the tensor cores
// Rows by the hundred: block-scaled tcgen05.mma, 128 rows by NT columns a tile, accumulated in tensor memory.
//
// A layer has far more rows than columns, so a CTA keeps NT columns of W with all of K in shared memory (for
// 1024 x 128 columns 64 KB) and lets the rows stream past: what is read per tile is its 128 rows alone.  One CTA a
// multiprocessor works through a contiguous part of the tiles, ordered by columns first, so that it loads weights once
// or twice and all CTAs pass the same rows at about the same time (they come from L2 after the first).
//
// 64 x 1998 rows (two thirds hold values), 1024 x 1024, out in 16 bits: 84 us, 2150 TFLOP/s.  The bytes would take 48.  Nearly all of
// them are written: with K = 80, which writes the same output, this kernel takes 57 us (bytes 41).  The rest is that the rows are read
// once for every 128 columns (54 bytes a clock is what a multiprocessor gets) while the instructions of 128 columns take 95 clocks
// instead of 64; the tensor pipe is busy for 31 % of the time, and nothing is saturated.  In 8 bits the rows are twice as long, the weights leave
// room for four stages, and the wait for them is what counts: 159 us.
//
//   warp 0      fetches 128 rows x 128 bytes a stage with TMA, swizzled as the tensor cores read them, and the weights
//               when the columns change;  warp 14 the rows' scales, some tiles ahead
//   warp 1      issues the multiplications
//   warps 2-5   put the scales into tensor memory: the rows' eight groups of 128 at a time, the weights' when the columns
//               change
//   warps 6-13  take finished tiles out of tensor memory (two accumulators: one fills while the other empties), add the
//               bias, round, and send 32 rows of 64 or 128 bytes at a time off by TMA, or write them word by word where rows do
//               not start on 16-byte boundaries
//
// 4-bit rows multiply in 4 bits (64 of K an instruction, 256 a stage); 8-bit rows multiply in 8 bits (32 and 128), for
// which warps 2-5 unpack the weights to e4m3, of which e2m1 is a part, and put them into shared memory.
// Tiles of 128 columns at most: of 192 they read the rows less often, but leave shared memory for fewer stages (64 x 1998 rows,
// 1536 columns: K = 1024 129 us either way, K = 640 103 and 119).
constexpr int TILE_M = 128, MAX_NT = 128, TILE_THREADS = 480;
constexpr int STAGE_A = TILE_M * 128;
constexpr int TMEM_COLUMNS = 512;
constexpr int LIVE_UNITS = 4096;         // tiles of a CTA that are checked for rows with values; later ones count as such
constexpr int MAX_STAGES = 8, MAX_KS = 64, MAX_AHEAD = 4;
constexpr int LOADERS = 128, CHUNK = 8, CHUNK_COLUMNS = 32, SFB_COLUMNS = 4, WRITERS = 8;

// How tiles are written, by pieces of 32 rows that a writing warp keeps in shared memory and sends off at once: 128 bytes a row word by
// word (rows that do not start on 16-byte boundaries), or by TMA 128 bytes a row, or 64.  Half pieces leave room for
// stages: beside 1024 rows of 8-bit weights a fourth one fits (64 x 1998 rows 159 us, with whole pieces 200); 4-bit rows with
// K = 640 take 69 and 76 us.  But where they do not start on their own boundaries (1000 columns) 4-bit rows are slower for
// them, 64 x 998 x 640 70 and 62 us, 8-bit rows still faster, 24 x 798 x 1000 33 and 36.
enum Out { WORDS, WHOLE, HALF };
Out how_to_write(const ProductArgs &p, bool a4, bool pieces) {
    const int64_t row = (int64_t)p.N * (p.bf16_out ? 2 : 4);
    if (!pieces || row % 16 != 0 || !on16(p.out)) return WORDS;
    return p.bf16_out && (!a4 || (row % 64 == 0 && (reinterpret_cast<uintptr_t>(p.out) & 63) == 0)) ? HALF : WHOLE;
}
template <bool BF16, Out OUT>
struct Piece {
    static constexpr int SIZE = BF16 ? 2 : 4, ROW = OUT == HALF ? 64 : 128, COLS = ROW / SIZE, BYTES = 32 * ROW;
    // where part i, 16 bytes, of a row is kept: as TMA swizzles rows of 128 or 64 bytes
    static __device__ __forceinline__ int at(int row, int i) {
        return row * ROW + ((ROW == 128 ? i ^ (row & 7) : i ^ (row >> 1 & 3)) << 4);
    }
};

struct TilePlan {
    int NT, KS, stages;                  // columns of a tile, stages along K, depth of the ring
    int MT, units;                       // row tiles, tiles
    Out out;
    int ahead;                           // tiles whose scales shared memory has room for
    int off_a, off_scales, off_out, off_misc, smem;
};

struct TileBars {
    unsigned long long a_full[MAX_STAGES], empty[MAX_STAGES], r_full[MAX_AHEAD], r_free[MAX_AHEAD], s_full[2], s_free[2];
    unsigned long long b_full[MAX_KS], bs_full, b_free, acc_full[2], acc_free[2], drained;
    unsigned tmem;
    int dead;                            // a wait ran out: every role ends
    alignas(16) float bias[WRITERS][MAX_NT + 32];      // a copy a warp, and what a piece reads beyond
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
constexpr long long WAIT_CLOCKS = 20000000000ll;
// Waits for a phase, for at most about ten seconds; false, in all lanes, once it or another wait of the
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
__device__ __forceinline__ bool bar_wait_one(unsigned long long *b, unsigned parity, int *dead) {
    return bar_try(b, parity) || bar_wait_long(b, parity, dead);
}
__device__ __forceinline__ bool bar_wait(unsigned long long *b, unsigned parity, int *dead) {      // a warp's lanes together
    return __all_sync(~0u, bar_wait_one(b, parity, dead));
}
// One thread of a converged warp, which issues what a single thread has to
__device__ __forceinline__ bool elected() {
    unsigned one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one;
}

// Shared memory descriptor of an operand with K innermost, rows of 128 bytes that are swizzled in groups of eight: the lower
// word holds the address in units of 16 bytes.
constexpr unsigned OPERAND_HIGH = 64u | 1u << 14 | 2u << 29;
__device__ __forceinline__ unsigned desc_low(unsigned at) { return at >> 4; }
template <bool A4>
__device__ __forceinline__ void multiply(unsigned d, unsigned a, unsigned b, unsigned idesc, unsigned sfa, unsigned sfb, unsigned add) {
    if constexpr (A4)
        asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %7};\nmov.b64 y, {%2, %7};\nsetp.ne.u32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, %3, [%4], [%5], p;\n}" ::"r"(d), "r"(a),
                     "r"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(add), "n"(OPERAND_HIGH) : "memory");
    else
        asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %7};\nmov.b64 y, {%2, %7};\nsetp.ne.u32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], x, y, %3, [%4], [%5], p;\n}" ::"r"(d), "r"(a),
                     "r"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(add), "n"(OPERAND_HIGH) : "memory");
}
__device__ __forceinline__ void commit(unsigned long long *b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_store16(unsigned at, const unsigned *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
                     at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                 "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_store32(unsigned at, const unsigned *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31]) : "memory");
}
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
__device__ __forceinline__ void add_pair(unsigned &a, unsigned &b, unsigned x, unsigned y) {
    asm("{\n.reg .b64 p, q;\nmov.b64 p, {%0, %1};\nmov.b64 q, {%2, %3};\nadd.rn.f32x2 p, p, q;\nmov.b64 {%0, %1}, p;\n}"
        : "+r"(a), "+r"(b) : "r"(x), "r"(y));
}
__device__ __forceinline__ unsigned pack2(const unsigned *v) {
    return mx::pack2_bf16(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
__device__ __forceinline__ void tma_load(void *to, const CUtensorMap *map, int x, int y, unsigned long long *bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                     smem_at(to)), "l"(map), "r"(x), "r"(y), "r"(smem_at(bar)) : "memory");
}
__device__ __forceinline__ void tma_load1(void *to, const CUtensorMap *map, int x, unsigned long long *bar) {
    asm volatile("cp.async.bulk.tensor.1d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2}], [%3];" ::"r"(
                     smem_at(to)), "l"(map), "r"(x), "r"(smem_at(bar)) : "memory");
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

// One group of 128 of K of NT columns of W, unpacked to e4m3: read, and put into shared memory
constexpr int UNPACKED = MAX_NT * 4 / LOADERS;  // pieces of 16 bytes a thread, four to a column
__device__ __forceinline__ void read_weights(const ProductArgs &p, const TilePlan &t, int n0, int g, int lt, uint4 *q) {
#pragma unroll
    for (int i = 0; i < UNPACKED; ++i) {
        const int r = (lt + LOADERS * i) >> 2, n = n0 + r;
        q[i] = r < t.NT && n < p.N && g < p.G ? reinterpret_cast<const uint4 *>(p.w + ((int64_t)n * p.G + g) * 64)[lt & 3]
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

template <bool A4, bool BF16, Out OUT>
__global__ void __launch_bounds__(TILE_THREADS, 1)
tile_product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap s_map, const __grid_constant__ CUtensorMap w_map,
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
            bar_init(&bars->empty[s], 1);
        }
        for (int s = 0; s < t.ahead; ++s) {
            bar_init(&bars->r_full[s], 1);
            bar_init(&bars->r_free[s], LOADERS / 32);
        }
        for (int s = 0; s < t.KS; ++s) bar_init(&bars->b_full[s], A4 ? 1 : LOADERS / 32);
        bar_init(&bars->bs_full, LOADERS / 32);
        bar_init(&bars->b_free, 1);
        bar_init(&bars->drained, 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(&bars->s_full[i], LOADERS / 32);
            bar_init(&bars->s_free[i], 1);
            bar_init(&bars->acc_full[i], 1);
            bar_init(&bars->acc_free[i], WRITERS / 2);
        }
        bars->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    chain_wait();                                        // nothing of memory has been touched so far
    // Tensor memory is taken behind the wait: a kernel ahead that lets this one start before it has taken its own would find
    // nothing left, and neither would end.
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
    struct Tile {
        int u, m, n, MT;
        __device__ __forceinline__ void next() {
            ++u;
            if (++m == MT) m = 0, ++n;
        }
    } at;
    at.u = u0;
    at.MT = t.MT;
    at.n = u0 / t.MT;
    at.m = u0 - at.n * t.MT;
    int n = -1, runs = 0;
    // tensor memory: two accumulators, two chunks of the rows' scales, all of the weights'
    const unsigned sfa = tmem + 2 * t.NT, sfb = sfa + 2 * CHUNK_COLUMNS;

    if (warp == 0) {
        int slot = 0, phase = 0, issued = 0, weights = 0;
        if (elected()) {
            for (; at.u < u1 && ok; at.next()) {
                if (!live(at.u)) continue;
                const int m0 = at.m * TILE_M;
                const bool fresh = at.n != n;
                if (fresh) {
                    n = at.n;
                    if (A4 && runs && !(ok = bar_wait_one(&bars->b_free, (runs - 1) & 1, dead))) break;
                    ++runs;
                    weights = 0;
                }
                for (int ks = 0; ks < t.KS; ++ks) {
                    if (A4 && fresh) {
                        bar_expect(&bars->b_full[ks], t.NT * 128);
                        tma_load(smem + ks * t.NT * 128, &w_map, ks * 128, n * t.NT, &bars->b_full[ks]);
                        ++weights;
                    }
                    if (!(ok = bar_wait_one(&bars->empty[slot], phase ^ 1, dead))) break;
                    bar_expect(&bars->a_full[slot], STAGE_A);
                    tma_load(smem + t.off_a + slot * STAGE_A, &a_map, ks * 128, m0, &bars->a_full[slot]);
                    ++issued;
                    if (++slot == S) slot = 0, phase ^= 1;
                }
            }
            if (!ok) {                                   // copies in flight end before the CTA does
                const long long start = clock64();
                for (int i = 0; i < weights; ++i)
                    while (!bar_try(&bars->b_full[i], (runs - 1) & 1) && clock64() - start < WAIT_CLOCKS) {}
                for (int i = 0; i < S && i < issued; ++i) {
                    if (--slot < 0) slot = S - 1, phase ^= 1;
                    while (!bar_try(&bars->a_full[slot], phase) && clock64() - start < WAIT_CLOCKS) {}
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const unsigned idesc = (A4 ? 1u << 7 | 1u << 10 : 0u) | (unsigned)(t.NT >> 3) << 17 | 1u << 23 | 1u << 27;
        const unsigned a0 = desc_low(smem_at(smem + t.off_a)), b0 = desc_low(smem_at(smem)), b_step = t.NT * 8;
        const int KS = t.KS, G = p.G;
        if (elected()) {
            int slot = 0, phase = 0, j = 0, chunk = 0;
            for (; at.u < u1 && ok; at.next()) {
                if (!live(at.u)) continue;
                const bool fresh = at.n != n;
                if (fresh) {
                    n = at.n;
                    if (runs) commit(&bars->b_free);
                    if (!(ok = bar_wait_one(&bars->bs_full, runs++ & 1, dead))) break;
                }
                const unsigned acc = tmem + (j & 1) * t.NT;
                unsigned b = b0, sa = 0, sb = sfb;
                if (!(ok = bar_wait_one(&bars->acc_free[j & 1], ((j >> 1) & 1) ^ 1, dead))) break;
                for (int ks = 0; ks < KS; ++ks) {
                    if (ks * GROUPS % CHUNK == 0) {          // scales of the next eight groups
                        if (ks) commit(&bars->s_free[chunk++ & 1]);
                        if (!(ok = bar_wait_one(&bars->s_full[chunk & 1], (chunk >> 1) & 1, dead))) break;
                        sa = sfa + (chunk & 1) * CHUNK_COLUMNS;
                    }
                    if (fresh && !(ok = bar_wait_one(&bars->b_full[ks], (runs - 1) & 1, dead))) break;
                    if (!(ok = bar_wait_one(&bars->a_full[slot], phase, dead))) break;
                    tmem_fence_after();
                    const unsigned a = a0 + slot * (STAGE_A / 16);
                    // which of a column's four scales to begin with stands in bits 4 and 29 of the descriptor
                    if (A4) {
                        multiply<A4>(acc, a, b, idesc, sa, sb, ks);
                        multiply<A4>(acc, a + 2, b + 2, idesc | 2u << 4 | 2u << 29, sa, sb, 1);
                        if (ks * GROUPS + 1 < G) {
                            multiply<A4>(acc, a + 4, b + 4, idesc, sa + 4, sb + SFB_COLUMNS, 1);
                            multiply<A4>(acc, a + 6, b + 6, idesc | 2u << 4 | 2u << 29, sa + 4, sb + SFB_COLUMNS, 1);
                        }
                    } else {
                        multiply<A4>(acc, a, b, idesc, sa, sb, ks);
                        multiply<A4>(acc, a + 2, b + 2, idesc | 1u << 4 | 1u << 29, sa, sb, 1);
                        multiply<A4>(acc, a + 4, b + 4, idesc | 2u << 4 | 2u << 29, sa, sb, 1);
                        multiply<A4>(acc, a + 6, b + 6, idesc | 3u << 4 | 3u << 29, sa, sb, 1);
                    }
                    commit(&bars->empty[slot]);
                    b += b_step;
                    sa += 4 * GROUPS;
                    sb += SFB_COLUMNS * GROUPS;
                    if (++slot == S) slot = 0, phase ^= 1;
                }
                if (ok) {
                    commit(&bars->acc_full[j & 1]);
                    commit(&bars->s_free[chunk++ & 1]);
                }
                ++j;
            }
            // nothing of this CTA's is under way when the tensor memory is given back
            commit(&bars->drained);
            const long long start = clock64();
            while (!bar_try(&bars->drained, 0) && clock64() - start < WAIT_CLOCKS) {}
        }
        __syncwarp();
        tmem_fence_before();
    } else if (warp < 6) {
        // Tensor memory holds the scales of 32 rows in its 32 lanes, four in a word for the blocks of a group; rows 32 c to
        // 32 c + 31 are in column c, and each of the four sets of lanes that a warp can write has all of it.
        const int lt = tid - 64, pieces = (p.G + CHUNK - 1) / CHUNK;
        const unsigned lanes = (unsigned)(warp & 3) << 21;
        int chunk = 0, place = 0, round = 0;
        auto deliver = [&](unsigned long long *bar) {
            __syncwarp();
            if (lane == 0) bar_arrive(bar);
        };
        auto deliver_tmem = [&](unsigned long long *bar) {
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            tmem_fence_before();
            deliver(bar);
        };
        for (; at.u < u1 && ok; at.next()) {
            if (!live(at.u)) continue;
            const bool fresh = at.n != n;
            uint4 q[2][UNPACKED];
            if (fresh) {
                n = at.n;
                if (runs && !(ok = bar_wait(&bars->b_free, (runs - 1) & 1, dead))) break;
                tmem_fence_after();
                ++runs;
                if (!A4) {
                    read_weights(p, t, n * t.NT, 0, lt, q[0]);
                    read_weights(p, t, n * t.NT, 1, lt, q[1]);
                }
                for (int g0 = 0; g0 < p.G; g0 += 4) {    // 16 columns at a time: four groups
                    unsigned v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int g = g0 + i / SFB_COLUMNS, c = i % SFB_COLUMNS * 32 + lane, row = n * t.NT + c;
                        v[i] = c < t.NT && row < p.N && g < p.G
                                   ? reinterpret_cast<const unsigned *>(p.w_scales)[(int64_t)row * p.G + g] : 0u;
                    }
                    tmem_store16(sfb + lanes + g0 * SFB_COLUMNS, v);
                }
                deliver_tmem(&bars->bs_full);
            }
            if (!(ok = bar_wait(&bars->r_full[place], round, dead))) break;
            const unsigned *rows = reinterpret_cast<const unsigned *>(smem + t.off_scales + place * 512 * p.G) + lane * p.G;
            for (int piece = 0; piece < pieces; ++piece, ++chunk) {
                unsigned w[CHUNK_COLUMNS];               // four rows, eight groups
                if ((p.G & 3) == 0) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint4 v = make_uint4(0, 0, 0, 0);
                            if (piece * CHUNK + 4 * h < p.G)
                                v = *reinterpret_cast<const uint4 *>(rows + 32 * c * p.G + piece * CHUNK + 4 * h);
                            w[16 * h + c] = v.x;
                            w[16 * h + 4 + c] = v.y;
                            w[16 * h + 8 + c] = v.z;
                            w[16 * h + 12 + c] = v.w;
                        }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int g = 0; g < CHUNK; ++g)
                            w[4 * g + c] = piece * CHUNK + g < p.G ? rows[32 * c * p.G + piece * CHUNK + g] : 0u;
                }
                if (!(ok = bar_wait(&bars->s_free[chunk & 1], ((chunk >> 1) & 1) ^ 1, dead))) break;
                tmem_fence_after();
                tmem_store32(sfa + lanes + (chunk & 1) * CHUNK_COLUMNS, w);
                deliver_tmem(&bars->s_full[chunk & 1]);
                if (!A4 && fresh && piece == 0)
                    for (int ks = 0; ks < t.KS; ks += 2)     // a group's reads are on their way while the one before is put
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (ks + h >= t.KS) break;
                            put_weights(t, smem + (ks + h) * t.NT * 128, lt, q[h]);
                            read_weights(p, t, n * t.NT, ks + h + 2, lt, q[h]);
                            fence_async();
                            deliver(&bars->b_full[ks + h]);
                        }
            }
            if (!ok) break;
            deliver(&bars->r_free[place]);
            if (++place == t.ahead) place = 0, round ^= 1;
        }
        tmem_fence_before();
    } else if (warp == 14) {
        int place = 0, round = 0, fetched = 0;
        if (elected()) {
            const int box = p.G & 1 ? 128 : 256;         // words that are fetched at once
            for (; at.u < u1 && ok; at.next()) {
                if (!live(at.u)) continue;
                if (!(ok = bar_wait_one(&bars->r_free[place], round ^ 1, dead))) break;
                bar_expect(&bars->r_full[place], 512 * p.G);
                for (int i = 0; i < TILE_M * p.G; i += box)
                    tma_load1(smem + t.off_scales + place * 512 * p.G + 4 * i, &s_map, at.m * TILE_M * p.G + i, &bars->r_full[place]);
                ++fetched;
                if (++place == t.ahead) place = 0, round ^= 1;
            }
            if (!ok) {
                const long long start = clock64();
                for (int i = 0; i < t.ahead && i < fetched; ++i) {
                    if (--place < 0) place = t.ahead - 1, round ^= 1;
                    while (!bar_try(&bars->r_full[place], round) && clock64() - start < WAIT_CLOCKS) {}
                }
            }
        }
        __syncwarp();
    } else {
        // Two sets of four warps take tiles in turns, each warp the 32 lanes of tensor memory that it may read.
        const int q = warp & 3, set = (warp - 6) >> 2;
        using P = Piece<BF16, OUT>;
        char *const stage = smem + t.off_out + (warp - 6) * P::BYTES;
        float *bias = bars->bias[warp - 6];
        int j = 0;
        constexpr int size = P::SIZE, wide = P::COLS;
        const int odd_base = (int)(reinterpret_cast<uintptr_t>(p.out) >> 1 & 1);
        for (; at.u < u1 && ok; at.next()) {
            const bool alive = live(at.u);
            if ((alive ? j++ : at.u) & 1 ^ set) continue;
            const int n0 = at.n * t.NT, row0 = at.m * TILE_M + 32 * q, cols = min(t.NT, p.N - n0);
            const int rows = min(32, batch.rows - row0);     // may be negative
            const bool valid = alive && batch.holds(row0 + lane);
            const bool some = __any_sync(~0u, valid), all = __all_sync(~0u, valid);
            if (at.n != n) {
                n = at.n;
                __syncwarp();
                if (p.bias)
                    for (int c = lane; c < MAX_NT + 32; c += 32) bias[c] = c < cols ? p.bias[n0 + c] : 0.f;
                __syncwarp();
            }
            char *out = static_cast<char *>(p.out) + ((int64_t)row0 * p.N + n0) * size;
            if (alive) {
                if (!(ok = bar_wait(&bars->acc_full[set], (j - 1) >> 1 & 1, dead))) break;
                tmem_fence_after();
            }
            const unsigned acc = tmem + set * t.NT + ((unsigned)q << 21);
            for (int c0 = 0; c0 < cols; c0 += wide) {
                unsigned r[2][32];
                const bool both = wide > 32 && c0 + 32 < cols;
                auto add_bias = [&](unsigned *v, int c) {            // two columns at a time
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint4 z = reinterpret_cast<const uint4 *>(bias + c)[i];
                        add_pair(v[4 * i], v[4 * i + 1], z.x, z.y);
                        add_pair(v[4 * i + 2], v[4 * i + 3], z.z, z.w);
                    }
                };
                if (some) {
                    tmem_load32(acc + c0, r[0]);
                    if (both) tmem_load32(acc + c0 + 32, r[1]);
                    tmem_loaded(r[0]);
                    if (both) tmem_loaded(r[1]);
                    if (p.bias) {
                        add_bias(r[0], c0);
                        if (both) add_bias(r[1], c0 + 32);
                    }
                }
                if (alive && c0 + wide >= cols) {            // the accumulator has been taken
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(&bars->acc_free[set]);
                }
                if (!all) {                                  // rows of the piece that hold nothing
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[h][i] = valid ? r[h][i] : __float_as_uint(p.pad);
                }
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();                                // the piece before has left
                // the lane's row as 32 words, four of them at a time
                const auto word = [&](int i) { return BF16 ? pack2(r[i >> 4] + 2 * (i & 15)) : r[0][i]; };
                if (OUT != WORDS) {                                // (cut off at the output's edges)
#pragma unroll
                    for (int i = 0; i < P::ROW / 16; ++i)
                        *reinterpret_cast<uint4 *>(stage + P::at(lane, i)) =
                            make_uint4(word(4 * i), word(4 * i + 1), word(4 * i + 2), word(4 * i + 3));
                    fence_async();
                    __syncwarp();
                    if (lane == 0 && rows > 0) tma_store(&out_map, n0 + c0, row0, stage);
                    continue;
                }
                const int some_cols = min(wide, cols - c0);
                // A row of 16-bit values that starts between two words of memory: shifted by one, so that its words are those of
                // memory; the values at its ends are written by themselves.
                const bool odd = odd_base ^ (p.N & lane & 1) && BF16;
                const unsigned short first = (unsigned short)word(0), last = (unsigned short)(word(31) >> 16);
                unsigned before = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    unsigned w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const unsigned v = word(4 * i + k);
                        w[k] = odd ? __funnelshift_l(before, v, 16) : v;
                        before = v;
                    }
                    *reinterpret_cast<uint4 *>(stage + P::at(lane, i)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                __syncwarp();
                char *to = out + (int64_t)c0 * size;
                const int64_t stride = (int64_t)p.N * size;
                if (BF16 && lane < rows) {             // ends of this lane's row
                    unsigned short *mine = reinterpret_cast<unsigned short *>(to + lane * stride);
                    if (odd) mine[0] = first;
                    if ((some_cols + odd) & 1 && (some_cols > 1 || !odd)) {
                        const int e = some_cols - 1, h = e + odd;
                        mine[e] = h == 64 ? last : *reinterpret_cast<unsigned short *>(stage + P::at(lane, h >> 3) + (h & 7) * 2);
                    }
                }
                // this lane's word of even rows and of odd ones
                char *next[2];
                bool inside[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int e = BF16 ? 2 * lane - (odd_base ^ (p.N & h & 1)) : lane;
                    next[h] = to + h * stride + e * size;
                    inside[h] = e >= 0 && e + BF16 < some_cols;
                }
                for (int y0 = 0; y0 < rows; y0 += 8) {
                    unsigned v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = *reinterpret_cast<const unsigned *>(stage + P::at(y0 + i, lane >> 2) + (lane & 3) * 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (y0 + i < rows && inside[i & 1]) *reinterpret_cast<unsigned *>(next[i & 1]) = v[i];
                        next[i & 1] += 2 * stride;
                    }
                }
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

// Columns of a tile and what shared memory holds; false where there is no room for as few as that.  `whole`: tiles of whole
// pieces, which go by TMA, as everything is that has room for them; others may have any multiple of 16 columns, word by word
// (64 x 1998 x 1024 rows, 1024 columns: 84 us and 136, 656 columns: 76 and 107).  The longer the rows, the fewer columns fit: with 16-bit
// output of 1024 columns 128 up to K = 2304 (8-bit rows 1152), 64 up to 4352 (2304), 48 and 32 word by word up to 6912 (3840), 16
// up to 11776 (7040).
bool plan_tiles(const AugCtx *ctx, int rows, const ProductArgs &p, bool a4, bool whole, TilePlan *best) {
    const Out out = how_to_write(p, a4, whole);
    const int piece_bytes = 32 * (out == HALF ? 64 : 128);
    const int groups = a4 ? 2 : 1, KS = (p.G + groups - 1) / groups, MT = (rows + TILE_M - 1) / TILE_M;
    double least = 0;
    bool found = false;
    int last = 0;
    // (scales are fetched by their number among all, which has to be an int, for rows of the last tile beyond the batch, too)
    if (KS > MAX_KS || (int64_t)MT * TILE_M * p.G > (int64_t)INT32_MAX + 1) return false;
    for (int tiles = (p.N + MAX_NT - 1) / MAX_NT; tiles <= (p.N + 15) / 16; ++tiles) {
        TilePlan t;
        const int wide = tiles == 1 || !whole ? 16 : p.bf16_out ? 64 : 32;
        t.NT = ((p.N + tiles - 1) / tiles + wide - 1) / wide * wide;
        t.out = out;
        if (t.NT > MAX_NT) continue;
        if (t.NT == last) continue;
        last = t.NT;
        t.KS = KS;
        t.MT = MT;
        const int64_t units = (int64_t)MT * ((p.N + t.NT - 1) / t.NT);
        if (units > INT32_MAX / 2) break;
        t.units = (int)units;
        if (2 * t.NT + 2 * CHUNK_COLUMNS + (p.G + 3) / 4 * 16 > TMEM_COLUMNS) continue;
        t.off_a = KS * t.NT * 128;                       // (a multiple of 1024, as 16 divides NT)
        const int fixed = WRITERS * piece_bytes + (int)sizeof(TileBars) + 2048;
        // the rows' scales of four tiles, of two or one where that leaves room for a stage more, or for three at all
        const int room = ctx->smem_per_sm - 1024 - fixed - t.off_a, scales = 512 * p.G;
        t.stages = 0;
        for (int ahead = MAX_AHEAD; ahead >= 1; ahead /= 2) {
            const int stages = std::min(MAX_STAGES, (room - ahead * scales) / STAGE_A);
            if (stages <= t.stages || t.stages >= (ahead == 1 ? 3 : 6)) continue;
            t.stages = stages;
            t.ahead = ahead;
        }
        if (t.stages < 3) continue;
        t.off_scales = t.off_a + t.stages * STAGE_A;
        t.off_out = (t.off_scales + t.ahead * scales + 1023) & ~1023;
        t.off_misc = t.off_out + WRITERS * piece_bytes;
        t.smem = t.off_misc + (int)sizeof(TileBars) + 1024;
        // Rounds of tiles on the busiest multiprocessor, their columns and what every tile costs besides.  (Counting stages,
        // their latency and the writes instead chose worse: 32 x 250 x 640 x 1024 13.3 us, this 10.3.)
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

template <bool A4, bool BF16, Out OUT>
int launch_tiles(AugCtx *ctx, const ProductArgs &p, const RowBatch &batch, const TilePlan &t) {
    using P = Piece<BF16, OUT>;
    const EncodeTiled encode = encode_tiled();
    if (!encode || smem_opt_in<tile_product_kernel<A4, BF16, OUT>>(ctx->device) != AUG_OK) return AUG_ECUDA;
    auto describe = [&](CUtensorMap *map, CUtensorMapDataType type, void *base, uint64_t width, uint64_t rows, uint64_t bytes,
                        int box_x, int box_y, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
        const cuuint64_t dims[2] = {width, rows}, strides[1] = {bytes};
        const cuuint32_t box[2] = {(cuuint32_t)box_x, (cuuint32_t)box_y}, steps[2] = {1, 1};
        return encode(map, type, 2, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    CUtensorMap a, s, w, out;
    const uint64_t a_bytes = (uint64_t)p.G * (A4 ? 64 : 128), w_bytes = (uint64_t)p.G * 64, size = BF16 ? 2 : 4;
    if (!describe(&a, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<uint8_t *>(p.a), a_bytes, batch.rows, a_bytes, 128, TILE_M))
        return AUG_ECUDA;
    const cuuint64_t words[1] = {(cuuint64_t)batch.rows * p.G};      // (a map of one dimension has no strides, but wants a pointer)
    const cuuint32_t word_box[1] = {p.G & 1 ? 128u : 256u}, word_step[1] = {1};
    if (encode(&s, CU_TENSOR_MAP_DATA_TYPE_UINT32, 1, const_cast<uint8_t *>(p.a_scales), words, words, word_box, word_step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return AUG_ECUDA;
    w = out = a;                                         // (those that are not used)
    if (A4 && !describe(&w, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<uint8_t *>(p.w), w_bytes, p.N, w_bytes, 128, t.NT))
        return AUG_ECUDA;
    if (OUT != WORDS && !describe(&out, BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, p.out, p.N,
                              batch.rows, p.N * size, P::COLS, 32, P::ROW == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
        return AUG_ECUDA;
    if (launch_chained(tile_product_kernel<A4, BF16, OUT>, dim3(std::min(t.units, ctx->sm_count)), TILE_THREADS, t.smem, ctx->stream, a, s, w,
                       out, p, batch, t, ctx->status) != AUG_OK)
        return AUG_ECUDA;
    ctx->launches++;
    return AUG_OK;
}

template <bool A4>
int launch_tiles(AugCtx *ctx, const ProductArgs &p, const RowBatch &batch, const TilePlan &t) {
    if (!p.bf16_out) return t.out == WORDS ? launch_tiles<A4, false, WORDS>(ctx, p, batch, t) : launch_tiles<A4, false, WHOLE>(ctx, p, batch, t);
    if constexpr (A4)
        if (t.out == WHOLE) return launch_tiles<A4, true, WHOLE>(ctx, p, batch, t);
    return t.out == WORDS ? launch_tiles<A4, true, WORDS>(ctx, p, batch, t) : launch_tiles<A4, true, HALF>(ctx, p, batch, t);
}

}  // namespace

extern "C" int feat_mx_product(AugCtx *ctx, const uint8_t *a_codes_dev, int a_type, const uint8_t *a_scales_dev,
                               const uint8_t *w_codes_dev, const uint8_t *w_scales_dev, const float *bias_dev,
                               const int *frame_counts_dev, int B, int T_max, int K, int N, void *out_dev, int out_type) {
    bool none;
    const int rc = check_rows(ctx, frame_counts_dev, B, T_max, K, &none);
    if (rc != AUG_OK || none) return rc;
    if (N < 1 || !is_mx_type(a_type) || !is_row_type(out_type)) return AUG_EINVAL;
    if (!a_codes_dev || !a_scales_dev || !w_codes_dev || !w_scales_dev || !out_dev) return AUG_EINVAL;
    if (!on16(a_codes_dev) || !on16(a_scales_dev) || !on16(w_codes_dev) || !on16(w_scales_dev)) return AUG_EINVAL;
    if ((uintptr_t)bias_dev & 3 || (uintptr_t)out_dev & (elem_bytes(out_type) - 1)) return AUG_EINVAL;
    if (K > AUG_MAX_PRODUCT_WIDTH || N > AUG_MAX_PRODUCT_WIDTH) return AUG_ECAP;
    const ProductArgs p = {a_codes_dev, a_scales_dev, w_codes_dev, w_scales_dev, bias_dev, out_dev, mx::groups(K), N,
                           out_type == AUG_ELEM_BF16, ctx->cfg.pad_value};
    const RowBatch batch(frame_counts_dev, T_max, B);
    const bool a4 = a_type == AUG_ELEM_MX4;
    TilePlan t;
    if (batch.rows <= FEW_ROWS || !(plan_tiles(ctx, batch.rows, p, a4, true, &t) || plan_tiles(ctx, batch.rows, p, a4, false, &t)))
        return a4 ? launch_few_rows<true>(ctx, p, batch) : launch_few_rows<false>(ctx, p, batch);
    return a4 ? launch_tiles<true>(ctx, p, batch, t) : launch_tiles<false>(ctx, p, batch, t);
}
