"""What can be told of the row operators' kernels from their source alone."""
import os
import re
import subprocess

import pytest

from paper_1912_11040_b200 import binding


def kernels(name):
    """(name, body without comments) of the file's kernels."""
    text = open(os.path.join(os.path.dirname(binding.__file__), "csrc", name)).read()
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    for k in text.split("__global__")[1:]:
        body = k.split("\n}\n")[0]
        yield re.search(r"(\w+_kernel)\(", body).group(1), body


def test_tensor_memory_is_taken_behind_the_kernels_ahead():
    """Tensor memory is waited for without a limit.  A CTA that held it while it waits for the kernel ahead on the stream
    could keep that kernel, and so itself, from ever ending."""
    taken = [(name, body) for name, body in kernels("product.cu") if "tcgen05.alloc" in body]
    assert [name for name, _ in taken] == ["tile_product_kernel"]
    for _, body in taken:
        assert 0 <= body.index("chain_wait();") < body.index("tcgen05.alloc")


PLANS = r"""
#include "product.cu"
#include <cstdio>
// every way a product of these sizes is planned, by the kind of rows and the type of the output
int main() {
    AugCtx ctx;
    memset(&ctx, 0, sizeof ctx);
    ctx.sm_count = 148;
    ctx.smem_per_sm = 233472;
    const int groups[] = {1, 2, 3, 8, 9, 16, 18, 33, 54, 55, 56, 61, 62, 91, 92, 93, 104, 105, 128};
    const int columns[] = {1, 16, 48, 100, 1000, 1001, 1024, 4096, 16384};
    for (int G : groups)
        for (int N : columns)
            for (int kind = 0; kind < 4; ++kind) {
                const int full = INT32_MAX / G, most = full < AUG_MAX_ROWS ? full : AUG_MAX_ROWS;
                const int rows[] = {9, 128, 129, 8192, most - 128, most - 1, most};
                for (int r : rows) {
                    ProductArgs p = {};
                    p.out = reinterpret_cast<void *>(1024);
                    p.G = G;
                    p.N = N;
                    p.bf16_out = kind & 1;
                    TilePlan t;
                    if (!plan_tiles(&ctx, r, p, kind & 2, true, &t) && !plan_tiles(&ctx, r, p, kind & 2, false, &t)) t.NT = 0;
                    printf("%d %d %d %d %d %d %d %d\n", G, N, kind, r, t.NT, t.NT ? t.smem : 0, t.NT ? t.stages : 0, t.NT ? t.MT : 0);
                }
            }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """(groups, columns, kind, rows, columns of a tile or 0, bytes of shared memory, stages, row tiles) of many products."""
    at = tmp_path_factory.mktemp("plans")
    (at / "plans.cu").write_text(PLANS)
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17",
                    "-I", csrc, "-o", str(at / "plans"), str(at / "plans.cu")], check=True)
    out = subprocess.run([str(at / "plans")], check=True, capture_output=True, text=True).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_tiles_of_a_product_fit(plans):
    """Shared memory, tensor memory (two accumulators, the scales of eight groups of rows twice, all of the weights')."""
    for groups, columns, kind, rows, nt, smem, stages, tiles in plans:
        if nt:
            assert smem <= 227 * 1024 and 3 <= stages <= 8 and nt % 16 == 0 and nt <= 128
            assert 2 * nt + 64 + -(-groups // 4) * 16 <= 512
            assert tiles == -(-rows // 128)


def test_scales_of_a_products_rows_are_fetched_by_numbers_that_an_int_holds(plans):
    """128 or 256 words at a time by the number of the first, for all 128 rows of a tile, the last one's too."""
    seen = 0
    for groups, columns, kind, rows, nt, smem, stages, tiles in plans:
        if nt:
            assert tiles * 128 * groups - 128 < 2 ** 31, (groups, rows)
            seen += rows > 10 ** 6
    assert seen > 100
