"""The operators on rows where they had not been looked at: more rows than the device holds at a time, eps beside squares at
either end of fp32, codes of rows that are not finite, lengths at the ends of the product's tiles."""
import numpy as np
import pytest

import row_reference as ref
from paper_1912_11040_b200 import binding
from test_gpu_row_operators import (BF16, EPS, F32, HALF, MX4, MX8, U32, check_grad, check_norm, check_product, context, guarded, host,
                                    on_device, rows, to_counts, torch_type)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return context(max_batch=4096)


# ----------------------------------------------------------------------------- norm to codes
def check_norm_codes(ctx, B, T, D, counts, t, kind, residual, shift=0, seed=0, spoil=None):
    """Sum, codes and scales against the sum and the fp32 norm quantised, those against 64 bits."""
    import torch
    rng = np.random.default_rng(seed)
    x = rows(rng, B, T, D, counts, t)
    r = rows(rng, B, T, D, counts, t) if residual else None
    if spoil:
        spoil(x)
    w = rng.normal(size=D).astype(np.float32)
    c, ok = to_counts(counts), ref.holds(counts, B, T)
    args = (on_device(x, t, shift), on_device(r, t, shift) if residual else None, t, torch.from_numpy(w).cuda(), c, B, T, D, EPS)
    y = torch.empty(B, T, D, device="cuda")
    sums = [guarded((B, T, D), torch_type(t), 3.0, shift) if residual else (None, lambda: True) for _ in range(2)]
    size = (B, T, binding.feat_mx_code_bytes(kind, D)), (B, T, binding.feat_mx_scale_bytes(D))
    out = [[guarded(s, torch.uint8, 0xAB) for s in size] for _ in range(2)]
    ctx.feat_rms_norm(*args, sums[0][0], y, F32)
    ctx.feat_mx_quantize(y, F32, c, B, T, D, out[0][0][0], kind, out[0][1][0])
    ctx.feat_rms_norm(*args, sums[1][0], out[1][0][0], kind, out[1][1][0])
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):             # (infinity times zero)
        h, want = ref.rms_norm(x, r, w, EPS)
    good = ok & np.isfinite(want).all(-1)
    # the sum of squares, 1/sqrt and the products as in check_norm
    assert np.all(np.abs(host(y) - want)[good] <= (np.abs(want) * (41 * U32))[good])
    for s, intact in sums:
        if residual:
            assert np.all(np.abs(host(s) - h)[good] <= (np.abs(h) * (U32 + HALF[t]))[good]) and intact()
    for a, b in zip(*out):
        assert torch.equal(a[0], b[0]) and a[1]() and b[1]()
    codes, scales = (v[0].cpu().numpy() for v in out[1])
    beyond = -(-D // ref.BLOCK)
    assert not scales[..., beyond:].any() and not codes[~ok].any() and not scales[~ok].any()
    return scales, ok


@pytest.mark.parametrize("D", [8, 40, 100, 128, 129, 257, 264, 640, 1000, 1025, 4100])
@pytest.mark.parametrize("kind", [MX8, MX4])
@pytest.mark.parametrize("t,shift", [(F32, 0), (BF16, 0), (BF16, 1)])
def test_norm_to_codes_of_what_is_not_finite(ctx, D, kind, t, shift):
    """Blocks that lie wholly beyond the width are zeros with a scale byte of 0, whatever the row holds."""
    def spoil(x):
        x[0, 0, 3], x[0, 1, -1], x[0, 2, 0], x[2, 1, D // 2] = np.nan, np.inf, -np.inf, np.nan
    scales, ok = check_norm_codes(ctx, 3, 4, D, [4, 0, 2], t, kind, False, shift, D, spoil)
    assert (scales[0, 0, : -(-D // ref.BLOCK)] == 255).all() and (scales[0, 3, : -(-D // ref.BLOCK)] != 255).all()


# ----------------------------------------------------------------------------- eps at the ends of fp32
@pytest.mark.parametrize("D", [1, 8, 40, 257, 1024, 4096, 10001])
@pytest.mark.parametrize("scale,eps", [(2e18, 1e37), (1e19, 1e38), (1e19, 3e38), (3e19, 1e36), (1e20, 1.0)])
def test_norm_with_eps_beside_squares_beyond_fp32(ctx, D, scale, eps):
    import torch
    rng = np.random.default_rng(D)
    x = host(torch.from_numpy(scale * rng.uniform(0.5, 1.5, (5, D))).float())
    y = torch.full((5, D), 3.0, device="cuda")
    ctx.feat_rms_norm(on_device(x, F32), None, F32, None, None, 1, 5, D, eps, None, y, F32)
    want = ref.rms_norm(x, None, None, float(np.float32(eps)))[1]
    # as in check_norm; the scaling is by powers of two
    assert np.all(np.abs(host(y) - want) <= np.abs(want) * (41 * U32))


LEAST = 2.0 ** -126                     # the smallest normal number of fp32


@pytest.mark.parametrize("D", [8, 40, 257, 1024])
def test_smallest_eps(ctx, D):
    """Squares lose what lies below 2^-149 of them, which is 2^-24 of the smallest eps at most."""
    import torch
    rng = np.random.default_rng(D)
    h = rng.normal(size=(6, D)) * np.array([0.0, 1e-21, 1e-19, 3e-19, 1e-15, 1.0])[:, None]
    h = host(torch.from_numpy(h).float())
    dy = host(torch.from_numpy(rng.normal(size=(6, D))).float())
    y, dx = (torch.full((6, D), 3.0, device="cuda") for _ in range(2))
    dw, part = torch.empty(D, device="cuda"), torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    ctx.feat_rms_norm(on_device(h, F32), None, F32, None, None, 1, 6, D, LEAST, None, y, F32)
    ctx.feat_rms_norm_grad(on_device(h, F32), on_device(dy, F32), None, F32, None, None, 1, 6, D, LEAST, dx, dw, part)
    want = ref.rms_norm(h, None, None, LEAST)[1]
    # as in check_norm, and the mean of squares off by two more units: what each square loses, and the mean itself
    assert np.all(np.abs(host(y) - want) <= np.abs(want) * (43 * U32))
    dx_want, dw_want, size, dw_size = ref.rms_norm_grad(h, dy, None, None, LEAST)
    assert np.all(np.abs(host(dx) - dx_want) <= size * (94 * U32))       # as in check_grad, and the same two, twice
    assert np.all(np.abs(host(dw) - dw_want) <= dw_size * (6 + 440 + 3) * U32)


@pytest.mark.parametrize("eps", [2.0 ** -127, 1e-40, 2.0 ** -149])
def test_eps_below_the_smallest_normal_number_is_refused(ctx, eps):
    import torch
    x, dx = torch.zeros(2, 64, device="cuda"), torch.full((2, 64), 3.0, device="cuda")
    dw, part = torch.full((64,), 3.0, device="cuda"), torch.empty(binding.feat_rms_norm_partial_floats(64), device="cuda")
    assert ctx.feat_rms_norm(x, None, F32, None, None, 1, 2, 64, eps, None, dx, F32, check=False) == binding.AUG_EINVAL
    assert ctx.feat_rms_norm_grad(x, x, None, F32, None, None, 1, 2, 64, eps, dx, dw, part, check=False) == binding.AUG_EINVAL
    assert (dx == 3).all() and (dw == 3).all()


# ----------------------------------------------------------------------------- the gradient's sums
def test_sums_of_the_gradient_are_in_four_parts(ctx):
    """A thread has sixteen neighbours by eights.  Of each sixteen the first value is 1 and the others are 2^-12, whose squares are
    half a unit of it: behind it in one sum all fifteen are lost, in four parts three."""
    import torch
    D, eps = 1024, 2.0 ** -20
    h = torch.full((1, D), 2.0 ** -12, device="cuda")
    h[0, 0:512:8] = 1.0
    h, one = h.bfloat16(), torch.ones(1, D, device="cuda").bfloat16()
    dx, dw = torch.empty_like(h), torch.empty(D, device="cuda")
    part = torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    ctx.feat_rms_norm_grad(h, one, None, BF16, None, None, 1, 1, D, eps, dx, dw, part)
    want = ref.rms_norm_grad(host(h), np.ones((1, D)), None, None, eps)[1]
    # the parts lose 3 U32 of the sum, the sums of threads are exact, the mean with eps is one U32: halved by the square
    # root, which is good to 2 U32 (its last bit but one); h and dy are powers of two
    assert np.all(np.abs(host(dw) - want) <= np.abs(want) * ((3 + 1) / 2 + 2) * U32)


# ----------------------------------------------------------------------------- more rows than the device holds at a time
def some_counts(B, T, seed):
    return [int(c) for c in np.random.default_rng(seed).integers(-1, T + 2, B)]


MANY = [(4000, 15, 40), (2400, 15, 128), (2000, 12, 257), (800, 15, 1024), (300, 10, 4100), (100, 10, 8192), (60, 10, 16384)]


@pytest.mark.parametrize("B,T,D", MANY)
@pytest.mark.parametrize("t,yt", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_of_many_rows(ctx, B, T, D, t, yt, shift):
    check_norm(ctx, B, T, D, [max(c, 0) for c in some_counts(B, T, D)], t, yt, shift=shift)


@pytest.mark.parametrize("B,T,D", MANY)
@pytest.mark.parametrize("t,kind,shift", [(F32, MX4, 0), (F32, MX8, 1), (BF16, MX8, 0), (BF16, MX4, 1)])
def test_norm_of_sums_to_codes(ctx, B, T, D, t, kind, shift):
    check_norm_codes(ctx, B, T, D, some_counts(B, T, D), t, kind, True, shift)


@pytest.mark.parametrize("D", [8, 40, 128, 136, 257, 384, 512, 640, 768, 1000, 1024, 1536, 2048, 2050, 4096, 4100, 8192])
@pytest.mark.parametrize("kind", [MX8, MX4])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_of_few_sums_to_codes(ctx, D, kind, shift):
    for t in (F32, BF16):
        check_norm_codes(ctx, 3, 4, D, [4, 0, 3], t, kind, True, shift, D)


@pytest.mark.parametrize("B,T,D", [(4000, 15, 40), (4000, 10, 80), (2400, 15, 128), (2000, 8, 257), (600, 10, 1024), (100, 8, 4100),
                                   (60, 10, 10001)])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
def test_grad_of_many_rows(ctx, B, T, D, t, shift):
    check_grad(ctx, B, T, D, some_counts(B, T, D), t, shift=shift)


@pytest.mark.parametrize("B,T,D", [(4000, 15, 40), (4000, 10, 80), (2400, 15, 128), (2000, 8, 257), (600, 10, 1024), (100, 8, 4100),
                                   (60, 10, 10001)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_grad_of_the_weights_counts_every_row_once(ctx, B, T, D, t):
    """h = +-1 and eps = 3, so that mean(h^2) + eps is 4 (the nearest number to it, whatever 1 / D is rounded to) and n is h / 2;
    whole numbers as dy: all terms are multiples of 1/2 whose sums stay below 2^23, so that dw is exact."""
    import torch
    rng = np.random.default_rng(D)
    counts = some_counts(B, T, D)
    ok = ref.holds(counts, B, T)
    h, dy = rng.choice([-1.0, 1.0], (B, T, D)), rng.integers(-8, 9, (B, T, D)).astype(float)
    want = (dy * h * ok[..., None]).sum((0, 1)) / 2
    h[~ok], dy[~ok] = np.nan, np.nan
    dx, dw = torch.empty(B, T, D, dtype=torch_type(t), device="cuda"), torch.empty(D, device="cuda")
    part = torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    ctx.feat_rms_norm_grad(on_device(h, t), on_device(dy, t), None, t, None, to_counts(counts), B, T, D, 3.0, dx, dw, part)
    assert np.array_equal(host(dw), want)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("B,T,D", [(4000, 15, 40), (2000, 12, 257), (800, 15, 1024), (60, 10, 16384)])
def test_many_rows_in_place(ctx, B, T, D, t):
    """Rows that are read ahead are not those that are written meanwhile."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(D)
    new = lambda: torch.randn(B, T, D, device="cuda", generator=gen).to(torch_type(t))
    x, r, w = new(), new(), torch.randn(D, device="cuda", generator=gen)
    c = to_counts(some_counts(B, T, D))
    y, s, y0, s0 = (torch.empty_like(x) for _ in range(4))
    ctx.feat_rms_norm(x, r, t, w, c, B, T, D, EPS, s, y, t)
    ctx.feat_rms_norm(x, None, t, w, c, B, T, D, EPS, s0, y0, t)            # a sum of one
    ok = torch.arange(T, device="cuda")[None, :] < c[:, None]
    assert torch.equal(s0[ok], x[ok])
    x1, r1 = x.clone(), r.clone()
    ctx.feat_rms_norm(x1, r1, t, w, c, B, T, D, EPS, r1, x1, t)
    assert torch.equal(x1, y) and torch.equal(r1, s)
    x1 = x.clone()
    ctx.feat_rms_norm(x1, None, t, w, c, B, T, D, EPS, None, x1, t)
    assert torch.equal(x1, y0)
    part = torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    dx, dw, dw1, ds = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda"), new()
    ctx.feat_rms_norm_grad(x, r, ds, t, w, c, B, T, D, EPS, dx, dw, part)
    for k in range(3):
        v = [x.clone(), r.clone(), ds.clone()]
        ctx.feat_rms_norm_grad(*v, t, w, c, B, T, D, EPS, v[k], dw1, part)
        assert torch.equal(v[k], dx) and torch.equal(dw1, dw)


def test_more_values_than_an_int_counts():
    """2^21 rows and some of 1024 values: the last rows begin beyond 2^31 values (beyond 2^32 bytes of any type but codes)."""
    import torch
    D, N, T = 1024, 1024, (1 << 21) + 300
    ctx = context(max_batch=1)
    at = [0, 1, 148 * 7, (1 << 20) - 1, 1 << 20, (1 << 21) - 1, 1 << 21, (1 << 21) + 127, T - 2, T - 1]
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    gain = 1 + 0.1 * torch.randn(D, device="cuda", generator=gen)
    y = torch.empty_like(x)
    ctx.feat_rms_norm(x, None, BF16, gain, None, 1, T, D, EPS, None, y, BF16)
    some, w = host(x[at]), host(gain)
    want = ref.rms_norm(some, None, w, EPS)[1]
    assert np.all(np.abs(host(y[at]) - want) <= np.abs(want) * (40 * U32 + HALF[BF16]))
    codes = torch.empty(T, binding.feat_mx_code_bytes(MX8, D), dtype=torch.uint8, device="cuda")
    scales = torch.empty(T, binding.feat_mx_scale_bytes(D), dtype=torch.uint8, device="cuda")
    ctx.feat_rms_norm(x, None, BF16, gain, None, 1, T, D, EPS, None, codes, MX8, scales)
    normed = [c[at].clone() for c in (codes, scales)]
    f = torch.empty(len(at), D, device="cuda")
    few = [torch.empty_like(c) for c in normed]
    ctx.feat_rms_norm(x[at].contiguous(), None, BF16, gain, None, 1, len(at), D, EPS, None, f, F32)
    ctx.feat_mx_quantize(f, F32, None, 1, len(at), D, few[0], MX8, few[1])
    assert all(torch.equal(a, b) for a, b in zip(normed, few))
    ctx.feat_mx_quantize(x, BF16, None, 1, T, D, codes, MX8, scales)
    raw_c, raw_s = ref.quantize(some, "mx8")
    got_c, got_s = codes[at].cpu().numpy(), scales[at].cpu().numpy()
    assert np.array_equal(got_s, raw_s) and np.array_equal(np.where(got_c == 128, 0, got_c), np.where(raw_c == 128, 0, raw_c))
    a = ref.dequantize(got_c, got_s, "mx8", D)
    ctx.feat_mx_dequantize(codes, MX8, scales, None, 1, T, D, y, BF16)
    assert np.all(np.abs(host(y[at]) - a) <= np.abs(a) * HALF[BF16])
    w_codes = torch.empty(N, binding.feat_mx_code_bytes(MX4, D), dtype=torch.uint8, device="cuda")
    w_scales = torch.empty(N, binding.feat_mx_scale_bytes(D), dtype=torch.uint8, device="cuda")
    ctx.feat_mx_quantize(torch.randn(N, D, device="cuda", generator=gen), F32, None, 1, N, D, w_codes, MX4, w_scales)
    ctx.feat_mx_product(codes, MX8, scales, w_codes, w_scales, None, None, 1, T, D, N, y, BF16)
    wv = ref.dequantize(ref.unpacked(w_codes.cpu().numpy(), "mx4"), w_scales.cpu().numpy(), "mx4", D)
    want, size = a @ wv.T, np.abs(a) @ np.abs(wv).T
    assert np.all(np.abs(host(y[at]) - want) <= size * ((D + 1) * 2 * U32) + np.abs(want) * HALF[BF16])
    out = torch.empty(T, N - 1, dtype=torch.bfloat16, device="cuda")         # rows that start anywhere
    ctx.feat_mx_product(codes, MX8, scales, w_codes, w_scales, None, None, 1, T, D, N - 1, out, BF16)
    assert torch.equal(out[at], y[at][:, :-1])
    dx, dw, part = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    ctx.feat_rms_norm_grad(x, y, None, BF16, gain, None, 1, T, D, EPS, dx, dw, part)
    dx_want, _, size, _ = ref.rms_norm_grad(some, host(y[at]), None, w, EPS)
    assert np.all(np.abs(host(dx[at]) - dx_want) <= size * (90 * U32) + np.abs(dx_want) * HALF[BF16])
    assert ctx.aug_last_status() == (-1, 0)


# ----------------------------------------------------------------------------- the product's longest rows
@pytest.mark.parametrize("kind,K", [(MX4, 2304), (MX4, 2305), (MX4, 4353), (MX4, 6913), (MX4, 11776), (MX4, 11777), (MX4, 13312), (MX4, 13313),
                                    (MX8, 1152), (MX8, 1153), (MX8, 2305), (MX8, 3841), (MX8, 7040), (MX8, 7041), (MX8, 7808),
                                    (MX8, 7809)])
@pytest.mark.parametrize("N,t", [(16, BF16), (200, F32)])
def test_product_at_the_ends_of_its_tiles(ctx, kind, K, N, t):
    """Where tiles get narrower for the length of the rows, and where the rows go another way."""
    check_product(ctx, 1, 140, K, N, None, kind, t, seed=K + N)
