"""Norm, gradient, microscaled conversion and product of the rows of padded batches, against 64 bits."""
import numpy as np
import pytest

import row_reference as ref
from helpers import Device
from paper_1912_11040_b200 import binding, synth

pytestmark = pytest.mark.gpu

EPS = 1e-5
F32, BF16, MX8, MX4 = binding.ELEM_F32, binding.ELEM_BF16, binding.ELEM_MX8, binding.ELEM_MX4
U32 = 2.0 ** -24                                  # half a step of fp32, relative
HALF = {F32: U32, BF16: 2.0 ** -8}                # of the types
KIND = {MX8: "mx8", MX4: "mx4"}
# widths: one value, less than a block, blocks and groups and one more or less, every split of a row over threads,
# with and without 128-bit accesses
WIDTHS = [1, 3, 8, 31, 32, 33, 40, 100, 128, 129, 136, 257, 264, 513, 640, 1000, 1024, 1031, 1536, 2050, 4096, 4100, 6000, 10001,
          16384]
PAD = -7.0


def context(stream=None, max_batch=64, pad=PAD):
    config = binding.AugConfig(
        fs=16000, win=400, hop=160, n_fft=512, n_mel=40, f_lo=0.0, f_hi=8000.0, rir_taps=1, max_order=0, max_sources=1,
        frac_half_width=40, sound_speed=343.0, log_floor=1e-7, pad_value=pad, compression=0, max_batch=max_batch,
        max_samples=400)
    return binding.AugContext(config, stream)


@pytest.fixture(scope="module")
def ctx():
    return context()


def torch_type(t):
    import torch
    return {F32: torch.float32, BF16: torch.bfloat16}[t]


def on_device(x, t, shift=0):
    """A tensor of type t with x's values (rounded), `shift` elements behind a 16-byte boundary."""
    import torch
    flat = torch.zeros(x.size + shift, dtype=torch_type(t), device="cuda")
    out = flat[shift:].view(x.shape)
    out.copy_(torch.from_numpy(np.ascontiguousarray(x)))
    return out


def host(t):
    return t.detach().double().cpu().numpy()


def guarded(shape, dtype, value, shift=0):
    """(tensor of `shape` filled with `value`, check that nothing around it was written)"""
    import torch
    n, edge = int(np.prod(shape)), 64
    flat = torch.full((n + 2 * edge + shift,), value, dtype=dtype, device="cuda")
    mine = flat[edge + shift: edge + shift + n].view(shape)

    def intact():
        return bool((flat[: edge + shift] == value).all()) and bool((flat[edge + shift + n:] == value).all())
    return mine, intact


def to_counts(counts):
    import torch
    return None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")


def rows(rng, B, T, D, counts, t, scale=1.0):
    """Values rounded to t, with NaN in the rows that hold none."""
    import torch
    x = scale * rng.normal(size=(B, T, D)) * np.exp(rng.normal(size=D))
    x = host(torch.from_numpy(x).to(torch_type(t)))
    x[~ref.holds(counts, B, T)] = np.nan
    return x


# ----------------------------------------------------------------------------- norm
def check_norm(ctx, B, T, D, counts, t, yt, residual=True, weight=True, shift=0, seed=0, scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    x = rows(rng, B, T, D, counts, t, scale)
    r = rows(rng, B, T, D, counts, t, scale) if residual else None
    w = rng.normal(size=D).astype(np.float32) if weight else None
    y, y_ok = guarded((B, T, D), torch_type(yt), 3.0, shift)
    s, s_ok = guarded((B, T, D), torch_type(t), 3.0, shift)
    ctx.feat_rms_norm(on_device(x, t, shift), on_device(r, t, shift) if residual else None, t,
                      None if w is None else torch.from_numpy(w).cuda(), to_counts(counts), B, T, D, EPS,
                      s if residual else None, y, yt)
    torch.cuda.synchronize()
    ok = ref.holds(counts, B, T)
    h, want = ref.rms_norm(x, r, w, EPS)
    got = host(y)
    # The sum of D squares takes at most 32 additions in a thread, 5 between lanes and 16 between warps, each off by
    # U32 at most, and half of that reaches 1/sqrt, itself good to 2 units (4 U32); h (its square counts twice,
    # halved again), mean, eps and the two products are one U32 each: 27 + 4 + 6.
    tol = np.abs(want) * (40 * U32 + HALF[yt])
    assert np.all(np.abs(got - want)[ok] <= tol[ok])
    assert np.all(got[~ok] == PAD) and y_ok()
    if residual:
        assert np.all(np.abs(host(s) - h)[ok] <= (np.abs(h) * (U32 + HALF[t]))[ok])
        assert np.all(host(s)[~ok] == PAD) and s_ok()


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("t,yt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
def test_norm_widths(ctx, D, t, yt):
    check_norm(ctx, 3, 5, D, [5, 0, 2], t, yt, seed=D)


@pytest.mark.parametrize("B,T,counts", [(1, 1, None), (1, 1, [0]), (1, 1, [1]), (64, 1, None), (2, 301, [301, 17]),
                                        (5, 37, [-3, 99, 37, 0, 1])])
@pytest.mark.parametrize("D", [40, 257, 1024])
def test_norm_batches(ctx, B, T, counts, D):
    check_norm(ctx, B, T, D, None if counts is None else [min(c, T) for c in counts], BF16, F32)
    check_norm(ctx, B, T, D, counts, F32, F32, residual=False, weight=False)


@pytest.mark.parametrize("D", [8, 128, 1024, 4096])
@pytest.mark.parametrize("t", [F32, BF16])
def test_norm_of_rows_beside_16_byte_boundaries(ctx, D, t):
    check_norm(ctx, 2, 3, D, [3, 1], t, t, shift=1)


@pytest.mark.parametrize("D", [40, 257, 1024, 4096])
def test_norm_of_squares_beyond_fp32(ctx, D):
    check_norm(ctx, 2, 3, D, [3, 1], F32, F32, scale=1e20)
    check_norm(ctx, 2, 3, D, [3, 1], F32, F32, scale=1e-30)


def test_norm_of_what_is_not_finite(ctx):
    import torch
    x = torch.ones(1, 4, 64, device="cuda")
    x[0, 1, 5] = float("inf")
    x[0, 2, 7] = float("nan")
    y = torch.empty_like(x)
    ctx.feat_rms_norm(x, None, F32, None, None, 1, 4, 64, EPS, None, y, F32)
    y = y.cpu()
    assert torch.isfinite(y[0, 0]).all() and torch.isfinite(y[0, 3]).all()       # other rows keep clear of it
    assert torch.isnan(y[0, 1, 5]) and (y[0, 1, :5] == 0).all()                  # inf / inf, 1 / inf
    assert torch.isnan(y[0, 2]).all()


def test_norm_of_zeros_is_zero(ctx):
    import torch
    x = torch.zeros(1, 2, 40, device="cuda")
    y = torch.full_like(x, 3.0)
    ctx.feat_rms_norm(x, x, F32, None, None, 1, 2, 40, EPS, None, y, F32)
    assert (y == 0).all()


@pytest.mark.parametrize("D", [40, 257, 1024])
def test_norm_in_place(ctx, D):
    """The sum over the residual stream, the output over the input."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, r = (torch.randn(4, 9, D, device="cuda", generator=gen).bfloat16() for _ in range(2))
    counts = to_counts([9, 0, 4, 1])
    s, y = torch.empty_like(x), torch.empty_like(x)
    ctx.feat_rms_norm(x, r, BF16, None, counts, 4, 9, D, EPS, s, y, BF16)
    ctx.feat_rms_norm(x, r, BF16, None, counts, 4, 9, D, EPS, r, x, BF16)
    assert torch.equal(s, r) and torch.equal(y, x)


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("kind", [MX8, MX4])
def test_norm_to_codes_is_the_norm_quantised(ctx, D, kind):
    import torch
    B, T, counts = 3, 4, [4, 0, 3]
    rng = np.random.default_rng(D)
    for t in (F32, BF16):
        x = on_device(rows(rng, B, T, D, counts, t), t)
        w = torch.from_numpy(rng.normal(size=D).astype(np.float32)).cuda()
        y = torch.empty(B, T, D, device="cuda")
        size = (B, T, binding.feat_mx_code_bytes(kind, D)), (B, T, binding.feat_mx_scale_bytes(D))
        out = [[guarded(s, torch.uint8, 0xAB, 0) for s in size] for _ in range(2)]
        c = to_counts(counts)
        ctx.feat_rms_norm(x, None, t, w, c, B, T, D, EPS, None, y, F32)
        ctx.feat_mx_quantize(y, F32, c, B, T, D, out[0][0][0], kind, out[0][1][0])
        ctx.feat_rms_norm(x, None, t, w, c, B, T, D, EPS, None, out[1][0][0], kind, out[1][1][0])
        for a, b in zip(*out):
            assert torch.equal(a[0], b[0]) and a[1]() and b[1]()
        assert (out[0][0][0][1] == 0).all() and (out[0][1][0][1] == 0).all()      # an utterance without frames


# ----------------------------------------------------------------------------- gradients
def check_grad(ctx, B, T, D, counts, t, dsum=True, weight=True, shift=0, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    h, dy = (rows(rng, B, T, D, counts, t) for _ in range(2))
    ds = rows(rng, B, T, D, counts, t) if dsum else None
    w = rng.normal(size=D).astype(np.float32) if weight else None
    dx, dx_ok = guarded((B, T, D), torch_type(t), 3.0, shift)
    dw, dw_ok = guarded((D,), torch.float32, 3.0)
    part, part_ok = guarded((binding.feat_rms_norm_partial_floats(D),), torch.float32, 3.0)
    args = (on_device(h, t, shift), on_device(dy, t, shift), on_device(ds, t, shift) if dsum else None, t,
            None if w is None else torch.from_numpy(w).cuda(), to_counts(counts), B, T, D, EPS)
    ctx.feat_rms_norm_grad(*args, dx, dw, part)
    torch.cuda.synchronize()
    ok = ref.holds(counts, B, T)
    want, dw_want, size, dw_size = ref.rms_norm_grad(*(None if v is None else np.where(ok[..., None], v, 0.0)
                                                       for v in (h, dy, ds)), w, EPS)
    got = host(dx)
    # two sums of D terms like the norm's (53 U32 of the magnitudes each), 1/sqrt three times over, ten products
    assert np.all(np.abs(got - want)[ok] <= (size * (90 * U32) + np.abs(want) * HALF[t])[ok])
    assert np.all(got[~ok] == 0) and dx_ok()
    # every addition of a column is off by U32 of the magnitudes at most: one a row, and 400 between CTAs and warps at
    # the most; the terms themselves by 40 U32
    assert np.all(np.abs(host(dw) - dw_want) <= dw_size * ((B * T + 440) * U32)) and dw_ok() and part_ok()
    first = dx.clone(), dw.clone()
    ctx.feat_rms_norm_grad(*args, dx, dw, part)
    assert torch.equal(first[0], dx) and torch.equal(first[1], dw)


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("t", [F32, BF16])
def test_grad_widths(ctx, D, t):
    check_grad(ctx, 3, 5, D, [5, 0, 2], t, seed=D)


@pytest.mark.parametrize("B,T,counts", [(1, 1, None), (1, 1, [0]), (64, 1, None), (3, 1500, [1500, 0, 700])])
@pytest.mark.parametrize("D", [40, 257, 1024, 1536])
def test_grad_batches(ctx, B, T, counts, D):
    check_grad(ctx, B, T, D, counts, BF16)
    check_grad(ctx, B, T, D, counts, F32, dsum=False, weight=False)


@pytest.mark.parametrize("t", [F32, BF16])
def test_grad_of_rows_beside_16_byte_boundaries(ctx, t):
    check_grad(ctx, 2, 3, 512, [3, 1], t, shift=1)


def test_grad_in_place_and_of_no_utterances(ctx):
    import torch
    D = 264
    gen = torch.Generator(device="cuda").manual_seed(1)
    h, dy, ds = (torch.randn(2, 6, D, device="cuda", generator=gen) for _ in range(3))
    dw, part = torch.empty(D, device="cuda"), torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    dx = torch.empty_like(h)
    ctx.feat_rms_norm_grad(h, dy, ds, F32, None, None, 2, 6, D, EPS, dx, dw, part)
    for k in range(3):
        v = [h.clone(), dy.clone(), ds.clone()]
        dw2 = torch.empty_like(dw)
        ctx.feat_rms_norm_grad(*v, F32, None, None, 2, 6, D, EPS, v[k], dw2, part)
        assert torch.equal(v[k], dx) and torch.equal(dw2, dw)
    ctx.feat_rms_norm_grad(None, None, None, F32, None, None, 0, 6, D, EPS, None, dw, None)
    assert (dw == 0).all()


# ----------------------------------------------------------------------------- microscaled numbers
def awkward(rng, rows_, D, t):
    """Values over the types' whole range: powers of two and their neighbours, ties, zeros, denormals."""
    import torch
    x = rng.normal(size=(rows_, D)) * np.exp2(rng.integers(-150, 120, (rows_, 1)).astype(float))
    k = rng.integers(0, 6, (rows_, D))
    ties = rng.choice([0.25, 0.75, 1.25, 2.5, 3.5, 5.0, 1.0625, 1.1875, 464.0, 2.0 ** -10], (rows_, D))
    x = np.where(k == 0, ties * np.sign(x), x)
    x = np.where(k == 1, 0.0, x)
    x[0] = 0.0
    if rows_ > 2:
        x[1, :: 3] = np.exp2(np.floor(rng.uniform(-100, 100)))
        x[2, 0] = np.inf
        x[2, -1] = np.nan
    with np.errstate(over="ignore"):
        return host(torch.from_numpy(x).to(torch_type(t)))


@pytest.mark.parametrize("D", [1, 31, 32, 33, 40, 128, 129, 136, 257, 640, 1000])
@pytest.mark.parametrize("kind", [MX8, MX4])
@pytest.mark.parametrize("t", [F32, BF16])
def test_quantise_and_back_bit_by_bit(ctx, D, kind, t):
    import torch
    B, T, counts = 3, 7, [7, 0, 5]
    rng = np.random.default_rng(D)
    for shift in (0, 1):
        x = awkward(rng, B * T, D, t).reshape(B, T, D)
        ok = ref.holds(counts, B, T)
        codes, c_ok = guarded((B * T, binding.feat_mx_code_bytes(kind, D)), torch.uint8, 0xAB)
        scales, s_ok = guarded((B * T, binding.feat_mx_scale_bytes(D)), torch.uint8, 0xAB)
        ctx.feat_mx_quantize(on_device(x, t, shift), t, to_counts(counts), B, T, D, codes, kind, scales)
        want_c, want_s = ref.quantize(np.where(ok[..., None], x, 0.0).reshape(B * T, D), KIND[kind])
        got_c, got_s = ref.unpacked(codes.cpu().numpy(), KIND[kind]), scales.cpu().numpy()
        assert np.array_equal(got_s, want_s)
        sign = 128 if kind == MX8 else 8
        assert np.array_equal(np.where(got_c == sign, 0, got_c), np.where(want_c == sign, 0, want_c))   # (-0 is 0)
        assert c_ok() and s_ok()
        values = ref.dequantize(got_c, got_s, KIND[kind], D).reshape(B, T, D)
        for back in (F32, BF16):
            v, v_ok = guarded((B, T, D), torch_type(back), 3.0, shift)
            ctx.feat_mx_dequantize(codes, kind, scales, to_counts(counts), B, T, D, v, back)
            v = host(v)
            assert np.array_equal(v[ok], values[ok], equal_nan=True)
            assert np.all(v[~ok] == PAD) and v_ok()


def test_dequantise_reads_every_code_and_scale(ctx):
    import torch
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(256, 1).contiguous()       # D = 256
    scales = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, 8).contiguous()
    v = torch.empty(256, 256, device="cuda")
    ctx.feat_mx_dequantize(codes, MX8, scales, None, 1, 256, 256, v, F32)
    want = ref.dequantize(codes.cpu().numpy(), scales.cpu().numpy(), "mx8", 256)
    with np.errstate(over="ignore"):
        assert np.array_equal(host(v), want.astype(np.float32), equal_nan=True)


# ----------------------------------------------------------------------------- product
def random_codes(rng, rows_, K, kind, spread=3):
    """Random microscaled rows: (raw codes, scales) as they lie in memory, and their values."""
    x = rng.normal(size=(rows_, K)) * np.exp2(rng.integers(-spread, spread + 1, (rows_, K)).astype(float))
    codes, scales = ref.quantize(x, KIND[kind])
    return ref.packed(codes, KIND[kind]), scales, ref.dequantize(codes, scales, KIND[kind], K)


def check_product(ctx, B, T, K, N, counts, kind, t, bias=True, shift=0, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    a_raw, a_scales, a = random_codes(rng, B * T, K, kind)
    w_raw, w_scales, w = random_codes(rng, N, K, MX4)
    ok = ref.holds(counts, B, T)
    a_raw[~ok.reshape(-1)] = 0x7F                   # rows that hold nothing hold anything: NaN among it
    a_scales[~ok.reshape(-1)] = 255
    b = rng.normal(size=N).astype(np.float32) if bias else None
    out, out_ok = guarded((B, T, N), torch_type(t), 3.0, shift)
    dev = [torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (a_raw, a_scales, w_raw, w_scales)]
    ctx.feat_mx_product(dev[0], kind, dev[1], dev[2], dev[3], None if b is None else torch.from_numpy(b).cuda(),
                        to_counts(counts), B, T, K, N, out, t)
    torch.cuda.synchronize()
    assert ctx.aug_last_status() == (-1, 0)
    a = a.reshape(B, T, K)
    want = a @ w.T + (0.0 if b is None else b)
    size = np.abs(a) @ np.abs(w).T + (0.0 if b is None else np.abs(b))
    got = host(out)
    # K + 1 additions, none off by more than a whole unit of the magnitudes (2 U32: sums may be cut rather than
    # rounded), and the rounding to the type
    tol = size * ((K + 1) * 2 * U32) + np.abs(want) * HALF[t]
    assert np.all(np.abs(got - want)[ok] <= tol[ok])
    assert np.all(got[~ok] == PAD) and out_ok()


@pytest.mark.parametrize("kind", [MX4, MX8])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("K,N", [(1, 1), (32, 16), (40, 33), (128, 128), (129, 257), (256, 64), (640, 1024), (1000, 1001),
                                 (1536, 100)])
@pytest.mark.parametrize("B,T,counts", [(1, 1, None), (3, 2, [2, 0, 1]), (2, 200, [200, 61])])
def test_product_shapes(ctx, kind, t, K, N, B, T, counts):
    check_product(ctx, B, T, K, N, counts, kind, t, seed=K + N)


@pytest.mark.parametrize("kind", [MX4, MX8])
@pytest.mark.parametrize("rows_", [1, 2, 4, 5, 8, 9, 16, 17, 31, 64, 127, 128, 129, 255, 300])
def test_product_row_counts(ctx, kind, rows_):
    check_product(ctx, 1, rows_, 384, 200, None, kind, F32, bias=False, seed=rows_)


@pytest.mark.parametrize("kind", [MX4, MX8])
@pytest.mark.parametrize("K", [2048, 4096, 8192, 16384])
def test_product_long_rows(ctx, kind, K):
    check_product(ctx, 1, 140, K, 48, None, kind, F32, seed=K)
    check_product(ctx, 1, 1, K, 48, None, kind, F32, seed=K)


@pytest.mark.parametrize("kind", [MX4, MX8])
def test_product_of_many_tiles(ctx, kind):
    check_product(ctx, 8, 700, 512, 1024, [700, 0, 1, 130, 699, 700, 0, 0], kind, BF16)
    check_product(ctx, 64, 1, 256, 4096, [1] * 20 + [0] * 44, kind, F32)
    check_product(ctx, 3, 6000, 128, 40, [5000, 0, 6000], kind, F32)


@pytest.mark.parametrize("kind", [MX4, MX8])
@pytest.mark.parametrize("t", [F32, BF16])
def test_product_of_long_rows_in_narrow_tiles(ctx, kind, t):
    """So long that shared memory holds fewer columns of weights than are written at once."""
    check_product(ctx, 2, 150, 4096, 300, [150, 9], kind, t)
    check_product(ctx, 1, 129, 6000, 77, None, kind, t)


@pytest.mark.parametrize("kind", [MX4, MX8])
def test_product_whose_weights_change_often(ctx, kind):
    """Few rows, many columns: a multiprocessor loads weights several times."""
    check_product(ctx, 2, 65, 256, 16384, [65, 64], kind, BF16)
    check_product(ctx, 1, 257, 40, 12000, None, kind, F32)


@pytest.mark.parametrize("kind", [MX4, MX8])
def test_product_of_mostly_nothing(ctx, kind):
    """Tiles, columns and multiprocessors without a row that holds values."""
    check_product(ctx, 64, 128, 200, 1024, [0] * 63 + [5], kind, BF16)
    check_product(ctx, 64, 100, 200, 520, [0] * 64, kind, F32)
    check_product(ctx, 64, 100, 520, 77, [0, 100] * 32, kind, BF16)


@pytest.mark.parametrize("N", [1, 2, 31, 33, 63, 64, 65, 127, 129, 193, 225])
@pytest.mark.parametrize("t,shift", [(F32, 0), (F32, 1), (BF16, 0), (BF16, 1)])
def test_product_ends_of_rows(ctx, N, t, shift):
    check_product(ctx, 1, 133, 96, N, [131], MX4, t, shift=shift, seed=N)


@pytest.mark.parametrize("t", [F32, BF16])
def test_product_beside_16_byte_boundaries(ctx, t):
    check_product(ctx, 2, 90, 256, 128, [90, 3], MX4, t, shift=1)


@pytest.mark.parametrize("kind", [MX4, MX8])
@pytest.mark.parametrize("shift", [8, 16, 32])
def test_product_between_64_byte_boundaries(ctx, kind, shift):
    check_product(ctx, 2, 190, 256, 320, [190, 3], kind, BF16, shift=shift)
    check_product(ctx, 2, 190, 256, 328, [190, 3], kind, F32, shift=shift // 2)


@pytest.mark.parametrize("rows_", [1, 130])
@pytest.mark.parametrize("kind", [MX4, MX8])
def test_product_of_a_block_that_is_not_finite(ctx, rows_, kind):
    import torch
    rng = np.random.default_rng(0)
    a_raw, a_scales, _ = random_codes(rng, rows_, 256, kind)
    w_raw, w_scales, _ = random_codes(rng, 40, 256, MX4)
    a_scales[0, 3] = 255
    dev = [torch.from_numpy(v).cuda() for v in (a_raw, a_scales, w_raw, w_scales)]
    out = torch.zeros(rows_, 40, device="cuda")
    ctx.feat_mx_product(dev[0], kind, dev[1], dev[2], dev[3], None, None, 1, rows_, 256, 40, out, F32)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1:]).all()
    dev[1][0, 3] = 100
    dev[3][7, 0] = 255
    ctx.feat_mx_product(dev[0], kind, dev[1], dev[2], dev[3], None, None, 1, rows_, 256, 40, out, F32)
    bad = torch.isnan(out)
    assert bad[:, 7].all() and bad.sum() == rows_


@pytest.mark.parametrize("rows_", [1, 130])
@pytest.mark.parametrize("kind", [MX4, MX8])
def test_product_of_far_apart_scales(ctx, rows_, kind):
    """2^-120 times 2^120, and 2^100 times 2^-100: nothing overflows or is lost on the way."""
    import torch
    rng = np.random.default_rng(0)
    a_raw, a_scales, _ = random_codes(rng, rows_, 128, kind)
    w_raw, w_scales, _ = random_codes(rng, 40, 128, MX4)
    a_scales[:] = [7, 227, 127, 130]
    w_scales[:] = [247, 27, 127, 124]
    a = ref.dequantize(ref.unpacked(a_raw, KIND[kind]), a_scales, KIND[kind], 128)
    w = ref.dequantize(ref.unpacked(w_raw, "mx4"), w_scales, "mx4", 128)
    dev = [torch.from_numpy(v).cuda() for v in (a_raw, a_scales, w_raw, w_scales)]
    out = torch.zeros(rows_, 40, device="cuda")
    ctx.feat_mx_product(dev[0], kind, dev[1], dev[2], dev[3], None, None, 1, rows_, 128, 40, out, F32)
    assert np.all(np.abs(host(out) - a @ w.T) <= 129 * 2 * U32 * (np.abs(a) @ np.abs(w).T) + np.abs(a @ w.T) * U32)


# ----------------------------------------------------------------------------- together, and how they are called
def layer(ctx, feats, counts, B, T, D, N, w, kind, stream_rows, out):
    """Norm to codes, product, norm of its sum with a residual stream: two layers' seam."""
    import torch
    codes = torch.empty(B, T, binding.feat_mx_code_bytes(kind, D), dtype=torch.uint8, device="cuda")
    scales = torch.empty(B, T, binding.feat_mx_scale_bytes(D), dtype=torch.uint8, device="cuda")
    y = torch.empty(B, T, N, dtype=torch.bfloat16, device="cuda")
    ctx.feat_rms_norm(feats, None, F32, w["gain"], counts, B, T, D, EPS, None, codes, kind, scales)
    ctx.feat_mx_product(codes, kind, scales, w["codes"], w["scales"], w["bias"], counts, B, T, D, N, y, BF16)
    ctx.feat_rms_norm(y, stream_rows, BF16, None, counts, B, T, N, EPS, stream_rows, out, BF16)
    return codes, scales, y


def layer_weights(ctx, D, N, gen):
    import torch
    w = {"gain": 1 + 0.1 * torch.randn(D, device="cuda", generator=gen), "bias": torch.randn(N, device="cuda", generator=gen),
         "codes": torch.empty(N, binding.feat_mx_code_bytes(MX4, D), dtype=torch.uint8, device="cuda"),
         "scales": torch.empty(N, binding.feat_mx_scale_bytes(D), dtype=torch.uint8, device="cuda")}
    ctx.feat_mx_quantize(torch.randn(N, D, device="cuda", generator=gen) / D ** 0.5, F32, None, 1, N, D, w["codes"], MX4,
                         w["scales"])
    return w


@pytest.mark.parametrize("kind", [MX8, MX4])
def test_features_through_a_layer(kind):
    """The features of a batch, as the pipeline leaves them, through norm, product and the next norm."""
    import torch
    w = synth.make_workload(1, batch=5, dur_scale=0.6)
    w.lengths[1] = 300                               # no frames
    dev = Device(w)
    F, counts, _ = dev.pipeline(want_wave=False)
    B, T, D, N = w.B, dev.T_max, dev.M, 96
    gen = torch.Generator(device="cuda").manual_seed(3)
    weights = layer_weights(dev.ctx, D, N, gen)
    stream = torch.randn(B, T, N, device="cuda", generator=gen).bfloat16()
    before = host(stream)
    out = torch.empty_like(stream)
    codes, scales, y = layer(dev.ctx, F, counts, B, T, D, N, weights, kind, stream, out)
    torch.cuda.synchronize()
    ok = ref.holds(counts.cpu().numpy(), B, T)
    assert ok.sum() == int(counts.sum()) and not ok[1].any()
    normed = ref.rms_norm(host(F), None, host(weights["gain"]), EPS)[1]
    raw = ref.unpacked(codes.cpu().numpy().reshape(B * T, -1), KIND[kind])
    a = ref.dequantize(raw, scales.cpu().numpy().reshape(B * T, -1), KIND[kind], D).reshape(B, T, D)
    # a block's values are off by half a step of its largest: 2^-4 or 2^-2 of it, a quarter where they saturate
    blocks = np.zeros((B, T, 64))
    blocks[..., :D] = np.where(ok[..., None], normed, 0.0)
    top = np.repeat(np.abs(blocks.reshape(B, T, 2, 32)).max(-1), 32, -1)[..., :D]
    assert np.all(np.abs(a - normed)[ok] <= (top * (0.126 if kind == MX8 else 0.251))[ok])
    wv = ref.dequantize(ref.unpacked(weights["codes"].cpu().numpy(), "mx4"), weights["scales"].cpu().numpy(), "mx4", D)
    want = a @ wv.T + host(weights["bias"])
    size = np.abs(a) @ np.abs(wv).T + np.abs(host(weights["bias"]))
    assert np.all(np.abs(host(y) - want)[ok] <= (size * (D + 1) * 2 * U32 + np.abs(want) * HALF[BF16])[ok])
    h, z = ref.rms_norm(host(y), before, None, EPS)
    assert np.all(np.abs(host(out) - z)[ok] <= (np.abs(z) * (40 * U32 + HALF[BF16]))[ok])
    assert np.all(np.abs(host(stream) - h)[ok] <= (np.abs(h) * (U32 + HALF[BF16]))[ok])
    assert np.all(host(out)[~ok] == dev.cfg.pad_value)


@pytest.mark.parametrize("T", [1, 150])
def test_captured_replayed_and_on_another_stream(T):
    import torch
    B, D, N = 3, 264, 80
    counts = to_counts([T, 0, max(1, T // 2)])
    gen = torch.Generator(device="cuda").manual_seed(T)
    s = torch.cuda.Stream()
    ctx = context(s.cuda_stream)
    with torch.cuda.stream(s):
        weights = layer_weights(ctx, D, N, gen)
        feats = torch.randn(B, T, D, device="cuda", generator=gen)
        stream0 = torch.randn(B, T, N, device="cuda", generator=gen).bfloat16()
        want, got = torch.empty_like(stream0), torch.empty_like(stream0)
        dx, dw = torch.empty_like(feats), torch.empty(D, device="cuda")
        part = torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
        dx_want, dw_want = torch.empty_like(dx), torch.empty_like(dw)
        run = stream0.clone()
        layer(ctx, feats, counts, B, T, D, N, weights, MX4, run, want)
        ctx.feat_rms_norm_grad(feats, feats, None, F32, weights["gain"], counts, B, T, D, EPS, dx_want, dw_want, part)
        run.copy_(stream0)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        layer(ctx, feats, counts, B, T, D, N, weights, MX4, run, got)
        ctx.feat_rms_norm_grad(feats, feats, None, F32, weights["gain"], counts, B, T, D, EPS, dx, dw, part)
    for _ in range(3):
        run.copy_(stream0)
        got.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(dx, dx_want) and torch.equal(dw, dw_want)
    del g


def test_operators_back_to_back_wait_for_one_another():
    """Every kernel here writes what the next one reads, over what the one before it has read: the same bits as with a
    wait for the device after every call."""
    import torch
    with torch.cuda.stream(torch.cuda.Stream()):
        back_to_back(context(torch.cuda.current_stream().cuda_stream))


def back_to_back(ctx):
    import torch
    B, T, D, N = 16, 500, 264, 264
    gen = torch.Generator(device="cuda").manual_seed(9)
    w = layer_weights(ctx, D, N, gen)
    counts = to_counts([T, 3, 0, 499] * 4)
    first = torch.randn(B, T, D, device="cuda", generator=gen)
    gain, dw = w["gain"].clone(), torch.empty(D, device="cuda")
    partial = torch.empty(binding.feat_rms_norm_partial_floats(D), device="cuda")
    codes = torch.empty(B, T, binding.feat_mx_code_bytes(MX8, D), dtype=torch.uint8, device="cuda")
    scales = torch.empty(B, T, binding.feat_mx_scale_bytes(D), dtype=torch.uint8, device="cuda")

    def passes(after):
        x, y = first.clone(), torch.empty(B, T, N, device="cuda")
        gain.copy_(w["gain"])
        for _ in range(6):
            ctx.feat_rms_norm(x, None, F32, gain, counts, B, T, D, EPS, None, codes, MX8, scales)
            after()
            ctx.feat_mx_product(codes, MX8, scales, w["codes"], w["scales"], gain, counts, B, T, D, N, y, F32)
            after()
            ctx.feat_rms_norm_grad(x, y, None, F32, gain, counts, B, T, D, EPS, x, dw, partial)
            after()
            ctx.feat_rms_norm(dw, None, F32, None, None, 1, 1, D, EPS, None, gain, F32, None)
            after()
            ctx.feat_mx_quantize(x, F32, counts, B, T, D, codes, MX8, scales)
            after()
            ctx.feat_mx_dequantize(codes, MX8, scales, counts, B, T, D, x, F32)
            after()
        torch.cuda.synchronize()
        return host(x), host(y), host(gain)

    want = passes(torch.cuda.synchronize)
    for _ in range(5):
        for a, b in zip(passes(lambda: None), want):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("captured", [False, True])
def test_operators_after_two_streams_join(captured):
    """The rows are quantised on one stream, the weights on another; the product waits for both, again and again over
    the same buffers."""
    import torch
    B, T, D, N = 8, 400, 512, 512
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn(B, T, D, device="cuda", generator=gen), torch.randn(N, D, device="cuda", generator=gen)
    bytes_, sbytes = binding.feat_mx_code_bytes(MX4, D), binding.feat_mx_scale_bytes(D)
    new = lambda *shape: torch.empty(*shape, dtype=torch.uint8, device="cuda")
    a, sa, q, sq = new(B * T, bytes_), new(B * T, sbytes), new(N, bytes_), new(N, sbytes)
    y = torch.empty(B, T, N, device="cuda")
    s, side = torch.cuda.Stream(), torch.cuda.Stream()
    ctx, beside = context(s.cuda_stream), context(side.cuda_stream)

    def step():
        side.wait_stream(s)
        beside.feat_mx_quantize(w, F32, None, 1, N, D, q, MX4, sq)
        ctx.feat_mx_quantize(x, F32, None, B, T, D, a, MX4, sa)
        s.wait_stream(side)
        ctx.feat_mx_product(a, MX4, sa, q, sq, None, None, B, T, D, N, y, F32)

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    want = y.clone()
    raw = [ref.dequantize(ref.unpacked(c.cpu().numpy(), "mx4"), sc.cpu().numpy(), "mx4", D) for c, sc in ((a, sa), (q, sq))]
    exact = (raw[0] @ raw[1].T).reshape(B, T, N)
    # sums in fp32 of D products: D steps of 2^-24 of the sum of their sizes at most
    assert (np.abs(host(want) - exact) <= D * 2.0 ** -24 * (np.abs(raw[0]) @ np.abs(raw[1]).T).reshape(B, T, N)).all()
    if captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
    for k in range(6):
        with torch.cuda.stream(s):
            for t in (a, sa, q, sq, y):
                t.zero_()
            g.replay() if captured else step()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_two_contexts_at_once():
    """Two streams, the same operators, nothing shared but the weights."""
    import torch
    B, T, D, N = 2, 400, 512, 512
    gen = torch.Generator(device="cuda").manual_seed(0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [context(s.cuda_stream) for s in streams]
    main = context()
    weights = layer_weights(main, D, N, gen)
    feats = [torch.randn(B, T, D, device="cuda", generator=gen) for _ in range(2)]
    zero = lambda: torch.zeros(B, T, N, dtype=torch.bfloat16, device="cuda")
    wants = []
    for f in feats:
        wants.append(zero())
        layer(main, f, None, B, T, D, N, weights, MX8, zero(), wants[-1])
    torch.cuda.synchronize()
    outs = [zero() for _ in range(2)]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                layer(ctxs[i], feats[i], None, B, T, D, N, weights, MX8, zero(), outs[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))


def test_no_utterances_and_refusals(ctx):
    import torch
    x = torch.zeros(4, 1024, device="cuda")
    u = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    f = torch.zeros(296 * 64, device="cuda")
    E, C = binding.AUG_EINVAL, binding.AUG_ECAP
    norm = lambda **k: ctx.feat_rms_norm(*(dict(x=x, r=None, t=F32, w=None, c=None, B=1, T=2, D=64, eps=EPS, s=None, y=x,
                                                yt=F32, sc=None) | k).values(), check=False)
    assert norm() == 0 and norm(B=0) == 0 and norm(B=0, x=None, y=None) == 0
    for bad in (dict(x=None), dict(y=None), dict(t=MX8), dict(t=9), dict(yt=7), dict(yt=-1), dict(T=0), dict(D=0), dict(B=-1),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(yt=MX8),
                dict(sc=u), dict(yt=BF16), dict(s=x), dict(c=u[1:]), dict(yt=MX4, y=u[4:], sc=u), dict(yt=MX4, y=u, sc=u[4:]), dict(x=u[1:]), dict(w=u[2:])):
        assert norm(**bad) == E, bad
    for cap in (dict(B=65), dict(D=16385), dict(T=(1 << 30) + 1), dict(B=64, T=1 << 25)):
        assert norm(**cap) == C, cap
    grad = lambda **k: ctx.feat_rms_norm_grad(*(dict(h=x, dy=x, ds=None, t=F32, w=None, c=None, B=1, T=2, D=64, eps=EPS,
                                                     dx=x, dw=f, p=f) | k).values(), check=False)
    assert grad(dw=torch.zeros(64, device="cuda")) == 0
    for bad in (dict(h=None), dict(dy=None), dict(dx=None), dict(dw=None), dict(p=None), dict(t=MX4), dict(eps=0.0),
                dict(D=-5), dict(p=u[2:]), dict(ds=u[2:])):
        assert grad(**bad) == E, bad
    assert grad(B=65) == C and grad(D=16385) == C
    quant = lambda **k: ctx.feat_mx_quantize(*(dict(x=x, t=F32, c=None, B=1, T=2, D=64, q=u, k=MX8, s=u) | k).values(),
                                             check=False)
    back = lambda **k: ctx.feat_mx_dequantize(*(dict(q=u, k=MX8, s=u, c=None, B=1, T=2, D=64, x=x, t=F32) | k).values(),
                                              check=False)
    for call in (quant, back):
        assert call() == 0 and call(B=0) == 0
        for bad in (dict(x=None), dict(q=None), dict(s=None), dict(t=MX8), dict(k=F32), dict(q=u[8:]), dict(s=u[4:]),
                    dict(x=u[1:]), dict(T=-1), dict(D=0)):
            assert call(**bad) == E, bad
        assert call(B=65) == C and call(T=(1 << 30) + 1) == C
    prod = lambda **k: ctx.feat_mx_product(*(dict(a=u, k=MX8, s=u, w=u, ws=u, b=None, c=None, B=1, T=2, K=64, N=8, o=x, t=F32)
                                             | k).values(), check=False)
    assert prod() == 0 and prod(B=0) == 0
    for bad in (dict(a=None), dict(s=None), dict(w=None), dict(ws=None), dict(o=None), dict(k=BF16), dict(t=MX8), dict(N=0),
                dict(K=0), dict(a=u[8:]), dict(w=u[8:]), dict(ws=u[4:]), dict(s=u[4:]), dict(b=u[2:]), dict(o=u[2:])):
        assert prod(**bad) == E, bad
    assert prod(K=16385) == C and prod(N=16385) == C and prod(B=65) == C
    torch.cuda.synchronize()
    assert ctx.aug_last_status() == (-1, 0)
