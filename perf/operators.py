"""What a model's first layers do with a batch of features, as cases to time.

A recogniser that is fed by this library takes padded feature rows [B][T_max][D] with frame
counts.  Before its first matrix product it normalises the rows (root mean square, with the
addition of the residual stream from the second layer on), and in low precision it holds
them, and its weights, microscaled: blocks of 32 values along a row share a power of two, the
values themselves have 8 bits (e4m3) or 4 (e2m1).  Four operators:

  norm      h = x + r,  y = h / sqrt(mean(h^2) + eps) * w, y in 32, 16 or 8 bits
  grad      the gradients of the norm with respect to h and w
  quantize  rows to microscaled codes and scales, and (4 bits) back to the values they stand for
  product   rows quantised on arrival, times microscaled 4-bit weights, plus a bias

Rows at and beyond an utterance's frame count are padding: they are not read, and receive zeros.

Sizes are those of the library's workloads (utterances of one frame to 60 s, 1 to 4096 of them,
40 / 80 / 128 bands and stacks of eight frames of them, spectra of 257 bins) and layer widths
up to 1536, four gates of 1024.
"""
import math
import random

import torch

own = False

EPS = 1e-5
BLOCK = 32                 # values that share a scale
GROUP = 128                # rows of codes are padded to whole groups of this many values
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------- the cases
_BASE = dict(op="norm", utts=1, frames=1, width=1024, out_width=0, type="bf16", out="bf16",
             residual=False)


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # streaming recognition: one frame of one stream, normalised for a product in 8 bits
        _case("norm one frame", residual=True, out="mx8"),
        # log-mel rows of 64 utterances of up to 20 s, on their way into a 16-bit model
        _case("norm mel batch", utts=64, frames=1998, width=80, type="f32"),
        # power spectra of a 512-point transform: 257 bins, rows that start anywhere
        _case("norm spectra", utts=16, frames=798, width=257, type="f32", out="f32", residual=True),
        # a layer of a large evaluation batch: residual stream in 16 bits, output in 8
        _case("norm large", utts=64, frames=1998, residual=True, out="mx8"),
        # training on short commands, first norm of the model
        _case("grad spectra", op="grad", utts=24, frames=198, width=257, type="f32"),
        # training, a layer inside the model
        _case("grad large", op="grad", utts=64, frames=998, width=1024, residual=True),
        # short commands to 8 bits
        _case("quantize short", op="quantize", utts=8, frames=198, width=40, type="f32", out="mx8"),
        # stacks of eight frames of 80 bands to 4 bits
        _case("quantize stacked", op="quantize", utts=128, frames=375, width=640, type="f32",
              out="mx4"),
        # streaming recognition: one frame into the four gates of 1024 cells
        _case("product one frame", op="product", width=1024, out_width=4096, out="mx4"),
        # a batch of stacked frames into a layer of 1024
        _case("product stacked", op="product", utts=32, frames=250, width=640, out_width=1024,
              type="f32", out="mx4"),
        # 8-bit rows, an output width that is no multiple of anything
        _case("product 8 bit", op="product", utts=24, frames=798, width=1000, out_width=1001,
              out="mx8"),
        # a large evaluation batch
        _case("product large", op="product", utts=64, frames=1998, width=1024, out_width=1024,
              out="mx4"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "grad", "quantize", "product", "product"])
    width = rng.choice([_log(rng, 8, 1536), rng.choice([40, 80, 128, 257, 320, 513, 640, 1024])])
    most = int(1.2e8 / max(width, 256))          # rows of a batch
    frames = _log(rng, 1, 1998)
    utts = _log(rng, 1, max(1, min(4096, most // frames)))
    out_width, out = 0, rng.choice(["f32", "bf16", "mx8"])
    if op == "product":
        out_width = _log(rng, 16, 4096)
        out = rng.choice(["mx4", "mx4", "mx8"])
        utts = max(1, min(utts, int(1.3e11 / (frames * width * out_width)),
                          int(1.2e8 / (frames * out_width))))
    elif op == "quantize":
        out = rng.choice(["mx4", "mx8"])
    elif op == "grad":
        utts = max(1, utts // 2)
        out = "bf16"
    return _case(op=op, utts=utts, frames=frames, width=width, out_width=out_width, out=out,
                 type=rng.choice(["f32", "bf16"]), residual=op in ("norm", "grad") and rng.random() < 0.6)


# ----------------------------------------------------------------------------- inputs
def _rows(shape, kind, gen):
    """Log-mel-like rows ("f32": bands of their own level, frames of their own loudness) or a
    layer's activations ("bf16": unit variance, a few loud channels)."""
    x = torch.randn(shape, device="cuda", generator=gen)
    if kind == "f32":
        band = torch.randn(shape[-1], device="cuda", generator=gen)
        loud = torch.randn(shape[:-1] + (1,), device="cuda", generator=gen)
        return (1.5 * x).add_(2.0 * band - 6.0).add_(loud)
    return x.mul_(torch.exp(1.2 * torch.randn(shape[-1], device="cuda", generator=gen))).to(torch.bfloat16)


def _counts(case, seed):
    """Frame counts: the first utterance fills the padded length, the others a third of it or more."""
    rng, T = random.Random(seed), case["frames"]
    return [T] + [rng.randint(max(1, T // 3), T) for _ in range(case["utts"] - 1)]


def _pow2(e):
    """2^e in fp32 by its bits, for -127 <= e <= 127 (a power function need not be exact)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _packed_weights(w):
    """Weights as a program keeps them: e2m1 codes, two to a byte, and scale bytes, from rows [N][K]."""
    N, K = w.shape
    G = -(-K // GROUP) * GROUP
    w = torch.nn.functional.pad(w, (0, G - K)).reshape(N, G // BLOCK, BLOCK)
    _, e = torch.frexp(w.abs().amax(-1, keepdim=True))
    e = torch.where(w.abs().amax(-1, keepdim=True) > 0, e - 3, -127).clamp_min(-127)
    v = w * _pow2(-e)
    m = v.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = (code + 8 * (v < 0)).reshape(N, G).to(torch.uint8)
    scales = (e + 127).to(torch.uint8).reshape(N, G // BLOCK)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=w.device)
    values = grid[(code & 7).long()] * (1.0 - 2.0 * (code >> 3)) * _pow2(e).expand(-1, -1, BLOCK).reshape(N, G)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scales.contiguous(), values[:, :K].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, T, D, N = case["utts"], case["frames"], case["width"], case["out_width"]
    st = dict(case, x=_rows((B, T, D), case["type"], gen),
              counts=torch.tensor(_counts(case, seed), dtype=torch.int32, device="cuda"))
    if case["op"] in ("norm", "grad"):
        st["weight"] = 1.0 + 0.2 * torch.randn(D, device="cuda", generator=gen)
        st["r"] = _rows((B, T, D), case["type"], gen) if case["residual"] else None
    if case["op"] == "grad":             # x is the sum; r is the gradient that comes down the stream
        st["dy"] = (0.01 * torch.randn((B, T, D), device="cuda", generator=gen)).to(st["x"].dtype)
        if case["residual"]:
            st["r"] = (0.01 * st["r"].float()).to(st["x"].dtype)
    if case["op"] == "product":
        w = torch.randn((N, D), device="cuda", generator=gen) / math.sqrt(D)
        st["w_codes"], st["w_scales"], st["w_values"] = _packed_weights(w)
        st["bias"] = 0.1 * torch.randn(N, device="cuda", generator=gen)
    return st


# ----------------------------------------------------------------------------- the plain forms
def _valid(st):
    return (torch.arange(st["frames"], device="cuda") < st["counts"][:, None])[:, :, None]


def _quantized(x, kind):
    """(values on the element's grid, exponents of the blocks) of fp32 rows, padded to whole groups.
    The block's exponent is that of its largest magnitude less the grid's largest one; the rest is
    rounded to nearest even and saturates."""
    D = x.shape[-1]
    G = -(-D // GROUP) * GROUP
    x = torch.nn.functional.pad(x, (0, G - D)).unflatten(-1, (G // BLOCK, BLOCK))
    amax = x.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 1 - (8 if kind == "mx8" else 2), -127).clamp_min(-127)
    v = x * _pow2(-e)
    if kind == "mx8":
        return v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).flatten(-2), e.squeeze(-1)
    m = v.abs()
    g = 0.5 * ((m > 0.25).float() + (m >= 0.75).float() + (m > 1.25).float() + (m >= 1.75).float()) \
        + (m > 2.5).float() + (m >= 3.5).float() + 2.0 * (m > 5.0).float()
    return (g * torch.sign(v)).flatten(-2), e.squeeze(-1)


def _dequantized(x, kind):
    v, e = _quantized(x, kind)
    return (v.float().unflatten(-1, (-1, BLOCK)) * _pow2(e)[..., None]).flatten(-2)[..., :x.shape[-1]]


def _scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _norm_plain(st):
    h = st["x"].float()
    if st["r"] is not None:
        h = h + st["r"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * st["weight"]
    ok = _valid(st)
    out = {}
    if st["r"] is not None:
        out["sum"] = torch.where(ok, h, 0.0).to(st["x"].dtype)
    y = torch.where(ok, y, 0.0)
    if st["out"] == "mx8":
        codes, e = _quantized(y, "mx8")
        return dict(out, y=codes, scales=_scales(e))
    return dict(out, y=y.to(_TYPES[st["out"]]))


def _grad_plain(st):
    ok = _valid(st)
    h = torch.where(ok, st["x"].float(), 0.0)
    dy = torch.where(ok, st["dy"].float(), 0.0)
    rs = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    g = dy * st["weight"]
    dx = rs * (g - h * (rs * rs * (g * h).mean(-1, keepdim=True)))
    if st["r"] is not None:
        dx = dx + torch.where(ok, st["r"].float(), 0.0)
    return {"dx": dx.to(st["x"].dtype), "dweight": (dy * h * rs).sum((0, 1))}


def _quantize_plain(st):
    x = torch.where(_valid(st), st["x"].float(), 0.0)
    if st["out"] == "mx8":
        codes, e = _quantized(x, "mx8")
        return {"codes": codes, "scales": _scales(e)}
    return {"values": _dequantized(x, "mx4").to(torch.bfloat16)}


def _product_plain(st):
    a = _dequantized(st["x"].float(), st["out"])
    y = a @ st["w_values"].T + st["bias"]
    return {"y": torch.where(_valid(st), y, 0.0).to(torch.bfloat16)}


# ----------------------------------------------------------------------------- the library's calls
_contexts = {}


def _context():
    """The program's context on the current device and stream; the operators need no workspace of it."""
    key = (torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)
    if key not in _contexts:
        from paper_1912_11040_b200 import binding
        config = binding.AugConfig(
            fs=16000, win=400, hop=160, n_fft=512, n_mel=80, f_lo=0.0, f_hi=8000.0, rir_taps=1,
            max_order=0, max_sources=1, frac_half_width=40, sound_speed=343.0, log_floor=1e-7,
            pad_value=0.0, compression=0, max_batch=4096, max_samples=400)
        _contexts[key] = (binding, binding.AugContext(config))
    return _contexts[key]


def _own_type(b, x):
    return b.ELEM_F32 if x.dtype == torch.float32 else b.ELEM_BF16


def _codes_like(b, kind, B, T, D):
    elem = b.ELEM_MX8 if kind == "mx8" else b.ELEM_MX4
    return (elem, torch.empty((B, T, b.feat_mx_code_bytes(elem, D)), dtype=torch.uint8, device="cuda"),
            torch.empty((B, T, b.feat_mx_scale_bytes(D)), dtype=torch.uint8, device="cuda"))


def _run_own(st):
    b, ctx = _context()
    B, T, D, N = st["utts"], st["frames"], st["width"], st["out_width"]
    x, counts = st["x"], st["counts"]
    kind = _own_type(b, x)
    if st["op"] == "norm":
        out = {}
        total = torch.empty_like(x) if st["r"] is not None else None
        if st["out"] == "mx8":
            elem, codes, scales = _codes_like(b, "mx8", B, T, D)
            ctx.feat_rms_norm(x, st["r"], kind, st["weight"], counts, B, T, D, EPS, total, codes, elem, scales)
            out = {"y": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}
        else:
            y = torch.empty((B, T, D), dtype=_TYPES[st["out"]], device="cuda")
            ctx.feat_rms_norm(x, st["r"], kind, st["weight"], counts, B, T, D, EPS, total, y, _own_type(b, y), None)
            out = {"y": y}
        return dict(out, sum=total) if total is not None else out
    if st["op"] == "grad":
        dx = torch.empty_like(x)
        dweight = torch.empty(D, device="cuda")
        partial = torch.empty(b.feat_rms_norm_partial_floats(D), device="cuda")
        ctx.feat_rms_norm_grad(x, st["dy"], st["r"], kind, st["weight"], counts, B, T, D, EPS, dx, dweight, partial)
        return {"dx": dx, "dweight": dweight}
    elem, codes, scales = _codes_like(b, st["out"], B, T, D)
    ctx.feat_mx_quantize(x, kind, counts, B, T, D, codes, elem, scales)
    if st["op"] == "quantize":
        if st["out"] == "mx8":
            return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}
        values = torch.empty((B, T, D), dtype=torch.bfloat16, device="cuda")
        ctx.feat_mx_dequantize(codes, elem, scales, counts, B, T, D, values, b.ELEM_BF16)
        return {"values": values}
    y = torch.empty((B, T, N), dtype=torch.bfloat16, device="cuda")
    ctx.feat_mx_product(codes, elem, scales, st["w_codes"], st["w_scales"], st["bias"], counts, B, T, D, N, y,
                        b.ELEM_BF16)
    return {"y": y}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm_plain, "grad": _grad_plain, "quantize": _quantize_plain,
            "product": _product_plain}[state["op"]](state)


# ----------------------------------------------------------------------------- in 64 bits
def _grid64(x, kind):
    """Elements and scales of rows by the formats' definition: an element's step is a power of two
    given by its own magnitude, no finer than that of the smallest normal number."""
    bits, low, top, most = (3, -6, 8, 448.0) if kind == "mx8" else (1, 0, 2, 6.0)
    shape = x.shape[:-1] + (-(-x.shape[-1] // GROUP) * GROUP // BLOCK, BLOCK)
    full = x.new_zeros(shape[:-2] + (shape[-2] * BLOCK,))
    full[..., : x.shape[-1]] = x
    full = full.reshape(shape)
    peak = full.abs().max(-1, keepdim=True).values
    power = lambda v: (v.view(torch.int64) >> 52 & 0x7FF) - 1023        # floor(log2) of a normal number
    two_to = lambda e: (e + 1023 << 52).view(torch.float64)
    scale = two_to((power(peak) - top).clamp(min=-127))                 # (zero has the lowest power)
    v = full / scale
    step = two_to(power(v).clamp(min=low) - bits)
    v = (torch.round(v / step) * step).clamp(-most, most)
    return v, scale


def exact(case, seed):
    st = prepare(case, seed)
    B, T, D = case["utts"], case["frames"], case["width"]
    keep = torch.zeros((B, T, 1), dtype=torch.float64, device="cuda")
    for u, n in enumerate(_counts(case, seed)):
        keep[u, :n] = 1.0
    x = st["x"].double() * keep
    if case["op"] in ("norm", "grad"):
        w = st["weight"].double()
        r = st["r"].double() * keep if st["r"] is not None else torch.zeros_like(x)
    if case["op"] == "norm":
        h = x + r
        y = w * h / torch.sqrt((h * h).sum(-1, keepdim=True) / D + EPS)
        out = {"sum": h} if case["residual"] else {}
        if case["out"] == "mx8":
            v, scale = _grid64(y, "mx8")
            return dict(out, y=v.flatten(-2), scales=scale.squeeze(-1))
        return dict(out, y=y)
    if case["op"] == "grad":
        dy = st["dy"].double() * keep
        size = torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS)
        n = x / size
        dn = dy * w
        dx = (dn - n * (dn * n).sum(-1, keepdim=True) / D) / size + r
        return {"dx": dx, "dweight": torch.einsum("btd,btd->d", dy, n)}
    v, scale = _grid64(x, case["out"])
    if case["op"] == "quantize" and case["out"] == "mx8":
        return {"codes": v.flatten(-2), "scales": scale.squeeze(-1)}
    a = (v * scale).flatten(-2)[..., :D]
    if case["op"] == "quantize":
        return {"values": a}
    return {"y": (torch.matmul(a, st["w_values"].double().t()) + st["bias"].double()) * keep}


# ----------------------------------------------------------------------------- work
def work(case):
    """Valid rows (two thirds of the padded ones; all of a single frame's) read once, all rows of
    the outputs written once; weights read once in 4 bits."""
    B, T, D, N = case["utts"], case["frames"], case["width"], case["out_width"]
    rows = B * T
    valid = T + (B - 1) * (T + max(1, T // 3)) / 2
    size = 4 if case["type"] == "f32" else 2
    mx = {"mx8": D + D / 32, "mx4": D / 2 + D / 32}
    out = mx[case["out"]] if case["out"] in mx else D * (4 if case["out"] == "f32" else 2)
    streams = 2 if case["residual"] else 1
    if case["op"] == "norm":
        nbytes = valid * D * size * streams + rows * (out + (D * size if case["residual"] else 0)) + 4 * D
        return {"bytes": nbytes, "flops": 5.0 * valid * D}
    if case["op"] == "grad":
        return {"bytes": valid * D * size * (1 + streams) + rows * D * size + 8 * D, "flops": 12.0 * valid * D}
    if case["op"] == "quantize":
        nbytes = valid * D * size + rows * (D * 2 if case["out"] == "mx4" else out)
        return {"bytes": nbytes, "flops": 4.0 * valid * D}
    return {"bytes": valid * D * size + N * (D / 2 + D / 32) + 4 * N + rows * N * 2,
            "flops": 2.0 * valid * D * N}
