"""The operators on rows of a padded batch, in 64 bits and from their definitions (numpy)."""
import numpy as np

BLOCK, GROUP = 32, 128
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_values():
    """The 127 finite non-negative numbers of e4m3, by code."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(float) - 10))


GRIDS = {"mx8": (e4m3_values(), 8), "mx4": (E2M1, 2)}


def holds(counts, B, T):
    """[B][T] truth: the rows that hold values."""
    if counts is None:
        return np.ones((B, T), bool)
    return np.arange(T)[None, :] < np.asarray(counts)[:, None]


def nearest_code(v, grid):
    """Code of the number of `grid` that is nearest to |v|, ties to the even code, with the sign above it."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    sign = 8 if len(grid) == 8 else 128
    return (code + sign * np.signbit(v)).astype(np.uint8)


def quantize(x, kind):
    """(codes [rows][G 128] one to a byte, scale bytes [rows][G 4]) of rows x."""
    grid, top = GRIDS[kind]
    rows, D = x.shape
    G = -(-D // GROUP)
    full = np.zeros((rows, G * GROUP))
    full[:, :D] = x
    blocks = full.reshape(rows, G * 4, BLOCK)
    finite = np.isfinite(blocks).all(-1)
    safe = np.where(finite[..., None], blocks, 0.0)
    amax = np.abs(safe).max(-1)
    _, e = np.frexp(np.where(amax > 0, amax, 1.0))
    byte = np.where(amax > 0, np.maximum(e - 1 - top + 127, 0), 0)
    codes = nearest_code(np.ldexp(safe, (127 - byte)[..., None]), grid)
    codes = np.where(finite[..., None], codes, 0)
    return codes.reshape(rows, -1).astype(np.uint8), np.where(finite, byte, 255).astype(np.uint8)


def dequantize(codes, scales, kind, D):
    grid, _ = GRIDS[kind]
    n = len(grid) if kind == "mx4" else 128
    table = np.full(n, np.nan)
    table[: len(grid)] = grid
    v = table[codes % n] * np.where(codes >= n, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(len(codes), -1, BLOCK) * s[..., None]).reshape(len(codes), -1)[:, :D]


def packed(codes, kind):
    return codes if kind == "mx8" else codes[:, 0::2] | codes[:, 1::2] << 4


def unpacked(raw, kind):
    if kind == "mx8":
        return raw
    out = np.empty((raw.shape[0], 2 * raw.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = raw & 15, raw >> 4
    return out


def rms_norm(x, r, w, eps):
    h = x + (0.0 if r is None else r)
    rs = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h, h * rs * (1.0 if w is None else w)


def rms_norm_grad(h, dy, dsum, w, eps):
    """dx, dweight and, for the tolerances, the sums of magnitudes that they come from."""
    D = h.shape[-1]
    rs = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    n = h * rs
    g = dy * (1.0 if w is None else w)
    dx = rs * (g - n * (g * n).mean(-1, keepdims=True)) + (0.0 if dsum is None else dsum)
    size = rs * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(-1, keepdims=True)) + (0.0 if dsum is None else np.abs(dsum))
    dn = (dy * n).reshape(-1, D)
    return dx, dn.sum(0), size, np.abs(dn).sum(0)
