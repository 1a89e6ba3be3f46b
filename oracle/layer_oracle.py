"""fp64 CPU oracle of the operators around the attention: norms and position rotation of queries and keys with their
gradient, microscaled formats, and the linear layer on them.  Written from the definitions; shares no code with the kernels.
"""
import numpy as np

BLOCK = 32
TOP = {"mxfp4": 6.0, "mxfp8": 448.0}


def element_values(fmt):
    """The values of the non-negative element codes, ascending: e2m1 (bias 1) or e4m3 (bias 7, without its NaN)."""
    mantissa_bits, bias, count = (1, 1, 8) if fmt == "mxfp4" else (3, 7, 127)
    code = np.arange(count)
    e, m = code >> mantissa_bits, code & ((1 << mantissa_bits) - 1)
    frac = m / 2.0 ** mantissa_bits
    return np.where(e == 0, frac * 2.0 ** (1 - bias), (1 + frac) * 2.0 ** (e.astype(float) - bias))


def quantize_mx(x, fmt):
    """x [rows, cols] -> (element codes uint8 [rows, cols] with the sign in the top bit of four or eight, scale bytes uint8
    [rows, cols / 32]).  A block with an infinity or NaN: byte 255, codes unspecified (zero here)."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = x.reshape(rows, cols // BLOCK, BLOCK)
    bad = ~np.isfinite(blocks).all(-1)
    blocks = np.where(bad[..., None], 0.0, blocks)
    amax = np.abs(blocks).max(-1)
    e = np.full(amax.shape, -127)
    for k in range(-127, 128):  # the smallest exponent that fits, by trying them all
        e = np.where((e < k) & (amax > TOP[fmt] * 2.0 ** (k - 1)) & (amax > TOP[fmt] * 2.0 ** -127), k, e)
    q = blocks / 2.0 ** e[..., None].astype(float)
    grid = element_values(fmt)
    mag = np.abs(q)
    hi = np.minimum(np.searchsorted(grid, mag), len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    sign = np.signbit(q).astype(int) << (3 if fmt == "mxfp4" else 7)
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return (code | sign).astype(np.uint8).reshape(rows, cols), byte


def pack_codes(codes, fmt):
    return codes if fmt == "mxfp8" else (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def tile_scales(byte):
    """Scale bytes [rows, blocks] in tiles of 128 rows x 4 blocks; places past the matrix are zero."""
    rows, blocks = byte.shape
    out = np.zeros((-(-rows // 128), -(-blocks // 4), 32, 4, 4), dtype=np.uint8)
    for r in range(rows):
        for j in range(blocks):
            out[r // 128, j // 4, r % 32, (r % 128) // 32, j % 4] = byte[r, j]
    return out


def mx_values(codes, byte, fmt):
    """The values that element codes and scale bytes stand for."""
    sign_bit = 8 if fmt == "mxfp4" else 128
    v = element_values(fmt)[codes & (sign_bit - 1)] * np.where(codes & sign_bit, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(float) - 127))
    return v * np.repeat(scale, BLOCK, axis=1)


def _normed(x, norm, eps):
    if norm == "none":
        return x, np.ones(x.shape[:-1] + (1,))
    if norm == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def rotation(positions, dim, base):
    """Matrices [..., dim, dim] with y = R z for positions [..., axes]."""
    positions = np.asarray(positions, dtype=np.float64)
    axes = positions.shape[-1]
    half = dim // axes // 2
    R = np.zeros(positions.shape[:-1] + (dim, dim))
    for a in range(axes):
        for i in range(half):
            angle = positions[..., a] * base ** (-i / half)
            lo, hi = a * 2 * half + i, a * 2 * half + i + half
            R[..., lo, lo] = R[..., hi, hi] = np.cos(angle)
            R[..., lo, hi], R[..., hi, lo] = -np.sin(angle), np.sin(angle)
    return R


def qk_norm_rope(x, norm, weight, bias, eps, positions, base):
    """x [B, H, N, D]; positions [B, N, axes] or None."""
    z, _ = _normed(np.asarray(x, dtype=np.float64), norm, eps)
    if weight is not None:
        z = z * weight
    if bias is not None:
        z = z + bias
    return z if positions is None else np.einsum("bnij,bhnj->bhni", rotation(positions, x.shape[-1], base), z)


def qk_norm_rope_backward(x, dy, norm, weight, eps, positions, base):
    """(dx, d weight, d bias)"""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    g = dy if positions is None else np.einsum("bnij,bhni->bhnj", rotation(positions, x.shape[-1], base), dy)
    xh, r = _normed(x, norm, eps)
    dw, db = (g * xh).sum((0, 1, 2)), g.sum((0, 1, 2))
    gh = g if weight is None else g * weight
    if norm == "none":
        return gh, dw, db
    dx = gh - xh * (gh * xh).mean(-1, keepdims=True)
    if norm == "layer":
        dx = dx - gh.mean(-1, keepdims=True)
    return dx * r, dw, db
