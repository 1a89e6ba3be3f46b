"""The oracle of the operators around the attention against independent statements of the same mathematics, and what the entry
points refuse.  No GPU needed: nothing is enqueued."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2605_11354_b200 import binding as lt
from paper_2605_11354_b200 import build as lb


@pytest.fixture(scope="module", autouse=True)
def library():
    lb.build()
    return lt.lib()


# ------------------------------------------------------------------------------------------------------ oracle pins
def test_element_values():
    assert lo.element_values("mxfp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(lo.element_values("mxfp8"), e4m3)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_quantiser_of_the_oracle(fmt):
    g = np.random.default_rng(0)
    x = (g.standard_normal((40, 96)) * np.exp(3 * g.standard_normal((40, 1)))).astype(np.float32)
    x[3] = 0
    x[4, :32] = 6.0 * 2.0 ** -9
    x[5, 0] = 448.0 * 4
    codes, byte = lo.quantize_mx(x, fmt)
    v = lo.mx_values(codes, byte, fmt)
    scale = 2.0 ** (byte.astype(float) - 127)
    amax = np.abs(x.reshape(40, 3, 32)).max(-1)
    live = amax > 0
    # the smallest power of two under which nothing saturates
    assert (amax <= lo.TOP[fmt] * scale).all() and (amax > lo.TOP[fmt] * scale / 2)[live].all() and (byte[~live] == 0).all()
    q = x.astype(np.float64) / np.repeat(scale, 32, axis=1)
    if fmt == "mxfp8":  # torch's cast rounds to nearest even too
        ref = torch.from_numpy(np.ascontiguousarray(q.astype(np.float32))).to(torch.float8_e4m3fn)
        assert np.array_equal(codes, ref.view(torch.uint8).numpy())
    # off by at most half a step of the element's binade
    least, bits = (0, 1) if fmt == "mxfp4" else (-6, 3)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** least))), least) - bits)
    assert (np.abs(v / np.repeat(scale, 32, axis=1) - q) <= step / 2).all()


def test_ties_of_the_oracle_go_to_the_even_code():
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0] + [6.0] + [0.0] * 22)[None]
    codes, byte = lo.quantize_mx(ties, "mxfp4")
    assert byte[0, 0] == 127
    assert lo.mx_values(codes, byte, "mxfp4")[0, :9].tolist() == [0, 1, 1, 2, 2, 4, 4, 0, -4]


def test_scale_tiles_and_packing():
    byte = np.arange(130 * 5, dtype=np.int64).reshape(130, 5) % 251
    t = lo.tile_scales(byte.astype(np.uint8))
    assert t.shape == (2, 2, 32, 4, 4)
    assert t[0, 0, 5, 2, 3] == byte[69, 3] and t[1, 1, 1, 0, 0] == byte[129, 4] and t[1, 0, 2, 0, 0] == 0
    codes = np.array([[1, 2, 15, 8]], dtype=np.uint8)
    assert lo.pack_codes(codes, "mxfp4").tolist() == [[0x21, 0x8F]]


@pytest.mark.parametrize("norm,axes", [("layer", 2), ("rms", 1), ("none", 2), ("layer", 0)])
def test_gradient_of_the_oracle(norm, axes):
    """Against differences and against autograd of torch's own norms and complex rotations."""
    g = np.random.default_rng(1)
    B, H, N, D, base, eps = 2, 3, 4, 32, 100.0, 1e-5
    x, dy = g.standard_normal((B, H, N, D)), g.standard_normal((B, H, N, D))
    w, b = 1 + 0.3 * g.standard_normal(D), 0.2 * g.standard_normal(D)
    pos = g.integers(-50, 50, (B, N, axes)) if axes else None
    y = lo.qk_norm_rope(x, norm, w, b, eps, pos, base)

    tx, tw, tb = (torch.from_numpy(a).requires_grad_() for a in (x, w, b))
    if norm == "layer":
        z = torch.nn.functional.layer_norm(tx, (D,), tw, tb, eps)
    elif norm == "rms":
        z = torch.nn.functional.rms_norm(tx, (D,), tw, eps) + tb
    else:
        z = tx * tw + tb
    if axes:
        half = D // axes // 2
        parts = []
        for a in range(axes):
            c = torch.complex(z[..., 2 * half * a:2 * half * a + half], z[..., 2 * half * a + half:2 * half * (a + 1)])
            angle = torch.from_numpy(pos[..., a]).double()[:, None, :, None] * base ** (-torch.arange(half).double() / half)
            c = c * torch.polar(torch.ones_like(angle), angle)
            parts += [c.real, c.imag]
        z = torch.cat(parts, -1)
    assert np.allclose(z.detach().numpy(), y, atol=1e-12)
    ref = torch.autograd.grad(z, [tx, tw, tb], torch.from_numpy(dy))
    got = lo.qk_norm_rope_backward(x, dy, norm, w, eps, pos, base)
    for r, o in zip(ref, got):
        assert np.allclose(r.numpy(), o, atol=1e-11)

    loss = lambda x, w, b: float((lo.qk_norm_rope(x, norm, w, b, eps, pos, base) * dy).sum())  # noqa: E731
    h = 1e-5
    for where in [(0, 1, 2, 3), (1, 2, 0, 31), (1, 0, 3, 8)]:
        xp, xm = x.copy(), x.copy()
        xp[where] += h
        xm[where] -= h
        assert abs((loss(xp, w, b) - loss(xm, w, b)) / (2 * h) - got[0][where]) < 1e-6
    for i in (0, 17):
        d = np.zeros(D)
        d[i] = h
        assert abs((loss(x, w + d, b) - loss(x, w - d, b)) / (2 * h) - got[1][i]) < 1e-5
        assert abs((loss(x, w, b + d) - loss(x, w, b - d)) / (2 * h) - got[2][i]) < 1e-5


def test_rotation_depends_on_differences_of_positions():
    g = np.random.default_rng(2)
    q, k = g.standard_normal(64), g.standard_normal(64)
    R = lambda p: lo.rotation(np.array(p), 64, 100.0)  # noqa: E731
    assert abs((R([5, 9]) @ q) @ (R([2, 11]) @ k) - (R([3, -2]) @ q) @ k) < 1e-10


# ------------------------------------------------------------------------------------------------------ refusals
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 1 << 20  # stands for a device pointer; nothing is launched


def source(stride_b=4096, stride_h=64, stride_n=128, dtype=1, ptr=P):
    return lt.TENSOR.pack(ptr or 0, dtype, stride_b, stride_h, stride_n)


def how(**change):
    fields = dict(batch=2, q_heads=2, k_heads=2, tokens=8, head_dim=64, norm=2, eps=1e-5, q_weight=0, q_bias=0,
                  k_weight=0, k_bias=0, axes=2, positions=P, position_stride_b=16, position_stride_n=2, base=100.0)
    return lt.ROPE.pack(*(x or 0 for x in {**fields, **change}.values()))


def grads(q_weight=None, q_bias=None, k_weight=None, k_bias=None):
    return lt.ROPE_GRADS.pack(q_weight or 0, q_bias or 0, k_weight or 0, k_bias or 0)


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), INVALID), (dict(q_heads=0), INVALID), (dict(k_heads=-1), INVALID), (dict(tokens=0), INVALID),
    (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(norm=3), UNSUPPORTED), (dict(axes=3), UNSUPPORTED),
    (dict(axes=-1), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(positions=None), INVALID), (dict(positions=P + 2), INVALID), (dict(position_stride_n=-2), INVALID),
    (dict(base=0.0), INVALID), (dict(base=float("nan")), INVALID), (dict(base=float("inf")), INVALID),
    (dict(base=-5.0), INVALID), (dict(base=1e-31), INVALID), (dict(base=1e31), INVALID),
    (dict(q_weight=P + 4), INVALID), (dict(k_bias=P + 8), INVALID)])
def test_rope_refuses_settings(library, change, status):
    s = source()
    assert library.lite3r_qk_norm_rope(s, s, how(**change), s, s, None) == status
    back = library.lite3r_qk_norm_rope_backward(s, s, s, s, how(**change), s, s, grads(), P, 1 << 30, None)
    assert back == status


@pytest.mark.parametrize("bad,status,as_result", [
    (source(ptr=None), INVALID, True), (source(ptr=P + 8), INVALID, True), (source(dtype=0), UNSUPPORTED, True),
    (source(dtype=7), UNSUPPORTED, True), (source(stride_n=100), INVALID, True), (source(stride_h=-64), INVALID, True),
    (source(stride_h=0), INVALID, False), (source(stride_b=1016), INVALID, False), (source(stride_n=64), INVALID, False),
    (source(stride_n=0), INVALID, False)])
def test_rope_refuses_tensors(library, bad, status, as_result):
    """as_result False: allowed as a source (broadcast, overlapping rows), refused as a result."""
    s, h = source(), how()
    assert library.lite3r_qk_norm_rope(s, s, h, s, bad, None) == status
    assert library.lite3r_qk_norm_rope_backward(s, s, s, s, h, s, bad, grads(), P, 1 << 30, None) == status
    if as_result:
        assert library.lite3r_qk_norm_rope(s, bad, h, s, s, None) == status
        assert library.lite3r_qk_norm_rope_backward(s, s, s, bad, h, s, s, grads(), P, 1 << 30, None) == status


def test_rope_refuses_halves(library):
    s = source()
    assert library.lite3r_qk_norm_rope(None, s, how(), s, s, None) == INVALID
    assert library.lite3r_qk_norm_rope(s, None, how(), s, s, None) == INVALID
    assert library.lite3r_qk_norm_rope(s, s, how(k_heads=0), s, s, None) == INVALID
    assert library.lite3r_qk_norm_rope(s, s, None, s, s, None) == INVALID
    back = library.lite3r_qk_norm_rope_backward
    need = lt.lite3r_qk_norm_rope_workspace(64)
    assert back(s, s, s, s, how(), s, s, grads(), None, need, None) == INVALID
    assert back(s, s, s, s, how(), s, s, grads(), P + 16, need, None) == INVALID
    assert back(s, s, s, s, how(), s, s, grads(), P, need - 1, None) == WORKSPACE
    assert back(s, s, s, s, how(), s, s, None, P, need, None) == INVALID
    assert back(s, None, s, None, how(k_heads=0), s, None, grads(k_weight=P), P, need, None) == INVALID
    with pytest.raises(lt.Lite3rError, match="unsupported"):
        lt.lite3r_qk_norm_rope_workspace(96)


@pytest.mark.parametrize("fmt,rows,cols,status", [(0, 0, 32, INVALID), (0, 4, 0, INVALID), (1, 4, 48, UNSUPPORTED), (2, 4, 32, UNSUPPORTED),
                                                  (0, 1 << 31, 32, INVALID), (-1, 4, 32, UNSUPPORTED)])
def test_microscaled_shapes(library, fmt, rows, cols, status):
    rows = C.c_int(rows).value if rows < 1 << 31 else -(1 << 31)
    size = C.c_size_t()
    assert library.lite3r_mx_sizes(fmt, rows, cols, C.byref(size), None) == status
    assert library.lite3r_quantize_mx(P, 1, 4096, rows, cols, fmt, P, P, None) == status
    assert library.lite3r_dequantize_mx(P, P, fmt, rows, cols, P, 1, 4096, None) == status


def test_microscaled_sizes():
    assert lt.lite3r_mx_sizes("mxfp8", 130, 160) == (130 * 160, 2 * 2 * 512)
    assert lt.lite3r_mx_sizes("mxfp4", 128, 128) == (128 * 64, 512)
    with pytest.raises(lt.Lite3rError, match="format"):
        lt.lite3r_mx_sizes("mxfp6", 128, 128)


@pytest.mark.parametrize("x,dtype,stride,codes,scales,status", [
    (None, 1, 64, P, P, INVALID), (P + 8, 1, 64, P, P, INVALID), (P, 3, 64, P, P, UNSUPPORTED), (P, 1, 60, P, P, INVALID),
    (P, 1, 32, P, P, INVALID), (P, 1, -64, P, P, INVALID), (P, 1, 64, None, P, INVALID), (P, 1, 64, P + 8, P, INVALID),
    (P, 1, 64, P, None, INVALID), (P, 1, 64, P, P + 4, INVALID)])
def test_microscaled_arguments(library, x, dtype, stride, codes, scales, status):
    assert library.lite3r_quantize_mx(x, dtype, stride, 5, 64, 0, codes, scales, None) == status
    assert library.lite3r_dequantize_mx(codes, scales, 1, 5, 64, x, dtype, stride, None) == status


def test_linear_layer_arguments(library):
    f = library.lite3r_linear_mxfp4
    good = [P, P, P, P, P, 5, 64, 24, P, 1, 24, P, None]
    for i, value, status in [(0, None, INVALID), (1, P + 8, INVALID), (2, P + 4, INVALID), (3, None, INVALID), (4, P + 2, INVALID),
                             (5, 0, INVALID), (6, 48, UNSUPPORTED), (6, 0, INVALID), (7, 0, INVALID), (8, None, INVALID),
                             (8, P + 8, INVALID), (9, 5, UNSUPPORTED), (10, 16, INVALID), (10, 28, INVALID), (11, P + 2, INVALID)]:
        args = list(good)
        args[i] = value
        assert f(*args) == status, (i, value)


def test_backward_arguments(library):
    good = [P, 24, P, P, 1, 5, 64, 24, P, 1, 64, P, None]
    for i, value, status in [(0, None, INVALID), (0, P + 8, INVALID), (1, 16, INVALID), (1, 28, INVALID), (2, None, INVALID),
                             (3, P + 8, INVALID), (4, 2, UNSUPPORTED), (5, 0, INVALID), (6, 40, UNSUPPORTED), (7, 0, INVALID),
                             (8, None, INVALID), (9, 3, UNSUPPORTED), (10, 56, INVALID), (11, P + 1, INVALID)]:
        args = list(good)
        args[i] = value
        assert library.lite3r_linear_mx_dgrad(*args) == status, (i, value)
    need = lt.lite3r_linear_mx_workspace(5, 64, 24)
    good = [P, 24, P, P, 1, 5, 64, 24, P, P, P, need, P, None]
    for i, value, status in [(0, None, INVALID), (1, 16, INVALID), (2, None, INVALID), (4, 5, UNSUPPORTED), (5, -1, INVALID),
                             (6, 33, UNSUPPORTED), (7, 0, INVALID), (8, None, INVALID), (8, P + 8, INVALID), (9, P + 2, INVALID),
                             (10, None, INVALID), (10, P + 128, INVALID), (11, need - 1, WORKSPACE), (12, P + 2, INVALID)]:
        args = list(good)
        args[i] = value
        assert library.lite3r_linear_mx_wgrad(*args) == status, (i, value)
    with pytest.raises(lt.Lite3rError, match="unsupported"):
        lt.lite3r_linear_mx_workspace(5, 40, 24)


def test_host_tensors_are_refused():
    x = torch.zeros((2, 2, 4, 64))
    with pytest.raises(lt.Lite3rError, match="CUDA"):
        lt.lite3r_qk_norm_rope(x, x, x, x)
    with pytest.raises(lt.Lite3rError, match="CUDA"):
        lt.lite3r_quantize_mx(torch.zeros((4, 64)))
    t = lt.alloc_mx(4, 64, "mxfp4", "cpu")
    with pytest.raises(lt.Lite3rError, match="CUDA"):
        lt.lite3r_linear_mxfp4(t, t, None, torch.zeros((4, 4)))
    with pytest.raises(lt.Lite3rError, match="CUDA"):
        lt.lite3r_linear_mx_dgrad(torch.zeros((4, 4), dtype=torch.bfloat16), t, torch.zeros((4, 64)))
    with pytest.raises(lt.Lite3rError, match="matrix"):
        lt.MxTensor(t.codes[:, 1:], t.scales, 4, 64).check("here")
    with pytest.raises(lt.Lite3rError, match="format"):
        lt.MxTensor(t.codes, t.scales, 4, 64, "mxfp3").check("here")
