"""Norms and rotation of queries and keys, microscaled formats, the 4-bit linear layer and its backward pass against the fp64
oracle.

Tolerances, with u = 2^-24 (half a step of fp32) and half_step(T) of the result's own rounding:
  rows     a mean of D <= 256 values, a variance, a reciprocal root (2 ulp), an affine map and a rotation (angle off by at
           most 3 u, sine and cosine 2 ulp) are some thirty roundings, each at most u of the row's largest intermediate; for
           16-bit types sine and cosine come from the special function unit, off by 2^-21.4 and 2^-21.2 (7 u each) of two
           products: 14 u more
  sums     n terms in fp32 in any order: n u times the sum of magnitudes
  products exact terms; a running sum that is cut off at fp32 loses at most 2 u of the sum of magnitudes per instruction of
           K = 64 (4-bit) or 16 (bf16) terms, and what is added after
"""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from oracle import sla_oracle as orc
from paper_2605_11354_b200 import binding as lt

import parity_util as pu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}  # half a step below fp16's smallest normal value
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def f64(t):
    return t.detach().double().cpu().numpy()


def workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda")


def within(got, ref, tol, dtype, what):
    """Values that round beyond the type's largest (fp16: from 65520 = 65504 + half a step on) have to be infinite."""
    got, tol = f64(got), np.broadcast_to(tol, ref.shape)
    end = torch.finfo(dtype).max * (1 + HALF_STEP[dtype] / (2 - 2 * HALF_STEP[dtype]))
    over, under = np.abs(ref) - tol >= end, np.abs(ref) + tol < end
    assert (got[over] == np.sign(ref[over]) * np.inf).all() and np.isfinite(got[under]).all(), what
    got, ref, tol = got[under], ref[under], tol[under]
    tol = tol + HALF_STEP[dtype] * (np.abs(ref) + tol) + TINY[dtype]
    worst = (np.abs(got - ref) / np.maximum(tol, 1e-300)).max() if got.size else 0.0
    assert worst <= 1.0, (what, worst)


# ------------------------------------------------------------------------------------------------------ norms and rotation
def rope_inputs(seed, B, H, K, N, D, dtype, layout):
    g = torch.Generator().manual_seed(seed)
    if layout == "packed":
        packed = torch.randn((B, N, H + 2 * K, D), generator=g).to(dtype).cuda()
        return packed[:, :, :H].permute(0, 2, 1, 3), packed[:, :, H:H + K].permute(0, 2, 1, 3)
    return torch.randn((B, H, N, D), generator=g).to(dtype).cuda(), torch.randn((B, K, N, D), generator=g).to(dtype).cuda()


def affine(seed, D):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.3 * torch.randn(D, generator=g)).cuda(), (0.2 * torch.randn(D, generator=g)).cuda(),
            (1 + 0.3 * torch.randn(D, generator=g)).cuda(), (0.2 * torch.randn(D, generator=g)).cuda()]


def check_rows(got, x, norm, w, b, eps, pos, base, what):
    x64 = f64(x)
    ref = lo.qk_norm_rope(x64, norm, None if w is None else f64(w), None if b is None else f64(b), eps, pos, base)
    r = lo._normed(x64, norm, eps)[1]
    top = np.abs(x64).max(-1, keepdims=True) * r * (1.0 if w is None else float(w.abs().max())) + (0.0 if b is None else float(b.abs().max()))
    within(got, ref, (32 if got.dtype == torch.float32 else 46) * U * top, got.dtype, what)


def check_row_grads(got, x, dy, norm, w, eps, pos, base, what):
    x64, dy64 = f64(x), f64(dy)
    w64 = None if w is None else f64(w)
    ref = lo.qk_norm_rope_backward(x64, dy64, norm, w64, eps, pos, base)
    r = lo._normed(x64, norm, eps)[1]
    top = np.abs(x64).max(-1, keepdims=True) * r
    a = 2 * np.abs(dy64).max(-1, keepdims=True) * (1.0 if w is None else float(w.abs().max()))  # a pair turns into at most sqrt 2 each
    within(got[0], ref[0], 64 * U * r * a * (1 + top + top * top), x.dtype, what + " dx")
    g, _, db = np.abs(lo.qk_norm_rope_backward(x64, dy64, "none", None, eps, pos, base)[0]), None, None
    xh = np.abs(lo._normed(x64, norm, eps)[0])
    n = x64.shape[0] * x64.shape[1] * x64.shape[2]
    slack = 32 * U * (2 * np.abs(dy64).max(-1, keepdims=True))  # of a turned gradient
    if got[1] is not None:
        within(got[1], ref[1], ((n + 64) * U * g * (xh + top) + slack * (xh + top)).sum((0, 1, 2)), torch.float32, what + " dw")
    if got[2] is not None:
        within(got[2], ref[2], ((n + 64) * U * g + slack).sum((0, 1, 2)), torch.float32, what + " db")


ROPE_CASES = [  # B, H, K, N, D, axes, norm, dtype, layout, weights
    (1, 1, 1, 1, 64, 2, "layer", "bf16", "heads", True),
    (2, 16, 16, 37, 64, 2, "layer", "bf16", "packed", True),
    (3, 5, 1, 131, 64, 1, "rms", "f32", "packed", True),
    (1, 8, 2, 1, 128, 1, "rms", "f16", "heads", True),
    (2, 4, 4, 33, 32, 2, "layer", "f32", "heads", False),
    (1, 3, 3, 50, 256, 2, "rms", "bf16", "packed", True),
    (1, 2, 1, 65, 256, 1, "none", "f32", "heads", True),
    (2, 7, 7, 19, 128, 0, "layer", "f16", "packed", True),
    (1, 24, 8, 700, 64, 2, "layer", "bf16", "heads", True),
    (1, 2, 2, 2000, 32, 1, "none", "bf16", "packed", False),
]


@pytest.mark.parametrize("B,H,K,N,D,axes,norm,dtype,layout,weights", ROPE_CASES)
def test_norm_and_rotation(B, H, K, N, D, axes, norm, dtype, layout, weights):
    q, k = rope_inputs(1, B, H, K, N, D, DTYPES[dtype], layout)
    qw, qb, kw, kb = affine(2, D) if weights else [None] * 4
    base, eps = 100.0, 1e-5
    pos = torch.randint(-40, 1400, (B, N, axes), generator=torch.Generator().manual_seed(3)).int() if axes else None
    p64 = pos.numpy() if axes else None
    pos = pos.cuda() if axes else None
    how = dict(norm=norm, positions=pos, base=base, eps=eps)
    qo, ko = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda"), torch.full(k.shape, 9.0, dtype=k.dtype, device="cuda")
    lt.lite3r_qk_norm_rope(q, k, qo, ko, q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb, **how)
    check_rows(qo, q, norm, qw, qb, eps, p64, base, "q")
    check_rows(ko, k, norm, kw, kb, eps, p64, base, "k")
    # in place, and through another call with the queries alone
    q2, k2 = q.clone(), k.clone()
    lt.lite3r_qk_norm_rope(q2, k2, q2, k2, q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb, **how)
    q3 = torch.empty_like(qo)
    lt.lite3r_qk_norm_rope(q, None, q3, None, q_weight=qw, q_bias=qb, **how)
    assert torch.equal(q2, qo) and torch.equal(k2, ko) and torch.equal(q3, qo)

    dqo, dko = rope_inputs(4, B, H, K, N, D, DTYPES[dtype], layout)
    dq, dk = torch.empty_like(qo), torch.empty_like(ko)
    ws = workspace(lt.lite3r_qk_norm_rope_workspace(D))
    grads = {n: torch.full((D,), 7.0, device="cuda") for n in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
    lt.lite3r_qk_norm_rope_backward(q, k, dqo, dko, dq, dk, ws, q_weight=qw, k_weight=kw, **grads, **how)
    check_row_grads((dq, grads["dq_weight"], grads["dq_bias"]), q, dqo, norm, qw, eps, p64, base, "q")
    check_row_grads((dk, grads["dk_weight"], grads["dk_bias"]), k, dko, norm, kw, eps, p64, base, "k")
    # the same bits again, in place of the incoming gradients
    first = {n: t.clone() for n, t in grads.items()}
    lt.lite3r_qk_norm_rope_backward(q, k, dqo, dko, dqo, dko, ws, q_weight=qw, k_weight=kw, **grads, **how)
    assert torch.equal(dqo, dq) and torch.equal(dko, dk) and all(torch.equal(first[n], grads[n]) for n in grads)


def test_gradient_is_that_of_the_forward():
    """<dy, y(x + h d) - y(x - h d)> / 2h against <dx, d>, and the same for the weights: the two calls belong together."""
    B, H, N, D = 1, 2, 9, 64
    g = torch.Generator().manual_seed(5)
    q = torch.randn((B, H, N, D), generator=g).cuda()
    w, b = affine(6, D)[:2]
    dy, d, e = (torch.randn(s, generator=g).cuda() for s in ((B, H, N, D), (B, H, N, D), (D,)))
    pos = torch.randint(0, 40, (N, 2), generator=g).int().cuda()

    def y(x, w, b):
        out = torch.empty_like(x)
        lt.lite3r_qk_norm_rope(x, None, out, None, q_weight=w, q_bias=b, positions=pos)
        return (out.double() * dy.double()).sum().item()

    dx, dw, db = torch.empty_like(q), torch.empty_like(w), torch.empty_like(b)
    lt.lite3r_qk_norm_rope_backward(q, None, dy, None, dx, None, workspace(lt.lite3r_qk_norm_rope_workspace(D)), q_weight=w,
                                    dq_weight=dw, dq_bias=db, positions=pos)
    h = 2.0 ** -7
    # a difference of two sums of B H N D terms, each off by 32 u of values of a few units, over 2 h; third derivatives h^2
    n = B * H * N * D
    slack = 2 * 32 * U * 8 * float(dy.abs().sum()) / (2 * h)
    for diff, inner in (((y(q + h * d, w, b) - y(q - h * d, w, b)) / (2 * h), float((dx.double() * d.double()).sum())),
                        ((y(q, w + h * e, b) - y(q, w - h * e, b)) / (2 * h), float((dw.double() * e.double()).sum())),
                        ((y(q, w, b + h * e) - y(q, w, b - h * e)) / (2 * h), float((db.double() * e.double()).sum()))):
        assert abs(diff - inner) <= slack + 40 * h * h * n ** 0.5, (diff, inner)


def test_special_rows_stay_by_themselves():
    q = torch.randn((1, 2, 6, 64), generator=torch.Generator().manual_seed(7)).cuda()
    q[0, 0, 1] = 3.0            # no variance
    q[0, 0, 2] = 0.0
    q[0, 1, 3, 5] = float("nan")
    q[0, 1, 4, 9] = float("inf")
    pos = torch.arange(6).int().cuda()[:, None]
    out = torch.empty_like(q)
    lt.lite3r_qk_norm_rope(q, None, out, None, positions=pos)
    assert not out[0, 0, 1].any() and not out[0, 0, 2].any()
    assert out[0, 1, 3].isnan().all() and out[0, 1, 4].isnan().any()
    clean = q.clone()
    clean[0, 1, 3:5] = 0
    ref = torch.empty_like(q)
    lt.lite3r_qk_norm_rope(clean, None, ref, None, positions=pos)
    keep = torch.ones(2, 6, dtype=torch.bool)
    keep[1, 3:5] = False
    assert torch.equal(out[0][keep], ref[0][keep])


def test_far_and_shared_positions_and_broadcast_sources():
    D, N, base = 64, 5, 10000.0
    row = torch.randn((1, 1, 1, D), generator=torch.Generator().manual_seed(8)).cuda()
    q = row.expand(3, 4, N, D)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).int()
    out = torch.empty((3, 4, N, D), device="cuda")
    lt.lite3r_qk_norm_rope(q, None, out, None, positions=pos.cuda()[:, None], base=base)
    ref = lo.qk_norm_rope(f64(q), "layer", None, None, 1e-5, np.broadcast_to(pos.numpy()[None, :, None], (3, N, 1)), base)
    # an angle of 2^31 radians in fp64 is off by half a step of 2^-22 on either side (here and in the oracle)
    far = np.abs(pos.numpy().astype(np.float64))[None, None, :, None] * 2.0 ** -52
    within(out, ref, (32 * U + far) * np.abs(ref).max(), torch.float32, "far")
    # the gradient of the broadcast source is the sum of its rows' gradients
    dy = torch.randn((3, 4, N, D), generator=torch.Generator().manual_seed(9)).cuda()
    dx = torch.empty_like(dy)
    lt.lite3r_qk_norm_rope_backward(q, None, dy, None, dx, None, workspace(lt.lite3r_qk_norm_rope_workspace(D)), positions=pos.cuda()[:, None],
                                    base=base)
    ref = lo.qk_norm_rope_backward(f64(q), f64(dy), "layer", None, 1e-5, np.broadcast_to(pos.numpy()[None, :, None], (3, N, 1)), base)[0]
    within(dx, ref, (64 * U + far) * 40 * np.abs(f64(dy)).max(), torch.float32, "broadcast")


def test_results_inside_larger_buffers():
    """Rows of a cache next to those written stay as they were."""
    k = torch.randn((2, 3, 4, 64), generator=torch.Generator().manual_seed(10)).bfloat16().cuda()
    cache = torch.full((2, 3, 20, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(7, 11).int().cuda()[:, None]
    lt.lite3r_qk_norm_rope(k, None, cache[:, :, 7:11], None, positions=pos)
    ref = torch.empty_like(k)
    lt.lite3r_qk_norm_rope(k, None, ref, None, positions=pos)
    assert torch.equal(cache[:, :, 7:11], ref) and (cache[:, :, :7] == 5).all() and (cache[:, :, 11:] == 5).all()


def test_rows_past_32_bit_offsets():
    """Element offsets beyond 2^32: a batch stride of three thousand million elements (two short sequences, far apart)."""
    far = 3 << 30
    buf = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((2, 2, 8, 64), (far, 64, 128, 1))
    small = torch.randn((2, 2, 8, 64), generator=torch.Generator().manual_seed(11)).bfloat16().cuda()
    q.copy_(small)
    pos = torch.arange(8).int().cuda()[:, None]
    ref = torch.empty_like(small)
    lt.lite3r_qk_norm_rope(small, None, ref, None, positions=pos)
    lt.lite3r_qk_norm_rope(q, None, q, None, positions=pos)
    assert torch.equal(q, ref)


# ------------------------------------------------------------------------------------------------------ microscaled formats
def mx_input(seed, rows, cols, dtype):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, cols)) * np.exp(2 * g.standard_normal((rows, 1)))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("rows,cols,dtype", [(1, 32, "f32"), (127, 96, "bf16"), (129, 1184, "f32"), (300, 128, "f16"), (256, 160, "bf16"),
                                             (5, 4096, "bf16")])
def test_quantiser_is_exact(fmt, rows, cols, dtype):
    x = mx_input(1, rows, cols, DTYPES[dtype]).cuda()
    t = lt.lite3r_quantize_mx(x, fmt)
    codes, byte = lo.quantize_mx(f64(x), fmt)
    assert np.array_equal(t.scales.cpu().numpy(), lo.tile_scales(byte))
    assert np.array_equal(t.codes.cpu().numpy(), lo.pack_codes(codes, fmt))
    for out_dtype in DTYPES.values():
        out = lt.lite3r_dequantize_mx(t, torch.empty((rows, cols), dtype=out_dtype, device="cuda"))
        assert torch.equal(out.cpu(), torch.from_numpy(lo.mx_values(codes, byte, fmt)).to(out_dtype)), out_dtype


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_quantiser_at_the_borders(fmt):
    """Largest magnitudes at and next to top * 2^k, ties, zeros of both signs, the smallest and largest numbers of fp32."""
    top = lo.TOP[fmt]
    rows = []
    for k in (-140, -127, -126, -20, 0, 1, 60, 119):
        base = np.float32(top) * np.float32(2.0) ** np.float32(k) if k > -127 else np.float32(top * 2.0 ** k)
        for m in (base, np.nextafter(base, np.float32(np.inf)), np.nextafter(base, np.float32(0))):
            row = np.linspace(-1, 1, 32).astype(np.float32) * m
            row[-1] = m
            rows.append(row)
    grid = lo.element_values(fmt)
    mids = (grid[1:] + grid[:-1]) / 2
    row = np.zeros(32, np.float32)
    row[:7] = mids[-7:]
    row[7:14] = -mids[:7]
    row[14] = top
    row[15] = -0.0
    rows += [row, np.zeros(32, np.float32), np.full(32, -0.0, np.float32), np.full(32, 1e-45, np.float32),
             np.full(32, np.finfo(np.float32).max, np.float32), np.float32(1e-40) * np.arange(32, dtype=np.float32)]
    x = np.stack(rows)
    t = lt.lite3r_quantize_mx(torch.from_numpy(x).cuda(), fmt)
    codes, byte = lo.quantize_mx(x, fmt)
    assert np.array_equal(t.scales.cpu().numpy(), lo.tile_scales(byte))
    assert np.array_equal(t.codes.cpu().numpy(), lo.pack_codes(codes, fmt))
    out = lt.lite3r_dequantize_mx(t, torch.empty(x.shape, device="cuda"))
    with np.errstate(over="ignore"):
        ref = lo.mx_values(codes, byte, fmt).astype(np.float32)
    assert np.array_equal(f64(out), ref.astype(np.float64))


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_infinities_and_nan_take_their_block_alone(fmt, dtype):
    x = mx_input(2, 40, 128, DTYPES[dtype])
    x[3, 40] = float("inf")
    x[5, 0] = float("nan")
    x[7, 127] = -float("inf")
    t = lt.lite3r_quantize_mx(x.cuda(), fmt)
    out = f64(lt.lite3r_dequantize_mx(t, torch.empty((40, 128), device="cuda"))).reshape(40, 4, 32)
    codes, byte = lo.quantize_mx(f64(x), fmt)
    ref = lo.mx_values(codes, byte, fmt).reshape(40, 4, 32)
    bad = np.zeros((40, 4), dtype=bool)
    bad[3, 1] = bad[5, 0] = bad[7, 3] = True
    assert np.isnan(out[bad]).all() and np.array_equal(out[~bad], ref[~bad])


def test_strided_rows_and_given_buffers():
    wide = mx_input(3, 50, 200, torch.float32).cuda()
    x = wide[:, 8:136]
    a, b = lt.lite3r_quantize_mx(x), lt.lite3r_quantize_mx(x.contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    out = lt.alloc_mx(50, 128, "mxfp8", "cuda")
    assert lt.lite3r_quantize_mx(x, "mxfp8", out=out) is out
    target = torch.full((50, 200), 3.0, device="cuda")
    lt.lite3r_dequantize_mx(out, target[:, 8:136])
    assert (target[:, :8] == 3).all() and (target[:, 136:] == 3).all() and (target[:, 8:136] - x).abs().max() < x.abs().max() / 8
    for bad in (lambda: lt.lite3r_quantize_mx(x, "mxfp4", out=out), lambda: lt.lite3r_dequantize_mx(out, target),
                lambda: lt.lite3r_quantize_mx(wide[:, :40]), lambda: lt.lite3r_quantize_mx(wide.double()),
                lambda: lt.lite3r_quantize_mx(wide.t()), lambda: lt.lite3r_quantize_mx(wide[:, 2:34])):
        with pytest.raises(lt.Lite3rError):
            bad()


# ------------------------------------------------------------------------------------------------------ the linear layer
def mx_matrix(seed, rows, cols, fmt, spread=1.0):
    """(MxTensor on the GPU, its values in fp64)"""
    g = np.random.default_rng(seed)
    x = (g.standard_normal((rows, cols)) * np.exp(spread * g.standard_normal((rows, 1)))).astype(np.float32)
    codes, byte = lo.quantize_mx(x, fmt)
    t = lt.MxTensor(torch.from_numpy(lo.pack_codes(codes, fmt)).cuda(), torch.from_numpy(lo.tile_scales(byte)).cuda(), rows, cols, fmt)
    return t, lo.mx_values(codes, byte, fmt)


LINEAR_CASES = [(1, 32, 1, "f32", True), (70, 64, 9, "bf16", True), (33, 160, 131, "f16", True), (1, 1024, 1024, "bf16", True), (129, 96, 65, "f32", True), (300, 1184, 1000, "f32", False),
                (513, 2048, 136, "f16", True), (128, 64, 8, "bf16", False), (17, 128, 4096, "f32", True), (2000, 416, 1300, "bf16", True),
                (130, 544, 320, "f32", True), (10007, 288, 1003, "bf16", True), (5001, 544, 2056, "f32", False), (9000, 1120, 648, "f16", True)]


@pytest.mark.parametrize("rows,d_in,d_out,dtype,with_bias", LINEAR_CASES)
def test_linear_mxfp4(rows, d_in, d_out, dtype, with_bias):
    x, xv = mx_matrix(1, rows, d_in, "mxfp4")
    w, wv = mx_matrix(2, d_out, d_in, "mxfp4")
    bias = torch.randn(d_out, generator=torch.Generator().manual_seed(3)).cuda() if with_bias else None
    pitch = -(-d_out // 8) * 8 + 8
    buf = torch.full((rows + 3, pitch), 5.0, dtype=DTYPES[dtype], device="cuda")
    y = buf[:rows, :d_out]
    status = torch.ones(1, dtype=torch.int32, device="cuda")
    lt.lite3r_linear_mxfp4(x, w, bias, y, status)
    assert int(status.item()) == 0
    ref = xv @ wv.T + (f64(bias) if with_bias else 0.0)
    size = np.abs(xv) @ np.abs(wv).T + (np.abs(f64(bias)) if with_bias else 0.0)
    within(y, ref, 2 * U * (d_in / 64 + 2) * size, DTYPES[dtype], "y")
    assert (buf[rows:] == 5).all() and (buf[:, d_out:] == 5).all()  # nothing beside the result is touched
    again = torch.empty((rows, pitch), dtype=DTYPES[dtype], device="cuda")[:, :d_out]
    lt.lite3r_linear_mxfp4(x, w, bias, again)
    assert torch.equal(again, y)


def test_linear_mxfp4_with_scales_far_apart_and_nan_blocks():
    rows, d_in, d_out = 140, 256, 72
    g = np.random.default_rng(4)
    x = (g.standard_normal((rows, d_in)) * 2.0 ** g.integers(-40, 40, (rows, 1))).astype(np.float32)
    w = (g.standard_normal((d_out, d_in)) * 2.0 ** g.integers(-20, 20, (d_out, d_in // 32)).repeat(32, 1)).astype(np.float32)
    x[131, 70] = np.nan
    w[66, 10] = np.inf
    qx, qw = lt.lite3r_quantize_mx(torch.from_numpy(x).cuda()), lt.lite3r_quantize_mx(torch.from_numpy(w).cuda())
    y = torch.empty((rows, d_out), device="cuda")
    lt.lite3r_linear_mxfp4(qx, qw, None, y)
    xv, wv = (lo.mx_values(*lo.quantize_mx(a, "mxfp4"), "mxfp4") for a in (x, w))
    assert y[131].isnan().all() and y[:, 66].isnan().all()
    keep_r, keep_c = np.arange(rows) != 131, np.arange(d_out) != 66
    xv, wv = xv[keep_r], wv[keep_c]
    within(y[keep_r][:, keep_c], xv @ wv.T, 2 * U * (d_in / 64 + 2) * (np.abs(xv) @ np.abs(wv).T), torch.float32, "y")


BACK_CASES = [  # rows, d_in, d_out, dx dtype, weight format, checkpoint format, bias
    (1, 32, 8, "f32", "mxfp4", "mxfp8", True), (129, 96, 72, "bf16", "mxfp4", "mxfp8", True), (777, 1184, 1000, "f32", "mxfp4", "mxfp8", True),
    (2500, 160, 136, "f16", "mxfp8", "mxfp4", False), (65, 512, 2504, "f32", "mxfp4", "mxfp8", True), (300, 288, 5, "bf16", "mxfp8", "mxfp8", True),
    (4133, 256, 128, "bf16", "mxfp4", "mxfp8", True), (64, 1056, 264, "f32", "mxfp8", "mxfp4", True)]


@pytest.mark.parametrize("rows,d_in,d_out,dtype,w_fmt,x_fmt,with_bias", BACK_CASES)
def test_linear_backward(rows, d_in, d_out, dtype, w_fmt, x_fmt, with_bias):
    x, xv = mx_matrix(1, rows, d_in, x_fmt)
    w, wv = mx_matrix(2, d_out, d_in, w_fmt)
    pitch = -(-d_out // 8) * 8 + 16
    dy = torch.randn((rows, pitch), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    dy[:, d_out:] = float("nan")  # beside the gradient; it must not be read
    dy = dy[:, :d_out]
    g = f64(dy)
    status = torch.ones(1, dtype=torch.int32, device="cuda")
    buf = torch.full((rows + 2, d_in + 8), 5.0, dtype=DTYPES[dtype], device="cuda")
    dx = buf[:rows, :d_in]
    lt.lite3r_linear_mx_dgrad(dy, w, dx, status)
    assert int(status.item()) == 0
    within(dx, g @ wv, 2 * U * (d_out / 16 + 8) * (np.abs(g) @ np.abs(wv)), DTYPES[dtype], "dx")
    assert (buf[rows:] == 5).all() and (buf[:, d_in:] == 5).all()
    dw, db = torch.full((d_out + 1, d_in), 5.0, device="cuda"), torch.full((d_out,), 5.0, device="cuda") if with_bias else None
    ws = workspace(lt.lite3r_linear_mx_workspace(rows, d_in, d_out))
    status.fill_(1)
    lt.lite3r_linear_mx_wgrad(dy, x, dw[:d_out], db, ws, status)
    assert int(status.item()) == 0
    within(dw[:d_out], g.T @ xv, 2 * U * (min(rows, 2048) / 16 + rows / 1024 + 8) * (np.abs(g).T @ np.abs(xv)), torch.float32, "dw")
    assert (dw[d_out:] == 5).all()
    if with_bias:
        within(db, g.sum(0), (rows / 8 + 80) * U * np.abs(g).sum(0), torch.float32, "db")
    first = dw.clone()
    ws.fill_(0xFF)  # what a workspace holds does not matter
    lt.lite3r_linear_mx_wgrad(dy, x, dw[:d_out], None, ws)
    assert torch.equal(first, dw)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_backward_with_scales_far_apart(fmt):
    """Block scales from 2^-100 to 2^100, which bf16 has: values beyond what one factor could restore."""
    g = np.random.default_rng(6)
    n, d = 64, 128
    w = (g.standard_normal((n, d)) * 2.0 ** g.integers(-100, 100, (n, d // 32)).repeat(32, 1)).astype(np.float32)
    t = lt.lite3r_quantize_mx(torch.from_numpy(w).cuda(), fmt)
    wv = lo.mx_values(*lo.quantize_mx(w, fmt), fmt)
    eye = torch.eye(n, dtype=torch.bfloat16, device="cuda")
    dx = torch.empty((n, d), device="cuda")
    lt.lite3r_linear_mx_dgrad(eye, t, dx)
    assert np.array_equal(f64(dx), wv)
    dw = torch.empty((n, d), device="cuda")
    lt.lite3r_linear_mx_wgrad(eye, t, dw, None, workspace(lt.lite3r_linear_mx_workspace(n, d, n)))
    assert np.array_equal(f64(dw), wv)


def test_nan_in_gradients_weights_and_checkpoints():
    """A NaN of dy is in its row of dx and its column's row of dw; a NaN block of the weight or the checkpoint in its columns."""
    rows, d_in, d_out = 200, 192, 136
    g = np.random.default_rng(7)
    w, x = g.standard_normal((d_out, d_in)).astype(np.float32), g.standard_normal((rows, d_in)).astype(np.float32)
    w[130, 40] = np.nan
    x[150, 100] = np.inf
    dy = torch.from_numpy(g.standard_normal((rows, d_out))).bfloat16().cuda()
    dy[7, 9] = float("nan")
    dx, dw, db = torch.empty((rows, d_in), device="cuda"), torch.empty((d_out, d_in), device="cuda"), torch.empty(d_out, device="cuda")
    for w_fmt, x_fmt in (("mxfp4", "mxfp8"), ("mxfp8", "mxfp4")):
        qw, qx = lt.lite3r_quantize_mx(torch.from_numpy(w).cuda(), w_fmt), lt.lite3r_quantize_mx(torch.from_numpy(x).cuda(), x_fmt)
        lt.lite3r_linear_mx_dgrad(dy, qw, dx)
        lt.lite3r_linear_mx_wgrad(dy, qx, dw, db, workspace(lt.lite3r_linear_mx_workspace(rows, d_in, d_out)))
        nan_x, nan_w = np.zeros((rows, d_in), bool), np.zeros((d_out, d_in), bool)
        nan_x[7], nan_x[:, 32:64], nan_w[9], nan_w[:, 96:128] = True, True, True, True
        assert np.array_equal(np.isnan(f64(dx)), nan_x) and np.array_equal(np.isnan(f64(dw)), nan_w)
        assert np.array_equal(np.isnan(f64(db)), np.arange(d_out) == 9)


def test_few_steps_in_many_parts_of_the_device():
    """Contractions of one to four steps (fewer than there are converting groups) in more tiles than there are pairs, and the
    same calls many times over: the same bits each time."""
    for rows, d_in, d_out in ((1, 4096, 2048), (64, 2080, 4096), (100, 4096, 2504), (250, 1024, 4096), (4000, 4096, 40), (2000, 1056, 200)):
        dy = torch.randn((rows, d_out), generator=torch.Generator().manual_seed(rows)).bfloat16().cuda()
        w, wv = mx_matrix(1, d_out, d_in, "mxfp4")
        x, xv = mx_matrix(2, rows, d_in, "mxfp8")
        dx, dw, db = torch.empty((rows, d_in), device="cuda"), torch.empty((d_out, d_in), device="cuda"), torch.empty(d_out, device="cuda")
        ws = workspace(lt.lite3r_linear_mx_workspace(rows, d_in, d_out))
        lt.lite3r_linear_mx_dgrad(dy, w, dx)
        lt.lite3r_linear_mx_wgrad(dy, x, dw, db, ws)
        g = f64(dy)
        within(dx, g @ wv, 2 * U * (d_out / 16 + 8) * (np.abs(g) @ np.abs(wv)), torch.float32, "dx")
        within(dw, g.T @ xv, 2 * U * (min(rows, 2048) / 16 + rows / 1024 + 8) * (np.abs(g).T @ np.abs(xv)), torch.float32, "dw")
        within(db, g.sum(0), (rows / 8 + 80) * U * np.abs(g).sum(0), torch.float32, "db")
        first = [t.clone() for t in (dx, dw, db)]
        differing = torch.zeros(3, device="cuda", dtype=torch.int64)
        for _ in range(200):
            lt.lite3r_linear_mx_dgrad(dy, w, dx)
            lt.lite3r_linear_mx_wgrad(dy, x, dw, db, ws)
            differing += torch.stack([(a != b).sum() for a, b in zip((dx, dw, db), first)])
        assert not differing.any(), (rows, d_in, d_out, differing)


def test_long_sums_do_not_drift():
    """All terms positive over 40000 rows: a running sum that is cut off at every step would be low by 4e-9 x 2500."""
    rows, d_in, d_out = 40000, 64, 64
    x = lt.lite3r_quantize_mx((1 + torch.rand((rows, d_in), generator=torch.Generator().manual_seed(1))).cuda(), "mxfp8")
    xv = f64(lt.lite3r_dequantize_mx(x, torch.empty((rows, d_in), device="cuda")))
    dy = (1 + torch.rand((rows, d_out), generator=torch.Generator().manual_seed(2))).bfloat16().cuda()
    dw = torch.empty((d_out, d_in), device="cuda")
    lt.lite3r_linear_mx_wgrad(dy, x, dw, None, workspace(lt.lite3r_linear_mx_workspace(rows, d_in, d_out)))
    ref = f64(dy).T @ xv
    # at most 128 products of 16 rows in a running sum, each cut off by less than 2 u of it, half that on average along
    # the way; twenty sums of them rounded
    assert (np.abs(f64(dw) - ref) <= (2 * U * 128 / 2 + 20 * U) * ref).all()
    assert np.abs(f64(dw) / ref - 1).max() < 2.5e-6


def test_more_refusals_on_the_device():
    x, w = mx_matrix(1, 8, 64, "mxfp4")[0], mx_matrix(2, 8, 96, "mxfp4")[0]
    y = torch.empty((8, 8), device="cuda")
    dy = torch.zeros((8, 8), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1 << 16)
    q = torch.zeros((1, 2, 4, 64), device="cuda")
    for bad in (lambda: lt.lite3r_linear_mxfp4(x, w, None, y),                        # d_in differs
                lambda: lt.lite3r_linear_mxfp4(x, mx_matrix(2, 8, 64, "mxfp8")[0], None, y),
                lambda: lt.lite3r_linear_mxfp4(x, x, None, y[:, :4]), lambda: lt.lite3r_linear_mxfp4(x, x, y[0, :4], y),
                lambda: lt.lite3r_linear_mxfp4(x, x, None, y.double()), lambda: lt.lite3r_linear_mxfp4(x, x, None, y.t()),
                lambda: lt.lite3r_linear_mx_dgrad(dy.float(), x, torch.empty((8, 64), device="cuda")),
                lambda: lt.lite3r_linear_mx_dgrad(dy, x, y), lambda: lt.lite3r_linear_mx_wgrad(dy[:4], x, y, None, ws),
                lambda: lt.lite3r_linear_mx_wgrad(dy, x, torch.empty((8, 64), device="cuda"), None, ws[:8]),
                lambda: lt.lite3r_linear_mx_wgrad(dy, x, torch.empty((8, 64), device="cuda"), None, ws[1:]),
                lambda: lt.lite3r_linear_mxfp4(x, x, None, y, torch.zeros(1, device="cuda")),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, None), lambda: lt.lite3r_qk_norm_rope(q, q, q, q[:, :1]),
                lambda: lt.lite3r_qk_norm_rope(q, q.half(), q, q.half()), lambda: lt.lite3r_qk_norm_rope(q, q[:, :, :2], q, q[:, :, :2]),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, norm="batch"),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, q_weight=torch.ones(32, device="cuda")),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, positions=torch.zeros((4, 1), device="cuda")),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, positions=torch.zeros((3, 1), dtype=torch.int32, device="cuda")),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, positions=torch.zeros((4, 3), dtype=torch.int32, device="cuda")),
                lambda: lt.lite3r_qk_norm_rope(q, q, q, q, positions=torch.zeros((4, 1), dtype=torch.int32)),
                lambda: lt.lite3r_qk_norm_rope(q, None, q[:1].expand(1, 2, 4, 64).expand(1, 2, 4, 64)[:, :, :1].expand(1, 2, 4, 64), None)):
        with pytest.raises(lt.Lite3rError):
            bad()
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------ together
def layer_buffers(B, N, H, d):
    g = torch.Generator().manual_seed(21)
    rows = B * N
    s = {"x": torch.randn((rows, d), generator=g).bfloat16().cuda(),
         "w": (torch.randn((3 * H * 64, d), generator=g) / d ** 0.5).cuda(), "bias": (0.1 * torch.randn(3 * H * 64, generator=g)).cuda(),
         "affine": affine(22, 64), "pos": torch.randint(0, 38, (N, 2), generator=g).int().cuda(),
         "dout": (0.1 * torch.randn((B, N, 3 * H, 64), generator=g)).bfloat16().cuda()}
    s["wq"] = lt.lite3r_quantize_mx(s["w"], "mxfp4")
    s["xq"], s["kept"] = lt.alloc_mx(rows, d, "mxfp4", "cuda"), lt.alloc_mx(rows, d, "mxfp8", "cuda")
    s["qkv"] = torch.empty((B, N, 3 * H, 64), dtype=torch.bfloat16, device="cuda")
    s["turned"] = torch.empty((2, B, H, N, 64), dtype=torch.bfloat16, device="cuda")
    s["dqkv"] = torch.empty_like(s["qkv"])
    s["dx"], s["dw"], s["db"] = torch.empty((rows, d), device="cuda"), torch.empty((3 * H * 64, d), device="cuda"), torch.empty(3 * H * 64, device="cuda")
    s["grads"] = {n: torch.empty(64, device="cuda") for n in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
    s["ws"] = workspace(max(lt.lite3r_linear_mx_workspace(rows, d, 3 * H * 64), lt.lite3r_qk_norm_rope_workspace(64)))
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["engine"] = lt.SlaForward(B, H, N, 64, 0.3, 0.3)
    s["proj"] = (torch.randn((H, 64, 64), generator=g) / 8).cuda()
    return s


def layer_step(s, H, stream=None):
    """Projection in 4 bits, norms and rotation, sparse linear attention; checkpoint in 8 bits; backward to the projection."""
    heads = lambda t, i: t[:, :, i * H:(i + 1) * H].permute(0, 2, 1, 3)  # noqa: E731
    qw, qb, kw, kb = s["affine"]
    B, N = s["qkv"].shape[:2]
    lt.lite3r_quantize_mx(s["x"], "mxfp4", out=s["xq"], stream=stream)
    lt.lite3r_quantize_mx(s["x"], "mxfp8", out=s["kept"], stream=stream)
    lt.lite3r_linear_mxfp4(s["xq"], s["wq"], s["bias"], s["qkv"].view(B * N, -1), s["status"], stream)
    q, k, v = (heads(s["qkv"], i) for i in range(3))
    lt.lite3r_qk_norm_rope(q, k, s["turned"][0], s["turned"][1], q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb, positions=s["pos"],
                           stream=stream)
    s["engine"].run(s["turned"][0], s["turned"][1], v, s["proj"], stream=stream)
    dq, dk, dv = (heads(s["dqkv"], i) for i in range(3))
    gq, gk, _ = (heads(s["dout"], i) for i in range(3))
    lt.lite3r_qk_norm_rope_backward(q, k, gq, gk, dq, dk, s["ws"], q_weight=qw, k_weight=kw, positions=s["pos"], stream=stream, **s["grads"])
    lt.lite3r_linear_mx_dgrad(s["dqkv"].view(B * N, -1), s["wq"], s["dx"], s["status"], stream)
    lt.lite3r_linear_mx_wgrad(s["dqkv"].view(B * N, -1), s["kept"], s["dw"], s["db"], s["ws"], s["status"], stream)


RESULTS = ("qkv", "turned", "dqkv", "dx", "dw", "db")


def test_a_layer_forward_and_backward():
    B, N, H, d = 2, 157, 4, 256
    s = layer_buffers(B, N, H, d)
    heads = lambda t, i: t[:, :, i * H:(i + 1) * H].permute(0, 2, 1, 3)  # noqa: E731
    s["dqkv"].copy_(s["dout"])  # the values' gradient goes through as it is
    layer_step(s, H)
    torch.cuda.synchronize()
    assert int(s["status"].item()) == 0 and int(s["engine"].status.item()) == 0
    x, w = f64(s["x"]), f64(s["w"])
    xv, wv, kept = (lo.mx_values(*lo.quantize_mx(a, f), f) for a, f in ((x, "mxfp4"), (w, "mxfp4"), (x, "mxfp8")))
    within(s["qkv"].view(B * N, -1), xv @ wv.T + f64(s["bias"]), 2 * U * 8 * (np.abs(xv) @ np.abs(wv).T), torch.bfloat16, "qkv")
    qw, qb, kw, kb = s["affine"]
    pos = np.broadcast_to(s["pos"].cpu().numpy()[None], (B, N, 2))
    q, k, v = (heads(s["qkv"], i) for i in range(3))
    check_rows(s["turned"][0], q, "layer", qw, qb, 1e-5, pos, 100.0, "q")
    check_rows(s["turned"][1], k, "layer", kw, kb, 1e-5, pos, 100.0, "k")
    ref = orc.sla_forward_from_source(*(f64(t).astype(np.float32) for t in (s["turned"][0], s["turned"][1], v)), s["proj"].cpu().numpy(),
                                      64, 0.3, 0.3)
    rel, _ = pu.output_errors(s["engine"].out.cpu().numpy(), ref["out"])
    assert rel <= pu.REL_L2_TOL
    for i, (src, wt, n) in enumerate(((q, qw, "q"), (k, kw, "k"))):
        check_row_grads((heads(s["dqkv"], i), s["grads"][f"d{n}_weight"], s["grads"][f"d{n}_bias"]), src, heads(s["dout"], i), "layer", wt, 1e-5,
                        pos, 100.0, n)
    assert torch.equal(heads(s["dqkv"], 2), heads(s["dout"], 2))
    g = f64(s["dqkv"]).reshape(B * N, -1)
    within(s["dx"], g @ wv, 2 * U * (g.shape[1] / 16 + 8) * (np.abs(g) @ np.abs(wv)), torch.float32, "dx")
    within(s["dw"], g.T @ kept, 2 * U * (B * N / 16 + 8) * (np.abs(g).T @ np.abs(kept)), torch.float32, "dw")
    within(s["db"], g.sum(0), (B * N + 80) * U * np.abs(g).sum(0), torch.float32, "db")


def test_a_layer_on_another_stream_and_captured():
    """The same bits from a side stream, from a captured graph whose inputs change between replays, and from two streams at
    once with buffers of their own."""
    B, N, H, d = 1, 200, 4, 256
    s, t = layer_buffers(B, N, H, d), layer_buffers(B, N, H, d)
    for a in (s, t):
        a["dqkv"].copy_(a["dout"])
    layer_step(s, H)
    torch.cuda.synchronize()
    first = {n: s[n].clone() for n in RESULTS}
    out = s["engine"].out.clone()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for n in RESULTS[:2] + RESULTS[3:]:
        s[n].fill_(3.0)
    torch.cuda.synchronize()
    for _ in range(3):
        layer_step(s, H, one)
        layer_step(t, H, two)
    torch.cuda.synchronize()
    for n in RESULTS:
        assert torch.equal(s[n], first[n]) and torch.equal(t[n], first[n]), n
    assert torch.equal(s["engine"].out, out) and torch.equal(t["engine"].out, out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(one):
        graph.capture_begin()
        layer_step(s, H, one)
        graph.capture_end()
    new = torch.randn(s["x"].shape, generator=torch.Generator().manual_seed(30)).bfloat16().cuda()
    for a in (s, t):
        a["x"].copy_(new)
    graph.replay()
    layer_step(t, H)
    torch.cuda.synchronize()
    assert not torch.equal(t["qkv"], first["qkv"])
    for n in RESULTS:
        assert torch.equal(s[n], t[n]), n
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s[n], t[n]) for n in RESULTS)
