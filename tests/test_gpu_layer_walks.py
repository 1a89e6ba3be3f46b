"""The parts of the operators around the attention that only large calls run -- several heads to a group of lanes, several
steps of the grid, pairs of CTAs over many tiles -- and the settings at the ends of what the calls accept.

The rows of test_gpu_layer_ops are few enough that every head of a token has a group of lanes of its own; here they are not.
References are in fp64, by complex numbers on the device; sums over rows are of whole numbers, which fp32 adds exactly, so that one
row too many or too few is seen.
"""
import numpy as np
import pytest
import torch

import test_gpu_layer_ops as base
from paper_2605_11354_b200 import binding as lt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = base.DTYPES


def turned(z, positions, base_, back=False):
    """The rotation of z [B, H, N, D] (fp64) by positions [B, N, axes]: a pair is a complex number."""
    axes = positions.shape[-1]
    half = z.shape[-1] // axes // 2
    angle = positions.double()[:, None, :, :, None] * base_ ** (-torch.arange(half, device=z.device, dtype=torch.float64) / half)
    a, b = z.view(*z.shape[:3], axes, 2, half).unbind(-2)
    c = torch.complex(a, b) * torch.polar(torch.ones_like(angle), -angle if back else angle)
    return torch.stack([c.real, c.imag], -2).reshape(z.shape)


def normed(x, norm, eps):
    if norm == "none":
        return x, torch.ones_like(x[..., :1])
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return x * r, r


def all_within(got, ref, tol, dtype, what):
    """As within() of the other file, on the device; nothing here comes near the end of a type."""
    half = torch.finfo(dtype).eps / 2
    tol = tol + half * (ref.abs() + tol) + base.TINY[dtype]
    worst = ((got.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, (what, worst)


# ------------------------------------------------------------------------------------------------------ walks over heads
# B, H, K, N, D, axes, norm, dtype.  With 148 SMs the forward gives a group of lanes
#   4 of 10 heads and 2 of 5;   12 of 24 and all 7;   all 16;   all 7 and all 3;   all 5 and 12 of 24;   4 of 10 and 2 of 5;   all 5
# and the gradient 4 and 2;  4 and 4;  4;  4 and 3;  3 and 4;  4 and 3;  3, in two to nine steps of the grid.
WALKS = [(3, 10, 5, 3001, 64, 1, "rms", "bf16"), (2, 24, 7, 10000, 64, 2, "layer", "bf16"), (1, 16, 16, 32003, 64, 2, "layer", "f16"),
         (1, 7, 3, 10007, 128, 1, "rms", "f16"), (4, 5, 24, 10001, 32, 2, "layer", "f32"), (3, 10, 5, 3001, 64, 0, "layer", "f32"),
         (1, 5, 5, 9001, 256, 2, "none", "f32")]


@pytest.mark.parametrize("B,H,K,N,D,axes,norm,dtype", WALKS)
def test_rows_of_a_walk(B, H, K, N, D, axes, norm, dtype):
    eps, turn_base = 1e-5, 100.0
    q, k = base.rope_inputs(41, B, H, K, N, D, DTYPES[dtype], "packed")
    dqo, dko = base.rope_inputs(42, B, H, K, N, D, DTYPES[dtype], "heads")
    qw, qb, kw, kb = base.affine(43, D)
    pos = torch.randint(-40, 1400, (B, N, axes), generator=torch.Generator().manual_seed(44)).int().cuda() if axes else None
    how = dict(norm=norm, positions=pos, base=turn_base, eps=eps)
    out = [torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda") for x in (q, k)]
    lt.lite3r_qk_norm_rope(q, k, *out, q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb, **how)
    grads = [torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda") for x in (q, k)]
    lt.lite3r_qk_norm_rope_backward(q, k, dqo, dko, *grads, base.workspace(lt.lite3r_qk_norm_rope_workspace(D)), q_weight=qw, k_weight=kw, **how)
    roundings = 32 if dtype == "f32" else 46  # the counts of test_gpu_layer_ops
    for x, y, dy, dx, w, b, name in ((q, out[0], dqo, grads[0], qw, qb, "q"), (k, out[1], dko, grads[1], kw, kb, "k")):
        for h in range(x.shape[1]):
            x64, dy64 = x[:, h:h + 1].double(), dy[:, h:h + 1].double()
            xh, r = normed(x64, norm, eps)
            z = xh * w + b
            ref = z if pos is None else turned(z, pos, turn_base)
            top = x64.abs().amax(-1, keepdim=True) * r
            all_within(y[:, h:h + 1], ref, roundings * U * (top * w.abs().max() + b.abs().max()), y.dtype, (name, h))
            g = dy64 if pos is None else turned(dy64, pos, turn_base, back=True)
            gh = g * w
            d = gh
            if norm != "none":
                d = gh - xh * (gh * xh).mean(-1, keepdim=True)
                d = (d - gh.mean(-1, keepdim=True) if norm == "layer" else d) * r
            a = 2 * dy64.abs().amax(-1, keepdim=True) * w.abs().max()
            all_within(dx[:, h:h + 1], d, 64 * U * r * a * (1 + top + top * top), dx.dtype, (name, h, "dx"))


def whole_rows(seed, shape, dtype):
    """Rows of as many 1 as -1: no mean, variance 1, whole numbers after either norm without an epsilon."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.rand(shape, generator=g, device="cuda").argsort(-1)
    return (1 - 2 * (order % 2)).to(dtype)


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("B,H,K,N,D,dtype", [(1, 1, 1, 3, 64, "f32"), (2, 3, 2, 37, 32, "bf16"), (1, 8, 2, 1, 256, "f16"), (1, 5, 1, 130, 128, "bf16"),
                                             (3, 10, 5, 3001, 64, "bf16"), (3, 10, 5, 3001, 64, "f32"), (2, 24, 7, 10000, 64, "f16"),
                                             (4, 5, 24, 10001, 32, "bf16"), (1, 7, 3, 20011, 128, "f16")])
def test_sums_without_an_epsilon_count_every_row_once(B, H, K, N, D, dtype, norm):
    """Gradients of whole numbers in some rows -- the first and last of every head and sequence among them -- and zeros in
    the rest: adding a zero is exact, and some 300 terms of at most 4 in fp32 in any order, with a root that is off by 2 ulp, are
    off by at most (300 + 4) u of a sum of magnitudes below 1200: 0.03.  A row lost, doubled or taken from its
    neighbour is off by 1 or more in half of the elements.  Rows of zeros have no deviation: at eps = 0 they may not be looked at."""
    args = []
    for heads, seed in ((H, 1), (K, 2)):
        x = whole_rows(seed, (B, heads, N, D), DTYPES[dtype])
        g = torch.Generator().manual_seed(seed)
        dy = torch.zeros(B * heads * N, D)
        ends = [(b * heads + h) * N + n for b in {0, B - 1} for h in range(heads) for n in (0, N - 1)]
        rows = torch.unique(torch.cat([torch.tensor(ends), torch.randint(0, B * heads * N, (150,), generator=g)]))
        assert len(rows) <= 300
        dy[rows] = torch.randint(1, 5, (len(rows), D), generator=g).float()
        args.append((x, dy.view(B, heads, N, D).to(DTYPES[dtype]).cuda()))
    total = [((x.double() * dy.double()).sum((0, 1, 2)), dy.double().sum((0, 1, 2))) for x, dy in args]
    grads = {n: torch.full((D,), 7.0, device="cuda") for n in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
    for positions in (None, torch.zeros((N, 2), dtype=torch.int32, device="cuda")):  # a turn by nothing is exact, too
        dx = [torch.empty_like(x) for x, _ in args]
        lt.lite3r_qk_norm_rope_backward(args[0][0], args[1][0], args[0][1], args[1][1], *dx, base.workspace(lt.lite3r_qk_norm_rope_workspace(D)),
                                        norm=norm, eps=0.0, positions=positions, **grads)
        for (dw, db), name in zip(total, "qk"):
            assert torch.equal(grads[f"d{name}_bias"].double(), db), name
            off = (grads[f"d{name}_weight"].double() - dw).abs().max().item()
            assert off <= (0.0 if norm == "none" else 0.03), (name, off)  # (a NaN compares false)
        assert all(t.isfinite().all() for t in dx)


def test_dense_sums_of_whole_numbers():
    """Every row has a gradient: sums of whole numbers below 2^24 are exact in fp32 in any order."""
    for B, H, K, N, D, dtype in ((3, 10, 5, 3001, 64, torch.bfloat16), (1, 16, 4, 40003, 64, torch.float16), (2, 6, 6, 9001, 128, torch.float32)):
        g = torch.Generator(device="cuda").manual_seed(3)
        ints = lambda heads: torch.randint(-3, 4, (B, heads, N, D), generator=g, device="cuda").to(dtype)  # noqa: E731
        q, k, dqo, dko = ints(H), ints(K), ints(H), ints(K)
        grads = {n: torch.full((D,), 7.0, device="cuda") for n in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
        lt.lite3r_qk_norm_rope_backward(q, k, dqo, dko, torch.empty_like(q), torch.empty_like(k),
                                        base.workspace(lt.lite3r_qk_norm_rope_workspace(D)), norm="none", **grads)
        for x, dy, name in ((q, dqo, "q"), (k, dko, "k")):
            assert torch.equal(grads[f"d{name}_weight"].double(), (x.double() * dy.double()).sum((0, 1, 2)))
            assert torch.equal(grads[f"d{name}_bias"].double(), dy.double().sum((0, 1, 2)))


def test_more_heads_than_a_grid_has_parts():
    """Heads of a token are parts of the grid's second dimension, of which there are 65535: 70000 and 40000 go by threes and twos."""
    H, K, D = 70000, 40000, 32
    q, k = base.rope_inputs(5, 1, H, K, 1, D, torch.bfloat16, "heads")
    pos = torch.tensor([[7]], dtype=torch.int32, device="cuda")
    out, few = [torch.full_like(x, 9.0) for x in (q, k)], [torch.empty_like(x) for x in (q, k)]
    lt.lite3r_qk_norm_rope(q, k, *out, positions=pos)
    for h in range(0, H, 20000):  # as calls of fewer heads
        lt.lite3r_qk_norm_rope(q[:, h:h + 20000], None, few[0][:, h:h + 20000], None, positions=pos)
    for h in range(0, K, 20000):
        lt.lite3r_qk_norm_rope(k[:, h:h + 20000], None, few[1][:, h:h + 20000], None, positions=pos)
    assert torch.equal(out[0], few[0]) and torch.equal(out[1], few[1])
    dq, dk = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    dw = {n: torch.empty(D, device="cuda") for n in ("dq_weight", "dk_weight")}
    lt.lite3r_qk_norm_rope_backward(q, k, q, k, dq, dk, base.workspace(lt.lite3r_qk_norm_rope_workspace(D)), norm="none", positions=pos, **dw)
    for x, d, name in ((q, dq, "q"), (k, dk, "k")):
        x64, p = x.double(), pos.view(1, 1, 1)
        g = turned(x64, p, 100.0, back=True)
        all_within(d, g, 46 * U * 2 * x64.abs().amax(-1, keepdim=True), d.dtype, name)
        n = x.shape[1]
        size = (g.abs() * x64.abs()).sum((0, 1, 2))
        all_within(dw[f"d{name}_weight"], (g * x64).sum((0, 1, 2)), (n + 64) * U * size, torch.float32, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_sums_have_sines_of_fp32(dtype):
    """The weight and bias gradients are fp32 results of 16-bit sources, too.  A gradient of (1, 0) in every pair of a single row
    makes the bias gradient (cos, -sin).  The angle is rounded to 24 bits below half a turn: off by at most 2^-26 turns, 1.58 u;
    sine and cosine are good to one ulp, at most u below 1; nothing is rounded after that."""
    D, turn_base = 256, 100.0
    x = torch.ones((1, 1, 1, D), dtype=DTYPES[dtype], device="cuda")
    dy = torch.zeros_like(x)
    dy[..., :D // 2] = 1
    dx, db, ws = torch.empty_like(x), torch.empty(D, device="cuda"), base.workspace(lt.lite3r_qk_norm_rope_workspace(D))
    worst = 0.0
    for p in np.random.default_rng(6).integers(-1400, 1400, 60):
        lt.lite3r_qk_norm_rope_backward(x, None, dy, None, dx, None, ws, norm="none", dq_bias=db, base=turn_base,
                                        positions=torch.tensor([[p]], dtype=torch.int32, device="cuda"))
        angle = p * turn_base ** (-np.arange(D // 2) / (D // 2))
        worst = max(worst, np.abs(base.f64(db) - np.concatenate([np.cos(angle), -np.sin(angle)])).max())
    assert worst <= 2.7 * U, worst / U


# ------------------------------------------------------------------------------------------------------ pairs of CTAs
@pytest.mark.parametrize("rows,d_in,d_out,dtype", [(20000, 256, 1024, "bf16"), (10007, 288, 1003, "f32"), (5001, 2080, 2056, "f16"),
                                                   (43968, 64, 256, "bf16"), (2048, 4096, 5120, "f32")])
def test_pairs_give_the_same_bits_each_time(rows, d_in, d_out, dtype):
    """Many tiles of 256 x 256 to a pair, from one stage of operands to a tile to many: what one CTA hands to the other, and the
    columns that two accumulators share.  A part of the rows and columns against the definition."""
    x, xv = base.mx_matrix(1, rows, d_in, "mxfp4")
    w, wv = base.mx_matrix(2, d_out, d_in, "mxfp4")
    pitch = -(-d_out // 8) * 8
    first, y = (torch.full((rows, pitch), 5.0, dtype=DTYPES[dtype], device="cuda")[:, :d_out] for _ in range(2))
    lt.lite3r_linear_mxfp4(x, w, None, first)
    r, c = (np.unique(np.concatenate([np.arange(0, n, max(1, n // 150)), [n - 1]])) for n in (rows, d_out))
    ref, size = xv[r] @ wv[c].T, np.abs(xv[r]) @ np.abs(wv[c]).T
    base.within(first[torch.from_numpy(r).cuda()][:, torch.from_numpy(c).cuda()], ref, 2 * U * (d_in / 64 + 2) * size, DTYPES[dtype], "y")
    differing = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(100):
        lt.lite3r_linear_mxfp4(x, w, None, y)
        differing += (y != first).sum()
    assert int(differing.item()) == 0


@pytest.mark.parametrize("rows,d_in,d_out,w_fmt,x_fmt", [(3000, 1024, 4096, "mxfp4", "mxfp8"), (5003, 2080, 1000, "mxfp8", "mxfp4"),
                                                         (20000, 512, 264, "mxfp4", "mxfp8")])
def test_backward_pairs_give_the_same_bits_each_time(rows, d_in, d_out, w_fmt, x_fmt):
    """Contractions long enough to go round the rings of stages many times, from two streams at once."""
    w, wv = base.mx_matrix(1, d_out, d_in, w_fmt)
    x, xv = base.mx_matrix(2, rows, d_in, x_fmt)
    dy = torch.randn((rows, d_out), generator=torch.Generator().manual_seed(rows)).bfloat16().cuda()
    ws = [base.workspace(lt.lite3r_linear_mx_workspace(rows, d_in, d_out)) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def results():
        return [torch.full(s, 5.0, dtype=t, device="cuda") for s, t in (((rows, d_in), torch.bfloat16), ((d_out, d_in), torch.float32),
                                                                        ((d_out,), torch.float32))]

    first, again = results(), [results() for _ in range(2)]
    lt.lite3r_linear_mx_dgrad(dy, w, first[0])
    lt.lite3r_linear_mx_wgrad(dy, x, first[1], first[2], ws[0])
    r, c = np.arange(0, rows, max(1, rows // 150)), np.arange(0, d_out, max(1, d_out // 150))
    g = base.f64(dy)
    base.within(first[0][torch.from_numpy(r).cuda()], g[r] @ wv, 2 * U * (d_out / 16 + 8) * (np.abs(g[r]) @ np.abs(wv)), torch.bfloat16, "dx")
    base.within(first[1][torch.from_numpy(c).cuda()], g[:, c].T @ xv, 2 * U * (min(rows, 2048) / 16 + rows / 1024 + 8) * (np.abs(g[:, c]).T @ np.abs(xv)),
                torch.float32, "dw")
    torch.cuda.synchronize()
    differing = [torch.zeros(3, dtype=torch.int64, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(50):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                lt.lite3r_linear_mx_dgrad(dy, w, again[i][0])
                lt.lite3r_linear_mx_wgrad(dy, x, again[i][1], again[i][2], ws[i])
                differing[i] += torch.stack([(a != b).sum() for a, b in zip(again[i], first)])
    torch.cuda.synchronize()
    assert not any(d.any() for d in differing), differing


# ------------------------------------------------------------------------------------------------------ very long contractions
def places(n, seed):
    """Some hundred places below n, the first and last among them."""
    p = np.random.default_rng(seed).integers(0, n, 300)
    return torch.from_numpy(np.unique(np.concatenate([p, [0, 1, n // 2, n - 1]]))).cuda()


def test_a_product_that_takes_seconds():
    """One row by one column of 3 x 2^29 elements: one sum of 6 million steps, longer than a wait on a barrier may take otherwise.  Nearly
    all elements are zero, so the sum of the others, multiples of 1/4, is exact."""
    n = 3 << 29
    at = places(n // 2, 1)  # bytes of two codes
    g = torch.Generator(device="cuda").manual_seed(2)
    values, operands = [], []
    for _ in range(2):
        codes = torch.zeros((1, n // 2), dtype=torch.uint8, device="cuda")
        byte = torch.randint(0, 256, (len(at),), generator=g, device="cuda").to(torch.uint8)
        codes[0, at] = byte
        scales = torch.zeros((1, n // 128, 32, 4, 4), dtype=torch.uint8, device="cuda")
        scales[:, :, 0, 0] = 127
        operands.append(lt.MxTensor(codes, scales, 1, n))
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
        values.append(torch.stack([table[(byte & 15).long()], table[(byte >> 4).long()]]))
    y, status = torch.full((1, 8), 9.0, device="cuda")[:, :1], torch.ones(1, dtype=torch.int32, device="cuda")
    lt.lite3r_linear_mxfp4(operands[0], operands[1], None, y, status)
    assert int(status.item()) == 0
    assert float(y.item()) == float((values[0] * values[1]).sum())


def test_an_input_gradient_that_takes_seconds():
    """The same for a layer of 3 x 2^27 outputs and a 16-bit result (fp32 results are sums of 2048 steps of the contraction)."""
    n, d_in = 3 << 27, 32
    at = places(n, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    codes = torch.zeros((n, d_in // 2), dtype=torch.uint8, device="cuda")
    codes[at] = 0x24  # 1 in the odd columns and 2 in the even ones
    scales = torch.full((n // 128, 1, 32, 4, 4), 127, dtype=torch.uint8, device="cuda")
    dy = torch.zeros((1, n), dtype=torch.bfloat16, device="cuda")
    dy[0, at] = torch.randint(-4, 5, (len(at),), generator=g, device="cuda").bfloat16()
    dx, status = torch.full((1, d_in), 9.0, dtype=torch.float16, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    lt.lite3r_linear_mx_dgrad(dy, lt.MxTensor(codes, scales, n, d_in), dx, status)
    assert int(status.item()) == 0
    total = float(dy[0, at].double().sum())
    assert abs(total) < 1024
    assert dx[0, 0::2].tolist() == [2 * total] * 16 and dx[0, 1::2].tolist() == [total] * 16  # whole numbers below 2048


@pytest.mark.parametrize("rows,d_in,d_out", [(130, 65536, 72), (2000, 32768, 2504)])
def test_a_long_running_sum_of_the_4_bit_layer(rows, d_in, d_out):
    """All terms positive, block scales spread over 2^6: the running sum is cut off at fp32 after every product of 64 elements, by
    less than 2 u of what it is then, which is at most the result: 2 u d_in / 64 in all, and nothing is added after."""
    def operand(seed, n):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = (0.5 + torch.rand((n, d_in // 32, 32), generator=g, device="cuda")) * torch.exp2(torch.randint(0, 7, (n, d_in // 32, 1), generator=g,
                                                                                                         device="cuda").float())
        t = lt.lite3r_quantize_mx(x.view(n, d_in), "mxfp4")
        return t, lt.lite3r_dequantize_mx(t, torch.empty((n, d_in), device="cuda")).double()

    (x, xv), (w, wv) = operand(1, rows), operand(2, d_out)
    y = torch.empty((rows, d_out), device="cuda")
    lt.lite3r_linear_mxfp4(x, w, None, y)
    off = (y.double() / (xv @ wv.t()) - 1)
    assert off.abs().max().item() <= 2 * U * (d_in / 64 + 1), (off.min().item() / U, off.max().item() / U)
    print(f"off by {off.mean().item() / U / (d_in / 64):.3f} u a product, {off.min().item() / U:.1f} to {off.max().item() / U:.1f} u")


# ------------------------------------------------------------------------------------------------------ more than 2^31 elements
def test_matrices_of_more_elements_than_an_index_of_32_bits_has():
    rows, cols = 70001, 32768
    assert rows * cols > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 10000):
        x[r:r + 10000] = torch.randn((min(10000, rows - r), cols), generator=g, device="cuda", dtype=torch.bfloat16)
    # the last tile of 128 rows (and what is left of it) as a matrix of its own
    tail = rows // 128 * 128 - 128
    for fmt in ("mxfp4", "mxfp8"):
        t, part = lt.lite3r_quantize_mx(x, fmt), lt.lite3r_quantize_mx(x[tail:], fmt)
        assert torch.equal(t.codes[tail:], part.codes) and torch.equal(t.scales[tail // 128:], part.scales)
        back = lt.lite3r_dequantize_mx(t, torch.empty_like(x))
        assert torch.equal(back[tail:], lt.lite3r_dequantize_mx(part, torch.empty_like(x[tail:])))
        assert torch.equal(back[:300], lt.lite3r_dequantize_mx(lt.lite3r_quantize_mx(x[:300], fmt), torch.empty_like(x[:300])))
        del t, back
    del x
    # a result, an input gradient and a weight gradient of that size
    few = 64
    a, w = lt.lite3r_quantize_mx(torch.randn((rows, few), generator=g, device="cuda")), lt.lite3r_quantize_mx(torch.randn((cols, few), generator=g, device="cuda"))
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    lt.lite3r_linear_mxfp4(a, w, None, y)
    av, wv = (lt.lite3r_dequantize_mx(t, torch.empty((t.rows, few), device="cuda")).double() for t in (a, w))
    pick = torch.cat([torch.arange(200, device="cuda"), torch.arange(rows - 200, rows, device="cuda")])
    size = av[pick].abs() @ wv.abs().t()
    all_within(y[pick], av[pick] @ wv.t(), 2 * U * (few / 64 + 2) * size, y.dtype, "y")
    del y
    dy = torch.randn((rows, few), generator=g, device="cuda").bfloat16()
    wide = lt.lite3r_quantize_mx(torch.randn((few, cols), generator=g, device="cuda"), "mxfp4")
    dx = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    lt.lite3r_linear_mx_dgrad(dy, wide, dx)
    value = lt.lite3r_dequantize_mx(wide, torch.empty((few, cols), device="cuda")).double()
    d = dy[pick].double()
    all_within(dx[pick], d @ value, 2 * U * (few / 16 + 8) * (d.abs() @ value.abs()), dx.dtype, "dx")
    del dx
    outputs = rows // 8 * 8
    kept = lt.lite3r_quantize_mx(torch.randn((few, cols), generator=g, device="cuda"), "mxfp8")
    dy = torch.randn((few, outputs), generator=g, device="cuda").bfloat16()
    dw, db = torch.empty((outputs, cols), device="cuda"), torch.empty(outputs, device="cuda")
    lt.lite3r_linear_mx_wgrad(dy, kept, dw, db, base.workspace(lt.lite3r_linear_mx_workspace(few, cols, outputs)))
    value = lt.lite3r_dequantize_mx(kept, torch.empty((few, cols), device="cuda")).double()
    pick = torch.cat([torch.arange(200, device="cuda"), torch.arange(outputs - 200, outputs, device="cuda")])
    d = dy[:, pick].double().t()
    all_within(dw[pick], d @ value, 2 * U * (few / 16 + 8) * (d.abs() @ value.abs()), dw.dtype, "dw")
    all_within(db, dy.double().sum(0), (few + 8) * U * dy.double().abs().sum(0), db.dtype, "db")
