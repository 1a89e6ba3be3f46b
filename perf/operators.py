"""Performance cases of the operators around the attention of a layer: norms and position rotation of queries and keys,
microscaled 4-bit and 8-bit formats, the 4-bit linear layer, and a linear layer's backward pass from an 8-bit checkpoint.

Five kinds of case:

``rope``        norm of every head's queries and keys and the rotation by the tokens' positions, in one pass.
``rope_back``   its gradient: that of the queries and keys and of the norms' weights and biases.
``checkpoint``  an activation stored in microscaled 8 (or 4) bits and restored.
``linear``      a linear layer with microscaled 4-bit operands: the activations quantised per call, the weight kept as codes.
``linear_back`` the backward pass of that layer: gradient of its input from the 4-bit weight, gradient of its weight and bias
                from the 8-bit checkpoint of its input.

With ``own`` false everything is computed by elementary torch operations in 32 bits (angles in 64).

Microscaled format: blocks of 32 values along a row share a scale 2^E, E the smallest integer (at least -127) with
max|x| <= top * 2^E, kept as the byte E + 127; elements are e2m1 (top 6, two to a byte, the even one low) or e4m3 (top 448),
rounded to nearest even.  Scales lie in tiles of 128 rows x 4 blocks: the byte of row r, block j is
[r / 128, j / 4, r % 32, (r % 128) / 32, j % 4]; places past the matrix are zero.
"""
import math

import torch

own = False

FRAME = 1374  # tokens of one 518 x 518 frame: a camera token, four registers, 37 x 37 patches
SIDE, SPECIAL = 37, 5
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
TOP = {"mxfp4": 6.0, "mxfp8": 448.0}
MANTISSA = {"mxfp4": 1, "mxfp8": 3}  # bits behind the point
LOWEST = {"mxfp4": 0, "mxfp8": -6}   # exponent of the smallest normal value
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5
MOST_VALUES = 2 * 100 * FRAME * 16 * 64          # of the largest listed rotation
MOST_BACK_VALUES = 2 * 32 * FRAME * 16 * 64
MOST_STORED = 32 * FRAME * 4096
MOST_PRODUCTS = 32.0 * FRAME * 4096 * 1024
MOST_BACK_PRODUCTS = 8.0 * FRAME * 1024 * 4096


def rope(name, batch, heads, kv_heads, tokens, dim=64, norm="layer", axes=2, src="bf16", layout="tokens", base=100.0, offset=0,
         kind="rope"):
    """layout "tokens": views of one packed [B, N, heads, D] projection output; "heads": contiguous [B, H, N, D]."""
    return {"name": name, "kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "tokens": tokens, "dim": dim,
            "norm": norm, "axes": axes, "src": src, "layout": layout, "base": base, "offset": offset}


def checkpoint(name, rows, cols, fmt="mxfp8", src="bf16"):
    return {"name": name, "kind": "checkpoint", "rows": rows, "cols": cols, "format": fmt, "src": src}


def linear(name, rows, d_in, d_out, src="bf16", out="bf16", bias=True):
    return {"name": name, "kind": "linear", "rows": rows, "d_in": d_in, "d_out": d_out, "src": src, "out": out, "bias": bias}


def linear_back(name, rows, d_in, d_out, out="bf16"):
    return {"name": name, "kind": "linear_back", "rows": rows, "d_in": d_in, "d_out": d_out, "out": out}


def listed():
    return [
        # one new token of each of four sequences with grouped heads, far into a long cache: latency counts
        rope("rope_token", 4, 16, 4, 1, dim=128, norm="rms", axes=1, base=10000.0, offset=900000),
        # frame attention: 32 frames, packed projection output, 2-D positions
        rope("rope_frame32", 32, 16, 16, FRAME),
        # global attention over a hundred frames
        rope("rope_stress100", 1, 16, 16, 100 * FRAME, layout="heads"),
        # training in 32 bits on odd sizes: grouped heads, root mean square norm, positions along one axis
        rope("rope_back_odd", 3, 10, 5, 3001, norm="rms", axes=1, src="f32", layout="heads", base=10000.0, kind="rope_back"),
        # training on 32 frames
        rope("rope_back_frame32", 32, 16, 16, FRAME, kind="rope_back"),
        # the input of a small 4-bit layer on an odd number of fp32 rows
        checkpoint("store4_odd", 1001, 1184, fmt="mxfp4", src="f32"),
        # the widest activation of a transformer layer (its MLP) on 32 frames, kept for the backward pass
        checkpoint("store8_mlp32", 32 * FRAME, 4096),
        # the output projection of a single token
        linear("linear_token", 1, 1024, 1024),
        # odd sizes, 32-bit input and output
        linear("linear_odd", 777, 1184, 1000, src="f32", out="f32"),
        # the second matrix of the MLP on 32 frames
        linear("linear_mlp32", 32 * FRAME, 4096, 1024),
        # backward pass on odd sizes with a 32-bit input gradient
        linear_back("back_odd", 777, 1184, 1000, out="f32"),
        # backward pass of the first matrix of the MLP on eight frames
        linear_back("back_mlp8", 8 * FRAME, 1024, 4096),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over their logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _tokens(rng, low, high):
    n = _spread(rng, low, high)
    return n // FRAME * FRAME if n > FRAME and rng.random() < 0.4 else n


def draw(rng):
    kind = rng.choice(["rope", "rope", "rope_back", "checkpoint", "linear", "linear", "linear_back"])
    if kind in ("rope", "rope_back"):
        most = MOST_VALUES if kind == "rope" else MOST_BACK_VALUES
        axes, norm = rng.choice([2, 2, 1]), rng.choice(["layer", "layer", "rms", "none"])
        if norm != "none" and rng.random() < 0.2:
            axes = 0
        src = rng.choice(["bf16", "bf16", "f16", "f32"])
        while True:
            heads = rng.choice([1, 2, 5, 8, 12, 16, 16, 24])
            kv_heads = rng.choice([h for h in (1, 2, 4, 5, 8, 12, 16, 24) if heads % h == 0])
            case = rope("", rng.choice([1, 1, 2, 3, 8, 32]), heads, kv_heads, _tokens(rng, 1, 100 * FRAME),
                        dim=rng.choice([64, 64, 64, 32, 128]), norm=norm, axes=axes,
                        src=src, layout=rng.choice(["tokens", "heads"]), base=100.0 if axes == 2 else 10000.0,
                        offset=_spread(rng, 1, 1 << 20) if axes == 1 else 0, kind=kind)
            values = case["batch"] * (heads + kv_heads) * case["tokens"] * case["dim"]
            if values * (2 if src == "f32" else 1) <= most:
                break
    elif kind == "checkpoint":
        while True:
            case = checkpoint("", _spread(rng, 1, 32 * FRAME), 32 * _spread(rng, 1, 256), fmt=rng.choice(["mxfp8", "mxfp8", "mxfp4"]),
                              src=rng.choice(["bf16", "bf16", "f32"]))
            if case["rows"] * case["cols"] * (2 if case["src"] == "f32" else 1) <= MOST_STORED:
                break
    else:
        most = MOST_PRODUCTS if kind == "linear" else MOST_BACK_PRODUCTS
        while True:
            rows, d_in, d_out = _spread(rng, 1, 32 * FRAME), 32 * _spread(rng, 2, 128), 8 * _spread(rng, 4, 512)
            if float(rows) * d_in * d_out <= most:
                break
        if kind == "linear":
            case = linear("", rows, d_in, d_out, src=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]),
                          bias=rng.random() < 0.7)
        else:
            case = linear_back("", rows, d_in, d_out, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------------ preparation
def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _positions(case):
    """int32 [B, N, axes], each sequence with its own offset along one axis; rows and columns of the patches along two (a
    frame's camera and register tokens are at 0)."""
    B, N, axes = case["batch"], case["tokens"], case["axes"]
    if axes == 0:
        return None
    n = torch.arange(N, device="cuda")
    if axes == 1:
        return (n + case["offset"] + 17 * torch.arange(B, device="cuda")[:, None]).to(torch.int32)[..., None].contiguous()
    p = n % FRAME - SPECIAL
    grid = torch.stack([torch.div(p, SIDE, rounding_mode="floor") + 1, p % SIDE + 1], -1)
    return torch.where(p[:, None] < 0, 0, grid).to(torch.int32).expand(B, N, 2).contiguous()


def _heads(g, case, scale=1.0):
    """Queries and keys as views [B, H, N, D] in the case's type and layout."""
    B, H, K, N, D = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim"))
    dtype = FLOAT[case["src"]]
    if case["layout"] == "tokens":  # (q | k | v) of a packed projection
        packed = _normal(g, (B, N, H + 2 * K, D), dtype).mul_(scale)
        return packed[:, :, :H].permute(0, 2, 1, 3), packed[:, :, H:H + K].permute(0, 2, 1, 3)
    return _normal(g, (B, H, N, D), dtype).mul_(scale), _normal(g, (B, K, N, D), dtype).mul_(scale)


def _outputs(case):
    B, H, K, N, D = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim"))
    return [torch.empty((B, h, N, D), dtype=FLOAT[case["src"]], device="cuda") for h in (H, K)]


def _activation(g, rows, cols, dtype):
    """Tokens differ in magnitude, and some channels are much larger than the rest."""
    x = _normal(g, (rows, cols)) * torch.exp(0.5 * _normal(g, (rows, 1)))
    return x.mul_(torch.exp(0.7 * _normal(g, (1, cols)))).to(dtype)


def _tile_scales(e):
    """The bytes of E [rows, blocks] in tiles of 128 rows x 4 blocks."""
    rows, blocks = e.shape
    rt, bt = -(-rows // 128), -(-blocks // 4)
    full = torch.zeros((rt * 128, bt * 4), dtype=torch.uint8, device=e.device)
    full[:rows, :blocks] = (e + 127).to(torch.uint8)
    return full.view(rt, 4, 32, bt, 4).permute(0, 3, 2, 1, 4).contiguous()


def _pack(x, fmt):
    """(codes, scales) of a matrix, laid out as the format says."""
    values, e = _quantised(x.float(), fmt)
    elements = values / _power(e)
    if fmt == "mxfp8":
        codes = elements.view(x.shape).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        table = torch.tensor(E2M1, device=x.device)
        nibble = torch.bucketize(elements.abs(), table).to(torch.uint8) | (elements < 0).to(torch.uint8) * 8
        nibble = nibble.view(x.shape[0], -1, 2)
        codes = nibble[..., 0] | nibble[..., 1] << 4
    return codes.contiguous(), _tile_scales(e[..., 0])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("rope", "rope_back"):
        s["q"], s["k"] = _heads(g, case, 2.0)
        s["positions"] = _positions(case)
        if case["norm"] != "none":
            for x in "qk":
                s[x + "_weight"] = 1.0 + 0.2 * _normal(g, (case["dim"],))
                s[x + "_bias"] = 0.1 * _normal(g, (case["dim"],)) if case["norm"] == "layer" else None
        if kind == "rope_back":
            s["dq_out"], s["dk_out"] = _heads(g, case, 0.01)
        s["out"] = _outputs(case)
    elif kind == "checkpoint":
        s["x"] = _activation(g, case["rows"], case["cols"], FLOAT[case["src"]])
        s["out"] = torch.empty_like(s["x"])
    else:
        rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
        s["w"] = _pack(_normal(g, (d_out, d_in)) / math.sqrt(d_in), "mxfp4")
        if kind == "linear":
            s["x"] = _activation(g, rows, d_in, FLOAT[case["src"]])
            s["bias"] = 0.1 * _normal(g, (d_out,)) if case["bias"] else None
            s["y"] = torch.empty((rows, d_out), dtype=FLOAT[case["out"]], device="cuda")
        else:
            s["x"] = _pack(_activation(g, rows, d_in, torch.bfloat16), "mxfp8")
            s["dy"] = _normal(g, (rows, d_out), torch.bfloat16).mul_(0.01)
            s["dx"] = torch.empty((rows, d_in), dtype=FLOAT[case["out"]], device="cuda")
            s["dw"] = torch.empty((d_out, d_in), device="cuda")
            s["db"] = torch.empty((d_out,), device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ plain forms
def _power(e):
    """2^e in fp32 by its bits; a block of 2^-127 holds nothing in these cases but zeros, for which 2^-126 is as good."""
    return (e.clamp(min=-126).add_(127) << 23).view(torch.float32)


def _quantised(x, fmt):
    """fp32 [rows, cols] -> (the values its microscaled form stands for [rows, blocks, 32], exponents [rows, blocks, 1])."""
    x = x.view(x.shape[0], -1, 32)
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)           # amax = m 2^e, m in [0.5, 1)
    mt, et = math.frexp(TOP[fmt])
    e = torch.where(amax > 0, (e - et + (m > mt)).clamp_(min=-127), -127)
    scale = _power(e)
    q = x / scale
    step = _power(torch.frexp(q)[1].sub_(1).clamp_(min=LOWEST[fmt]).sub_(MANTISSA[fmt]))
    return torch.round(q / step) * step * scale, e


def _unpacked(codes, scales, fmt):
    """The values of codes and tiled scales, fp32 [rows, cols]."""
    if fmt == "mxfp8":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        nibble = torch.stack([codes & 15, codes >> 4], -1).view(codes.shape[0], -1).int()
        v = torch.tensor(E2M1, device=codes.device)[nibble & 7] * (1 - 2 * (nibble >> 3))
    rows, cols = v.shape
    rt, bt = scales.shape[:2]
    e = scales.permute(0, 3, 2, 1, 4).reshape(rt * 128, bt * 4)[:rows, :cols // 32].int() - 127
    return (v.view(rows, -1, 32) * _power(e)[..., None]).view(rows, cols)


def _angles(case, positions):
    """cos, sin [B, 1, N, axes, D / axes / 2] in fp32, the angles in fp64."""
    half = case["dim"] // case["axes"] // 2
    freq = case["base"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    a = positions.double()[:, None, :, :, None] * freq
    return a.cos().float(), a.sin().float()


def _rotate(x, case, positions, back=False):
    if case["axes"] == 0:
        return x
    cos, sin = _angles(case, positions)
    if back:
        sin = -sin
    a, b = x.view(*x.shape[:3], case["axes"], 2, -1).unbind(-2)
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -2).view(x.shape)


def _normed(x, norm):
    """(normalised values, reciprocal of the deviation)"""
    if norm == "none":
        return x, None
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_rope(s, x, weight, bias):
    z, _ = _normed(x.float().contiguous(), s["case"]["norm"])
    if weight is not None:
        z = z * weight
    if bias is not None:
        z = z + bias
    return _rotate(z, s["case"], s["positions"]).to(x.dtype)


def _plain_rope_back(s, x, grad, weight, bias):
    """(dx, d weight, d bias)"""
    norm = s["case"]["norm"]
    g = _rotate(grad.float().contiguous(), s["case"], s["positions"], back=True)
    if norm == "none":
        return g.to(x.dtype), None, None
    xh, r = _normed(x.float().contiguous(), norm)
    dw = (g * xh).sum((0, 1, 2))
    db = g.sum((0, 1, 2)) if bias is not None else None
    gh = g * weight
    d = gh - xh * (gh * xh).mean(-1, keepdim=True)
    if norm == "layer":
        d = d - gh.mean(-1, keepdim=True)
    return (d * r).to(x.dtype), dw, db


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    affine = [(s.get(x + "_weight"), s.get(x + "_bias")) for x in "qk"]
    if kind == "rope":
        return {"q": _plain_rope(s, s["q"], *affine[0]), "k": _plain_rope(s, s["k"], *affine[1])}
    if kind == "rope_back":
        q = _plain_rope_back(s, s["q"], s["dq_out"], *affine[0])
        k = _plain_rope_back(s, s["k"], s["dk_out"], *affine[1])
        out = {"dq": q[0], "dk": k[0], "dq_weight": q[1], "dq_bias": q[2], "dk_weight": k[1], "dk_bias": k[2]}
        return {name: t for name, t in out.items() if t is not None}
    if kind == "checkpoint":
        return {"x": _quantised(s["x"].float(), case["format"])[0].view(s["x"].shape).to(s["x"].dtype)}
    w = _unpacked(*s["w"], "mxfp4")
    if kind == "linear":
        y = _quantised(s["x"].float(), "mxfp4")[0].view(s["x"].shape) @ w.t()
        return {"y": (y if s["bias"] is None else y + s["bias"]).to(s["y"].dtype)}
    dy = s["dy"].float()
    return {"dx": (dy @ w).to(s["dx"].dtype), "dw": dy.t() @ _unpacked(*s["x"], "mxfp8"), "db": dy.sum(0)}


# ------------------------------------------------------------------------------------------------------ the framework's calls
def _own_rope(s):
    from paper_2605_11354_b200 import binding as lt
    case = s["case"]
    how = {"norm": case["norm"], "eps": EPS, "base": case["base"], "positions": s["positions"]}
    q_weight, q_bias, k_weight, k_bias = (s.get(n) for n in ("q_weight", "q_bias", "k_weight", "k_bias"))
    q, k = s["out"]
    if case["kind"] == "rope":
        lt.lite3r_qk_norm_rope(s["q"], s["k"], q, k, q_weight=q_weight, q_bias=q_bias, k_weight=k_weight, k_bias=k_bias, **how)
        return {"q": q, "k": k}
    if "workspace" not in s:
        s["workspace"] = torch.empty(lt.lite3r_qk_norm_rope_workspace(case["dim"]), dtype=torch.uint8, device="cuda")
        s["grads"] = {"d" + n: torch.empty_like(s[n]) for n in ("q_weight", "q_bias", "k_weight", "k_bias") if s.get(n) is not None}
    lt.lite3r_qk_norm_rope_backward(s["q"], s["k"], s["dq_out"], s["dk_out"], q, k, q_weight=q_weight, k_weight=k_weight,
                                    workspace=s["workspace"], **s["grads"], **how)
    return {"dq": q, "dk": k, **s["grads"]}


def _own_matrix(s):
    from paper_2605_11354_b200 import binding as lt
    case = s["case"]
    if case["kind"] == "checkpoint":
        kept = lt.lite3r_quantize_mx(s["x"], case["format"])
        return {"x": lt.lite3r_dequantize_mx(kept, s["out"])}
    rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
    w = lt.MxTensor(*s["w"], d_out, d_in, "mxfp4")
    if case["kind"] == "linear":
        lt.lite3r_linear_mxfp4(lt.lite3r_quantize_mx(s["x"], "mxfp4"), w, s["bias"], s["y"])
        return {"y": s["y"]}
    if "workspace" not in s:
        s["workspace"] = torch.empty(lt.lite3r_linear_mx_workspace(rows, d_in, d_out), dtype=torch.uint8, device="cuda")
    lt.lite3r_linear_mx_dgrad(s["dy"], w, s["dx"])
    lt.lite3r_linear_mx_wgrad(s["dy"], lt.MxTensor(*s["x"], rows, d_in, "mxfp8"), s["dw"], s["db"], s["workspace"])
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def run(s):
    if not own:
        return _plain(s)
    return _own_rope(s) if s["case"]["kind"] in ("rope", "rope_back") else _own_matrix(s)


# ------------------------------------------------------------------------------------------------------ what it takes
def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_back"):
        B, H, K, N, D = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim"))
        values, tensors = B * (H + K) * N * D, 2 if kind == "rope" else 3
        affine = 0 if case["norm"] == "none" else 2 * D * 4 * (2 if case["norm"] == "layer" else 1) * (1 if kind == "rope" else 2)
        return {"bytes": values * tensors * BYTES[case["src"]] + 4 * B * N * case["axes"] + affine,
                "flops": values * (14.0 if kind == "rope" else 26.0)}
    if kind == "checkpoint":
        values = case["rows"] * case["cols"]
        stored = values * (8 if case["format"] == "mxfp8" else 4) // 8 + values // 32
        return {"bytes": 2 * values * BYTES[case["src"]] + 2 * stored, "flops": 4.0 * values}
    r, i, o = case["rows"], case["d_in"], case["d_out"]
    weight = i * o // 2 + i * o // 32
    if kind == "linear":
        return {"bytes": r * i * BYTES[case["src"]] + weight + 4 * o * case["bias"] + r * o * BYTES[case["out"]],
                "flops": 2.0 * r * i * o}
    return {"bytes": 2 * r * o + weight + r * i + r * i // 32 + r * i * BYTES[case["out"]] + 4 * i * o + 4 * o, "flops": 4.0 * r * i * o}


# ------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_values(x, fmt):
    """The microscaled form of a matrix by search: the scale among neighbouring powers of two, an element among all values
    of its type, the one whose code is even where two are as near."""
    if fmt == "mxfp4":
        grid = torch.tensor(E2M1, device="cuda", dtype=torch.float64)
    else:
        grid = torch.arange(127, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    for r0 in range(0, x.shape[0], 8192):
        b = x[r0:r0 + 8192].double().view(-1, 32)
        amax = b.abs().amax(1)
        near = torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0) / TOP[fmt]))[:, None] + torch.arange(-1, 3, device="cuda")
        fits = amax[:, None] <= TOP[fmt] * torch.exp2(near)
        e = torch.where(fits, near, math.inf).amin(1, keepdim=True).clamp_(min=-127.0)
        q = b / torch.exp2(e)
        low = (torch.searchsorted(grid, q.abs().contiguous(), right=True) - 1).clamp_(max=grid.numel() - 2)
        up, down = grid[low + 1] - q.abs(), q.abs() - grid[low]
        code = low + ((up < down) | ((up == down) & (low % 2 == 1))).long()
        out[r0:r0 + 8192] = (torch.copysign(grid[code], q) * torch.exp2(e)).view(-1, x.shape[1])
    return out


def _exact_rope(x, weight, bias, case, positions):
    """By complex numbers: the pair (i, i + half) of an axis turns by e^(i angle)."""
    if case["norm"] == "layer":
        x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
    elif case["norm"] == "rms":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    if weight is not None:
        x = x * weight
    if bias is not None:
        x = x + bias
    if case["axes"] == 0:
        return x
    half = case["dim"] // (2 * case["axes"])
    parts = []
    for axis in range(case["axes"]):
        c = torch.complex(x[..., 2 * half * axis:][..., :half], x[..., 2 * half * axis + half:][..., :half])
        angle = positions[:, None, :, axis, None].double() * torch.tensor([case["base"] ** (-i / half) for i in range(half)],
                                                                         dtype=torch.float64, device="cuda")
        c = c * torch.polar(torch.ones_like(angle), angle)
        parts += [c.real, c.imag]
    return torch.cat(parts, -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "checkpoint":
        return {"x": _exact_values(s["x"], case["format"])}
    if kind == "linear":
        y = _exact_values(s["x"], "mxfp4") @ _unpacked(*s["w"], "mxfp4").double().t()
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    if kind == "linear_back":
        dy = s["dy"].double()
        return {"dx": dy @ _unpacked(*s["w"], "mxfp4").double(), "dw": dy.t() @ _unpacked(*s["x"], "mxfp8").double(), "db": dy.sum(0)}
    out = {}
    for x in "qk":
        weight, bias = (s[x + n].double() if s.get(x + n) is not None else None for n in ("_weight", "_bias"))
        if kind == "rope":  # one head at a time
            out[x] = torch.cat([_exact_rope(h.double(), weight, bias, case, s["positions"]) for h in s[x].split(1, 1)], 1)
            continue
        leaves = [t.requires_grad_() for t in (weight, bias) if t is not None]
        grads, sums = [], [torch.zeros_like(t) for t in leaves]
        for h, dh in zip(s[x].split(1, 1), s["d" + x + "_out"].split(1, 1)):
            h = h.double().requires_grad_()
            d = torch.autograd.grad(_exact_rope(h, weight, bias, case, s["positions"]), [h, *leaves], dh.double())
            grads.append(d[0])
            sums = [a + b for a, b in zip(sums, d[1:])]
        out["d" + x] = torch.cat(grads, 1)
        for name, total in zip(("_weight", "_bias"), sums):
            out["d" + x + name] = total
    return out
