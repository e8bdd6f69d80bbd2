"""The operators on both sides of the attention call whose speed counts: the products that make Q, K and V from the hidden
states and take the attention's output back (weights and rows in microscaled 4-bit floating point), and what stands between
the first product and the attention: each head's norm of Q and K, the rotation by the token's place in the clip, and the FP8
operands, with the gradient of norm and rotation.

A case is described by plain values.  `op` says which operator a pass calls:
  rotate       norm and rotation, out in raster order            x -> y
  operand      norm and rotation into packed E4M3, one scale per 3D tile, and the values that those stand for
  rotate_grad  the gradient of `rotate`                          x, dy -> dx, dweight
  linear       y = x W^T + bias, x quantised in the call, W kept in 4 bits
  values       rows to 4 bits and back (what a product sees of them)
Fields of the first three:
  B, heads, T, H, W          batch, heads and token grid (128 channels a head)
  fused                      x is Q's or K's share of a projection's rows [B, tokens, 3 heads 128]; otherwise it is in raster
                             order [B, heads, tokens, 128]
  f32                        fp32 tensors instead of bf16
  halves                     channel i turns with i + 64 instead of 2i with 2i + 1
  per_head                   a norm weight for each head instead of one for all
  start                      first frame's place (a later chunk of a long clip)
  Tt, Th, Tw, key            (operand) the tile, and K's operand layout instead of Q's
Fields of the others:
  rows, K, N                 rows, their length and, for linear, the row length of the result
  from_heads, to_heads       the rows are a tensor in raster order, K = heads * 128 (the attention's output); the result is
                             written as one (the attention's input)
  bias
"""
from __future__ import annotations

import math

import torch

own = False

HEAD_DIM, PAIRS, SPLIT = 128, 64, (22, 21, 21)          # pairs that turn with the frame, the row and the column
EPS, BASE = 1e-6, 10000.0
# The largest listed cases: one product of 4 Tflop, one tensor of 387 M elements.  Drawn ones stay below.
MAX_FLOPS, MAX_ELEMENTS = 3.9e12, 380e6


def _attention_side(name, op, heads, grid, **more):
    c = dict(name=name, op=op, B=1, heads=heads, T=grid[0], H=grid[1], W=grid[2], fused=True, f32=False, halves=False,
             per_head=False, start=0)
    if op == "operand":
        c.update(Tt=1, Th=8, Tw=16, key=False)
    c.update(more)
    return c


def _product_side(name, op, rows, K, N, **more):
    c = dict(name=name, op=op, rows=rows, K=K, N=N, from_heads=False, to_heads=False, bias=True)
    c.update(more)
    return c


def listed():
    small, large = (21, 30, 52), (21, 45, 80)           # 480p and 720p clips
    return [
        # one token of a clip that is made token by token: two microseconds of work, latency counts
        _attention_side("rotate-one-token", "rotate", 12, (1, 1, 1), start=977),
        # a small clip with a ragged grid in fp32, weights of each head, the other pairing
        _attention_side("rotate-ragged-f32", "rotate", 5, (5, 23, 37), B=2, fused=False, f32=True, halves=True, per_head=True),
        # Q of the large model, as its projection leaves it, into raster order
        _attention_side("rotate-720p", "rotate", 40, large),
        # K of the small model straight into FP8 operands, and a coarse tile (more than one workgroup's share)
        _attention_side("operand-480p", "operand", 12, small, key=True),
        _attention_side("operand-480p-tile-488", "operand", 12, small, Tt=8, Th=8, Tw=8, halves=True, fused=False),
        # Q of the large model
        _attention_side("operand-720p", "operand", 40, large),
        # training: the gradient for a preview clip in fp32, and for Q of the small model
        _attention_side("grad-ragged-f32", "rotate_grad", 5, (5, 23, 37), B=2, f32=True, per_head=True, halves=True),
        _attention_side("grad-480p", "rotate_grad", 12, small),
        # the step embedding's six modulation vectors: one row, the weights are all there is to read
        _product_side("linear-one-row", "linear", 1, 5120, 30720),
        # Q, K, V of a preview clip's ragged rows, written in the attention's order
        _product_side("linear-qkv-preview", "linear", 851, 1536, 4608, to_heads=True),
        # the output projection of the large model, read in the attention's order: the largest product
        _product_side("linear-out-720p", "linear", 75600, 5120, 5120, from_heads=True),
        # what 4 bits leave of the small model's rows
        _product_side("values-480p", "values", 32760, 1536, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another call of the same kinds over the ranges of the listed ones."""
    op = rng.choice(["rotate", "operand", "rotate_grad", "linear", "linear", "values"])
    if op in ("linear", "values"):
        while True:
            heads_in, heads_out = rng.random() < 0.3, rng.random() < 0.3
            c = _product_side("", op, _log_int(rng, 1, 75600), 0, 0, from_heads=heads_in, to_heads=heads_out and op == "linear",
                              bias=rng.random() < 0.5)
            c["K"] = 128 * rng.randint(1, 40) if heads_in else _log_int(rng, 64, 20480)
            c["N"] = 0 if op == "values" else 128 * rng.randint(1, 120) if c["to_heads"] else _log_int(rng, 64, 30720)
            del c["name"]
            if 2.0 * c["rows"] * c["K"] * max(1, c["N"]) <= MAX_FLOPS and c["rows"] * max(c["K"], c["N"]) <= MAX_ELEMENTS:
                return c
    while True:
        tokens = _log_int(rng, 1, 75600)
        T = max(1, min(21, tokens, _log_int(rng, 1, 21)))
        H = max(1, int(round(math.sqrt(tokens / T) * rng.uniform(0.6, 1.1))))
        W = max(1, int(round(tokens / (T * H))))
        c = _attention_side("", op, _log_int(rng, 1, 40), (T, H, W), B=rng.choice([1, 1, 1, 2]), fused=rng.random() < 0.7,
                            f32=op != "operand" and rng.random() < 0.25, halves=rng.random() < 0.4,
                            per_head=rng.random() < 0.3, start=rng.choice([0, 0, rng.randint(1, 5000)]))
        if op == "operand":
            c.update(zip(("Tt", "Th", "Tw"), rng.choice([(1, 8, 16), (1, 8, 16), (2, 4, 4), (3, 4, 4), (1, 7, 15), (2, 8, 16),
                                                         (6, 8, 8), (4, 16, 16)])), key=rng.random() < 0.5)
        del c["name"]
        if _elements(c) <= MAX_ELEMENTS:
            return c


def _elements(c):
    return c["B"] * c["heads"] * c["T"] * c["H"] * c["W"] * HEAD_DIM


def _tiles(c):
    return [-(-c[g] // c[t]) for g, t in (("T", "Tt"), ("H", "Th"), ("W", "Tw"))]


def work(case):
    """Inputs read once, outputs written once, at the width that they have in memory: 2 or 4 bytes, in 4 bits 17/32 of a byte
    (a code, and one byte of scale for 32 of them).  Norm and rotation are some ten operations an element, a product two for each of its terms."""
    c = case
    if c["op"] == "linear":
        rows, K, N = c["rows"], c["K"], c["N"]
        return {"bytes": 2 * rows * K + N * K * 17 // 32 + 2 * rows * N + (4 * N if c["bias"] else 0), "flops": 2 * rows * K * N}
    if c["op"] == "values":
        return {"bytes": 4 * c["rows"] * c["K"], "flops": 4 * c["rows"] * c["K"]}
    n, width = _elements(c), 4 if c["f32"] else 2
    passes = 3 if c["op"] == "rotate_grad" else 2
    small = 4 * HEAD_DIM * (c["heads"] if c["per_head"] else 1) * (2 if c["op"] == "rotate_grad" else 1)
    if c["op"] == "operand":
        small += 4 * c["B"] * c["heads"] * math.prod(_tiles(c))
    return {"bytes": passes * width * n + small, "flops": 10 * n}


# ---- inputs ---------------------------------------------------------------------------------------
def _angles(c, dtype=torch.float64, device="cpu"):
    """The angle of every place of every axis: [T,22], [H,21], [W,21]."""
    out = []
    for size, pairs, first in zip((c["T"], c["H"], c["W"]), SPLIT, (c["start"], 0, 0)):
        place = torch.arange(first, first + size, dtype=dtype, device=device)
        out.append(place[:, None] * BASE ** (-torch.arange(pairs, dtype=dtype, device=device) / pairs))
    return out


def _activations(gen, rows, cols, dev):
    """Rows of unit variance in which a few channels are 8 times the others, as hidden states have them."""
    x = torch.randn(rows, cols, generator=gen, device=dev)
    pick = torch.rand(cols, generator=gen, device=dev).topk(max(1, cols // 48)).indices
    x[:, pick] *= 8.0
    return x.to(torch.bfloat16)


def prepare(case, seed):
    """Activations, norm weights near one, weights of the size that training starts from, the rotation's tables, and the
    buffers that a program keeps: with weights that are held in 4 bits, as it holds them."""
    c = case
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if c["op"] in ("linear", "values"):
        rows, K, N = c["rows"], c["K"], c["N"]
        s = {"case": c, "x": _activations(gen, rows, K, dev)}
        if c["from_heads"]:                              # [1, heads, rows, 128]
            s["x"] = s["x"].view(1, rows, K // HEAD_DIM, HEAD_DIM).transpose(1, 2).contiguous()
        if c["op"] == "linear":
            w = (torch.randn(N, K, generator=gen, device=dev) / math.sqrt(K)).to(torch.bfloat16)
            s["bias"] = torch.randn(N, generator=gen, device=dev) if c["bias"] else None
            s["out"] = torch.empty((1, N // HEAD_DIM, rows, HEAD_DIM) if c["to_heads"] else (rows, N), dtype=torch.bfloat16, device=dev)
            if own:
                from paper_2506_04648_amd import fps
                s["weight"] = fps.mx4_quantize(w)
                s["workspace"] = torch.empty(fps.mx4_linear_bytes(rows, K), dtype=torch.uint8, device=dev)
            else:
                s["weight"] = _to_four_bits(w.float())
        elif own:
            from paper_2506_04648_amd import fps
            s["packed"] = torch.empty(fps.mx4_bytes(rows, K), dtype=torch.uint8, device=dev)
            s["out"] = torch.empty_like(s["x"])
        return s
    B, heads, N = c["B"], c["heads"], c["T"] * c["H"] * c["W"]
    dt = torch.float32 if c["f32"] else torch.bfloat16

    def tensor(width):
        if c["fused"]:                                   # the projection's rows; Q is their first third
            t = torch.randn(B, N, width, heads, HEAD_DIM, generator=gen, device=dev, dtype=dt)[:, :, 0].transpose(1, 2)
        else:
            t = torch.randn(B, heads, N, HEAD_DIM, generator=gen, device=dev, dtype=dt)
        return t

    s = {"case": c, "x": tensor(3)}
    s["x"] *= torch.exp(0.5 * torch.randn(heads, 1, HEAD_DIM, generator=gen, device=dev)).to(dt)
    s["weight"] = 1.0 + 0.2 * torch.randn((heads, HEAD_DIM) if c["per_head"] else (HEAD_DIM,), generator=gen, device=dev)
    s["table"] = torch.cat([torch.stack((a.cos(), a.sin()), -1).reshape(-1, 2) for a in _angles(c)]).float().to(dev)
    raster = (B, heads, c["T"], c["H"], c["W"], HEAD_DIM)
    if c["op"] == "rotate_grad":
        s["dy"] = torch.randn(raster, generator=gen, device=dev, dtype=dt)
        s["dx"] = torch.empty(B, N, heads, HEAD_DIM, device=dev, dtype=dt).transpose(1, 2) if c["fused"] else torch.empty_like(s["x"])
        s["dweight"] = torch.empty_like(s["weight"])
    else:
        s["out"] = torch.empty(raster, device=dev, dtype=dt)
    if own:
        from paper_2506_04648_amd import fps
        tile = (c["Tt"], c["Th"], c["Tw"]) if c["op"] == "operand" else (1, 1, 1)
        s["shape"] = fps.make_shape(heads, (c["T"], c["H"], c["W"]), tile, B=B)
        s["norm"] = fps.make_norm(s["weight"], EPS)
        s["rotation"] = fps.make_rotation(s["table"], SPLIT, halves=c["halves"])
        if c["op"] == "operand":
            s["packed"] = torch.empty(fps.packed_bytes(s["shape"], fps.PREC_FP8), dtype=torch.uint8, device=dev)
            s["scales"] = torch.empty(B, heads, fps.num_groups(s["shape"]), device=dev)
        elif c["op"] == "rotate_grad":
            s["workspace"] = torch.empty(fps.norm_rotate_bwd_bytes(s["shape"], s["norm"]), dtype=torch.uint8, device=dev)
    return s


# ---- one pass -------------------------------------------------------------------------------------
def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2506_04648_amd import fps
        if c["op"] == "rotate":
            return fps.norm_rotate(s["shape"], s["x"], s["norm"], s["rotation"], out=s["out"])
        if c["op"] == "operand":
            role = fps.ROLE_K if c["key"] else fps.ROLE_Q
            fps.norm_rotate_operand(s["shape"], s["x"], role, fps.PREC_FP8, s["norm"], s["rotation"], out=s["packed"], scales=s["scales"])
            return {"values": fps.dequantize(s["shape"], s["packed"], s["scales"], role, out=s["out"]), "scales": s["scales"]}
        if c["op"] == "rotate_grad":
            dx, dweight = fps.norm_rotate_bwd(s["shape"], s["x"], s["dy"], s["norm"], s["rotation"], dx=s["dx"], dweight=s["dweight"],
                                              workspace=s["workspace"])
            return {"dx": dx, "dweight": dweight}
        if c["op"] == "linear":
            return fps.mx4_linear(s["x"], s["weight"], c["N"], bias=s["bias"], out=s["out"], workspace=s["workspace"])
        return fps.mx4_dequantize(fps.mx4_quantize(s["x"], out=s["packed"]), c["rows"], c["K"], out=s["out"])
    if c["op"] in ("linear", "values"):
        values = _to_four_bits(_matrix(s["x"], c).float())
        if c["op"] == "values":
            return _from_matrix(values, c["from_heads"]).to(torch.bfloat16)
        y = values @ s["weight"].t()
        if s["bias"] is not None:
            y = y + s["bias"]
        return _from_matrix(y, c["to_heads"]).to(torch.bfloat16)
    x, weight = s["x"].float(), _weight_of_heads(s["weight"], c)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    turn = _turn_of_tokens(s["table"], c)                # [tokens, 64, 2]
    if c["op"] == "rotate_grad":
        back = _turned(s["dy"].float().reshape(x.shape), turn[..., 0], -turn[..., 1], c["halves"])
        dweight = (back * x * r).sum((0, 2) if c["per_head"] else (0, 1, 2))
        back = back * weight
        dx = r * (back - x * r.square() * (back * x).mean(-1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dweight": dweight}
    y = _turned(x * r * weight, turn[..., 0], turn[..., 1], c["halves"]).reshape(s["out"].shape)
    if c["op"] == "rotate":
        return y.to(s["out"].dtype)
    # each tile's largest magnitude to 448; a tile that the grid's edge cuts counts what it has
    tiles = _tiles(c)
    pad = [0, 0]
    for g, t in (("W", "Tw"), ("H", "Th"), ("T", "Tt")):
        pad += [0, -c[g] % c[t]]
    top = torch.nn.functional.pad(y.abs().amax(-1), pad[2:])
    top = top.reshape(c["B"], c["heads"], tiles[0], c["Tt"], tiles[1], c["Th"], tiles[2], c["Tw"]).amax((3, 5, 7))
    scales = torch.where(top == 0, torch.ones_like(top), top / 448.0)
    each = scales.repeat_interleave(c["Tt"], 2).repeat_interleave(c["Th"], 3).repeat_interleave(c["Tw"], 4)
    each = each[:, :, :c["T"], :c["H"], :c["W"], None]
    values = (y / each).to(torch.float8_e4m3fn).float() * each
    return {"values": values.to(torch.bfloat16), "scales": scales.reshape(c["B"], c["heads"], -1)}


def _matrix(x, c):
    """Rows of a tensor in raster order: channel h * 128 + i of row r is channel i of row r of head h."""
    return x[0].transpose(0, 1).reshape(c["rows"], c["K"]) if c["from_heads"] else x


def _from_matrix(y, to_heads):
    return y.reshape(1, y.shape[0], -1, HEAD_DIM).transpose(1, 2).contiguous() if to_heads else y


def _to_four_bits(x):
    """The values that blocks of 32 have in microscaled E2M1: a power of two for each block, two above which its largest
    magnitude lies, and 1 sign, 2 exponent and 1 mantissa bits an element, rounded to even, at most 6."""
    rows, K = x.shape
    blocks = torch.nn.functional.pad(x, (0, -K % 32)).reshape(rows, -1, 32)
    top = blocks.abs().amax(-1, keepdim=True)
    power = (torch.frexp(top).exponent - 3).clamp(-127, 127)      # floor(log2) - 2
    power = torch.where(top == 0, torch.zeros_like(power), power)
    v = torch.ldexp(blocks, -power)
    size = v.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    v = ((v / step).round() * step).clamp(-6, 6)
    return torch.ldexp(v, power).reshape(rows, -1)[:, :K]


def _weight_of_heads(weight, c):
    return weight[None, :, None, :] if c["per_head"] else weight


def _turn_of_tokens(table, c):
    """Cosine and sine of every token's 64 pairs from the tables of the axes: [tokens, 64, 2]."""
    grid, first, parts = (c["T"], c["H"], c["W"]), 0, []
    for axis, (size, pairs) in enumerate(zip(grid, SPLIT)):
        part = table[first:first + size * pairs].reshape([size if a == axis else 1 for a in range(3)] + [pairs, 2])
        parts.append(part.expand(*grid, pairs, 2))
        first += size * pairs
    return torch.cat(parts, 3).reshape(-1, PAIRS, 2)


def _turned(x, cos, sin, halves):
    if halves:
        a, b = x[..., :PAIRS], x[..., PAIRS:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _nearest_e2m1(v):
    """Index of the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, halfway cases to the even index."""
    at = torch.zeros_like(v)
    for i, middle in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        at += (v > middle) if i % 2 == 0 else (v >= middle)
    return at.long()


def _exact_four_bits(x):
    x = x.double()
    rows, K = x.shape
    out = torch.empty_like(x)
    levels = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    part = max(1, (1 << 26) // K)
    for r in range(0, rows, part):
        b = x[r:r + part]
        n = b.shape[0]
        b = torch.cat((b, b.new_zeros(n, -K % 32)), 1).view(n, -1, 32)
        top = b.abs().max(2, keepdim=True).values
        unit = torch.where(top > 0, 2.0 ** (top.clamp_min(1e-300).log2().floor() - 2).clamp(-127, 127), torch.ones_like(top))
        out[r:r + part] = (levels[_nearest_e2m1(b.abs() / unit)] * b.sign() * unit).view(n, -1)[:, :K]
    return out


def _exact_rotated(x, c, turn_back=False):
    """x [B, heads, tokens, 128] in 64 bits, each pair as a complex number times the token's."""
    grid = torch.meshgrid(*[torch.arange(n, device=x.device) for n in (c["T"], c["H"], c["W"])], indexing="ij")
    at = [g.reshape(-1) for g in grid]
    angle = torch.cat([a[i] for a, i in zip(_angles(c, device=x.device), at)], 1)          # [tokens, 64]
    turn = torch.polar(torch.ones_like(angle), -angle if turn_back else angle)
    if c["halves"]:
        z = torch.complex(x[..., :PAIRS].contiguous(), x[..., PAIRS:].contiguous()) * turn
        return torch.cat((z.real, z.imag), -1)
    z = torch.view_as_complex(x.reshape(x.shape[:-1] + (PAIRS, 2)).contiguous()) * turn
    return torch.view_as_real(z).reshape(x.shape)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] in ("linear", "values"):
        x = s["x"][0].permute(1, 0, 2).reshape(c["rows"], c["K"]) if c["from_heads"] else s["x"]
        y = _exact_four_bits(x)
        if c["op"] == "linear":
            y = torch.mm(y, s["weight"].double().t())    # the weights are the values that 4 bits hold
            if c["bias"]:
                y += s["bias"].double()
        heads = c["to_heads"] or (c["op"] == "values" and c["from_heads"])
        return y.reshape(1, c["rows"], -1, HEAD_DIM).permute(0, 2, 1, 3).contiguous() if heads else y
    w = s["weight"].double()
    w = w.reshape(1, c["heads"], 1, HEAD_DIM) if c["per_head"] else w
    if c["op"] == "rotate_grad":
        x = s["x"].double()
        size = (x.pow(2).sum(-1, keepdim=True) / HEAD_DIM + EPS).sqrt()
        g = _exact_rotated(s["dy"].double().reshape(x.shape), c, turn_back=True)
        unit = x / size
        dweight = (g * unit).sum(2).sum(0)
        gw = g * w
        dx = (gw - unit * (gw * unit).sum(-1, keepdim=True) / HEAD_DIM) / size
        return {"dx": dx, "dweight": dweight if c["per_head"] else dweight.sum(0)}
    y = torch.empty(s["x"].shape, dtype=torch.float64, device=s["x"].device)
    for h in range(c["heads"]):
        x = s["x"][:, h:h + 1].double()
        unit = x / (x.pow(2).sum(-1, keepdim=True) / HEAD_DIM + EPS).sqrt()
        y[:, h:h + 1] = _exact_rotated(unit * (w[:, h:h + 1] if c["per_head"] else w), c)
    y = y.reshape(s["out"].shape)
    if c["op"] == "rotate":
        return y
    nT, nH, nW = _tiles(c)
    scales = torch.ones(c["B"], c["heads"], nT, nH, nW, dtype=torch.float64, device=y.device)
    for t in range(nT):
        for h in range(nH):
            for v in range(nW):
                box = (slice(None), slice(None), slice(t * c["Tt"], (t + 1) * c["Tt"]), slice(h * c["Th"], (h + 1) * c["Th"]),
                       slice(v * c["Tw"], (v + 1) * c["Tw"]))
                top = y[box].abs().amax((2, 3, 4, 5))
                scales[:, :, t, h, v] = torch.where(top > 0, top / 448, torch.ones_like(top))
                unit = scales[:, :, t, h, v, None, None, None, None]
                q = y[box] / unit
                step = 2.0 ** (q.abs().clamp_min(2.0 ** -6).log2().floor() - 3)
                y[box] = (q / step).round() * step * unit
    return {"values": y, "scales": scales.reshape(c["B"], c["heads"], -1)}
