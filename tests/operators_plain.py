"""The operators around the attention in 64 bits, from their definitions, with torch's elementary operations on whatever device
the inputs are, and bounds on what fp32 arithmetic may add.  (Test code; it calls nothing of the library.)"""
import math

import torch

F32 = 2.0 ** -24                       # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- norm and rotation --------------------------------------------------------------------------
def turn_of_tokens(table, grid, split):
    """(cos, sin) of every token's 64 pairs [.., tokens, 64] from tables [.., entries, 2]; pairs that stay: (1, 0)."""
    T, H, W = grid
    table = table.double()
    lead = table.shape[:-2]
    at, parts = 0, []
    for axis, (n, c) in enumerate(zip(grid, split)):
        part = table[..., at:at + n * c, :].reshape(lead + tuple(n if a == axis else 1 for a in range(3)) + (c, 2))
        parts.append(part.expand(lead + (T, H, W, c, 2)))
        at += n * c
    rest = torch.zeros(lead + (T, H, W, 64 - sum(split), 2), dtype=torch.float64, device=table.device)
    rest[..., 0] = 1.0
    turn = torch.cat(parts + [rest], -2).reshape(lead + (T * H * W, 64, 2))
    return turn[..., 0], turn[..., 1]


def pairs(x, halves):
    return (x[..., :64], x[..., 64:]) if halves else (x[..., 0::2], x[..., 1::2])


def unpaired(a, b, halves):
    return torch.cat((a, b), -1) if halves else torch.stack((a, b), -1).flatten(-2)


def turned(x, cos, sin, halves):
    a, b = pairs(x, halves)
    return unpaired(a * cos - b * sin, a * sin + b * cos, halves)


def of_pair(x, halves):
    """|a| + |b| of the pair that a channel belongs to, for both of its channels."""
    a, b = pairs(x.abs(), halves)
    return unpaired(a + b, a + b, halves)


class Turning:
    """x [B, heads, tokens, 128]; weight None, [128] or [heads, 128]; turn None or (cos, sin) [tokens, 64] or [B, tokens, 64]."""

    def __init__(self, weight, eps, turn, halves, norm=True):
        self.w = None if weight is None else weight.double().reshape(1, -1, 1, 128)
        self.eps, self.halves, self.norm = eps, halves, norm
        self.turn = turn if turn is None or turn[0].dim() == 2 else tuple(t[:, None] for t in turn)

    def r(self, x):
        return (x.square().mean(-1, keepdim=True) + self.eps).rsqrt() if self.norm else torch.ones_like(x[..., :1])

    def forward(self, x):
        """y and a bound on fp32's error of it.  With n = x r w: the squares' sum over a row of 128 is at most 16 + 3 roundings deep
        (half of that in r), eps, the reciprocal root (1 ulp = 2), r w x two products: 15 half steps of n; the rotation adds
        two roundings of each product and sum: 18 (|a| + |b|).  Taken as 24."""
        x = x.double()
        n = x * self.r(x) * (1.0 if self.w is None else self.w)
        y = n if self.turn is None else turned(n, *self.turn, self.halves)
        return y, 24 * F32 * of_pair(n, self.halves)

    def backward(self, x, dy):
        """dx, the terms of dweight [B, heads, tokens, 128], and bounds: g = R^T dy to 3 (|a| + |b|); a term, g x r, to 15 more; in
        dx = r (g w - x r^2 m) the mean m of 128 products to 16 + 3 + 5 of the magnitudes' mean, r^2 to 24, r to 12: 48 of all
        magnitudes.  Taken as 24 and 64."""
        x, dy = x.double(), dy.double()
        cos, sin = self.turn if self.turn is not None else (None, None)
        g = dy if cos is None else turned(dy, cos, -sin, self.halves)
        size = of_pair(dy, self.halves)
        r = self.r(x)
        w = 1.0 if self.w is None else self.w
        terms, terms_size = g * x * r, size * (x * r).abs()
        if self.norm:
            dx = r * (g * w - x * r.square() * (g * w * x).mean(-1, keepdim=True))
            dx_size = r * (size * abs(w) + x.abs() * r.square() * (size * abs(w) * x.abs()).mean(-1, keepdim=True))
        else:
            dx, dx_size = g * w, size * abs(w)
        return dx, 64 * F32 * dx_size, terms, terms_size


def within(got, want, bound, dtype):
    """got is want to `bound`, rounded once to dtype: the largest excess over what is allowed, in units of it (<= 1)."""
    allowed = bound + half_step(dtype) * (want.abs() + bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    return float(((got.double() - want).abs() / allowed).max())


# ---- E4M3 ---------------------------------------------------------------------------------------
def e4m3_half_step(q):
    """Half the distance of the codes around q (|q| <= 448)."""
    return 2.0 ** (q.abs().clamp_min(2.0 ** -6).log2().floor() - 4)


def tiles_of(grid, tile):
    return [-(-g // t) for g, t in zip(grid, tile)]


def group_of_tokens(grid, tile, qtile=None):
    """Scale group of every token [T*H*W] and the number of groups: tiles in raster order, sub-tiles within them."""
    q = qtile or tile
    n = tiles_of(grid, tile)
    ns = [t // s for t, s in zip(tile, q)]
    t, h, w = torch.meshgrid(*[torch.arange(g) for g in grid], indexing="ij")
    at = [t, h, w]
    u = s = 0
    for a in range(3):
        u = u * n[a] + at[a] // tile[a]
        s = s * ns[a] + at[a] % tile[a] // q[a]
    NS = math.prod(ns)
    return (u * NS + s).reshape(-1), math.prod(n) * NS


# ---- microscaled 4-bit floating point -----------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def mx4_values(x):
    """What blocks of 32 along the last axis of x [rows, K] stand for, by the definition: NaN in a block with anything not finite."""
    rows, K = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -K % 32)).reshape(rows, -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    bad = ~top.isfinite() | b.isnan().any(-1, keepdim=True)
    e = (torch.frexp(torch.where(bad, 1.0, top)).exponent - 3).clamp_min(-127)       # floor(log2) - 2
    unit = ((torch.where(top == 0, 0, e).long() + 1023) << 52).view(torch.float64)   # 2^e exactly; ldexp on a GPU is off by a step
    v = torch.where(bad, 0.0, b) / unit
    size = v.abs()
    index = torch.zeros_like(size)
    for i in range(7):                                       # middles: ties to the even index
        middle = (E2M1[i] + E2M1[i + 1]) / 2
        index += (size > middle) if i % 2 == 0 else (size >= middle)
    level = torch.tensor(E2M1, dtype=torch.float64, device=x.device)[index.long()]
    out = torch.where(bad, float("nan"), torch.where(v < 0, -level, level) * unit)
    return out.reshape(rows, -1)[:, :K]


def mx4_product(a, b, bias=None):
    """a [M, K], b [N, K] as values; the product and a bound on what the sums of the matrix instructions may be off: each adds 64
    products to the sum before it, dropping less than a step (2^-23) of their magnitudes together, and less than 16 partial sums are
    added at the end."""
    y, size = a @ b.t(), a.abs() @ b.abs().t()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, (-(-a.shape[1] // 64) + 16) * 2.0 ** -23 * size
