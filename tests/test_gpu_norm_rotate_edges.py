"""Norm and rotation of Q and K on the GPU where bits, ends of the range and long sums count."""
import pytest

from paper_2506_04648_amd import fps
from tests import operators_plain as op
from tests.test_gpu_norm_rotate import BF16, DEV, F32, OPERANDS, Case, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LONG = [dict(grid=(3, 9, 20), tile=(1, 8, 16), dt=BF16), dict(grid=(3, 9, 20), tile=(4, 16, 16), dt=F32, halves=True),
        dict(grid=(5, 18, 33), tile=(1, 8, 16), heads=9, dt=BF16, weight="per_head"),
        dict(grid=(9, 60, 70), tile=(1, 8, 16), heads=5, layout="fused")]


@pytest.mark.parametrize("case", LONG)
def test_rows_whose_squares_pass_fp32_are_infinitely_long(case):
    """r is 0 then: zeros out and no gradient, however large the row, its weights and its gradient are; other rows keep their bits."""
    say("long rows", case)
    c = Case(**case)
    c.weight.mul_(64.0)
    rows = torch.zeros(c.x.shape[:3], dtype=torch.bool, device=DEV)
    rows[0, 0, 17], rows[0, 1, 18], rows[0, 1, 19] = True, True, True
    x, dy = c.x.clone(), torch.randn(c.x.shape, generator=c.gen, device=DEV).to(c.dt)
    dy[rows] *= 1024.0
    x[0, 0, 17] = x[0, 0, 17].sign() * 3.3e38
    x[0, 1, 18] = x[0, 1, 18].sign() * 2.0 ** 80
    x[0, 1, 19, 5] = 2.0 ** 127
    short = torch.where(rows[..., None], torch.zeros_like(x), x)             # what the other rows are worth without those
    for out in (BF16, F32):
        y = fps.norm_rotate(c.shape, x, c.norm, c.rotation, out_dtype=out).reshape(x.shape)
        assert bool((y[rows] == 0).all()) and torch.equal(y, fps.norm_rotate(c.shape, short, c.norm, c.rotation, out_dtype=out).reshape(x.shape))
    for role in (fps.ROLE_Q, fps.ROLE_K):
        for prec in (fps.PREC_FP8, fps.PREC_BF16):
            (a, s), (b, t) = (fps.norm_rotate_operand(c.shape, v, role, prec, c.norm, c.rotation) for v in (x, short))
            if prec == fps.PREC_FP8:
                assert torch.equal(s, t)
                a, b = (fps.debug_unpack_q8(c.shape, v, role).view(torch.float8_e4m3fn).float() for v in (a, b))
            else:
                a, b = a.view(BF16), b.view(BF16)
            assert bool((a == b).all())                      # zeros of either sign
    dx, dw = fps.norm_rotate_bwd(c.shape, x, dy, c.norm, c.rotation)
    assert bool((dx[rows] == 0).all())
    quiet = torch.where(rows[..., None], torch.zeros_like(dy), dy)
    other, want = fps.norm_rotate_bwd(c.shape, short, quiet, c.norm, c.rotation)
    assert torch.equal(dx[~rows], other[~rows]) and torch.equal(dw, want)


@pytest.mark.parametrize("case", OPERANDS)
def test_fp8_scales_are_those_of_the_raster_values(case):
    """amax / 448 of what norm_rotate gives in fp32, bit for bit, whichever kernel a call takes.  (A quotient of two 24-bit numbers
    rounded to 53 bits and then to 24 is the one rounded once.)"""
    say("scales", case)
    c = Case(**case)
    y = fps.norm_rotate(c.shape, c.x, c.norm, c.rotation, out_dtype=F32).reshape(c.x.shape)
    group, n = op.group_of_tokens(c.grid, case["tile"], case.get("qtile"))
    top = torch.zeros(c.B, c.heads, n, device=DEV).scatter_reduce_(2, group.to(DEV).expand(c.B, c.heads, -1), y.abs().amax(-1), "amax")
    want = torch.where(top == 0, 1.0, (top.double() / 448).float())
    for role in (fps.ROLE_Q, fps.ROLE_K):
        assert torch.equal(fps.norm_rotate_operand(c.shape, c.x, role, fps.PREC_FP8, c.norm, c.rotation)[1], want)


@pytest.mark.parametrize("case", [c for c in OPERANDS if c.get("heads", 2) > 4])
def test_operands_of_a_head_do_not_depend_on_the_others(case):
    """Codes and scales of all heads in one call are those of each head in a call of its own."""
    say("heads", case)
    c = Case(**case)
    packed, scales = fps.norm_rotate_operand(c.shape, c.x, fps.ROLE_K, fps.PREC_FP8, c.norm, c.rotation)
    packed = packed.view(c.B, c.heads, -1)
    alone = fps.make_shape(1, c.grid, case["tile"], B=c.B, qtile=case.get("qtile"))
    for h in range(c.heads):
        norm = fps.make_norm(c.weight[h:h + 1].clone(), 1e-6) if case.get("weight") == "per_head" else c.norm
        p, s = fps.norm_rotate_operand(alone, c.x[:, h:h + 1], fps.ROLE_K, fps.PREC_FP8, norm, c.rotation)
        assert torch.equal(s[:, 0], scales[:, h]) and torch.equal(p.view(c.B, -1), packed[:, h]), h


@pytest.mark.parametrize("case", OPERANDS)
@pytest.mark.parametrize("role", [fps.ROLE_Q, fps.ROLE_K])
def test_fp8_codes_are_those_of_the_quotient(case, role):
    """Every code is the one nearest to the fp32 quotient of norm_rotate's value and the scale, halfway cases to even."""
    say("codes", case, role)
    c = Case(**case)
    y = fps.norm_rotate(c.shape, c.x, c.norm, c.rotation, out_dtype=F32).reshape(c.x.shape)
    group, _ = op.group_of_tokens(c.grid, case["tile"], case.get("qtile"))
    packed, scales = fps.norm_rotate_operand(c.shape, c.x, role, fps.PREC_FP8, c.norm, c.rotation)
    codes = fps.tile_unorder(c.shape, fps.debug_unpack_q8(c.shape, packed, role).view(torch.float8_e4m3fn).float()).reshape(y.shape)
    for h in range(c.heads):
        s = scales[:, h].gather(1, group.to(DEV).expand(c.B, -1))[..., None]
        want = (y[:, h].double() / s.double()).float().to(torch.float8_e4m3fn).float()
        assert bool((codes[:, h] == want).all()), (h, int((codes[:, h] != want).sum()))


@pytest.mark.parametrize("size", [3e-41, 1.4e-42, 1e-42, 3.2e-43, 2e-43, 1.5e-45])
@pytest.mark.parametrize("tile", [(1, 8, 16), (3, 4, 4), (8, 8, 8), (4, 16, 16)])
def test_scales_of_few_bits(size, tile):
    """Groups about the smallest fp32 numbers, zeros among them: the scale is amax / 448 rounded to what fp32 has there, 1 where that is
    nothing, and a quotient beyond 448, which is the scale's rounding, saturates."""
    c = Case(grid=(5, 18, 33), tile=tile, norm=False, rotate=False, dt=F32)
    c.x.copy_((c.x.double().clamp(-1, 1) * size).float())
    c.x[..., ::7] = 0.0
    c.x[0, 0, 40:60] = 0.0
    tiniest = 2.0 ** -149
    group, n = op.group_of_tokens(c.grid, tile)
    index = group.to(DEV).expand(1, c.heads, -1)
    top = torch.zeros(1, c.heads, n, dtype=torch.float64, device=DEV).scatter_reduce_(2, index, c.x.double().abs().amax(-1), "amax")
    want = (top / tiniest / 448).round() * tiniest
    want = torch.where(want == 0, torch.ones_like(want), want)
    s = want.gather(2, index)[..., None]
    codes64 = (c.x.double() / s).clamp(-448, 448).float().to(torch.float8_e4m3fn).float()
    for role in (fps.ROLE_Q, fps.ROLE_K):
        packed, scales = fps.norm_rotate_operand(c.shape, c.x, role)
        assert torch.equal(scales.double(), want)
        codes = fps.tile_unorder(c.shape, fps.debug_unpack_q8(c.shape, packed, role).view(torch.float8_e4m3fn).float()).reshape(c.x.shape)
        assert bool((codes == codes64).all())


@pytest.mark.parametrize("tile", [(1, 8, 16), (3, 4, 4), (2, 8, 16), (8, 8, 8), (4, 16, 16)])
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("norm", [True, False])
def test_groups_with_infinities_and_nans_have_such_a_scale(tile, dt, norm):
    """And the other groups are as they were."""
    c = Case(grid=(9, 18, 33), tile=tile, dt=dt, heads=3, norm=norm)
    group, n = op.group_of_tokens(c.grid, tile)
    packed, scales = fps.norm_rotate_operand(c.shape, c.x, fps.ROLE_K, fps.PREC_FP8, c.norm, c.rotation)
    bad = torch.zeros(1, 3, n, dtype=torch.bool)
    x = c.x.clone()
    for h, token, channel, value in ((0, 3, 5, float("nan")), (1, 700, 127, float("inf")), (2, c.N - 1, 0, float("-inf")), (2, 1500, 64, float("nan"))):
        x[0, h, token, channel] = value
        bad[0, h, group[token]] = True
    p, s = fps.norm_rotate_operand(c.shape, x, fps.ROLE_K, fps.PREC_FP8, c.norm, c.rotation)
    bad = bad.to(DEV)
    assert not bool(s[bad].isfinite().any()) and torch.equal(s[~bad], scales[~bad])
    if norm:
        assert bool(s[bad].isnan().all())
    of_token = bad.gather(2, group.to(DEV).expand(1, 3, -1))
    a, b = (fps.tile_unorder(c.shape, fps.debug_unpack_q8(c.shape, v, fps.ROLE_K).view(torch.float8_e4m3fn).float()).reshape(x.shape) for v in (p, packed))
    assert torch.equal(a[~of_token], b[~of_token])
    values = fps.dequantize(c.shape, p, s, fps.ROLE_K, out_dtype=F32).reshape(x.shape)
    assert bool((~values.isfinite()).any(-1)[0, 0, 3])


# ---- sums of the weights' gradient --------------------------------------------------------------
SUMS = [dict(grid=(9, 40, 64), heads=9, B=2), dict(grid=(9, 40, 64), heads=9, B=2, weight="per_head", layout="fused"),
        dict(grid=(9, 40, 64), heads=9, B=2, dt=F32, halves=True), dict(grid=(9, 40, 64), heads=5, B=2, dt=F32, weight="per_head"),
        dict(grid=(16, 61, 67), heads=9, halves=True, layout="fused"), dict(grid=(16, 61, 67), heads=9, weight="per_head"),
        dict(grid=(1, 1, 33), heads=5, halves=True, weight="per_head"), dict(grid=(21, 30, 52), heads=13)]


@pytest.mark.parametrize("case", SUMS)
def test_exact_sums_of_the_weights_gradient(case):
    """Rows of one magnitude, a power of two, small whole numbers as dy, quarter turns: x r is +-1, and every term and sum is a whole
    number below 2^24, so that the result is exact in any order of additions.  Up to nine parts of the rows a workgroup, the last one
    cut, and beyond the caches."""
    say("sums", case)
    split = (22, 21, 21)
    c = Case(rotate=False, eps=2.0 ** -40, **case)
    size = torch.exp2(torch.randint(-2, 4, c.x.shape[:3], generator=c.gen, device=DEV))[..., None]
    sign = 1.0 - 2.0 * torch.randint(2, c.x.shape, generator=c.gen, device=DEV)
    c.x.copy_(size * sign)
    dy = torch.randint(-3, 4, c.x.shape, generator=c.gen, device=DEV).to(c.dt)
    turn = torch.tensor([[1.0, 0.0], [0.0, 1.0], [-1.0, 0.0], [0.0, -1.0]], device=DEV)
    table = turn[torch.randint(4, (sum(n * k for n, k in zip(c.grid, split)),), generator=c.gen, device=DEV)].contiguous()
    rotation = fps.make_rotation(table, split, c.halves)
    cos, sin = op.turn_of_tokens(table, c.grid, split)
    axes = (0, 2) if c.weight.dim() == 2 else (0, 1, 2)
    want = (op.turned(dy.double(), cos, -sin, c.halves) * sign).sum(axes)
    assert float(want.abs().max()) < 2 ** 24 and 3 * c.B * c.N * c.heads < 2 ** 24
    dx, dw = fps.norm_rotate_bwd(c.shape, c.x, dy, c.norm, rotation)
    assert torch.equal(dw.double(), want)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("halves", [False, True])
def test_the_gradient_of_a_rotation_alone_does_not_see_x(dt, halves):
    say("rotation alone", dt, halves)
    c = Case(grid=(9, 18, 33), heads=9, dt=dt, norm=False, weight="none", halves=halves)
    dy = torch.randn(c.x.shape, generator=c.gen, device=DEV).to(dt)
    want, none = fps.norm_rotate_bwd(c.shape, c.x, dy, None, c.rotation)
    c.x[0, 3, 17, 5], c.x[0, 4, 18], c.x[0, 8, -1, 127] = float("inf"), float("nan"), float("-inf")
    dx, _ = fps.norm_rotate_bwd(c.shape, c.x, dy, None, c.rotation)
    assert none is None and torch.equal(dx, want) and bool(dx.isfinite().all())


# ---- tensors that are kept from call to call ----------------------------------------------------
def test_weights_and_tables_that_were_given_other_memory():
    say("other memory")
    c = Case(grid=(3, 9, 20), tile=(1, 8, 16), heads=3, weight="per_head")
    weight, table = torch.nn.Parameter(c.weight.clone(), requires_grad=False), c.rotation.tensor.clone()
    norm, rotation = fps.make_norm(weight, 1e-6), fps.make_rotation(table, (22, 21, 21))
    dy = torch.randn(c.x.shape, generator=c.gen, device=DEV).to(BF16)
    for _ in range(3):
        old = weight.data, table.data
        weight.data, table.data = torch.randn(3, 128, generator=c.gen, device=DEV), table.data.roll(5, 0).contiguous()
        old[0].fill_(7.0), old[1].fill_(7.0)
        want = fps.make_norm(weight.data.clone(), 1e-6), fps.make_rotation(table.data.clone(), (22, 21, 21))
        for call in (lambda n, r: (fps.norm_rotate(c.shape, c.x, n, r),), lambda n, r: fps.norm_rotate_operand(c.shape, c.x, fps.ROLE_Q, fps.PREC_FP8, n, r),
                     lambda n, r: fps.norm_rotate_bwd(c.shape, c.x, dy, n, r)):
            assert all(torch.equal(a, b) for a, b in zip(call(norm, rotation), call(*want)))
