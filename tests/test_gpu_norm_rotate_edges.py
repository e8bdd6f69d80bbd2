"""Norm and rotation of Q and K on the GPU where bits, ends of the range and long sums count."""
import pytest

from paper_2506_04648_amd import fps
from tests.test_gpu_norm_rotate import BF16, DEV, F32, Case, say

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
