"""Microscaled 4-bit floating point on the GPU: quantisation bit for bit, products against 64 bits."""
import sys

import pytest

from paper_2506_04648_amd import fps
from tests import operators_plain as op

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def rows_of(gen, rows, K, dt, spread=0.0):
    """Normal values; spread: of the blocks' sizes, in binary orders."""
    x = torch.randn(rows, K, generator=gen, device=DEV)
    if spread:
        x *= torch.exp2(spread * torch.randn(rows, -(-K // 32), generator=gen, device=DEV)).repeat_interleave(32, 1)[:, :K]
    return x.to(dt)


def same(got, want):
    """Equal values, NaN where NaN is; the sign of a zero does not count."""
    return bool(((got.double() == want) | (got.isnan() & want.isnan())).all())


# ---- quantisation -------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (1, 31), (3, 33), (32, 256), (33, 257), (31, 255), (5, 1000), (64, 64), (70, 1536), (129, 515)])
def test_values(rows, K, dt):
    say("values", rows, K, dt)
    gen = torch.Generator(device=DEV).manual_seed(rows * 1000 + K)
    x = rows_of(gen, rows, K, dt, spread=3.0)
    packed = fps.mx4_quantize(x)
    assert packed.numel() == fps.mx4_bytes(rows, K)
    want = op.mx4_values(x)
    for out in (BF16, F32):
        assert same(fps.mx4_dequantize(packed, rows, K, out_dtype=out), want)
    # rows with gaps in between, and an output with gaps, beside which nothing is written
    wide = torch.zeros(rows, K + 3, dtype=dt, device=DEV)
    wide[:, :K] = x
    assert torch.equal(fps.mx4_quantize(wide[:, :K]), packed)
    wide = torch.full((rows, K + 5), 7.0, dtype=dt, device=DEV)
    fps.mx4_dequantize(packed, rows, K, out=wide[:, :K])
    assert same(wide[:, :K], want) and bool((wide[:, K:] == 7).all())


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("B,heads,tokens,cols", [(1, 3, 7, 128), (2, 2, 33, 128), (2, 5, 11, 32), (3, 1, 9, 40), (3, 2, 1, 128), (40, 1, 1, 33)])
def test_values_of_views(B, heads, tokens, cols, dt):
    say("views", B, heads, tokens, cols, dt)
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x = torch.randn(B, heads, tokens, cols, generator=gen, device=DEV).to(dt)
    m = x.transpose(1, 2).reshape(B * tokens, heads * cols).contiguous()
    packed = fps.mx4_quantize(x)
    assert torch.equal(packed, fps.mx4_quantize(m))
    assert torch.equal(packed, fps.mx4_quantize(x.transpose(1, 2).contiguous().transpose(1, 2)))
    back = fps.mx4_dequantize(packed, B * tokens, heads * cols, out=torch.empty_like(x))
    assert same(back.transpose(1, 2).reshape(m.shape), op.mx4_values(m))


@pytest.mark.parametrize("dt,rows,K", [(BF16, 26400, 5137), (F32, 14000, 5003), (BF16, 1, 140000001), (BF16, 2200000, 65)])
def test_values_beyond_the_caches(dt, rows, K):
    """More than 256 MB of rows, which are read past the caches; with infinities and NaN in them."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    x = rows_of(gen, rows, K, dt, spread=3.0)
    x[rows // 2, K // 3], x[0, K - 1], x[rows - 1, 0] = float("nan"), float("inf"), float("-inf")
    packed = fps.mx4_quantize(x)
    assert same(fps.mx4_dequantize(packed, rows, K), op.mx4_values(x))
    part = min(rows, 4096)                                   # the same codes as of fewer rows
    assert torch.equal(fps.mx4_quantize(x[:part])[:fps.mx4_bytes(part, K) // 17 * 16], packed[:fps.mx4_bytes(part, K) // 17 * 16])
    if rows % 2 == 0:
        half = x.view(2, rows // 2, K)                       # in two parts of rows
        assert torch.equal(fps.mx4_quantize(half), packed)


def test_views_beyond_the_caches():
    gen = torch.Generator(device=DEV).manual_seed(9)
    x = torch.randn(2, 9, 60000, 128, generator=gen, device=DEV).to(BF16)
    m = x.transpose(1, 2).reshape(120000, 9 * 128).contiguous()
    assert torch.equal(fps.mx4_quantize(x), fps.mx4_quantize(m))
    assert torch.equal(fps.mx4_quantize(m[:, :1000]), fps.mx4_quantize(m[:, :1000].contiguous()))


def test_every_bf16_value_and_the_scales_ends():
    """Blocks that hold one value beside a largest one of every exponent; blocks of zeros, of subnormal numbers, of the largest
    number; infinities and NaN make a block NaN and no other."""
    bits = torch.arange(65536, device=DEV).to(torch.uint16).view(BF16)
    x = torch.zeros(65536, 64, dtype=BF16, device=DEV)
    x[:, 3], x[:, 32] = bits, 1.0
    for other in (0.0, 1.0, 3.3895e38, 1e-40, 6.0):
        x[:, 17] = other
        want = op.mx4_values(x)
        packed = fps.mx4_quantize(x)
        assert same(fps.mx4_dequantize(packed, 65536, 64, out_dtype=F32), want)
        assert same(fps.mx4_dequantize(fps.mx4_quantize(x.float()), 65536, 64, out_dtype=F32), want)
        assert bool((want[:, 32] == 1).all())
    wide = x.repeat(1, 33)                                   # read past the caches
    assert same(fps.mx4_dequantize(fps.mx4_quantize(wide), 65536, 64 * 33, out_dtype=F32)[:, -64:], want)
    assert same(fps.mx4_dequantize(fps.mx4_quantize(wide.float()), 65536, 64 * 33, out_dtype=F32)[:, -64:], want)


def test_every_quotient_near_a_tie_in_fp32():
    """fp32 values a step beside every middle, at several scales."""
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], device=DEV)
    near = torch.stack([torch.nextafter(middles, middles - 1), middles, torch.nextafter(middles, middles + 1)]).reshape(-1)
    x = torch.zeros(6, 32, device=DEV)
    for i, e in enumerate((-120, -20, 0, 1, 60, 120)):
        x[i, :24], x[i, 31] = near * 2.0 ** e, 4.0 * 2.0 ** e
    x[:, 8:16] *= -1
    assert same(fps.mx4_dequantize(fps.mx4_quantize(x), 6, 32, out_dtype=F32), op.mx4_values(x))


# ---- products -----------------------------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 64, 64), (1, 5120, 640), (2, 33, 100), (7, 160, 33), (32, 256, 256), (33, 300, 31), (40, 512, 512), (64, 1536, 96),
         (77, 100, 1000), (100, 2304, 372), (128, 128, 128), (255, 640, 257), (256, 256, 256), (300, 700, 520), (513, 1000, 384),
         (851, 1536, 640), (16, 9000, 64), (2000, 96, 2100), (1, 96, 5000), (1025, 2049, 1030)]
# From 112 tiles of 128 x 128 on they are what is multiplied, one step of K or more, the last tile cut; tiles of 256 where they fill the CUs
# better, up to several of them one after the other
SIZES += [(33, 300, 15000), (1400, 1100, 1501), (1500, 64, 1496), (15000, 200, 1), (5000, 257, 4100)]
SIZES += [(7000, 64, 2104), (7001, 300, 2103), (8200, 520, 4104), (6921, 1792, 2048), (12000, 256, 5128), (26333, 64, 5128)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_product(M, K, N):
    say("product", M, K, N)
    gen = torch.Generator(device=DEV).manual_seed(M + K + N)
    x, w = rows_of(gen, M, K, BF16, spread=1.0), rows_of(gen, N, K, BF16, spread=1.0)
    bias = torch.randn(N, generator=gen, device=DEV)
    a, b = fps.mx4_quantize(x), fps.mx4_quantize(w)
    va, vb = op.mx4_values(x), op.mx4_values(w)
    for add in (None, bias):
        want, bound = op.mx4_product(va, vb, add)
        y = fps.mx4_matmul(a, b, M, N, K, bias=add, out_dtype=F32)
        assert op.within(y, want, bound, F32) <= 1
        low = fps.mx4_matmul(a, b, M, N, K, bias=add)
        assert torch.equal(low, y.to(BF16))                  # rounded once, from the same sums
        wide = torch.full((M, N + 3), 7.0, dtype=BF16, device=DEV)
        assert torch.equal(fps.mx4_linear(x, b, N, bias=add, out=wide[:, :N]), low)
        assert bool((wide[:, N:] == 7).all())
        assert torch.equal(fps.mx4_linear(x.float(), b, N, bias=add, out_dtype=F32), y)


@pytest.mark.parametrize("B,heads_in,heads_out,tokens", [(1, 2, 3, 45), (2, 4, 5, 31), (3, 1, 2, 200), (1, 5, 12, 700), (2, 2, 12, 700), (1, 1, 17, 7000), (4, 2, 3, 1), (1500, 1, 12, 1),
                                                          (2, 3, 16, 3500)])
def test_product_between_the_attentions_layouts(B, heads_in, heads_out, tokens):
    say("layouts", B, heads_in, heads_out, tokens)
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    K, N = 128 * heads_in, 128 * heads_out
    x = torch.randn(B, heads_in, tokens, 128, generator=gen, device=DEV).to(BF16)
    w = fps.mx4_quantize(rows_of(gen, N, K, BF16))
    m = x.transpose(1, 2).reshape(B * tokens, K).contiguous()
    y = fps.mx4_linear(m, w, N)
    out = torch.empty(B, heads_out, tokens, 128, dtype=BF16, device=DEV)
    fps.mx4_linear(x, w, N, out=out)
    assert torch.equal(out.transpose(1, 2).reshape(B * tokens, N), y)
    three = torch.full((B, tokens, 3, heads_out, 128), 7.0, dtype=F32, device=DEV)           # a share of wider rows
    fps.mx4_linear(x, w, N, out=three[:, :, 1].transpose(1, 2))
    assert torch.equal(three[:, :, 1].reshape(B * tokens, N).to(BF16), y)
    assert bool((three[:, :, 0] == 7).all()) and bool((three[:, :, 2] == 7).all())


@pytest.mark.parametrize("M,K,N", [(1, 700, 96), (40, 700, 96), (600, 700, 520), (1400, 700, 1500), (7000, 300, 2104)])
def test_not_finite_blocks_make_their_rows_and_columns_nan(M, K, N):
    gen = torch.Generator(device=DEV).manual_seed(3)
    x, w = rows_of(gen, M, K, BF16), rows_of(gen, N, K, BF16)
    y = fps.mx4_linear(x, fps.mx4_quantize(w), N)
    x[M // 2, K - 1], w[N - 1, 5] = float("nan"), float("inf")
    z = fps.mx4_linear(x, fps.mx4_quantize(w), N)
    bad = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    bad[M // 2], bad[:, N - 1] = True, True
    assert bool(z[bad].isnan().all()) and torch.equal(z[~bad], y[~bad])


@pytest.mark.parametrize("M,N", [(1, 96), (33, 96), (300, 96), (15000, 96), (7000, 2104)])
def test_scales_of_very_different_size(M, N):
    """Blocks from 2^-100 to 2^60, products from 2^-127 to 2^120, in one row; the bound is on the magnitudes' sum."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    K = 640
    e = torch.linspace(-60, 55, K // 32, device=DEV).round()
    x = (rows_of(gen, M, K, F32) * torch.exp2(e).repeat_interleave(32)).to(BF16)
    w = (rows_of(gen, N, K, F32) * torch.exp2(e.flip(0) * 0.9).round(decimals=0).clamp_min(2.0 ** -60).repeat_interleave(32)).to(BF16)
    want, bound = op.mx4_product(op.mx4_values(x), op.mx4_values(w))
    y = fps.mx4_linear(x, fps.mx4_quantize(w), N, out_dtype=F32)
    assert op.within(y, want, bound, F32) <= 1


@pytest.mark.parametrize("M,K,N", [(513, 1792, 770), (1, 5120, 640), (1400, 1792, 1500), (7000, 1792, 2104)])
def test_exact_sums(M, K, N):
    """Small whole numbers: every sum is exact, whatever its order."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    pick = torch.tensor([0, 1, 2, 3, 4, 6], device=DEV)
    x = (pick[torch.randint(6, (M, K), generator=gen, device=DEV)] * (1 - 2 * torch.randint(2, (M, K), generator=gen, device=DEV))).to(BF16)
    w = (pick[torch.randint(6, (N, K), generator=gen, device=DEV)] * (1 - 2 * torch.randint(2, (N, K), generator=gen, device=DEV))).to(BF16)
    x[:, ::32], w[:, ::32] = 4, 6                            # the blocks' scales are 1
    y = fps.mx4_linear(x, fps.mx4_quantize(w), N, out_dtype=F32)
    assert torch.equal(y.double(), x.double() @ w.double().t())


def test_offsets_beyond_32_bits():
    """Rows, read and written, 2^31 + 8 elements apart, in a batch of two."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    far = torch.empty((1 << 31) + 8 + 3 * 640, dtype=BF16, device=DEV)
    m = rows_of(gen, 6, 640, BF16)
    w = fps.mx4_quantize(rows_of(gen, 640, 640, BF16))
    y = fps.mx4_linear(m, w, 640)
    x = far.as_strided((2, 3, 640), ((1 << 31) + 8, 640, 1))
    x.copy_(m.reshape(2, 3, 640))
    assert torch.equal(fps.mx4_linear(x, w, 640), y)
    fps.mx4_linear(m, w, 640, out=x)
    assert torch.equal(x.reshape(6, 640), y)


def test_packed_matrix_and_rows_of_the_result_beyond_4_gib():
    """600000 rows that repeat 96 of small whole numbers, whose sums are exact in any order; then a result with rows 2 MB apart."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    K, N, times = 16384, 256, 6250
    m, w = (torch.randint(-2, 3, (n, K), generator=gen, device=DEV).to(BF16) for n in (96, N))
    packed = fps.mx4_quantize(m.expand(times, 96, K))
    assert packed.numel() > 1 << 32
    want = (m.double() @ w.double().t()).to(BF16)
    for n in (40, N):                                        # tiles of 128, tiles of 256
        y = fps.mx4_matmul(packed, fps.mx4_quantize(w[:n].contiguous()), times * 96, n, K)
        assert bool((y.view(times, 96, n) == want[:, :n]).all())
    assert bool((fps.mx4_dequantize(packed, times * 96, K)[-96:] == m).all())
    del packed
    x, b = rows_of(gen, 7000, 64, BF16), fps.mx4_quantize(rows_of(gen, 2104, 64, BF16))
    y = fps.mx4_linear(x, b, 2104)
    far = torch.full((7000, 1 << 20), 7.0, dtype=BF16, device=DEV)
    fps.mx4_linear(x, b, 2104, out=far[:, :2104])
    assert torch.equal(far[:, :2104], y) and bool((far[:, 2104:2400] == 7).all())


def test_another_stream_and_replayed_graphs_that_share_a_workspace():
    """Two graphs captured with one workspace, replayed one after the other on new inputs, against eager calls."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    cases = []
    w = {}
    for M, K, N in ((1, 512, 320), (300, 512, 640), (1400, 512, 1504), (7000, 512, 2104)):
        w[N] = fps.mx4_quantize(rows_of(gen, N, K, BF16))
        cases.append((rows_of(gen, M, K, BF16), N, torch.empty(M, N, dtype=BF16, device=DEV)))
    workspace = torch.empty(fps.mx4_linear_bytes(7000, 512), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x, N, y in cases:
            fps.mx4_linear(x, w[N], N, out=y, workspace=workspace)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for x, N, y in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fps.mx4_linear(x, w[N], N, out=y, workspace=workspace)
        graphs.append(g)
    for k in range(4):
        for x, N, y in cases:
            x.copy_(rows_of(gen, *x.shape, BF16))
            y.fill_(7)
        eager = [fps.mx4_linear(x, w[N], N) for x, N, y in cases]
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for (x, N, y), e in zip(cases, eager):
            assert torch.equal(y, e), k
