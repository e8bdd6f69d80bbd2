"""From hidden states to hidden states: the projection in 4 bits, norm and rotation into operands, the attention, the projection back;
each stage against 64 bits, from what the stage before left."""
import pytest

from paper_2506_04648_amd import fps
from tests import operators_plain as op
from tests.accepted_set import ACC_EPS

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


class Layer:
    """One attention layer's weights and buffers; forward() runs it on the current stream."""

    def __init__(self, grid, tile, window, heads, prec, vscale, halves, seed=1, qtile=None):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.gen, self.grid, self.tile, self.window, self.heads, self.prec, self.vscale = gen, grid, tile, window, heads, prec, vscale
        self.shape = fps.make_shape(heads, grid, tile, qtile=qtile)
        self.N, self.C = grid[0] * grid[1] * grid[2], heads * 128
        N, C = self.N, self.C
        self.w = {n: (torch.randn(k * C, C, generator=gen, device=DEV) / C ** 0.5).to(BF16) for n, k in (("in", 3), ("out", 1))}
        self.packed = {n: fps.mx4_quantize(w) for n, w in self.w.items()}
        self.bias = {n: 0.1 * torch.randn(w.shape[0], generator=gen, device=DEV) for n, w in self.w.items()}
        self.gain = [1 + 0.2 * torch.randn(heads, 128, generator=gen, device=DEV) for _ in range(2)]
        self.norms = [fps.make_norm(g, 1e-6) for g in self.gain]
        split = (22, 21, 21)
        table = fps.rotation_table(self.shape, split).to(DEV)
        self.rotation = fps.make_rotation(table, split, halves)
        self.plain = [op.Turning(g, 1e-6, op.turn_of_tokens(table, grid, split), halves) for g in self.gain]
        self.x = torch.randn(N, C, generator=gen, device=DEV).to(BF16)
        bytes_ = fps.packed_bytes(self.shape, prec)
        groups = fps.num_groups(self.shape)
        self.qkv = torch.empty(1, 3 * heads, N, 128, dtype=BF16, device=DEV)
        self.operands = [torch.empty(bytes_, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.scales = [torch.empty(1, heads, groups, device=DEV) for _ in range(2)]
        self.o = torch.empty((1, heads) + grid + (128,), dtype=BF16, device=DEV)
        self.y = torch.empty(N, C, dtype=BF16, device=DEV)
        self.workspace = torch.empty(fps.mx4_linear_bytes(N, C), dtype=torch.uint8, device=DEV)

    def forward(self):
        C, heads, fp8 = self.C, self.heads, self.prec == fps.PREC_FP8
        fps.mx4_linear(self.x, self.packed["in"], 3 * C, bias=self.bias["in"], out=self.qkv, workspace=self.workspace)
        for i, role in enumerate((fps.ROLE_Q, fps.ROLE_K)):
            fps.norm_rotate_operand(self.shape, self.qkv[:, i * heads:(i + 1) * heads], role, self.prec, self.norms[i], self.rotation,
                                    out=self.operands[i], scales=self.scales[i])
        v = self.qkv[:, 2 * heads:].reshape((1, heads) + self.grid + (128,))
        if fp8:
            self.v, self.sv = fps.quantize_tiles(self.shape, v, fps.ROLE_V, vscale=self.vscale, raster=True)
        else:
            self.v, self.sv = fps.pack_tiles_bf16(self.shape, v, fps.ROLE_V, raster=True)
        fps.attn_fwd(self.shape, self.window, self.prec, *self.operands, self.v, *(self.scales if fp8 else (None, None)), self.sv,
                     vscale=self.vscale if fp8 else fps.VSCALE_TILE, out=self.o, raster_out=True)
        fps.mx4_linear(self.o.reshape(1, heads, self.N, 128), self.packed["out"], C, bias=self.bias["out"], out=self.y, workspace=self.workspace)
        return self.y

    def attention(self, q, k, v, p_step, p_tiniest):
        """In 64 bits, and a bound on the kernel's difference: a weight in its type is off by p_step of itself or by p_tiniest, a score
        by its sum's rounding in the matrix instructions (ACC_EPS of the products' magnitudes), which a weight and the sum of the weights
        follow; the output is rounded once more."""
        tile_of, _ = op.group_of_tokens(self.grid, self.tile)
        seen = torch.as_tensor(fps.tile_mask_host(self.shape, self.window)[0]).bool().to(DEV)[tile_of.to(DEV)][:, tile_of.to(DEV)]
        scores = q @ k.transpose(1, 2).contiguous() / 128 ** 0.5
        off = float((q.abs() @ k.abs().transpose(1, 2).contiguous()).max()) / 128 ** 0.5 * ACC_EPS + 2.0 ** -16
        scores = scores.masked_fill(~seen, float("-inf"))
        p = (scores - scores.amax(-1, keepdim=True)).exp()
        l = p.sum(-1, keepdim=True)
        o, size = p @ v / l, p @ v.abs() / l
        most = v.abs().amax(1, keepdim=True) * seen.sum(-1, dtype=torch.float64)[:, None]
        rel = p_step + 2 * off
        return o, 2 * rel * size + 2 * p_tiniest * (most + size) / l


LAYERS = [
    dict(grid=(3, 9, 20), tile=(1, 8, 16), window=(3, 3, 3, 0), heads=2, halves=False),
    dict(grid=(5, 18, 33), tile=(4, 16, 16), window=(3, 3, 3, 0), heads=3, halves=True),
    dict(grid=(4, 8, 10), tile=(2, 4, 4), window=(1, 3, 1, 0), heads=1, halves=False),
    dict(grid=(2, 13, 20), tile=(1, 8, 16), window=(1, 1, 3, 0), heads=12, halves=True),
    dict(grid=(1, 1, 1), tile=(1, 8, 16), window=(1, 1, 1, 0), heads=2, halves=False),
]


@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("prec,vscale", [(fps.PREC_FP8, fps.VSCALE_TILE), (fps.PREC_FP8, fps.VSCALE_CHANNEL), (fps.PREC_BF16, fps.VSCALE_TILE)])
def test_an_attention_layer(layer, prec, vscale):
    print(layer, prec, vscale, flush=True)
    m = Layer(prec=prec, vscale=vscale, **layer)
    y = m.forward()
    heads, N, C = m.heads, m.N, m.C
    # the projection
    want, bound = op.mx4_product(op.mx4_values(m.x), op.mx4_values(m.w["in"]), m.bias["in"])
    assert op.within(m.qkv[0].transpose(0, 1).reshape(N, 3 * C), want, bound, BF16) <= 1
    # norm, rotation and operands
    values = []
    for i, role in enumerate((fps.ROLE_Q, fps.ROLE_K)):
        turned, off = m.plain[i].forward(m.qkv[:, i * heads:(i + 1) * heads])
        if prec == fps.PREC_FP8:
            got = fps.dequantize(m.shape, m.operands[i], m.scales[i], role, out_dtype=F32).reshape(turned.shape).double()
            group, _ = op.group_of_tokens(m.grid, m.tile)
            s = m.scales[i].double().gather(2, group.to(DEV).expand(1, heads, -1))[..., None]
            code, slack = turned / s, off / s + 4 * op.F32 * (turned.abs() / s + 1)
            assert bool(((got / s - code).abs() <= op.e4m3_half_step((code.abs() + slack).clamp_max(448.0)) + slack).all())
        else:
            got = fps.norm_rotate(m.shape, m.qkv[:, i * heads:(i + 1) * heads], m.norms[i], m.rotation).reshape(turned.shape)
            assert op.within(got, turned, off, BF16) <= 1
            assert torch.equal(fps.pack_tiles_bf16(m.shape, got.reshape((1, heads) + m.grid + (128,)), role, raster=True)[0], m.operands[i])
            got = got.double()
        values.append(got[0])
    # the attention; a weight in FP8 is a code of weight * 448, with BF16 operands it is in fp16, as V is, by powers of two
    if prec == fps.PREC_FP8:
        v = fps.dequantize(m.shape, m.v, m.sv, fps.ROLE_V, vscale=vscale, out_dtype=F32).reshape(heads, N, 128).double()
        o, bound = m.attention(*values, v, 2.0 ** -4, 2.0 ** -10 / 448)
    else:
        v = m.qkv[0, 2 * heads:].double()
        o, bound = m.attention(*values, v, 2.0 ** -11, 2.0 ** -24)
    assert op.within(m.o.reshape(o.shape), o, bound, BF16) <= 1
    # the projection back
    rows = m.o.reshape(heads, N, 128).transpose(0, 1).reshape(N, C)
    want, bound = op.mx4_product(op.mx4_values(rows), op.mx4_values(m.w["out"]), m.bias["out"])
    assert op.within(y, want, bound, BF16) <= 1


@pytest.mark.parametrize("prec", [fps.PREC_FP8, fps.PREC_BF16])
def test_two_layers_at_once_and_replayed(prec):
    """Two layers on two streams, then each in a captured graph, replayed on new inputs: bits of eager calls alone."""
    layers = [Layer(prec=prec, vscale=fps.VSCALE_TILE, seed=i, **LAYERS[i]) for i in range(2)]
    alone = [m.forward().clone() for m in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for m, s in zip(layers, streams):
            with torch.cuda.stream(s):
                m.y.fill_(7)
                m.forward()
    torch.cuda.synchronize()
    for m, a in zip(layers, alone):
        assert torch.equal(m.y, a)
    graphs = []
    for m in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.forward()
        graphs.append(g)
    for k in range(3):
        for m in layers:
            m.x.copy_(torch.randn(m.x.shape, generator=m.gen, device=DEV))
        eager = [m.forward().clone() for m in layers]
        for m in layers:
            m.y.fill_(7)
        for g, s in zip(graphs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for m, e in zip(layers, eager):
            assert torch.equal(m.y, e), k


def test_gradients_of_q_and_k_through_a_layer():
    """dL/dx of norm and rotation by the library against autograd through the formulas in 64 bits, with L's gradient of the values given."""
    m = Layer(prec=fps.PREC_FP8, vscale=fps.VSCALE_TILE, **LAYERS[1])
    m.forward()
    dq = torch.randn(1, m.heads, m.N, 128, generator=m.gen, device=DEV).to(BF16)
    for i in range(2):
        x = m.qkv[:, i * m.heads:(i + 1) * m.heads]
        dx, dw = fps.norm_rotate_bwd(m.shape, x, dq, m.norms[i], m.rotation)
        leaf, gain = x.double().requires_grad_(), m.gain[i].double().requires_grad_()
        plain = op.Turning(gain, 1e-6, m.plain[i].turn, m.plain[i].halves)
        plain.forward(leaf)[0].backward(dq.double())
        want, off, terms, size = m.plain[i].backward(x, dq)
        assert float((leaf.grad - want).abs().max()) < 1e-9          # the formulas are the derivative's
        assert op.within(dx, leaf.grad, off, BF16) <= 1
        assert bool(((dw.double() - gain.grad).abs() <= (24 + 1000) * op.F32 * size.sum((0, 2))).all())
