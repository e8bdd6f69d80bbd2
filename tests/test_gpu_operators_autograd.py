"""The operators around the attention beside autograd: in a program's own Function, and on tensors that autograd has saved."""
import pytest

from paper_2506_04648_amd import fps
from tests import operators_plain as op

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def test_saved_tensors_that_a_call_writes_into():
    """backward() refuses them, as after any write in place."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    s, weight = fps.make_shape(2, (2, 3, 5), (1, 2, 2)), torch.ones(128, device=DEV)
    norm = fps.make_norm(weight)
    x = torch.randn(1, 2, 30, 128, generator=gen, device=DEV)
    packed, scales = fps.norm_rotate_operand(s, x, fps.ROLE_Q)
    rows = torch.randn(30, 256, generator=gen, device=DEV)
    w = fps.mx4_quantize(rows)
    writes = [lambda t: fps.norm_rotate(s, x, out=t), lambda t: fps.norm_rotate_bwd(s, x, x, dx=t), lambda t: fps.norm_rotate(s, t, out=t),
              lambda t: fps.dequantize(s, packed, scales, fps.ROLE_Q, out=t), lambda t: fps.mx4_dequantize(w, 30, 256, out=t),
              lambda t: fps.mx4_matmul(w, w[:fps.mx4_bytes(30, 256)], 30, 30, 256, out=t.view(-1)[:900].view(30, 30)),
              lambda t: fps.mx4_linear(rows, w, 30, out=t.view(-1)[:900].view(30, 30))]
    for write in writes:
        leaf, saved = torch.ones(1, device=DEV, requires_grad=True), torch.ones(1, 2, 30, 128, device=DEV)
        y = (leaf * saved).sum()
        write(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    for write, like in ((lambda t: fps.norm_rotate_bwd(s, x, x, norm, dweight=t), weight), (lambda t: fps.norm_rotate_operand(s, x, fps.ROLE_Q, scales=t), scales),
                        (lambda t: fps.norm_rotate_operand(s, x, fps.ROLE_Q, out=t), packed), (lambda t: fps.mx4_quantize(rows, out=t), w)):
        t = like.clone()
        before = t._version
        write(t)
        assert t._version > before


def test_a_function_of_the_programs_own():
    """Norm and rotation in a graph of autograd's, by the gradient's entry point, against autograd through the formulas in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    grid, heads, split = (3, 9, 11), 3, (22, 21, 21)
    s = fps.make_shape(heads, grid, (1, 8, 16))
    rotation = fps.make_rotation(fps.rotation_table(s, split).to(DEV), split)

    class NormRotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            ctx.save_for_backward(x, weight)
            return fps.norm_rotate(s, x, fps.make_norm(weight), rotation)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            x, weight = ctx.saved_tensors
            return fps.norm_rotate_bwd(s, x, dy, fps.make_norm(weight), rotation)

    for dt in (F32, BF16):
        x = torch.randn(1, heads, 297, 128, generator=gen, device=DEV).to(dt).requires_grad_()
        weight = torch.randn(heads, 128, generator=gen, device=DEV).requires_grad_()
        dy = torch.randn(1, heads, *grid, 128, generator=gen, device=DEV).to(dt)
        NormRotate.apply(x, weight).backward(dy)
        plain = op.Turning(weight.detach(), 1e-6, op.turn_of_tokens(rotation.tensor, grid, split), False)
        dx, off, terms, size = plain.backward(x.detach(), dy.reshape(x.shape))
        assert op.within(x.grad, dx, off, dt) <= 1
        # a term to 24 half steps, a sum of 297 terms no deeper than 297 additions
        assert bool(((weight.grad.double() - terms.sum((0, 2))).abs() <= (24 + 297) * op.F32 * size.sum((0, 2))).all())
