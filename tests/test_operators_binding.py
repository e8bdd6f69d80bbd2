"""CPU-only checks of what the binding does with the tensors that the operators around the attention are given."""
import pytest

from paper_2506_04648_amd import fps

torch = pytest.importorskip("torch")
BF16, U8 = torch.bfloat16, torch.uint8


def shape(heads=2, grid=(2, 3, 5)):
    return fps.make_shape(heads, grid, (1, 2, 2))


# ---- workspaces ---------------------------------------------------------------------------------
@pytest.mark.parametrize("workspace", [lambda n: torch.empty(1, dtype=U8).expand(n), lambda n: torch.empty(2 * n, dtype=U8)[::2],
                                       lambda n: torch.empty(1, 64, dtype=U8).expand(-(-n // 64), 64),
                                       lambda n: torch.empty(1, dtype=torch.float32).expand(-(-n // 4))])
def test_a_workspace_owns_its_bytes(workspace):
    """As many elements as the call needs, on fewer bytes or with gaps: the kernels would write over what follows."""
    x, w = torch.zeros(5, 70), torch.zeros(fps.mx4_bytes(9, 70), dtype=U8)
    with pytest.raises(ValueError, match="workspace"):
        fps.mx4_linear(x, w, 9, workspace=workspace(fps.mx4_linear_bytes(5, 70)))
    s, norm = shape(), fps.make_norm(torch.ones(128))
    x = torch.zeros(1, 2, 30, 128, dtype=BF16)
    with pytest.raises(ValueError, match="workspace"):
        fps.norm_rotate_bwd(s, x, x, norm, workspace=workspace(fps.norm_rotate_bwd_bytes(s, norm)))


# ---- tensors that are kept from call to call ----------------------------------------------------
def calls(s, norm, rotation):
    x = torch.zeros(1, 2, 30, 128, dtype=BF16)
    return (lambda: fps.norm_rotate(s, x, norm, rotation), lambda: fps.norm_rotate_operand(s, x, fps.ROLE_Q, fps.PREC_FP8, norm, rotation),
            lambda: fps.norm_rotate_bwd(s, x, x, norm, rotation))


@pytest.mark.parametrize("heads", [0, 2])
def test_weights_and_tables_are_read_where_they_lie(heads):
    """A parameter's memory is another one after an assignment to .data, a cast there and back, or a load that assigns."""
    s, size = shape(), (heads, 128) if heads else (128,)
    weight, table = torch.nn.Parameter(torch.ones(size), requires_grad=False), torch.ones(10, 2)
    norm, rotation = fps.make_norm(weight), fps.make_rotation(table, (1, 1, 1))
    for i in range(3):
        old = weight.data, table.data                        # keeps the old memory, so that the new one is another
        weight.data, table.data = torch.zeros(size), torch.zeros(10, 2)
        norm.weight = rotation.table = 0x10000
        with pytest.raises(ValueError, match="current device"):
            calls(s, norm, rotation)[i]()
        assert norm.weight == weight.data_ptr() != old[0].data_ptr() and rotation.table == table.data_ptr() != old[1].data_ptr()


@pytest.mark.parametrize("change", [lambda t: t.to(BF16), lambda t: t.double(), lambda t: torch.ones(t.shape[:-1] + (2 * t.shape[-1],))[..., ::2],
                                    lambda t: torch.ones(t.shape[:-1] + (64,)), lambda t: torch.ones((3,) + t.shape)])
def test_weights_and_tables_that_became_something_else(change):
    s = shape()
    for of_norm in (True, False):
        weight, table = torch.ones(128), torch.ones(10, 2)
        norm, rotation = fps.make_norm(weight), fps.make_rotation(table, (1, 1, 1))
        t = weight if of_norm else table
        t.data = change(t.data)
        for call in calls(s, norm, rotation):
            with pytest.raises(ValueError, match="a norm's weight has become" if of_norm else "a rotation's table has become"):
                call()
    weight = torch.ones(128)
    norm = fps.make_norm(weight)
    weight.untyped_storage().resize_(0)                      # as sharded parameters have it between their uses
    with pytest.raises(ValueError, match="without memory"):
        calls(s, norm, None)[0]()


# ---- gradients ----------------------------------------------------------------------------------
def test_gradients_are_not_lost_in_silence():
    """These calls record nothing: a tensor that autograd waits for is refused, unless the program has said that it does not."""
    s, x, w = shape(), torch.zeros(1, 2, 30, 128, dtype=BF16), torch.zeros(fps.mx4_bytes(9, 256), dtype=U8)
    leaf, weight, rows = x.clone().requires_grad_(), torch.ones(128, requires_grad=True), torch.zeros(30, 256, requires_grad=True)
    norm, out = fps.make_norm(weight), torch.zeros(30, 9)
    asked = [lambda: fps.norm_rotate(s, leaf), lambda: fps.norm_rotate(s, leaf * 2), lambda: fps.norm_rotate(s, x, norm), lambda: fps.norm_rotate(s, x, out=leaf),
             lambda: fps.norm_rotate_operand(s, leaf, fps.ROLE_Q), lambda: fps.norm_rotate_operand(s, x, fps.ROLE_Q, norm=norm),
             lambda: fps.norm_rotate_bwd(s, leaf, x), lambda: fps.norm_rotate_bwd(s, x, leaf), lambda: fps.norm_rotate_bwd(s, x, x, norm),
             lambda: fps.mx4_quantize(rows), lambda: fps.mx4_linear(rows, w, 9), lambda: fps.mx4_linear(rows.detach(), w, 9, bias=torch.zeros(9, requires_grad=True)),
             lambda: fps.mx4_dequantize(w, 30, 9, out=rows[:, :9])]
    for call in asked:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        for quiet in (torch.no_grad, torch.inference_mode):
            with quiet(), pytest.raises(ValueError, match="current device"):
                call()
    with pytest.raises(ValueError, match="current device"):
        fps.norm_rotate(s, leaf.detach())

    class Own(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            return fps.norm_rotate(s, t)

    with pytest.raises(ValueError, match="current device"):
        Own.apply(leaf)


# ---- launches -----------------------------------------------------------------------------------
def test_calls_that_a_launch_has_not_the_threads_for():
    """2^32 threads and more are refused before anything is launched; the addresses are never followed."""
    L, at, many = fps.lib(), 0x10000, 1 << 20

    def view(B, heads, rows, cols=128, dt=fps.OUT_BF16):
        return fps.View(at, dt, B, heads, rows, cols, heads * rows * cols, rows * cols, cols)

    def refused(status):
        assert status == fps.FPS_ERR_UNSUPPORTED and "threads" in fps.last_error()

    s, v = fps.make_shape(1, (1, 16, 32), (1, 8, 16), B=many), view(many, 1, 512)            # 16 blocks of 32 rows
    refused(L.fps_norm_rotate(s, v, None, None, v, None))
    s, v = fps.make_shape(1, (1, 8, 128), (1, 8, 16), B=many), view(many, 1, 1024)           # 8 blocks of 128 slots, 512 threads each
    refused(L.fps_norm_rotate_operand(s, v, None, None, fps.ROLE_Q, fps.PREC_FP8, at, at, None))
    s, v = fps.make_shape(1, (1, 4, 8), (1, 1, 1), B=many), view(many, 1, 32)                # 32 blocks of 32 slots, 128 threads each
    refused(L.fps_norm_rotate_operand(s, v, None, None, fps.ROLE_K, fps.PREC_BF16, at, None, None))
    refused(L.fps_dequantize(s, at, at, fps.ROLE_Q, fps.VSCALE_TILE, fps.OUT_BF16, at, None))
    s, v, norm = fps.make_shape(1 << 18, (1, 1, 1), (1, 1, 1)), view(1, 1 << 18, 1), fps.Norm(at, 1, 1e-6)
    need = L.fps_norm_rotate_bwd_bytes(s, norm)
    refused(L.fps_norm_rotate_bwd(s, v, norm, None, v, v, at, at, need, None))
    refused(L.fps_mx4_matmul(1, at, at, None, view(1, 1, 1, 1 << 29), None))
    refused(L.fps_mx4_quantize(view(1, 1, 1 << 30, 512), at, None))
    refused(L.fps_mx4_dequantize(at, view(1, 1, 1 << 30, 512), None))
