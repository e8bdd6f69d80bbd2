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
