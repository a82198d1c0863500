"""Calls of linear layers and of norms between blocks that the other tests do not make (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_residual_norm import dol  # noqa: E402,F401


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gates", [1, 3])
def test_no_rows_leave_a_gate_without_gradient(dol, gates, dtype):
    """Sums over no rows are zeros, a gate's as well as gammas', in rows of any distance."""
    t = getattr(torch, dtype)
    u, gate = torch.empty(0, 40, dtype=t, device="cuda"), torch.ones(gates, 40, dtype=t, device="cuda")
    buf = torch.full((gates, 47), 5.0, dtype=t, device="cuda")
    gg, sums = buf[:, 3:43], [torch.full((40,), 5.0, device="cuda") for _ in range(2)]
    none = sums[0][:0]
    dol.residual_norm(u, u, None, gate, None, u, u)
    for first in ((u, u, None, gate, None), (u, None, gate, None, u)):
        gg.fill_(5.0)
        dol.residual_norm_backward(*first, none, none, u, u, u, u, sums[0], gg, sums[1])
        assert not gg.any() and not sums[0].any() and not sums[1].any()
    assert bool((buf[:, :3] == 5).all()) and bool((buf[:, 43:] == 5).all())
    gg.fill_(5.0)
    dol.residual_norm_backward(u, u, None, gate, None, none, none, u, u, u, u, None, gg, None)
    assert not gg.any()
