"""adamw_step writes to tensors that autograd may have kept: it has to notice, as it does after an update by PyTorch."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_adamw import a3po  # noqa: E402, F401


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("what", ["param", "copy"])
def test_a_backward_pass_through_updated_weights_is_refused(a3po, what, bits):  # noqa: F811
    master = torch.nn.Parameter(torch.randn(64, 3, device="cuda"))
    copy = torch.nn.Parameter(master.detach().bfloat16())
    other = torch.nn.Parameter(torch.randn(64, 3, device="cuda"))
    used = master if what == "param" else copy
    loss, untouched = used.square().sum(), other.square().sum()
    m, v, scales = a3po.adamw_state(master, bits)
    a3po.adamw_step([master], [torch.ones_like(master)], [m], [v], scales=None if scales is None else [scales], copies=[copy], step=1, lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    untouched.backward()
    # the next forward pass is as good as any
    used.grad = None
    used.square().sum().backward()
    assert torch.equal(used.grad, 2 * used.detach())


def test_tensors_without_versions(a3po):  # noqa: F811
    with torch.inference_mode():
        p = torch.ones(5, device="cuda")
        m, v, _ = a3po.adamw_state(p)
        a3po.adamw_step([p], [torch.ones_like(p)], [m], [v], step=1, lr=0.5)
    assert (p < 1).all()
