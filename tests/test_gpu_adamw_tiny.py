"""Updates whose running squares are so small that fp32 holds them with fewer bits, or as a few units of its smallest number."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_adamw import U, a3po  # noqa: E402, F401


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-24])
@pytest.mark.parametrize("bits", [32, 8])
def test_updates_are_those_of_the_states(a3po, bits, eps):  # noqa: F811
    """A first step from zero states, from gradients of 10^-21 (v is 7 units of 2^-149) to 10^-10.  The update is that of m and v in
    fp32, so v here is the fp32 product and sum's; the root's, reciprocal's, constants' and products' roundings are 16 * 2^-24 of
    the update, p adds one of itself.  Weights are of the updates' size, so that these show."""
    n, lr, beta1, beta2 = 4096, 1e-3, 0.9, 0.99
    g = torch.logspace(-21, -10, n) * torch.where(torch.arange(n) % 3 == 0, -1.0, 1.0)
    p = 1e-4 * torch.ones(n)
    w = p.cuda()
    m, v, scales = a3po.adamw_state(w, bits)
    a3po.adamw_step([w], [g.cuda()], [m], [v], scales=None if scales is None else [scales], step=1, lr=lr, beta1=beta1, beta2=beta2, eps=eps)
    fm, fv = (1 - beta1) * g, (1 - beta2) * g * g
    assert (fv > 0).all()
    if bits == 32:
        assert torch.equal(v.cpu(), fv) and torch.equal(m.cpu(), fm)
    update = lr / (1 - beta1) * fm.double() / (torch.sqrt(fv.double() / (1 - beta2)) + eps)
    assert ((w.cpu().double() - (p.double() - update)).abs() <= 16 * U * update.abs() + U * (p + update.abs())).all()
