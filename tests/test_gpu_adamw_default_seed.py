"""adamw_step called as its signature asks, without a seed: the roundings by chance still differ from step to step, so what they leave
has the value as its mean over steps."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_adamw import a3po  # noqa: E402, F401


@pytest.mark.parametrize("on_device", [False, True])
def test_running_squares_fall(a3po, on_device):  # noqa: F811
    """700 steps without gradients at beta2 = 0.999: the mean of 4,096 states falls to 0.999^700 = 0.496 of its start.  A step's rounding
    has at most a deviation of half a step of e5m2, an eighth of the value: 700 of them add up to 0.125 * 0.496 * sqrt(700) / sqrt(4,096) =
    0.026 at most if each were that; five of those bound the mean."""
    n, steps = 4096, 700
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v, scales = a3po.adamw_state(p, 8)
    a3po.adamw_step([p], [torch.rand(n, device="cuda") + 0.5], [m], [v], scales=[scales], step=1, lr=0.0)
    start = a3po.adamw_state_values(v, scales[1]).double().mean()
    number = torch.tensor([1], device="cuda")
    for step in range(2, steps + 2):
        number += 1
        a3po.adamw_step([p], [g], [m], [v], scales=[scales], step=number if on_device else step, lr=0.0)
    left = float(a3po.adamw_state_values(v, scales[1]).double().mean() / start)
    assert abs(left - 0.999 ** steps) <= 5 * 0.026


def test_bfloat16_weights_take_updates_below_their_last_bit(a3po):  # noqa: F811
    """300 equal updates of lr = 2^-12 (a gradient of one sign: mean over root is 1) from weights of 1, whose neighbours are 2^-8 below and
    2^-7 above: the mean of 4,096 weights falls by 300 * 2^-12 = 0.073; deviations of half a step of 2^-8 each add up to at most
    2^-9 * sqrt(300) / sqrt(4,096) = 0.00053, six of those, and 1 % for a mean over root that is only nearly 1."""
    n, steps = 4096, 300
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, device="cuda")
    m, v, _ = a3po.adamw_state(p)
    for step in range(1, steps + 1):
        a3po.adamw_step([p], [g], [m], [v], step=step, lr=2.0 ** -12)
    assert abs(float(1.0 - p.double().mean()) - steps * 2.0 ** -12) <= 6 * 0.00053 + 0.01 * steps * 2.0 ** -12


def test_the_default_is_the_step(a3po):  # noqa: F811
    n = 3000
    g = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    def run(step, **kw):
        p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
        m, v, scales = a3po.adamw_state(p, 8)
        a3po.adamw_step([p], [g], [m], [v], scales=[scales], step=step, lr=1e-3, **kw)
        return p, v.view(torch.uint8)
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert same(run(5), run(5, seed=5)) and not same(run(5), run(5, seed=0))
    assert same(run(torch.tensor([5], device="cuda")), run(torch.tensor([5], device="cuda"), seed=0))
