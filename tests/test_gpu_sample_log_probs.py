"""Log-probs are at most 0: in rows with one entry, and with one that has nearly all of the mass, sums in 64 bits may end a few units of
2^-52 below the entry's own weight, whose logarithm then is not the sum's."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sample import DT, a3po  # noqa: E402, F401


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cuts", ["", "temperature", "top_p", "top_k", "min_p", "temperature+top_k+top_p"])
@pytest.mark.parametrize("V", [1, 200, 40001])
def test_rows_of_one_token(a3po, V, cuts, dt):  # noqa: F811
    T = 512
    g = torch.Generator().manual_seed(V)
    z = torch.full((T, V), -math.inf)
    at = torch.randint(0, V, (T,), generator=g)
    z[torch.arange(T), at] = 20 * torch.randn(T, generator=g)
    if V > 1:
        z[T // 2:, 0].clamp_(min=-60.0)  # (another one far below in half of the rows)
    values = dict(temperature=torch.linspace(0.3, 2.0, T), top_p=torch.full((T,), 0.999), top_k=torch.full((T,), 3).int(), min_p=torch.full((T,), 1e-3))
    out = a3po.sample(z.to(DT[dt]).cuda(), torch.full((T,), 0.5).cuda(), want_logp_full=True, **{n: values[n].cuda() for n in cuts.split("+") if n})
    for n in ("logp", "logp_full"):
        assert (out[n] <= 0).all() and (out[n].cpu()[:T // 2].abs() <= 2.0 ** -35).all(), n
