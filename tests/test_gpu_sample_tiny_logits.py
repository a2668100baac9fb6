"""Rows whose logits and temperatures are among fp32's smallest numbers, where a bin is a few of them or less than one: the grid's borders
are found in floats that the type still tells apart."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sample import a3po  # noqa: E402, F401
from test_gpu_sample_cut import LISTED, check as check_cut  # noqa: E402
from test_gpu_sample_uncut import check as check_uncut  # noqa: E402

SMALLEST = 2.0 ** -149
TAU = [SMALLEST, 3 * SMALLEST, 100 * SMALLEST, 1e-41, 1e-39, 2.0 ** -126, 1e-37, 1e-30]


@pytest.mark.parametrize("top", [0.0, 40 * SMALLEST, -SMALLEST, 1e-39, -1e-38])
@pytest.mark.parametrize("only", ["", "k", "p", "min_p", "k+p+min_p"])
def test_logits_of_a_few_smallest_numbers(a3po, only, top):  # noqa: F811
    T, V = len(TAU), 9001
    g = torch.Generator().manual_seed(7)
    tau = torch.tensor(TAU, dtype=torch.float64)
    z = (top - 12.0 * tau[:, None] * torch.rand(T, V, generator=g, dtype=torch.float64)).float()
    z[:, ::5], z[:, 1::50], z[:, 77] = -math.inf, -1e-20, top
    u = torch.rand(T, generator=g)
    cuts = dict(k=torch.randint(1, 3000, (T,), generator=g).int(), p=0.1 + 0.85 * torch.rand(T, generator=g), min_p=torch.full((T,), 0.05))
    if only:
        check_cut(a3po, z.cuda(), u, LISTED, tau=tau.float(), **{n: cuts[n] for n in only.split("+")})
    else:
        check_uncut(a3po, z.cuda(), u, tau.float())
