"""What asking for the kept entries' bits must not change: the token, its log-probs and the count; and the bits of rows that nothing
cuts, which are the entries above -inf, beside cut rows and alone."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sample import DT, a3po, unpack_bits  # noqa: E402, F401
from test_gpu_sample_uncut import ENDS, check_row, make  # noqa: E402

NAMES = ("token", "logp", "logp_full", "kept")


def both(a3po, z, u, **cuts):  # noqa: F811
    args = dict(want_logp_full=True, want_kept=True, **{k: v.cuda() for k, v in cuts.items()})
    with_bits, without = a3po.sample(z, u.cuda(), want_allowed=True, **args), a3po.sample(z, u.cuda(), **args)
    for n in NAMES:
        assert torch.equal(with_bits[n].nan_to_num(9.0), without[n].nan_to_num(9.0)), n
    return with_bits


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 31, 33, 2049, 8193, 50001, 151936])
def test_uncut_rows(a3po, V, dt):  # noqa: F811
    z, u, tau = make(9, V, V, dt)
    if V > 40:
        z[3, :V // 2], z[4, V // 3:], z[5] = -math.inf, -math.inf, -math.inf
    zc = z.float().numpy()
    for t, named in ((torch.ones(9), {}), (tau, dict(temperature=tau)), (torch.ones(9), dict(top_p=torch.ones(9)))):
        for numbers in (u, torch.tensor(ENDS)):
            out = {k: v.cpu() for k, v in both(a3po, z.cuda(), numbers, **named).items() if k in NAMES + ("allowed",)}
            bits = unpack_bits(out["allowed"], V)
            assert np.array_equal(bits[:, :V].astype(bool), zc > -math.inf) and not bits[:, V:].any()
            for r in range(9):
                if V > 40 and r == 5:
                    assert out["token"][r] == -1 and out["kept"][r] == 0
                else:
                    check_row(zc[r], float(numbers[r]), float(t[r]), int(out["token"][r]), out["logp"][r].item(), out["logp_full"][r].item(), int(out["kept"][r]), f"row {r}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_uncut_rows_beside_cut_ones(a3po, dt):  # noqa: F811
    T, V = 40, 30011
    z, u, tau = make(T, V, 3, dt)
    z[7, :9000] = -math.inf
    k = torch.tensor([0, 5, 0, 8000, 0, 0, 0, 0] * 5).int()
    p = torch.tensor([1.0, 1.0, 0.5, 1.0, 1.0, 0.99, 1.0, 1.0] * 5)
    out = both(a3po, z.cuda(), u, top_k=k, top_p=p, temperature=tau)
    bits = unpack_bits(out["allowed"], V)[:, :V].astype(bool)
    for t in range(T):
        alone = a3po.sample(z[t:t + 1].cuda(), u[t:t + 1].cuda(), temperature=tau[t:t + 1].cuda(), top_k=k[t:t + 1].cuda(), top_p=p[t:t + 1].cuda(), want_logp_full=True, want_kept=True)
        assert all(torch.equal(alone[n][0], out[n][t]) for n in NAMES)
        if k[t] == 0 and p[t] == 1:
            assert np.array_equal(bits[t], z[t].float().numpy() > -math.inf)
        assert bits[t].sum() == out["kept"][t]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("depth", [28.0, 29.5, 30.5, 40.0])
def test_many_small_weights_count(a3po, depth, dt):  # noqa: F811
    """151,935 equal entries of e^-depth before one of 1, and drawn numbers within what they make up: weights that are each far below
    2^-36 of the sum, where rounding them to a multiple of 2^-44 would show in the token."""
    V, n = 151936, 16
    z = torch.full((n, V), -depth)
    z[:, -1] = 0.0
    share = (V - 1) * math.exp(-depth)
    u = (torch.arange(n) + 0.5) / n * share / (1 + share)
    zc = z.numpy()
    out = {k: v.cpu() for k, v in both(a3po, z.to(DT[dt]).cuda(), u).items() if k in NAMES}
    for r in range(n):
        check_row(zc[r], float(u[r]), 1.0, int(out["token"][r]), out["logp"][r].item(), out["logp_full"][r].item(), V, f"row {r}")
