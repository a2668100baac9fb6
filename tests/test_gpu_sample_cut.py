"""a3po_sample on cut rows, held to the figures that the header promises, with and without bits of the kept.

The kept entries are the definition's, but for a border of top_p that lies within `slack` of the sum of what it is a share of; the token is an
entry kept in any case, with a weight above zero, and the drawn number lies in its part of the kept sum or within `slack` of it, also where the
number is 0.  slack is 2^-35 of the sum where the entries down to the border are listed (at most 4,864 of them, or 9,728 in its bin):
4,864 roundings of 2^-49 of the largest weight are 2^-36.75, bins' sums are off by 2^-37 of themselves each for the rounding and 2^-38 for
the series.  In rows that go in passes each weight is rounded to 2^-(62 - ceil(log2 V)) of the largest: V half units of that."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sample import DT, a3po, unpack_bits  # noqa: E402, F401
from test_gpu_sample_uncut import ENDS, LAST, make, weights  # noqa: E402

LISTED = 2.0 ** -35


def passes(V):
    return LISTED + V * 2.0 ** -(63 - max(12, math.ceil(math.log2(V))))


def check(a3po, z, u, slack, tau=None, k=None, p=None, min_p=None):  # noqa: F811
    """z on the GPU, the rest on the CPU."""
    named = {n: t.cuda() for n, t in (("temperature", tau), ("top_k", k), ("top_p", p), ("min_p", min_p)) if t is not None}
    out = a3po.sample(z, u.cuda(), want_logp_full=True, want_kept=True, want_allowed=True, **named)
    bare = a3po.sample(z, u.cuda(), **named)
    assert torch.equal(bare["token"], out["token"]) and torch.equal(bare["logp"], out["logp"])
    token, logp, full, count = (out[n].cpu().numpy() for n in ("token", "logp", "logp_full", "kept"))
    V = z.shape[1]
    bits = unpack_bits(out["allowed"], V)
    assert not bits[:, V:].any()
    zc = z.float().cpu().numpy()
    for t in range(z.shape[0]):
        greedy = tau is not None and tau[t] == 0
        x = weights(zc[t], 1.0 if tau is None or greedy else float(tau[t]))
        w = np.exp(x)
        order = np.lexsort((np.arange(V), -zc[t].astype(np.float64)))
        order = order[zc[t][order] > -math.inf]
        most = 1 if greedy else int(k[t]) if k is not None and k[t] > 0 else V
        order = order[:most]
        n, doubt = order.size, (0, 0)
        upto = np.cumsum(w[order])
        if p is not None and p[t] < 1:
            need = max(float(p[t]), 0.0) * upto[-1]
            ends = [1 + int((upto[:-1] < need + s * slack * upto[-1]).sum()) for s in (-1, 0, 1)]
            n, doubt = ends[1], (ends[0], ends[2])
        if min_p is not None and min_p[t] > 0:
            m = int((x[order] >= math.log(min(float(min_p[t]), 1.0))).sum())
            n, doubt = min(n, m), tuple(min(d, m) for d in doubt)
        got = bits[t, :V].astype(bool)
        assert got.sum() == count[t], t
        if count[t] != n:
            assert doubt[0] <= count[t] <= doubt[1], f"row {t}: {count[t]} kept for {n}"
        kept = np.zeros(V, bool)
        kept[order[:count[t]]] = True
        assert np.array_equal(got, kept), f"row {t}: others are kept"
        y = int(token[t])
        assert 0 <= y < V and kept[y] and w[y] > 0, f"row {t}: token {y}"
        sums = np.cumsum(np.where(kept, w, 0.0))
        number, before = min(max(float(u[t]), 0.0), LAST) * sums[-1], sums[y] - w[y]
        assert before - slack * sums[-1] <= number < sums[y] + slack * sums[-1], f"row {t}: token {y}"
        for have, total in ((logp[t], sums[-1]), (full[t], w.sum())):
            want = x[y] - math.log(total)
            assert abs(have - want) <= 2.0 ** -24 * abs(want) + 2 * slack, t
    return out


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("entries", [100, 4000, 4860])
@pytest.mark.parametrize("depth", [26.0, 29.0, 31.3, 32.0])
def test_listed_entries_of_small_weights(a3po, depth, entries, dt):  # noqa: F811
    """So many equal entries of e^-depth before one of 1, and drawn numbers within what they make up, by a count and by a share."""
    V, n = 151936, 12
    z = torch.full((n, V), -60.0)
    z[:, 1000:1000 + entries] = -depth
    z[:, -1] = 0.0
    share = entries * math.exp(-depth)
    u = (torch.arange(n) + 0.5) / n * share / (1 + share)
    k = torch.full((n,), entries + 1).int()
    check(a3po, z.to(DT[dt]).cuda(), u, LISTED, k=k)
    # (e^-26.5 is 2^-38: a border that far down without top_k goes in passes, as bins of 1/16 power of two reach 2^-32)
    check(a3po, z.to(DT[dt]).cuda(), u, passes(V), min_p=torch.full((n,), math.exp(-depth - 0.5)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lead", ["nothing", "masked", "lowest"])
@pytest.mark.parametrize("only", ["k", "p", "min_p", "k+p", "p+min_p", "tau+k+p+min_p"])
def test_numbers_at_the_ends(a3po, only, lead, dt):  # noqa: F811
    V, T = 30001, len(ENDS)
    g = torch.Generator().manual_seed(4)
    z, _, tau = make(T, V, 11, dt)
    if lead != "nothing":
        z[:, :10000] = -math.inf if lead == "masked" else torch.finfo(DT[dt]).min
    cuts = dict(tau=tau, k=torch.randint(2, 4000, (T,), generator=g).int(), p=0.2 + 0.75 * torch.rand(T, generator=g), min_p=0.001 + 0.1 * torch.rand(T, generator=g))
    check(a3po, z.cuda(), torch.tensor(ENDS), LISTED, **{n: cuts[n] for n in only.split("+")})


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_numbers_at_the_ends_of_wide_nuclei(a3po, dt):  # noqa: F811
    """Borders in a bin of thousands (a nucleus of most of a flat row), and in passes (a count of 20,000 with a share of it)."""
    V, T = 60001, len(ENDS)
    z, _, tau = make(T, V, 12, dt, 0.7)
    z[:, :20000] = -math.inf
    check(a3po, z.cuda(), torch.tensor(ENDS), LISTED, p=torch.linspace(0.3, 0.95, T))
    check(a3po, z.cuda(), torch.tensor(ENDS), passes(V), p=torch.linspace(0.3, 0.95, T), k=torch.full((T,), 20000).int(), tau=tau)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [17, 2500, 20000, 151936, 262145])
def test_all_cuts(a3po, V, dt):  # noqa: F811
    T = 10
    g = torch.Generator().manual_seed(V)
    z, u, tau = make(T, V, V + 1, dt, 2.5)
    tau[3] = 0.0
    k, p = torch.randint(1, 4000, (T,), generator=g).int(), 0.1 + 0.89 * torch.rand(T, generator=g)
    check(a3po, z.cuda(), u, LISTED, k=k)
    check(a3po, z.cuda(), u, LISTED, k=k, p=p, tau=tau)
    check(a3po, z.cuda(), u, passes(V), p=p, tau=tau)
    check(a3po, z.cuda(), u, LISTED, p=torch.full((T,), 0.9), min_p=torch.full((T,), 0.3), tau=torch.full((T,), 2.0))
