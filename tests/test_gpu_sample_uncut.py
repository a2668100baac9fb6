"""a3po_sample on rows that nothing cuts (no cut at all, or temperature alone), by the kernels that draw such rows without bits of the
kept, and beside cut rows, against the definition in 64 bits.

Weights are off by 2^-42 of themselves at the most (series and table, sums in 64 bits of up to 2^10 terms a thread), NumPy's running sums by
2^-53 an entry, at most 2^-35 for 2^18 of them and far less as roundings go both ways; a token may differ where the drawn number lies
within 2^-36 of the sum of its ends, and with a drawn number of 0 not even there: it is the first entry of a weight above zero (2^-900 of the
sum: the kernels take what is below 2^-1000 of the largest weight as none).  It is an entry above -inf with a weight in any case.
Log-probs are computed in 64 bits and rounded once."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sample import DT, a3po, unpack_bits  # noqa: E402, F401

INF = math.inf
LAST = 1.0 - 2.0 ** -24


def weights(z, tau):
    z = z.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        x = np.where(z == z.max(), 0.0, (z - z.max()) / tau)
    return np.where(z > -INF, x, -INF)


def check_row(z, u, tau, token, logp, full, kept, where):
    x = weights(z, tau)
    w = np.exp(x)
    upto = np.cumsum(w)
    total = upto[-1]
    u = min(max(u, 0.0), LAST)
    assert 0 <= token < z.size and w[token] > 0, f"{where}: token {token}"
    before = upto[token - 1] if token else 0.0
    slack = (2.0 ** -36 if u > 0 else 2.0 ** -900) * total
    assert before - slack <= u * total < upto[token] + slack, f"{where}: token {token}"
    want = x[token] - math.log(total)
    for got in (logp, full):
        assert abs(got - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -36, where
    assert kept == (z > -INF).sum(), where


def check(a3po, z, u, tau=None, V=None):  # noqa: F811
    """z on the GPU; with and without the outputs that are not needed, with bits and without: the token is one."""
    V = z.shape[1] if V is None else V
    named = {} if tau is None else dict(temperature=tau.cuda())
    out = a3po.sample(z, u.cuda(), V, want_logp_full=True, want_kept=True, **named)
    bare = a3po.sample(z, u.cuda(), V, want_logp=False, **named)
    assert torch.equal(bare["token"], out["token"])
    zc = z.float().cpu().numpy()[:, :V]
    token, logp, full, kept = (out[n].cpu().numpy() for n in ("token", "logp", "logp_full", "kept"))
    for t in range(z.shape[0]):
        check_row(zc[t], float(u[t]), 1.0 if tau is None else float(tau[t]), int(token[t]), logp[t], full[t], kept[t], f"row {t}")
    return out


def make(T, V, seed, dt, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(T, V, generator=g)).to(DT[dt]), torch.rand(T, generator=g), 0.3 + 1.7 * torch.rand(T, generator=g)


ENDS = [0.0, -1.0, -INF, 2.0 ** -149, 2.0 ** -24, 0.5, LAST, 1.0, INF]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("with_tau", [False, True])
@pytest.mark.parametrize("begin", [1, 2047, 2048, 2049, 4096, 6144, 8191, 8192, 8200, 16384, 19999])
@pytest.mark.parametrize("lead", ["masked", "lowest"])
def test_numbers_at_the_ends_behind_entries_without_weight(a3po, lead, begin, with_tau, dt):  # noqa: F811
    """The row begins with masked entries, or such of the type's lowest value: a drawn number of 0 gives the first of the others."""
    V = 20000
    z, _, tau = make(len(ENDS), V, begin, dt)
    z[:, :begin] = -INF if lead == "masked" else torch.finfo(DT[dt]).min
    u = torch.tensor(ENDS)
    out = check(a3po, z.cuda(), u, tau if with_tau else None)
    assert (out["token"][:3] == begin).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("with_tau", [False, True])
def test_numbers_at_the_ends_with_one_entry_anywhere(a3po, with_tau, dt):  # noqa: F811
    """One entry a row, the rest masked, and one far below it behind or before it."""
    V = 30011
    at = [0, 1, 2047, 2048, 5000, 8191, 8192, 12288, 24575, 24576, 29999, 30000, 30010]
    for u in (0.0, 0.5, LAST):
        z = torch.full((3 * len(at), V), -INF)
        for i, e in enumerate(at):
            z[3 * i:3 * i + 3, e] = 5.0 * i - 30
            z[3 * i + 1, (e + 3000) % V] = -1e30
            z[3 * i + 2, (e + 27000) % V] = -1e30
        out = check(a3po, z.to(DT[dt]).cuda(), torch.full((z.shape[0],), u), torch.linspace(0.5, 1.5, z.shape[0]) if with_tau else None)
        assert out["token"].tolist() == [e for e in at for _ in range(3)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("u", [0.0, 2.0 ** -149, 0.3, LAST])
def test_parts_that_are_far_apart(a3po, u, dt):  # noqa: F811
    """Parts and quarters of parts whose weights are beyond what 64 bits hold beside others: 2^-1000 and less of the largest."""
    V, T = 40000, 8
    z, _, _ = make(T, V, 7, dt, 1.0)
    z[0, :20000] -= 2000
    z[1, 2048:] -= 5000
    z[2, :2048], z[2, 2048:4096] = -INF, z[2, 2048:4096] - 1500
    z[3] += 800
    z[3, 8192:] -= 1600
    z[4, :8192], z[4, 8192:] = -INF, z[4, 8192:] + 1e4
    z[5, :30000] = -1e30
    z[6] *= 1e4
    z[7, :4096] -= 720
    check(a3po, z.cuda(), torch.full((T,), u))
    check(a3po, z.cuda(), torch.full((T,), u), torch.linspace(0.25, 3.0, T))


WIDTHS = [1, 2, 3, 7, 31, 32, 33, 255, 257, 2047, 2049, 8191, 8193, 16385, 50001, 151936, 262145]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", WIDTHS)
def test_every_width(a3po, V, dt):  # noqa: F811
    z, u, tau = make(9, V, V, dt)
    check(a3po, z.cuda(), u)
    check(a3po, z.cuda(), u, tau)
    check(a3po, z.cuda(), torch.tensor(ENDS))


@pytest.mark.parametrize("V", [256 * 8192 - 5, 256 * 8192 + 1, 512 * 8192])
def test_rows_of_as_many_parts_as_there_are_threads(a3po, V):  # noqa: F811
    z, u, tau = make(2, V, 5, "bf16")
    check(a3po, z.cuda(), u)
    check(a3po, z.cuda(), u, tau)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("with_tau", [False, True])
def test_masks_lowest_values_and_logits_far_out(a3po, with_tau, dt):  # noqa: F811
    V, T = 40001, 14
    g = torch.Generator().manual_seed(6)
    z, u, _ = make(T, V, 5, dt)
    low = torch.finfo(DT[dt]).min
    for t in range(6):
        z[t, torch.rand(V, generator=g) < t / 5] = -INF
        z[t, (9973 * t) % V] = float(t)
    z[6] = low
    z[7, 1:], z[8, :-1] = low, low
    z[9, ::2], z[9, 1::2] = -INF, low
    z[10, 7] = -low
    z[11] += 1e4
    z[12] *= 1e30
    z[13] *= 1e-30
    check(a3po, z.cuda(), u, torch.linspace(0.5, 1.5, T) if with_tau else None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_temperatures_far_out(a3po, dt):  # noqa: F811
    """Up to infinity, where all entries that are not masked weigh the same."""
    tau = torch.tensor([1e-45, 1e-30, 1e-3, 1e3, 1e10, 1e28, 1e30, 3e38, INF])
    z, u, _ = make(9, 20001, 9, dt)
    z[:, ::3] = -INF
    check(a3po, z.cuda(), u, tau)
    check(a3po, z.cuda(), torch.zeros(9), tau[3:].repeat(2)[:9])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("with_tau", [False, True])
@pytest.mark.parametrize("V", [70, 20001])
def test_rows_without_a_policy(a3po, V, with_tau, dt):  # noqa: F811
    T = 16
    z, u, _ = make(T, V, 8, dt)
    z[1] = -INF
    z[3, V // 2], z[5, V - 1], z[7, 0] = math.nan, INF, math.nan
    z[9], z[9, V // 3] = -INF, math.nan
    z[11], z[11, V // 3] = torch.finfo(DT[dt]).min, math.nan
    u[10] = math.nan
    tau = torch.ones(T)
    nan = [3, 5, 7, 9, 10, 11]
    if with_tau:
        tau[12], tau[13] = -1.0, math.nan
        nan += [12, 13]
    named = dict(temperature=tau.cuda()) if with_tau else {}
    out = {k: v.cpu() for k, v in a3po.sample(z.cuda(), u.cuda(), want_logp_full=True, want_kept=True, **named).items() if k in ("token", "logp", "logp_full", "kept")}
    for t in range(T):
        if t in nan or t == 1:
            assert out["token"][t] == -1 and out["kept"][t] == 0
            assert all(v.isnan() if t in nan else v == -INF for v in (out["logp"][t], out["logp_full"][t]))
        else:
            check_row(z[t].float().numpy(), float(u[t]), 1.0, int(out["token"][t]), out["logp"][t].item(), out["logp_full"][t].item(), int(out["kept"][t]), f"row {t}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(1000, 24, 0), (1000, 25, 1), (4099, 13, 3), (33, 1, 1), (30001, 7, 5)])
def test_strides_and_unaligned_rows(a3po, V, pad, shift, dt):  # noqa: F811
    T = 7
    buf = torch.full((T * (V + pad) + shift,), 1e30, dtype=DT[dt], device="cuda")
    z = buf[shift:].view(T, V + pad)
    inner, u, tau = make(T, V, V, dt)
    z[:, :V] = inner.cuda()
    check(a3po, z, u, V=V)
    check(a3po, z, u, tau, V=V)


def test_more_rows_than_one_launch_takes(a3po):  # noqa: F811
    z, u, tau = make(2100, 900, 13, "bf16")
    check(a3po, z.cuda(), u)
    check(a3po, z.cuda(), u, tau)


def test_in_a_graph(a3po):  # noqa: F811
    z, u, tau = make(40, 33000, 30, "f32")
    z[:, :9000] = -INF
    z, u, tau = z.cuda(), u.cuda(), tau.cuda()
    for named in ({}, dict(temperature=tau)):
        call = lambda: a3po.sample(z, u, want_logp_full=True, want_kept=True, **named)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = call()
        for i in range(3):
            u.copy_(torch.rand(40, generator=torch.Generator().manual_seed(i)))
            u[i] = 0.0
            graph.replay()
            want = call()
            torch.cuda.synchronize()
            assert all(torch.equal(want[n], kept[n]) for n in ("token", "logp", "logp_full", "kept")), i
            assert kept["token"][i] == 9000
