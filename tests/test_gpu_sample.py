"""a3po_sample against the definition in 64 bits, row by row.

Kept entries and tokens are whole numbers and have to be the definition's.  The library's sums are off by at most V roundings of
2^-46 of the largest weight and by weights' errors of 2^-47 of themselves, below 2^-28 of the sum for V = 2^18, so a token (or a
border of top_p) may differ only where the drawn number (top_p's share) lies within 2^-28 of the sum of a border: each difference
is held to that, and the cases are few enough that none is expected.  Log-probs are computed in 64 bits and rounded once:
2^-24 |logp|, beside 2^-28 for the sums."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEAR = 2.0 ** -28


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def unpack_bits(words, V):
    return np.unpackbits(words.cpu().numpy().view(np.uint8), axis=1, bitorder="little")


def reference_row(z, u, tau, k, p, min_p):
    """(kept bool [V], token, logp, logp_full, distance of the nearest border that decided, relative to its sum)."""
    z = z.astype(np.float64)
    V = z.size
    if tau == 0:
        tau, k = 1.0, 1
    x = (z - z.max()) / tau
    w = np.exp(x)
    order = np.lexsort((np.arange(V), -z))
    order = order[z[order] > -np.inf]
    near = np.inf
    if k is not None and k > 0:
        order = order[:k]
    if p is not None and p < 1:
        upto = np.cumsum(w[order])
        ahead = upto - w[order]
        need = max(p, 0.0) * upto[-1]
        keep = ahead < need
        keep[0] = True
        near = min(near, np.abs(ahead[1:] - need).min() / upto[-1] if order.size > 1 else np.inf)
        order = order[keep]
    if min_p is not None and min_p > 0:
        order = order[(x[order] >= math.log(min(min_p, 1.0)))]
    kept = np.zeros(V, bool)
    kept[order] = True
    upto = np.cumsum(np.where(kept, w, 0.0))
    u = min(max(u, 0.0), 1 - 2.0 ** -24)
    token = int(np.searchsorted(upto, u * upto[-1], side="right"))
    near = min(near, np.abs(upto - u * upto[-1]).min() / upto[-1])
    return kept, token, x[token] - math.log(upto[-1]), x[token] - math.log(w.sum()), near


def check(a3po, z, u, tau=None, k=None, p=None, min_p=None, V=None):
    """z on the GPU, possibly with rows wider than V; the rest on the CPU."""
    V = z.shape[1] if V is None else V
    T = z.shape[0]
    cuda = lambda t: None if t is None else t.cuda()
    before = z.clone()
    out = a3po.sample(z, u.cuda(), V, temperature=cuda(tau), top_k=cuda(k), top_p=cuda(p), min_p=cuda(min_p),
                      want_logp_full=True, want_kept=True, want_allowed=True)
    assert torch.equal(before.view(torch.uint8), z.view(torch.uint8))
    token, logp, full, count = (out[n].cpu().numpy() for n in ("token", "logp", "logp_full", "kept"))
    bits = unpack_bits(out["allowed"], V)
    assert not bits[:, V:].any()
    zc = z.float().cpu().numpy()[:, :V]
    at = lambda t, i: None if t is None else float(t[i])
    for t in range(T):
        kept, y, lp, lf, near = reference_row(zc[t], float(u[t]), 1.0 if tau is None else float(tau[t]),
                                              None if k is None else int(k[t]), at(p, t), at(min_p, t))
        same = np.array_equal(bits[t, :V].astype(bool), kept) and token[t] == y
        assert same or near < NEAR, f"row {t}: token {token[t]} for {y}, {bits[t].sum()} kept for {kept.sum()}, border {near}"
        assert count[t] == bits[t].sum()
        if same:
            assert abs(logp[t] - lp) <= 2.0 ** -24 * abs(lp) + NEAR and abs(full[t] - lf) <= 2.0 ** -24 * abs(lf) + NEAR
    return out


def make(T, V, seed, dt="f32", scale=3.0):
    g = torch.Generator().manual_seed(seed)
    z = (scale * torch.randn(T, V, generator=g)).to(DT[dt])
    r = lambda lo, hi: lo + (hi - lo) * torch.rand(T, generator=g)
    return z, torch.rand(T, generator=g), dict(tau=r(0.3, 2.0), k=torch.randint(1, V + 2, (T,), generator=g).int(), p=r(0.2, 1.0),
                                               min_p=r(0.0, 0.3))


WIDTHS = [1, 2, 3, 7, 31, 32, 33, 64, 65, 255, 256, 257, 511, 513, 1000, 2049, 4097, 8191, 8193, 16385, 32000, 50001, 151936, 262145]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", WIDTHS)
def test_every_width(a3po, V, dt):
    z, u, cuts = make(5, V, V, dt)
    z = z.cuda()
    check(a3po, z, u)
    check(a3po, z, u, **cuts)
    check(a3po, z, u, p=cuts["p"])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.05, 0.7, 4.0, 30.0])
@pytest.mark.parametrize("only", ["tau", "k", "p", "min_p", "k+p", "p+min_p", "k+min_p", "tau+k+p+min_p"])
def test_cuts_alone_and_together(a3po, only, scale, dt):
    z, u, cuts = make(12, 9000, 3, dt, scale)
    check(a3po, z.cuda(), u, **{n: cuts[n] for n in only.split("+")})


@pytest.mark.parametrize("T", [1, 2, 17, 255, 300, 1500])
def test_numbers_of_rows(a3po, T):
    z, u, cuts = make(T, 700, T, "bf16")
    check(a3po, z.cuda(), u, **cuts)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_small_k_and_narrow_p_of_long_rows(a3po, dt):
    T, V = 24, 120001
    z, u, _ = make(T, V, 11, dt, 2.5)
    z[:, ::997] += 9
    k = torch.tensor([1, 2, 3, 5, 10, 20, 50, 64, 100, 200, 500, 1000] * 2).int()
    p = torch.linspace(0.01, 0.9999, T)
    z = z.cuda()
    check(a3po, z, u, k=k)
    check(a3po, z, u, p=p)
    check(a3po, z, u, p=p, k=k, tau=torch.linspace(0.2, 1.5, T))
    check(a3po, z, u, min_p=torch.logspace(-12, -0.001, T))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5000, 60001])
def test_equal_logits_go_by_their_index(a3po, V, dt):
    """Whole logits between -2 and 2, many of each: borders lie inside a group of equal ones."""
    T = 12
    g = torch.Generator().manual_seed(V)
    z = torch.randint(-2, 3, (T, V), generator=g).to(DT[dt])
    z[0], z[1] = 1.0, -0.0
    z[1, ::2] = 0.0  # 0 and -0 are one
    k = torch.randint(1, V, (T,), generator=g).int()
    u, p = torch.rand(T, generator=g), torch.rand(T, generator=g)
    z = z.cuda()
    for cuts in (dict(k=k), dict(p=p), dict(k=k, p=p), dict(min_p=torch.full((T,), math.exp(-1.5))), dict(min_p=torch.ones(T)),
                 dict(tau=torch.zeros(T))):
        check(a3po, z, u, **cuts)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 40000])
def test_masked_entries_are_never_kept_or_drawn(a3po, V, dt):
    T = 16
    z, u, cuts = make(T, V, 5, dt)
    g = torch.Generator().manual_seed(6)
    for t in range(T):
        z[t, torch.rand(V, generator=g) < t / (T - 1)] = -math.inf
        z[t, (7 * t) % V] = float(t)
    z = z.cuda()
    check(a3po, z, u)
    check(a3po, z, u, **cuts)
    check(a3po, z, torch.full((T,), 1.0 - 2.0 ** -24), k=cuts["k"])
    check(a3po, z, torch.zeros(T), p=cuts["p"])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("V", [70, 20001])
def test_rows_without_a_policy(a3po, V, cut, dt):
    """No entry above -inf; NaN, +inf; parameters that are none.  Their neighbours are not touched."""
    T = 14
    z, u, _ = make(T, V, 8, dt)
    tau, k, p, min_p = torch.ones(T), torch.full((T,), 5).int(), torch.full((T,), 0.9), torch.full((T,), 0.01)
    z[1] = -math.inf
    z[3, V // 2] = math.nan
    z[5, V - 1] = math.inf
    tau[7], p[8], min_p[9], u[10], tau[11] = -1.0, math.nan, math.nan, math.nan, math.nan
    named = dict(temperature=tau.cuda())
    if cut:
        named.update(top_k=k.cuda(), top_p=p.cuda(), min_p=min_p.cuda())
    out = a3po.sample(z.cuda(), u.cuda(), want_logp_full=True, want_kept=True, want_allowed=True, **named)
    nan = [3, 5, 7, 10, 11] + ([8, 9] if cut else [])
    token, kept, bits = out["token"].cpu(), out["kept"].cpu(), unpack_bits(out["allowed"], V)
    for name in ("logp", "logp_full"):
        v = out[name].cpu()
        assert v[1] == -math.inf and v[nan].isnan().all()
    for t in range(T):
        if t in nan or t == 1:
            assert token[t] == -1 and kept[t] == 0 and not bits[t].any()
        else:
            want = reference_row(z[t].float().numpy(), float(u[t]), 1.0, 5 if cut else None, float(p[t]) if cut else None, float(min_p[t]) if cut else None)
            assert token[t] == want[1] and np.array_equal(bits[t, :V].astype(bool), want[0])


def test_the_ends_of_the_parameters(a3po):
    T, V = 9, 3001
    z, u, _ = make(T, V, 9)
    big = torch.tensor([0, -1, -2 ** 31, 1, V, V + 1, 2 ** 31 - 1, 2, 3]).int()
    p = torch.tensor([0.0, -1.0, 1.0, 2.0, 1e-30, 1 - 2.0 ** -24, math.inf, 0.5, -math.inf])
    min_p = torch.tensor([0.0, -1.0, 1.0, 2.0, 1e-38, 1 - 2.0 ** -24, 1e-45, -math.inf, math.inf])
    tau = torch.tensor([1e-30, 1e30, 1e-45, 1.0, 0.0, 5.0, 1e-3, 3e38, 1e3])
    z = z.cuda()
    for cuts in (dict(k=big), dict(p=p), dict(min_p=min_p), dict(tau=tau), dict(tau=tau, p=p), dict(tau=tau, min_p=min_p, k=big)):
        check(a3po, z, u, **cuts)
    check(a3po, z, torch.tensor([0.0, -1.0, 1.0, 2.0, 1 - 2.0 ** -24, 2.0 ** -149, math.inf, -math.inf, 0.5]))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_logits_far_from_zero_and_far_apart(a3po, dt):
    T, V = 6, 10000
    z, u, cuts = make(T, V, 10, dt)
    z[0] += 1e4
    z[1] -= 3e4
    z[2] *= 1e30
    z[3] *= 1e-30
    z[4, 5000:] = -3e38 if dt == "f32" else -3.3e38
    z[5] = torch.linspace(-80, 0, V).to(DT[dt])
    z = z.cuda()
    check(a3po, z, u)
    check(a3po, z, u, **cuts)
    check(a3po, z, u, p=cuts["p"])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(1000, 24, 0), (1000, 25, 1), (4099, 13, 3), (33, 1, 1), (30001, 7, 5)])
def test_strides_and_unaligned_rows(a3po, V, pad, shift, dt):
    """Rows in a wider buffer, starting anywhere; what lies between them would win if it were read."""
    T = 7
    buf = torch.full((T * (V + pad) + shift,), 1e30, dtype=DT[dt], device="cuda")
    z = buf[shift:].view(T, V + pad)
    inner, u, cuts = make(T, V, V, dt)
    z[:, :V] = inner.cuda()
    check(a3po, z, u, V=V)
    check(a3po, z, u, V=V, **cuts)


def test_many_draws_follow_the_policy(a3po):
    """4,096 evenly spaced numbers: the share of each token is its probability to one part in 4,096."""
    n, V = 4096, 500
    row = (2.0 * torch.randn(V, generator=torch.Generator().manual_seed(2))).cuda()
    u = (torch.arange(n, device="cuda") + 0.5) / n
    out = a3po.sample(row.expand(n, V).contiguous(), u, top_k=torch.full((n,), 40, dtype=torch.int32, device="cuda"))
    share = torch.bincount(out["token"].long(), minlength=V).double().cpu() / n
    best = torch.topk(row.double().cpu(), 40)
    want = torch.zeros(V, dtype=torch.float64).index_copy(0, best.indices, torch.softmax(best.values, 0))
    assert (share - want).abs().max() <= 1.0 / n + 1e-9


def test_kept_bits_give_training_the_cut_policy(a3po):
    """sample -> adjust_logits with its bits -> loss gradient: log-probs agree (each to 1e-5 (1 + |logp|), the library's bar), and
    gradients of entries that were cut are 0."""
    T, V = 64, 30011
    z, u, cuts = make(T, V, 21, "bf16")
    z, u, tau = z.cuda(), u.cuda(), cuts["tau"].cuda()
    out = a3po.sample(z, u, temperature=tau, top_k=torch.full((T,), 60, dtype=torch.int32, device="cuda"), top_p=cuts["p"].cuda(),
                      want_allowed=True)
    adjusted = a3po.adjust_logits(z, chosen=out["token"], temperature=tau, allowed=out["allowed"], out_dtype=torch.float32)
    assert ((adjusted["logp"] - out["logp"]).abs() <= 1e-5 * (1 + out["logp"].abs())).all()
    ones = torch.ones(T, device="cuda")
    loss = a3po.loss_fwd_bwd(adjusted["out"], out["token"], out["logp"], torch.zeros(T, dtype=torch.int32, device="cuda"), 1, ones,
                             torch.ones(T, dtype=torch.uint8, device="cuda"), 0.2)
    assert abs(float(loss["loss"]) + 1.0) <= 1e-4  # on policy: the mean of ratios of 1
    bits = torch.from_numpy(unpack_bits(out["allowed"], V)[:, :V].copy()).bool()
    assert (loss["dlogits"].cpu()[~bits] == 0).all()


def test_on_another_stream_and_in_a_graph(a3po):
    T, V = 40, 33000
    z, u, cuts = make(T, V, 30)
    z, u, tau, k, p = z.cuda(), u.cuda(), cuts["tau"].cuda(), cuts["k"].cuda(), cuts["p"].cuda()
    call = lambda: a3po.sample(z, u, temperature=tau, top_k=k, top_p=p, want_logp_full=True, want_kept=True, want_allowed=True)
    names = ("token", "logp", "logp_full", "kept", "allowed")
    eager = {n: call()[n].clone() for n in names}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = call()
    stream.synchronize()
    assert all(torch.equal(eager[n], other[n]) for n in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = call()
    for i in range(3):
        u.copy_(torch.rand(T, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], kept[n]) for n in names), i


def test_identical_calls_and_subsets_of_rows_agree(a3po):
    T, V = 33, 151936
    z, u, cuts = make(T, V, 31, "bf16", 1.0)
    z, u, p = z.cuda(), u.cuda(), cuts["p"].cuda()
    a = a3po.sample(z, u, top_p=p, want_allowed=True)
    b = a3po.sample(z, u, top_p=p, want_allowed=True)
    assert all(torch.equal(a[n], b[n]) for n in ("token", "logp", "allowed"))
    for t in (0, 17, 32):
        c = a3po.sample(z[t:t + 1], u[t:t + 1], top_p=p[t:t + 1], want_allowed=True)
        assert torch.equal(c["token"], a["token"][t:t + 1]) and torch.equal(c["allowed"], a["allowed"][t:t + 1])


def test_empty_calls(a3po):
    z = torch.empty(0, 100, device="cuda")
    out = a3po.sample(z, torch.empty(0, device="cuda"), want_kept=True, want_allowed=True)
    assert out["token"].shape == (0,) and out["allowed"].shape == (0, 4)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_borders_among_many_entries(a3po, dt):
    """Nuclei and counts of thousands to tens of thousands, borders in bins of up to all entries: rows that are flat, equal but for a
    few, in two levels, with a border far below the rest, with both cuts at once."""
    V, T = 70001, 10
    g = torch.Generator().manual_seed(41)
    z = torch.randn(T, V, generator=g) * torch.logspace(-4, 1, T)[:, None]
    z[1, 100:] = 0.25
    z[2] = torch.where(torch.rand(V, generator=g) < 0.5, 1.0, 0.75)
    z[3, :3] = 40.0
    z = z.to(DT[dt]).cuda()
    u = torch.rand(T, generator=g)
    many = torch.tensor([4863, 4864, 4865, 9727, 9728, 9729, 30000, 69999, 70000, 70001]).int()
    check(a3po, z, u, k=many)
    check(a3po, z, u, k=many, p=torch.linspace(0.05, 0.95, T))
    check(a3po, z, u, k=many.flip(0), min_p=torch.full((T,), 1e-3))
    for p in (0.3, 0.9, 0.999, 1 - 2.0 ** -20):
        check(a3po, z, u, p=torch.full((T,), p))
        check(a3po, z, u, p=torch.full((T,), p), min_p=torch.full((T,), 0.2), tau=torch.linspace(0.3, 2.0, T))


@pytest.mark.parametrize("cut", [False, True])
def test_more_parts_than_threads(a3po, cut):
    """A row longer than the kernels that go by parts take."""
    V = 4300000
    z, u, _ = make(2, V, 51, "bf16", 1.5)
    check(a3po, z.cuda(), u, **(dict(p=torch.tensor([0.01, 0.7]), k=torch.tensor([0, 100000]).int()) if cut else {}))


def test_offsets_beyond_32_bits(a3po):
    """The last rows of logits that fill more than 4 GiB are drawn as they are alone."""
    T, V = 18000, 120001
    z = torch.randn(T, V, dtype=torch.bfloat16, device="cuda")
    u = torch.rand(T, device="cuda")
    p = torch.full((T,), 0.8, device="cuda")
    names = ("token", "logp", "kept", "allowed")
    for cuts in ({}, dict(top_p=p)):
        whole = a3po.sample(z, u, want_kept=True, want_allowed=bool(cuts), **cuts)
        for a, b in ((0, 3), (T - 5, T)):
            part = a3po.sample(z[a:b].clone(), u[a:b], want_kept=True, want_allowed=bool(cuts), **{k: v[a:b] for k, v in cuts.items()})
            assert all(torch.equal(whole[n][a:b], part[n]) for n in names if part[n] is not None)


def test_two_streams_at_once(a3po):
    T, V = 64, 50000
    z, u, cuts = make(T, V, 61)
    z, u, p = z.cuda(), u.cuda(), cuts["p"].cuda()
    want = a3po.sample(z, u, top_p=p, want_allowed=True)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got += [a3po.sample(z, u, top_p=p, want_allowed=True) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(want[n], o[n]) for o in got for n in ("token", "logp", "allowed"))


def test_outputs_that_are_not_asked_for(a3po):
    z, u, cuts = make(9, 3000, 71)
    z, u, p = z.cuda(), u.cuda(), cuts["p"].cuda()
    for more in ({}, dict(top_p=p)):
        full = a3po.sample(z, u, want_logp_full=True, want_kept=True, want_allowed=True, **more)
        bare = a3po.sample(z, u, want_logp=False, **more)
        assert torch.equal(full["token"], bare["token"]) and all(bare[n] is None for n in ("logp", "logp_full", "kept", "allowed"))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_masks_of_the_lowest_value(a3po, dt):
    """Entries at the type's lowest value are entries, of no weight beside others: kept where nothing cuts them, never drawn; a row of
    nothing else is flat."""
    V, T = 40001, 8
    g = torch.Generator().manual_seed(81)
    low = torch.finfo(DT[dt]).min
    z = (torch.randn(T, V, generator=g) * 3).to(DT[dt])
    z[0] = low
    z[1, 1:] = low
    z[2, :-1] = low
    z[3, 5:30000] = low
    z[4] = torch.where(torch.rand(V, generator=g) < 0.999, torch.tensor(low, dtype=DT[dt]), z[4])
    z[5, ::2] = float("-inf")
    z[5, 1::2] = low
    z[6, 7] = -low
    z[7, 100:] = low
    z, u = z.cuda(), torch.rand(T, generator=g)
    check(a3po, z, u)
    check(a3po, z, u, tau=torch.linspace(0.5, 1.5, T))
    check(a3po, z, u, k=torch.full((T,), 200).int())
    check(a3po, z, u, p=torch.full((T,), 0.9))
    check(a3po, z, u, min_p=torch.full((T,), 0.1), tau=torch.full((T,), 1e-3))
    check(a3po, z, u, k=torch.full((T,), 20000).int(), p=torch.full((T,), 0.5), min_p=torch.full((T,), 1e-30))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("gap", [5.0, 21.0, 23.0, 40.0, 86.0, 90.0, 200.0])
def test_counts_that_end_far_below_the_largest(a3po, gap, dt):
    """A few entries lead by `gap`; the k-th is among the many behind them, as it is in rows that are nearly certain of a token."""
    V, T = 20011, 9
    g = torch.Generator().manual_seed(91)
    z = torch.randn(T, V, generator=g)
    for t in range(T):
        z[t, torch.randperm(V, generator=g)[:1 + t]] += gap
    z = z.to(DT[dt]).cuda()
    u = torch.rand(T, generator=g)
    k = torch.tensor([1, 2, 3, 5, 40, 50, 1000, 2400, 5000]).int()
    check(a3po, z, u, k=k)
    check(a3po, z, u, k=k, p=torch.linspace(0.3, 0.999999, T))
    check(a3po, z, u, k=k, min_p=torch.full((T,), math.exp(-gap - 1)), tau=torch.full((T,), 1.25))
    check(a3po, z, u, k=k, p=torch.full((T,), 0.9), min_p=torch.full((T,), 0.02), tau=torch.linspace(0.4, 1.6, T))
