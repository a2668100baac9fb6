"""a3po_adjust_logits / a3po_adjust_logits_bwd against the definition in 64 bits, row by row.

Bars: an adjusted logit is at most eight fp32 operations on values no larger than M = (|z| max(rep, 1/rep) + frequency n +
presence + |bias|) / temperature: 8 * 2^-24 * M.  Log-sum-exp and log-probs are held to the library's 1e-5 (1 + |value|).  A
gradient element is three products: 4 * 2^-24 relative.  What is stored in a type D lies between D(value - bar) and
D(value + bar)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def within(got, ref, bar):
    """Rounding is monotone: what was rounded to got's type lies between the rounded ends of the bar."""
    return (got >= (ref - bar).to(got.dtype)) & (got <= (ref + bar).to(got.dtype))


def pack_bits(allowed):
    """bool [T, V] -> int32 words [T, ceil(V/32)]."""
    T, V = allowed.shape
    b = np.zeros((T, (V + 31) // 32 * 32), dtype=np.uint8)
    b[:, :V] = allowed.numpy()
    return torch.from_numpy(np.packbits(b, axis=1, bitorder="little").view(np.int32).copy())


def make(T, V, seed, most=200, bias="row", mask=True, prompt=True, share=False):
    """Logits and adjustments on the CPU.  Histories are ragged (empty ones among them) and hold tokens many times."""
    g = torch.Generator().manual_seed(seed)
    r = lambda lo, hi: lo + (hi - lo) * torch.rand(T, generator=g)
    n = torch.randint(0, most + 1, (T,), generator=g)
    n[torch.rand(T, generator=g) < 0.2] = 0
    start = torch.cumsum(n, 0) - n
    ids = (V * torch.rand(max(1, int(n.sum())), generator=g) ** 3).long().clamp_(max=V - 1)
    p = dict(history=ids.int(), hist_start=start.long(), hist_len=n.int(),
             prompt_len=(n * torch.rand(T, generator=g)).int() if prompt else None,
             repetition=r(0.8, 1.5), frequency=r(-0.2, 0.6), presence=r(-0.2, 0.8), temperature=r(0.5, 2.0), bias=None,
             allowed=None)
    if bias:
        p["bias"] = 3.0 * torch.randn(*((V,) if bias == "shared" else (T, V)), generator=g)
    ok = None
    if mask:
        ok = torch.rand(1 if share else T, V, generator=g) < 0.4
        p["allowed"] = pack_bits(ok)[0] if share else pack_bits(ok)
        ok = ok.expand(T, V)
    z = 4.0 * torch.randn(T, V, generator=g)
    return z, p, ok


def reference(z, p, ok):
    """u (64 bits), its bars, and the factor of the gradient."""
    T, V = z.shape
    u, M, f = z.double().clone(), torch.zeros(T, V, dtype=torch.float64), torch.ones(T, V, dtype=torch.float64)
    for t in range(T):
        count, seen = torch.zeros(V, dtype=torch.float64), torch.zeros(V, dtype=torch.bool)
        if p["history"] is not None:
            a, n = int(p["hist_start"][t]), int(p["hist_len"][t])
            k = int(p["prompt_len"][t]) if p["prompt_len"] is not None else 0
            total = p["history"].numel()
            tokens = p["history"][a:min(a + n, total)].long().tolist() if 0 <= a < total and n > 0 else []
            for i, v in enumerate(tokens):
                if 0 <= v < V:
                    seen[v] = True
                    count[v] += i >= k
        rep = 1.0 if p["repetition"] is None else float(p["repetition"][t])
        zt = z[t].double()
        f[t] = torch.where(seen, torch.where(zt > 0, 1.0 / rep, rep), torch.ones(()).double())
        off = (0.0 if p["frequency"] is None else float(p["frequency"][t])) * count
        off = off + (0.0 if p["presence"] is None else float(p["presence"][t])) * (count > 0)
        b = 0.0 if p["bias"] is None else (p["bias"] if p["bias"].dim() == 1 else p["bias"][t]).double()
        temp = 1.0 if p["temperature"] is None else float(p["temperature"][t])
        u[t] = (zt * f[t] - off + b) / temp
        M[t] = ((zt * f[t]).abs() + off.abs() + (b.abs() if torch.is_tensor(b) else 0.0)) / temp
        f[t] /= temp
    if ok is not None:
        u[~ok] = -math.inf
        f[~ok] = 0.0
    return u, 8 * U * M, f


def dev(p):
    return {k: None if v is None else v.cuda() for k, v in p.items()}


def check_forward(a3po, z, p, ok, ut, zg=None, out=None, write=True, V=None):
    T, n = z.shape
    u, bar, _ = reference(z, p, ok)
    g = torch.Generator().manual_seed(n)
    y = torch.randint(0, n, (T,), generator=g)
    if ok is not None and n > 1:
        y = torch.where(torch.rand(T, generator=g) < 0.8, torch.multinomial(ok.double() + 1e-9, 1, generator=g)[:, 0], y)
    r = a3po.adjust_logits(z.cuda() if zg is None else zg, V=V, chosen=y.int().cuda(), out=out, out_dtype=ut, write=write, **dev(p))
    torch.cuda.synchronize()
    if write:
        got = r["out"][:, :n].cpu()
        assert r["out"].dtype == ut and torch.equal(got.isinf(), u.isinf()) and torch.equal(got.isnan(), u.isnan())
        fine = u.isfinite()
        assert within(got[fine], u[fine], bar[fine] + 1e-37).all()
    else:
        assert r["out"] is None
    lse = torch.logsumexp(u, 1)
    above = u.amax(1).masked_fill(lse == -math.inf, 0.0)[:, None]   # (differences first: log n is nothing beside 1e38)
    logp = (u - above)[torch.arange(T), y] - torch.logsumexp(u - above, 1)
    logp = torch.where(lse == -math.inf, torch.full_like(lse, -math.inf), logp)
    for name, ref in (("lse", lse), ("logp", logp)):
        got = r[name].cpu().double()
        fine = ref.isfinite()
        assert torch.equal(got[~fine], ref[~fine]), name
        assert ((got - ref).abs()[fine] <= 1e-5 * (1 + ref.abs()[fine])).all(), name
    return r


def check_backward(a3po, z, p, ok, ut, du=None, dug=None, zg=None, out=None):
    T, V = z.shape
    _, _, f = reference(z, p, ok)
    if du is None:
        du = torch.randn(T, V, generator=torch.Generator().manual_seed(V)).to(ut)
    got = a3po.adjust_logits_bwd(du.cuda() if dug is None else dug, z.cuda() if zg is None else zg, dlogits=out, **dev(p))
    torch.cuda.synchronize()
    ref = du.double() * f
    assert got.dtype == z.dtype and within(got.cpu(), ref, 4 * U * ref.abs()).all()
    return got


# one part and many, every number of vectors a thread, ends inside a vector, fewer entries than lanes
WIDTHS = [1, 2, 7, 8, 31, 33, 500, 511, 513, 2047, 2049, 4097, 8191, 8193, 12289, 15872, 15873, 16385, 33003]


@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("zt,ut", PAIRS)
def test_every_width(a3po, V, zt, ut):
    z, p, ok = make(3, V, seed=V)
    z = z.to(DT[zt])
    check_forward(a3po, z, p, ok, DT[ut])
    check_backward(a3po, z, p, ok, DT[ut])


@pytest.mark.parametrize("T", [1, 2, 65, 300, 1100])
def test_numbers_of_rows(a3po, T):
    """From one row (many parts of one vector a thread) to rows that are one part or as few as fit."""
    V = 8200 if T <= 300 else 4200
    for zt, ut in PAIRS[:3]:
        z, p, ok = make(T, V, seed=T, most=60, bias="shared", share=T % 2 == 1)
        z = z.to(DT[zt])
        check_forward(a3po, z, p, ok, DT[ut])
        check_backward(a3po, z, p, ok, DT[ut])


def test_many_rows_of_the_widest_parts(a3po):
    z, p, ok = make(600, 40001, seed=8, most=900, bias=None)
    z = z.to(torch.bfloat16)
    check_forward(a3po, z, p, ok, torch.bfloat16)
    check_backward(a3po, z, p, ok, torch.bfloat16)
    check_forward(a3po, z, p, ok, torch.bfloat16, write=False)


FIELDS = ["history", "prompt_len", "repetition", "frequency", "presence", "temperature", "bias", "allowed"]


@pytest.mark.parametrize("only", FIELDS[2:] + [None])
@pytest.mark.parametrize("zt", ["bf16", "f32"])
def test_each_adjustment_alone(a3po, only, zt):
    z, p, ok = make(9, 3001, seed=11)
    z = z.to(DT[zt])
    keep = {only} | ({"history", "hist_start", "hist_len", "prompt_len"} if only in FIELDS[2:5] else set())
    p = {k: v if k in keep else None for k, v in p.items()}
    check_forward(a3po, z, p, ok if only == "allowed" else None, DT[zt])
    check_backward(a3po, z, p, ok if only == "allowed" else None, DT[zt])
    if only is None:  # nothing to adjust: the logits themselves, and what the log-prob kernel says of them
        r = a3po.adjust_logits(z.cuda(), chosen=torch.zeros(9, dtype=torch.int32, device="cuda"))
        lp, lse, _ = a3po.token_logprobs(z.cuda(), torch.zeros(9, dtype=torch.int32, device="cuda"))
        assert torch.equal(r["out"].cpu(), z) and torch.allclose(r["lse"], lse, rtol=1e-6) and torch.allclose(r["logp"], lp, rtol=1e-5)


def test_histories_of_all_kinds(a3po):
    """One token thousands of times, prompt and output of the same tokens, ids outside the vocabulary, ranges that leave the
    array at either end, negative lengths, rows that share their tokens."""
    V = 700
    z, p, ok = make(12, V, seed=12, mask=False)
    ids = torch.cat([torch.full((9000,), 5), torch.arange(-50, 2 * V), torch.arange(100).repeat(30)]).int()
    n = ids.numel()
    p["history"] = ids
    p["hist_start"] = torch.tensor([0, 0, 8990, 9000, 9000, n - 10, n - 1, n, -5, n + 100, 50, 10500])
    p["hist_len"] = torch.tensor([9000, n, 100, 1450, 700, 500, 2 ** 31 - 1, 10, 20, 5, -3, 3000], dtype=torch.int32)
    p["prompt_len"] = torch.tensor([8999, 0, 50, 1450, 2 ** 31 - 1, 5, 0, 0, 0, 0, 0, -7], dtype=torch.int32)
    for zt, ut in PAIRS:
        check_forward(a3po, z.to(DT[zt]), p, ok, DT[ut])
        check_backward(a3po, z.to(DT[zt]), p, ok, DT[ut])
    p["prompt_len"] = None
    check_forward(a3po, z, p, ok, torch.float32)


def test_sequences_that_share_their_tokens_as_growing_prefixes(a3po):
    T, V = 96, 5000
    z, p, ok = make(T, V, seed=13)
    p["history"] = torch.randint(0, V, (T,), dtype=torch.int32)
    p["hist_start"], p["hist_len"] = torch.arange(T) // 40 * 40, (torch.arange(T) % 40).int()
    p["prompt_len"] = p["hist_len"].clamp(max=6)
    check_forward(a3po, z, p, ok, torch.float32)
    check_backward(a3po, z, p, ok, torch.float32)


@pytest.mark.parametrize("zt", ["bf16", "f32"])
def test_masks_that_leave_little_or_nothing_and_extreme_logits(a3po, zt):
    V = 4500
    z, p, ok = make(10, V, seed=14, bias=None)
    p["history"] = None
    p["hist_start"] = p["hist_len"] = p["prompt_len"] = None
    ok = ok.clone()
    ok[0] = False                                   # nothing left
    ok[1] = False
    ok[1, V - 1] = True                             # the last entry alone
    ok[2] = True
    z = z.to(DT[zt])
    low = torch.finfo(DT[zt]).min
    z[3] = low                                      # masked by the type's lowest value
    z[4, ::2] = low
    z[5] = -math.inf
    z[6, ::3] = -math.inf
    z[7, ~ok[7]] = math.nan                         # whatever stands in a masked place
    z[8, ~ok[8]] = math.inf
    z[9] = 3e4
    p["temperature"] = torch.linspace(1.0, 2.0, 10)
    p["repetition"] = None
    p["allowed"] = pack_bits(ok)
    r = check_forward(a3po, z, p, ok, torch.float32)
    assert float(r["lse"][0]) == -math.inf and float(r["lse"][5]) == -math.inf
    du = torch.randn(10, V, generator=torch.Generator().manual_seed(1))
    du[7, ~ok[7]] = math.nan
    du[8, ~ok[8]] = math.inf
    got = a3po.adjust_logits_bwd(du.cuda(), None, dtype=DT[zt], **dev(p)).cpu()
    want = torch.where(ok, du.double() / p["temperature"].double()[:, None], torch.zeros(()).double())
    assert within(got, want, 4 * U * want.abs()).all()


def test_unmasked_nan_and_infinity_reach_their_own_row_only(a3po):
    z, p, ok = make(5, 3000, seed=15, mask=False)
    z[1, 2999], z[3, 5] = math.nan, math.inf
    r = a3po.adjust_logits(z.cuda(), **dev(p))
    lse = r["lse"].cpu()
    assert lse[[1, 3]].isnan().all() and lse[[0, 2, 4]].isfinite().all()
    assert r["out"][1, 2999].isnan() and r["out"][[0, 2, 4]].isfinite().all()


def test_invalid_chosen_ids_give_zero(a3po):
    z, p, _ = make(4, 1000, seed=16, mask=False)
    y = torch.tensor([-1, 1000, 2 ** 31 - 1, 999], dtype=torch.int32)
    logp = a3po.adjust_logits(z.cuda(), chosen=y.cuda(), **dev(p))["logp"].cpu()
    assert (logp[:3] == 0).all() and logp[3] < 0


@pytest.mark.parametrize("zt", ["bf16", "f32"])
@pytest.mark.parametrize("V,pad,shift", [(130, 5, 1), (9001, 3, 3), (20001, 0, 1)])
def test_strides_unaligned_rows_padding_and_in_place(a3po, zt, V, pad, shift):
    T = 4
    z, p, ok = make(T, V, seed=17)
    z = z.to(DT[zt])
    place = lambda fill, s: torch.full((T * (V + pad) + s,), fill, dtype=DT[zt], device="cuda")[s:].view(T, V + pad)
    zv, out = place(3.0, shift), place(7.0, 2 * shift)
    zv[:, :V] = z.cuda()
    check_forward(a3po, z, p, ok, DT[zt], zg=zv, out=out, V=V)
    assert (out[:, V:] == 7.0).all()
    check_forward(a3po, z, p, ok, DT[zt], zg=zv, out=zv, V=V)
    assert (zv[:, V:] == 3.0).all()
    du = torch.randn(T, V, generator=torch.Generator().manual_seed(2)).to(DT[zt])
    zv[:, :V] = z.cuda()
    out[:, :V] = du.cuda()
    check_backward(a3po, z, p, ok, DT[zt], du=du, dug=out[:, :V], zg=zv[:, :V], out=out[:, :V])
    assert pad == 0 or (out[:, V:] == 7.0).all()


def test_gradient_against_differences(a3po):
    """Of a smooth function of the adjusted logits, by central differences of the 64-bit definition."""
    T, V, h = 3, 40, 1e-5
    z, p, ok = make(T, V, seed=18, most=30)
    c = torch.randn(T, V, dtype=torch.float64, generator=torch.Generator().manual_seed(3))
    loss = lambda zz: (c * torch.exp(0.3 * reference(zz, p, ok)[0]))[ok].sum()
    u = reference(z.double(), p, ok)[0]
    du = torch.where(ok, 0.3 * c * torch.exp(0.3 * u.masked_fill(~ok, 0.0)), torch.zeros(()).double())
    got = a3po.adjust_logits_bwd(du.float().cuda(), z.cuda(), **dev(p)).cpu().double()
    for t in range(T):
        for v in range(V):
            lo, hi = z.double().clone(), z.double().clone()
            lo[t, v] -= h
            hi[t, v] += h
            d = float((loss(hi) - loss(lo)) / (2 * h))
            assert abs(float(got[t, v]) - d) <= 1e-5 * (1 + abs(d)), (t, v)


def test_gradient_through_the_adjusted_policy_s_loss(a3po):
    """Adjust, loss, gradient back, in place: the row gradients of log-probs of the adjusted policy."""
    T, V = 20, 6000
    z, p, ok = make(T, V, seed=19)
    ok = ok.clone()
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(4))
    ok[torch.arange(T), y] = True
    p["allowed"] = pack_bits(ok)
    d = dev(p)
    zg, yg = z.cuda(), y.int().cuda()
    u = a3po.adjust_logits(zg, chosen=yg, **d)
    f = lambda v: torch.full((T,), v, device="cuda")
    adv = torch.linspace(-1, 1, T).cuda()
    r = a3po.loss_fwd_bwd(u["out"], yg, u["logp"], None, 0, adv, torch.ones(T, dtype=torch.uint8, device="cuda"), 0.2,
                          dlogits=u["out"], prox_mode=2)
    assert torch.allclose(r["logp"], u["logp"], rtol=1e-5, atol=1e-5)
    got = a3po.adjust_logits_bwd(r["dlogits"], zg, dlogits=r["dlogits"], **d).cpu().double()
    ud, _, fac = reference(z, p, ok)
    onehot = torch.zeros(T, V, dtype=torch.float64)
    onehot[torch.arange(T), y] = 1.0
    want = -(adv.cpu().double() / T)[:, None] * (onehot - torch.softmax(ud, 1)) * fac
    assert ((got - want).abs() <= 2e-5 * (adv.cpu().double().abs() / T)[:, None] * fac.abs() + 1e-12).all()


def test_on_another_stream_and_in_a_graph(a3po):
    z, p, _ = make(8, 10000, seed=20)
    d = dev(p)
    zg = z.to(torch.bfloat16).cuda()
    out = torch.empty(8, 10000, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(a3po.workspace_bytes(8, 10000, which=a3po.A3PO_WS_ADJUST_LOGITS), dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(s):
        a3po.adjust_logits(zg, out=out, workspace=ws, **d)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = a3po.adjust_logits(zg, out=out, workspace=ws, **d)
    for i in range(3):
        zg.copy_(torch.randn(8, 10000, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))
        want = a3po.adjust_logits(zg, out_dtype=torch.float32, **d)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want["out"]) and torch.equal(r["lse"], want["lse"]), i


def test_empty_calls(a3po):
    e = torch.empty((0, 100), device="cuda")
    r = a3po.adjust_logits(e, temperature=torch.empty(0, device="cuda"))
    assert r["out"].shape == (0, 100) and r["lse"].shape == (0,)
    assert a3po.adjust_logits_bwd(e).shape == (0, 100)


@pytest.mark.parametrize("zt", ["f32", "bf16"])
@pytest.mark.parametrize("level,temperature", [(-1e30, 1.0), (1e9, 1.0), (-3e7, 1e-3), (7.0, 1e-12), (1e6, 1.0)])
def test_values_far_from_zero_whose_scaled_maximum_rounds_coarsely(a3po, zt, level, temperature):
    T, V = 4, 1500
    g = torch.Generator().manual_seed(3)
    z = (level * (1 + 1e-2 * torch.rand(T, V, generator=g))).to(DT[zt])
    z[1] = level                                    # ties throughout
    z[2, V // 2] = level + abs(level) / 2           # one ahead of the others
    p = dict(history=None, hist_start=None, hist_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
             temperature=torch.full((T,), temperature), bias=None, allowed=None)
    check_forward(a3po, z, p, None, torch.float32)


def test_more_rows_than_workgroups(a3po):
    T, V = (1 << 20) + 700, 9
    g = torch.Generator(device="cuda").manual_seed(1)
    z = 4 * torch.randn(T, V, device="cuda", generator=g)
    y = torch.randint(-1, V, (T,), device="cuda", generator=g, dtype=torch.int32)
    temperature = 0.5 + torch.rand(T, device="cuda", generator=g)
    r = a3po.adjust_logits(z, chosen=y, temperature=temperature, write=False)
    u = z.double() / temperature.double()[:, None]
    ref = torch.log_softmax(u, 1).gather(1, y.clamp(min=0).long()[:, None])[:, 0].masked_fill(y < 0, 0.0)
    for got, ref in ((r["logp"], ref), (r["lse"], torch.logsumexp(u, 1))):
        assert ((got.double() - ref).abs() <= 1e-5 * (1 + ref.abs())).all()


@pytest.mark.parametrize("T,V,zt,ut,write", [(600, 1000, "bf16", "bf16", True), (700, 517, "f32", "f32", True), (600, 1000, "bf16", "f32", False),
                                             (1025, 130, "f32", "bf16", True), (1025, 131, "bf16", "bf16", False), (300, 33001, "bf16", "bf16", True),
                                             (530, 66001, "bf16", "bf16", False)])
def test_many_rows_some_with_long_histories(a3po, T, V, zt, ut, write):
    """Rows enough for the smaller workgroups; histories with more tokens, and more distinct ones, than are noted or numbered at
    a time."""
    z, p, ok = make(T, V, seed=T + V, most=20)
    g = torch.Generator().manual_seed(T)
    longer = (V * torch.rand(14000, generator=g)).int()
    p["hist_start"][1], p["hist_len"][1] = p["history"].numel(), 14000
    p["hist_start"][T - 1], p["hist_len"][T - 1] = p["history"].numel() + 500, 9001
    p["prompt_len"][1], p["prompt_len"][T - 1] = 6000, 0
    p["history"] = torch.cat((p["history"], longer))
    check_forward(a3po, z.to(DT[zt]), p, ok, DT[ut], write=write)


@pytest.mark.parametrize("V", [700, 40001])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_row_s_nan_shows_in_the_log_prob_of_a_token_that_is_masked(a3po, V, bad):
    """NaN or +inf in an unmasked place: the row's log-sum-exp is NaN, and no log-prob of the row is a number, that of a masked
    token, or of one with -inf for a logit, among them.  Rows in one part and in many."""
    T = 6
    z, p, _ = make(T, V, seed=31, bias=None, mask=False)
    ok = torch.ones(T, V, dtype=torch.bool)
    ok[:, 3] = False
    z[:, 5] = -math.inf
    z[1::2, V - 2] = bad
    p["allowed"] = pack_bits(ok)
    for token in (3, 5):
        y = torch.full((T,), token, dtype=torch.int32, device="cuda")
        r = a3po.adjust_logits(z.cuda(), chosen=y, write=False, **dev(p))
        lse, logp = r["lse"].cpu(), r["logp"].cpu()
        assert lse[1::2].isnan().all() and logp[1::2].isnan().all(), token
        assert lse[::2].isfinite().all() and (logp[::2] == -math.inf).all(), token


# ---- rows whole at full vocabularies --------------------------------------------------------------------------------------


def _wide(T, V, zt, seed, tokens):
    """Logits and adjustments on the GPU, every row with `tokens` of history from one array, some with far more."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda lo, hi: lo + (hi - lo) * torch.rand(T, device="cuda", generator=g)
    z = 4.0 * torch.randn(T, V, device="cuda", generator=g, dtype=DT[zt])
    n = torch.randint(0, tokens + 1, (T,), device="cuda", generator=g, dtype=torch.int32)
    n[1], n[T // 2], n[T - 1] = 30000, 9001, 0      # (more than the lists and numbers of a workgroup hold, and nothing)
    ids = torch.cat(((V * torch.rand(20000, device="cuda", generator=g) ** 3).int(),
                     torch.randint(0, V, (20000,), device="cuda", generator=g, dtype=torch.int32)))
    start = torch.randint(0, 10000, (T,), device="cuda", generator=g)
    p = dict(history=ids, hist_start=start, hist_len=n, prompt_len=(n * rand(0, 1)).int(), repetition=rand(0.8, 1.5),
             frequency=rand(-0.2, 0.6), presence=rand(-0.2, 0.8), temperature=rand(0.5, 2.0),
             bias=3.0 * torch.randn(V, device="cuda", generator=g),
             allowed=torch.randint(-2 ** 31, 2 ** 31, (T, (V + 31) // 32), device="cuda", generator=g).int())
    y = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
    y[3] = ids[start[1] + 12000]
    rows = torch.unique(torch.cat((torch.tensor([0, 1, 2, 3, T // 2, T - 2, T - 1]), torch.randint(0, T, (8,)))))
    return z, p, y, rows.cuda()


def _rows_of(z, p, rows):
    """The rows' share of the arguments on the CPU, for `reference`."""
    ok = (p["allowed"][rows][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    own = {k: v if k in ("history", "bias") else v[rows] for k, v in p.items()}
    return z[rows].cpu(), {k: v.cpu() for k, v in own.items()}, ok.view(len(rows), -1)[:, :z.shape[1]].bool().cpu()


@pytest.mark.parametrize("T,V", [(1030, 70001), (1030, 131073), (1024, 151936), (1025, 262144), (1030, 262145)])
@pytest.mark.parametrize("zt,ut,write", [("bf16", "bf16", True), ("bf16", "f32", True), ("f32", "f32", True), ("bf16", "bf16", False)])
def test_rows_taken_whole_at_full_vocabularies(a3po, T, V, zt, ut, write):
    '''From 1,024 rows on they are one part each, up to 262,144 entries: the longest bits, half as many numbers, the shortest
    lists, and workgroups of 512 threads beyond 131,072.'''
    z, p, y, rows = _wide(T, V, zt, V, 600)
    r = a3po.adjust_logits(z, chosen=y, write=write, out_dtype=DT[ut], **p)
    zs, ps, ok = _rows_of(z, p, rows)
    u, bar, _ = reference(zs, ps, ok)
    if write:
        got = r["out"][rows].cpu()
        fine = u.isfinite()
        assert torch.equal(got[~fine].double(), u[~fine]) and within(got[fine], u[fine], bar[fine]).all()
    lse = torch.logsumexp(u, 1)
    logp = u[torch.arange(len(rows)), y[rows].long().cpu()] - lse
    for name, ref in (("lse", lse), ("logp", logp)):
        got, fine = r[name][rows].cpu().double(), ref.isfinite()
        assert torch.equal(got[~fine], ref[~fine]) and ((got - ref).abs()[fine] <= 1e-5 * (1 + ref.abs()[fine])).all(), name


@pytest.mark.parametrize("T,V,zt,ut", [(4100, 65535, "bf16", "bf16"), (2050, 131072, "bf16", "f32"), (1030, 151936, "f32", "f32"),
                                       (4100, 65537, "bf16", "f32")])
def test_gradients_of_the_widest_parts(a3po, T, V, zt, ut):
    z, p, _, rows = _wide(T, V, zt, V, 600)
    du = torch.randn(T, V, device="cuda", dtype=DT[ut], generator=torch.Generator(device="cuda").manual_seed(5))
    got = a3po.adjust_logits_bwd(du, z, **p)[rows].cpu()
    zs, ps, ok = _rows_of(z, p, rows)
    ref = du[rows].cpu().double() * reference(zs, ps, ok)[2]
    assert within(got, ref, 4 * U * ref.abs()).all()


@pytest.mark.parametrize("zt,ut", PAIRS)
@pytest.mark.parametrize("T,V", [(3, 9001), (300, 1025), (1100, 500)])
def test_what_is_not_finite_has_its_sign(a3po, zt, ut, T, V):
    '''A masked entry is -inf and nothing else, in the history or not, whatever stood there; an unmasked infinity keeps its sign.'''
    z, p, ok = make(T, V, seed=21, most=80)
    z = z.to(DT[zt])
    z[0, ~ok[0]] = math.inf
    z[1, ~ok[1]] = math.nan
    z[2, ::5] = -math.inf
    z[2, 2::5] = math.inf
    p["repetition"].clamp_(min=1.0)
    u, _, _ = reference(z, p, ok)
    got = a3po.adjust_logits(z.cuda(), out_dtype=DT[ut], **dev(p))["out"].cpu().double()
    assert torch.equal(got[~ok], torch.full_like(got[~ok], -math.inf))
    assert torch.equal(got.isposinf(), u.isposinf()) and torch.equal(got.isneginf(), u.isneginf())
    assert u.isposinf().any() and not got.isnan().any()


def test_gradient_on_another_stream_and_in_a_graph(a3po):
    z, p, _ = make(8, 10000, seed=22)
    d, zg = dev(p), z.to(torch.bfloat16).cuda()
    du, out = torch.randn(8, 10000, device="cuda"), torch.empty(8, 10000, dtype=torch.bfloat16, device="cuda")
    want = a3po.adjust_logits_bwd(du, zg, **d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a3po.adjust_logits_bwd(du, zg, dlogits=out, **d)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a3po.adjust_logits_bwd(du, zg, dlogits=out, **d)
    for i in range(3):
        du.copy_(torch.randn(8, 10000, generator=torch.Generator().manual_seed(i)))
        want = a3po.adjust_logits_bwd(du, zg, **d)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
