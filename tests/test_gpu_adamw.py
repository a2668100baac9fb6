"""a3po_grad_norm and a3po_adamw_step against the definition in 64 bits.

Bars.  The norm is a 64-bit sum rounded once: 2^-24, and 2^-40 for the sum's own roundings.  m is three fp32 operations on terms no
larger than M = beta1 |m| + (1 - beta1) |g|, with the clip factor (five roundings) nine of 2^-24 M; v, whose terms are all
positive, twice the factor's and four more: 14 * 2^-24 v.  The update u = size m / (root sqrt(v) + eps): the kernel's root and
reciprocal are off by 1 ulp = 2^-23 each, constants and products by 2^-24: m's bar scaled, and 16 * 2^-24 |u|; p adds two roundings
of |p|.  What is stored in bfloat16 or float8 to nearest lies between the rounded ends of its bar; what is rounded by chance is one
of the two neighbours of a value within its bar, and its mean over many seeds is the value."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def within(got, ref, bar):
    return (got >= (ref - bar).to(got.dtype)) & (got <= (ref + bar).to(got.dtype))


def grid_floor(x, bits, lowest):
    """x >= 0 (64 bits) cut to `bits` bits of mantissa, exponents not below `lowest`; and the distance to the next."""
    e = torch.clamp(torch.frexp(x).exponent.double() - 1, min=lowest)
    step = torch.exp2(e - (bits - 1))
    return torch.floor(x / step) * step, step


def neighbours(got, ref, bar, bits, lowest):
    """got is one of the two neighbours, on the grid, of something within the bar of ref (magnitudes)."""
    low, _ = grid_floor((ref - bar).clamp(min=0), bits, lowest)
    high, step = grid_floor(ref + bar, bits, lowest)
    return (got >= low) & (got <= high + step)


def unit_of(scale, n):
    return torch.exp2(scale.cpu().double() - 127).repeat_interleave(32)[:n]


def make(n, seed, param, grad, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    s = torch.exp(spread * torch.randn(n, generator=g))
    return dict(p=torch.randn(n, generator=g).to(DT[param]), g=(1e-2 * s * torch.randn(n, generator=g)).to(DT[grad]),
                m=2e-3 * s * torch.randn(n, generator=g), v=1e-4 * s * s * torch.rand(n, generator=g))


def state_of(a3po, x, bits):
    """m and v of x in the format, on the GPU (8 bits: by a first step from zero with them as what is added)."""
    if bits == 32:
        return x["m"].cuda(), x["v"].cuda(), None
    n = x["m"].numel()
    unit = lambda t, top: torch.exp2(torch.floor(torch.log2(torch.nn.functional.pad(t.abs(), (0, -n % 32)).view(-1, 32).amax(1).clamp(min=1e-30))) - top)
    um, uv = unit(x["m"], 7), unit(x["v"], 14)
    m = (x["m"] / um.repeat_interleave(32)[:n]).to(torch.float8_e4m3fn)
    v = (x["v"] / uv.repeat_interleave(32)[:n]).clamp(min=2.0 ** -16).to(torch.float8_e5m2)
    return m.cuda(), v.cuda(), tuple((torch.log2(u) + 127).to(torch.uint8).cuda() for u in (um, uv))


def reference(p, g, m, v, step, factor=1.0, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1):
    """p, m, v in 64 bits, and their bars."""
    g = g.double() * factor
    M = beta1 * m.abs() + (1 - beta1) * g.abs()
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    below = torch.sqrt(v / (1 - beta2 ** step)) + eps
    size = lr / (1 - beta1 ** step)
    u = size * m / below
    bm, bv = 9 * U * M + 2.0 ** -148, 14 * U * v + 2.0 ** -148
    bp = size * bm / below + (16 * U + 7 * U) * u.abs() + 2 * U * (p.double().abs() + u.abs())
    return p.double() * (1 - lr * weight_decay) - u, m, v, bp, bm, bv


def check_step(a3po, sizes, param, grad, bits, step=7, clip=False, copy=False, seed=5, shift=0):
    xs = [make(n, 31 * i + n, param, grad) for i, n in enumerate(sizes)]
    place = lambda t: torch.cat([t.new_zeros(shift), t]).cuda()[shift:]  # (not on a line's beginning)
    ps, gs = [place(x["p"]) for x in xs], [place(x["g"]) for x in xs]
    states = [state_of(a3po, x, bits) for x in xs]
    if bits == 32:
        states = [(place(x["m"]), place(x["v"]), None) for x in xs]
        olds = [(s[0].cpu().double(), s[1].cpu().double()) for s in states]
    else:
        states = [(place(m.view(torch.uint8)).view(m.dtype), place(v.view(torch.uint8)).view(v.dtype), s) for m, v, s in states]
        olds = [tuple(a3po.adamw_state_values(s[i], s[2][i]).cpu().double() for i in (0, 1)) for s in states]
    copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in ps] if copy else None
    norm, factor = None, 1.0
    total = math.sqrt(sum(float(x["g"].double().square().sum()) for x in xs))
    if clip:
        norm = a3po.grad_norm(gs)
        assert abs(float(norm) - total) <= (U + 2.0 ** -40) * total
        factor = min(1.0, 0.3 / (total + 1e-6))
    a3po.adamw_step(ps, gs, [s[0] for s in states], [s[1] for s in states], scales=[s[2] for s in states] if bits == 8 else None,
                    copies=copies, step=step, norm=norm, max_norm=0.3, seed=seed, **HYPER)
    for i, x in enumerate(xs):
        n = sizes[i]
        p, m, v, bp, bm, bv = reference(x["p"], x["g"], *olds[i], step, factor, **HYPER)
        got = ps[i].cpu()
        assert torch.equal(gs[i].cpu(), x["g"])
        if param == "f32":
            assert within(got, p, bp).all(), n
        else:
            assert (neighbours(got.double().abs(), p.abs(), bp, 8, -126.0) & ((got.double() * p >= 0) | (p.abs() <= bp))).all(), n
        if copy:
            assert torch.equal(copies[i], ps[i].to(torch.bfloat16))
        gm, gv, scales = states[i]
        if bits == 32:
            assert within(gm.cpu(), m, bm).all() and within(gv.cpu(), v, bv).all(), n
            continue
        # the largest of a block lies between 2^7 and 2^8 (2^14 and 2^15) of its unit, but for its bar
        for got8, scale, ref, bar, top in ((gm, scales[0], m, bm, 7), (gv, scales[1], v, bv, 14)):
            big = torch.nn.functional.pad(ref.abs(), (0, -n % 32)).view(-1, 32).amax(1)
            unit = torch.exp2(scale.cpu().double() - 127)
            assert (big * (1 + 1e-5) >= unit * 2.0 ** top).logical_or(scale.cpu() == 1).all() and (big * (1 - 1e-5) < unit * 2.0 ** (top + 1)).all()
        unit = unit_of(scales[0], n)
        lo, hi = (((m + s * bm) / unit).float().to(torch.float8_e4m3fn).double() for s in (-1, 1))
        assert ((gm.cpu().double() >= lo) & (gm.cpu().double() <= hi)).all(), n
        unit = unit_of(scales[1], n)
        got8 = gv.cpu().double()
        assert neighbours(got8, v / unit, bv / unit, 3, -14.0).all() and ((got8 > 0) | (v <= bv)).all(), n


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n", [1, 7, 8, 31, 32, 33, 255, 2047, 2048, 2049, 70001])
def test_every_size(a3po, n, param, grad, bits):
    check_step(a3po, [n], param, grad, bits)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[5, 4096, 1, 33, 9000, 2048], [64] * 39, [64] * 40, [65] * 41, [3000 - 7 * i for i in range(205)], [100, 0, 3, 0]])
def test_many_tensors(a3po, sizes, bits):
    """More than one launch takes, empty ones among them; each is its own."""
    check_step(a3po, sizes, "f32", "bf16", bits, clip=True, copy=True)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("shift", [1, 3])
def test_tensors_at_any_element(a3po, shift, param, grad, bits):
    check_step(a3po, [5000, 40, 33], param, grad, bits, shift=shift, copy=True, clip=True)


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 7])
def test_first_and_late_steps(a3po, step):
    check_step(a3po, [3001], "f32", "f32", 32, step=step)
    check_step(a3po, [3001], "f32", "f32", 8, step=step)


def test_a_training_run_against_64_bits(a3po):
    """20 steps from zero states: each step adds its bar, so 40 times one step's is ample."""
    n = 5000
    x = make(n, 3, "f32", "f32")
    p, (m, v, _) = x["p"].cuda(), a3po.adamw_state(x["p"].cuda())
    rp, rm, rv = x["p"].double(), torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    g = torch.Generator().manual_seed(1)
    for step in range(1, 21):
        grad = 1e-2 * torch.randn(n, generator=g)
        a3po.adamw_step([p], [grad.cuda()], [m], [v], step=step, **HYPER)
        rp, rm, rv, bp, _, _ = reference(rp, grad, rm, rv, step, **HYPER)
    assert ((p.cpu().double() - rp).abs() <= 40 * bp + 1e-3 * 40 * 40 * U).all()


@pytest.mark.parametrize("what", ["param", "state"])
def test_roundings_by_chance_have_the_value_as_their_mean(a3po, what):
    """400 seeds of 2,000 elements: a rounding between neighbours a step apart has a variance of at most a quarter of its square,
    the mean over 400 seeds a deviation of at most step / 40; six of them bound 2,000 means."""
    n, seeds = 2000, 400
    x = make(n, 9, "bf16", "f32", spread=0.3)
    total, first = torch.zeros(n, dtype=torch.float64), None
    for seed in range(seeds):
        p, g = x["p"].cuda(), x["g"].cuda()
        m, v, scales = state_of(a3po, x, 8)
        old = a3po.adamw_state_values(m, scales[0]).cpu().double(), a3po.adamw_state_values(v, scales[1]).cpu().double()
        a3po.adamw_step([p], [g], [m], [v], scales=[scales], step=7, seed=seed, **HYPER)
        got = p.cpu().double() if what == "param" else a3po.adamw_state_values(v, scales[1]).cpu().double()
        total += got
        if first is not None and seed == 1:
            assert not torch.equal(first, got)
        first = got if seed == 0 else first
    ref = reference(x["p"], x["g"], *old, 7, **HYPER)
    value = ref[0] if what == "param" else ref[2]
    if what == "param":
        step = grid_floor(value.abs(), 8, -126.0)[1]
    else:
        unit = unit_of(scales[1], n)
        step = grid_floor(value / unit, 3, -14.0)[1] * unit
    inside = value.abs() > 4 * step if what == "param" else value / unit > 2.0 ** -12
    assert inside.float().mean() > 0.9
    assert ((total / seeds - value).abs() <= 6 * step / 40)[inside].all()


def test_seeds_tensors_and_elements_have_bits_of_their_own(a3po):
    """The same numbers everywhere: v halfway between two values goes up in about half of all places, differently by tensor and seed."""
    n = 4096
    def run(seed):
        ps = [torch.zeros(n, device="cuda") for _ in range(2)]
        gs = [torch.full((n,), math.sqrt(1.125 / 0.01), device="cuda") for _ in range(2)]
        st = [a3po.adamw_state(p, 8) for p in ps]
        a3po.adamw_step(ps, gs, [s[0] for s in st], [s[1] for s in st], scales=[s[2] for s in st], step=1, seed=seed, **HYPER)
        return [a3po.adamw_state_values(s[1], s[2][1]).cpu() > 1.1 for s in st]
    a, b = run(1), run(2)
    for u in a + b:
        assert abs(float(u.float().mean()) - 0.5) < 6 * 0.5 / math.sqrt(n)
    for u, w in ((a[0], a[1]), (a[0], b[0]), (a[1], b[0])):
        assert abs(float((u == w).float().mean()) - 0.5) < 6 * 0.5 / math.sqrt(n)
    c = run(1)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_8_bit_states_of_zeros_of_wide_ranges_and_of_tiny_values(a3po):
    n = 320
    g = torch.zeros(n)
    g[32:64] = torch.logspace(-12, 3, 32)
    g[64:96] = torch.logspace(-25, -18, 32)
    g[100], g[130], g[131] = 1.0, -1e18, 1e-18
    p = torch.ones(n, device="cuda")
    m, v, scales = a3po.adamw_state(p, 8)
    assert not a3po.adamw_state_values(m, scales[0]).any()
    a3po.adamw_step([p], [g.cuda()], [m], [v], scales=[scales], step=1, **HYPER)
    z = torch.zeros(n, dtype=torch.float64)
    rp, rm, rv, bp, bm, bv = reference(torch.ones(n), g, z, z, 1, **HYPER)
    assert within(p.cpu(), rp, bp).all()
    gm, gv = (a3po.adamw_state_values(t, s).cpu().double() for t, s in zip((m, v), scales))
    assert not gm[:32].any() and not gv[:32].any()
    block = lambda t: t.abs().view(-1, 32).amax(1, keepdim=True).expand(-1, 32).reshape(-1)
    # half a step of e4m3 (3 bits), or of the smallest number, 2^-9 of what 2^8 is above the block's largest
    assert ((gm - rm).abs() <= bm + (2.0 ** -4 * rm.abs()).maximum(block(rm) * 2.0 ** -17)).all()
    # a whole step of e5m2, or of its smallest number, 2^-16, in a unit that is 2^-14 of the block's largest; units are 2^-126 at
    # least, their smallest number 2^-142, which is what every smaller one above zero becomes
    assert ((gv - rv).abs() <= bv + (2.0 ** -2 * rv.abs()).maximum(block(rv) * 2.0 ** -29) + 2.0 ** -142).all()
    seen = (rv > 2.0 ** -126) & (rv > block(rv) * 1e-30)
    assert (gv[seen & (rv > 2.0 ** -110)] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_step_whose_norm_is_not_finite_changes_nothing(a3po, bad, bits):
    n = 1000
    x = make(n, 4, "f32", "f32")
    x["g"][777] = bad
    p, g = x["p"].cuda(), x["g"].cuda()
    m, v, scales = state_of(a3po, x, bits)
    copy = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    keep = [t.clone() for t in (p, m, v, copy, *(scales or ()))]
    norm = a3po.grad_norm([g])
    assert not math.isfinite(float(norm))
    named = dict(scales=None if scales is None else [scales], copies=[copy], step=3, **HYPER)
    a3po.adamw_step([p], [g], [m], [v], norm=norm, **named)
    raw = lambda t: t.view(torch.uint8)
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(keep, (p, m, v, copy, *(scales or ()))))
    # without the norm the damage is the element's, or its block's
    a3po.adamw_step([p], [g], [m], [v], **named)
    hurt = torch.isfinite(p.cpu()).logical_not()
    assert hurt.nonzero()[:, 0].tolist() in ([777], [])
    if bits == 8:
        values = a3po.adamw_state_values(m, scales[0]).cpu()
        assert values[768:800].isnan().all() and values[:768].isfinite().all() and values[800:].isfinite().all()


def test_norms(a3po):
    g = torch.Generator().manual_seed(2)
    for dt in ("f32", "bf16"):
        for sizes in ([1], [8191, 8192, 8193], [5] * 201, [100000, 0, 3], [3000000], [0], []):
            gs = [torch.randn(n, generator=g).to(DT[dt]) for n in sizes]
            total = math.sqrt(sum(float(t.double().square().sum()) for t in gs))
            a, b = (float(a3po.grad_norm([t.cuda() for t in gs], scale=-0.5)) for _ in range(2))
            assert a == b and abs(a - 0.5 * total) <= (U + 2.0 ** -40) * 0.5 * total
    assert abs(float(a3po.grad_norm([torch.full((100,), 3e38, device="cuda")], scale=1e-10)) - 3e29) <= 4 * U * 3e29


@pytest.mark.parametrize("bits", [32, 8])
def test_rate_and_step_on_the_device_and_replayed_graphs(a3po, bits):
    n = 5001
    x = make(n, 6, "f32", "f32")
    def fresh():
        m, v, scales = state_of(a3po, x, bits)
        return x["p"].cuda(), x["g"].cuda(), m.clone(), v.clone(), scales
    step, lr = torch.tensor([3], device="cuda"), torch.tensor([HYPER["lr"]], device="cuda")
    named = {k: v for k, v in HYPER.items() if k != "lr"}
    def call(s, **kw):
        p, g, m, v, scales = s
        norm = a3po.grad_norm([g])
        a3po.adamw_step([p], [g], [m], [v], scales=None if scales is None else [scales], norm=norm, **named, **kw)
    a, b = fresh(), fresh()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(b, step=step, lr=lr)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(a, step=step, lr=lr)
    c = fresh()
    raw = lambda t: t.view(torch.uint8)
    for i in range(3):
        graph.replay()
        call(c, step=step, lr=lr)
        torch.cuda.synchronize()
        assert all(torch.equal(raw(u), raw(w)) for u, w in zip(a[:4], c[:4])), i
        if i == 0:
            assert all(torch.equal(raw(u), raw(w)) for u, w in zip(a[:4], b[:4]))
            d = fresh()
            call(d, step=3, lr=float(lr))
            # the same numbers, computed on the host
            assert ((a[0] - d[0]).abs() <= 4 * U * d[0].abs()).all()
        step += 1
        lr *= 0.5


def test_no_tensors(a3po):
    a3po.adamw_step([], [], [], [], step=1, lr=0.1)
    p = torch.empty(0, device="cuda")
    m, v, s = a3po.adamw_state(p)
    a3po.adamw_step([p], [p], [m], [v], step=1, lr=0.1)
    assert float(a3po.grad_norm([])) == 0.0


def test_more_elements_than_32_bits_count(a3po):
    """A tensor of 2^31 + 1,000 elements: its last ones are updated as they are alone."""
    n, last = 2 ** 31 + 1000, 5000
    g = torch.Generator(device="cuda").manual_seed(1)
    p = torch.randn(n, generator=g, device="cuda")
    grad = torch.randn(n, generator=g, device="cuda", dtype=torch.bfloat16)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    tail = [t[-last:].clone() for t in (p, grad, m, v)]
    a3po.adamw_step([p], [grad], [m], [v], step=2, **HYPER)
    a3po.adamw_step([tail[0]], [tail[1]], [tail[2]], [tail[3]], step=2, **HYPER)
    assert torch.equal(p[-last:], tail[0]) and torch.equal(m[-last:], tail[2]) and torch.equal(v[-last:], tail[3])
    total = float(grad[:n // 2].double().square().sum() + grad[n // 2:].double().square().sum())
    assert abs(float(a3po.grad_norm([grad])) - math.sqrt(total)) <= (U + 2.0 ** -40) * math.sqrt(total)


def test_parameters_and_shapes_of_modules(a3po):
    """Tensors of any shape, parameters that want gradients among them, states in their shape."""
    p = torch.nn.Parameter(torch.randn(7, 5, 3, device="cuda"))
    grad = torch.randn(7, 5, 3, device="cuda")
    flat = p.detach().clone().view(-1)
    for bits in (32, 8):
        m, v, s = a3po.adamw_state(p, bits)
        assert m.shape == v.shape == p.shape
        fm, fv, fs = a3po.adamw_state(flat, bits)
        a3po.adamw_step([p], [grad], [m], [v], scales=None if s is None else [s], step=1, **HYPER)
        a3po.adamw_step([flat], [grad.view(-1)], [fm], [fv], scales=None if fs is None else [fs], step=1, **HYPER)
        assert torch.equal(p.detach().view(-1), flat)


def test_a_replayed_graph_draws_new_bits(a3po):
    """v halfway between two numbers at each replay: about half of the places go up each time, and not the same ones."""
    n = 4000
    p, g, m = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda")
    start = torch.full((n,), 2.0 ** 14 * 1.25, device="cuda").to(torch.float8_e5m2)
    v, scales = start.clone(), tuple(torch.full((n // 32,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    step = torch.tensor([1], device="cuda")
    call = lambda: a3po.adamw_step([p], [g], [m], [v], scales=[scales], step=step, lr=0.1, beta2=0.9)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    seen = []
    for i in range(3):
        v.copy_(start)
        step.fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        seen.append(a3po.adamw_state_values(v, scales[1]) > 2.0 ** 14 * 1.1)
        # 1.125 lies halfway between 1 and 1.25; six deviations of 4,000 coins
        assert abs(float(seen[-1].float().mean()) - 0.5) <= 6 * 0.5 / math.sqrt(n)
        for other in seen[:-1]:
            assert abs(float((seen[-1] == other).float().mean()) - 0.5) <= 6 * 0.5 / math.sqrt(n)


@pytest.mark.parametrize("bits", [32, 8])
def test_tables_of_tensors_cut_anywhere(a3po, bits):
    """More tensors than a launch takes, empty ones among them: each is updated as its place in the list alone says."""
    sizes = [(37 * i * i) % 5000 if i % 7 else 0 for i in range(250)]
    g = torch.Generator(device="cuda").manual_seed(8)
    ps = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    gs = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    def run(keep):
        mine = [p.clone() if i in keep else torch.empty(0, device="cuda") for i, p in enumerate(ps)]
        st = [a3po.adamw_state(p, bits) for p in mine]
        a3po.adamw_step(mine, [x if i in keep else x[:0] for i, x in enumerate(gs)], [s[0] for s in st], [s[1] for s in st],
                        scales=[s[2] for s in st] if bits == 8 else None, step=1, **HYPER)
        return mine, st
    raw = lambda t: t.view(torch.uint8)
    mine, st = run(range(250))
    for keep in (range(79, 82), range(159, 250), [0, 249], [1]):
        part, pst = run(keep)
        for i in keep:
            assert torch.equal(part[i], mine[i]) and torch.equal(raw(pst[i][0]), raw(st[i][0])) and torch.equal(raw(pst[i][1]), raw(st[i][1]))
        assert not sizes[keep[0]] or not torch.equal(part[keep[0]], ps[keep[0]])
