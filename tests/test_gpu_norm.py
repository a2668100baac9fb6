"""a3po_norm_fwd / a3po_norm_bwd against the formulas in 64 bits.

Bars, with u = 2^-24 (fp32 arithmetic): a normed element carries the roundings of x - mean (u (|x| + mean|x|) rstd), of rstd and of the sums behind both, each of which is a tree
over at most 32 serial additions and ten levels: 128 u (1 + mean|x| rstd) relative.  Sums over rows are at most 128 serial
additions: 128 u of the sum of magnitudes.  An output stored in a type D lies between D(value - bar) and D(value + bar)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# one wavefront a row, every number of vectors; four and sixteen wavefronts a row; elements behind the last vector
WIDTHS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 511, 512, 513, 896, 1025, 1536, 2047, 2048, 2049, 2055, 2056, 4095, 4096, 4103,
          4104, 6145, 8191, 8192, 8200, 8211, 12289, 16383, 16384]


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


def _inputs(T, H, xt, pt, seed, offset=0.3, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, H + pad, generator=g) * (0.3 + 3.0 * torch.rand(T, 1, generator=g)) + offset).to(xt)
    w, b = (1.0 + 0.3 * torch.randn(H, generator=g)).to(pt), (0.2 * torch.randn(H, generator=g)).to(pt)
    return x, w, b, g


def _forward(x, w, b, eps, layer):
    x = x.double()
    mean = x.mean(1) if layer else torch.zeros(x.shape[0], dtype=torch.float64)
    c = x - mean[:, None]
    rstd = ((c * c).mean(1) + eps) ** -0.5
    xhat = c * rstd[:, None]
    return xhat * w.double() + (b.double() if b is not None else 0.0), mean, rstd, xhat


def _forward_bars(x, w, b, rstd, xhat, y):
    ax = x.double().abs()
    spread = 1.0 + ax.mean(1) * rstd
    wd = w.double().abs()
    bar = (128 * U * spread)[:, None] * (xhat.abs() * wd) + 64 * U * rstd[:, None] * (ax + ax.mean(1, keepdim=True)) * wd
    bar = bar + 4 * U * (y.abs() + (b.double().abs() if b is not None else 0.0)) + 1e-30
    return bar, 128 * U * spread


def _check_forward(a3po, x, w, b, layer, yt, eps=1e-6, out=None):
    dev = x.cuda() if out is None else out[0]
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    y, mean, rstd = a3po.norm_fwd(dev, w.cuda(), None if b is None else b.cuda(), eps=eps, kind=kind,
                                  out=None if out is None else out[1], out_dtype=yt)
    torch.cuda.synchronize()
    ref, m, r, xhat = _forward(x, w, b, eps, layer)
    bar, rel = _forward_bars(x, w, b, r, xhat, ref)
    assert y.dtype == yt and within(y.cpu(), ref, bar).all()
    assert ((rstd.cpu().double() - r).abs() <= rel * r).all()
    if layer:
        assert ((mean.cpu().double() - m).abs() <= 64 * U * x.double().abs().mean(1)).all()
    else:
        assert mean is None


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_forward_every_width(a3po, H, layer, xt, yt):
    x, w, b, _ = _inputs(5, H, DT[xt], DT[xt], seed=H)
    _check_forward(a3po, x, w, b if layer else None, layer, DT[yt])


@pytest.mark.parametrize("T", [1, 3, 4, 257, 5000])
def test_forward_numbers_of_rows_parameter_types_and_none(a3po, T):
    for pt in (torch.float32, torch.bfloat16):
        x, w, b, _ = _inputs(T, 130, torch.bfloat16, pt, seed=T)
        _check_forward(a3po, x, w, b, True, torch.bfloat16)
    y = a3po.norm_fwd(x.cuda(), kind=a3po.A3PO_NORM_RMS, want_stats=False)
    assert y[1] is None and y[2] is None
    ref, _, r, xhat = _forward(x, torch.ones(130), None, 1e-6, False)
    bar, _ = _forward_bars(x, torch.ones(130), None, r, xhat, ref)
    assert within(y[0].cpu(), ref, bar).all()


def test_more_rows_than_the_grid_has_workgroups(a3po):
    x, w, b, _ = _inputs(40000, 24, torch.float32, torch.float32, seed=9)
    _check_forward(a3po, x, w, b, True, torch.float32)


def test_rows_with_large_means_equal_rows_and_zero_rows(a3po):
    x, w, b, _ = _inputs(6, 300, torch.float32, torch.float32, seed=1)
    x[0] += 1e4          # the variance is that of the differences: digits are lost to x - mean alone
    x[1] = 7.25          # no spread: xhat 0, y = bias
    x[2] = 0.0
    _check_forward(a3po, x, w, b, True, torch.float32)
    _check_forward(a3po, x, w, None, False, torch.float32)
    y, _, rstd = a3po.norm_fwd(x.cuda(), w.cuda(), b.cuda())
    assert torch.equal(y[1].cpu(), b) and float(rstd[2]) == pytest.approx(1e3, rel=1e-5)


def test_non_finite_rows_stay_in_their_rows(a3po):
    x, w, b, _ = _inputs(8, 200, torch.float32, torch.float32, seed=2)
    x[3, 17], x[5, 199] = float("nan"), float("inf")
    y = a3po.norm_fwd(x.cuda(), w.cuda(), b.cuda())[0].cpu()
    assert y[3].isnan().all() and y[5].isnan().any() and y[[0, 1, 2, 4, 6, 7]].isfinite().all()


@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("H,pad,shift", [(65, 3, 1), (2049, 2, 1), (4100, 1, 3), (9000, 7, 5)])
def test_strides_unaligned_rows_and_in_place(a3po, xt, H, pad, shift):
    x, w, b, _ = _inputs(7, H, DT[xt], torch.float32, seed=3, pad=pad)
    flat = torch.empty(7 * (H + pad) + shift, dtype=DT[xt], device="cuda")
    view = flat[shift:].view(7, H + pad)
    view.copy_(x.cuda())
    before = view.cpu().clone()
    ldy = H + 5
    out = torch.full((7 * ldy + 1,), 7.0, dtype=DT[xt], device="cuda")[1:].view(7, ldy)
    _check_forward(a3po, x[:, :H], w, b, True, DT[xt], out=(view[:, :H], out[:, :H]))
    assert torch.equal(view.cpu(), before) and (out[:, H:] == 7.0).all()
    _check_forward(a3po, x[:, :H], w, b, True, DT[xt], out=(view[:, :H], view[:, :H]))
    assert torch.equal(view[:, H:].cpu(), before[:, H:])


# ---- backward --------------------------------------------------------------------------------------------------------


def _backward(dy, x, w, mean, rstd, layer):
    dy, x, r = dy.double(), x.double(), rstd.double()[:, None]
    xhat = (x - mean.double()[:, None]) * r if layer else x * r
    g = dy * w.double()
    along = (g * xhat).mean(1, keepdim=True)
    level = g.mean(1, keepdim=True) if layer else torch.zeros_like(along)
    dx = r * (g - level - xhat * along)
    # the bars: roundings of xhat, of the two means and of the difference
    m = mean.double().abs()[:, None] if layer else 0.0
    off = 64 * U * r * (x.abs() + m)
    terms = g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True)
    bar = r * (128 * U * terms + off * along.abs() + (g.abs() * off).mean(1, keepdim=True) * xhat.abs()) + 1e-30
    dw, db = (dy * xhat).sum(0), dy.sum(0)
    return dx, bar, dw, 128 * U * (dy * xhat).abs().sum(0) + (dy.abs() * off).sum(0) + 1e-30, db, \
        128 * U * dy.abs().sum(0) + 1e-30


def _check_backward(a3po, x, w, dy, layer, eps=1e-6, dx=None, dev=None):
    _, mean, rstd, _ = _forward(x, w, None, eps, layer)
    mean, rstd = mean.float(), rstd.float()
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    xg, dyg = (x.cuda(), dy.cuda()) if dev is None else dev
    out = a3po.norm_bwd(dyg, xg, w.cuda(), rstd.cuda(), mean=mean.cuda() if layer else None, kind=kind, want_dbias=layer, dx=dx)
    torch.cuda.synchronize()
    ref, bar, dw, dwbar, db, dbbar = _backward(dy, x, w, mean, rstd, layer)
    assert out["dx"].dtype == x.dtype and within(out["dx"].cpu(), ref, bar).all()
    assert ((out["dweight"].cpu().double() - dw).abs() <= dwbar).all()
    if layer:
        assert ((out["dbias"].cpu().double() - db).abs() <= dbbar).all()
    return out


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_backward_every_width(a3po, H, layer, xt, yt):
    x, w, _, g = _inputs(6, H, DT[xt], DT[xt], seed=H + 1)
    _check_backward(a3po, x, w, torch.randn(6, H, generator=g).to(DT[yt]), layer)


@pytest.mark.parametrize("T", [1, 2, 511, 512, 513, 2049, 5003])
@pytest.mark.parametrize("H", [72, 2304])
def test_backward_numbers_of_rows(a3po, T, H):
    x, w, _, g = _inputs(T, H, torch.bfloat16, torch.float32, seed=T)
    dy = torch.randn(T, H, generator=g).to(torch.bfloat16)
    a = _check_backward(a3po, x, w, dy, True)
    b = _check_backward(a3po, x, w, dy, True)
    for k in ("dx", "dweight", "dbias"):
        assert torch.equal(a[k], b[k]), k     # one order of summation


def test_backward_against_differences(a3po):
    """d/dx, d/dw, d/db of sum(dy * y) by central differences of the 64-bit forward pass (error h^2 = 1e-8 times third
    derivatives of order 10)."""
    T, H, h = 3, 13, 1e-4
    x, w, b, g = _inputs(T, H, torch.float32, torch.float32, seed=4)
    dy = torch.randn(T, H, generator=g)
    for layer in (True, False):
        f = lambda xx, ww, bb: (dy.double() * _forward(xx, ww, bb if layer else None, 1e-6, layer)[0]).sum()
        args = [x.double(), w.double(), b.double()]
        grads = []
        for i, a in enumerate(args):
            d = torch.zeros_like(a)
            for at in np.ndindex(*a.shape):
                lo, hi = a.clone(), a.clone()
                lo[at] -= h
                hi[at] += h
                d[at] = (f(*args[:i], hi, *args[i + 1:]) - f(*args[:i], lo, *args[i + 1:])) / (2 * h)
            grads.append(d)
        out = _check_backward(a3po, x, w, dy, layer)
        for name, d in zip(("dx", "dweight", "dbias") if layer else ("dx", "dweight"), grads):
            assert ((out[name].cpu().double() - d).abs() <= 1e-5 * (1 + d.abs())).all(), name


@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("H,pad,shift", [(65, 3, 1), (2049, 2, 1), (4100, 1, 3), (9000, 7, 5)])
def test_backward_strides_unaligned_rows_and_in_place(a3po, xt, H, pad, shift):
    T = 9
    x, w, _, g = _inputs(T, H, DT[xt], torch.float32, seed=5, pad=pad)
    dy = torch.randn(T, H, generator=g).to(DT[xt])
    place = lambda t, fill: torch.full((T * (H + pad) + shift,), fill, dtype=DT[xt], device="cuda")[shift:].view(T, H + pad)
    xv, dyv, dxv = place(x, 0.0), place(dy, 3.0), place(dy, 7.0)
    xv.copy_(x.cuda())
    dyv[:, :H] = dy.cuda()
    _check_backward(a3po, x[:, :H], w, dy, True, dx=dxv[:, :H], dev=(xv[:, :H], dyv[:, :H]))
    assert (dxv[:, H:] == 7.0).all()
    _check_backward(a3po, x[:, :H], w, dy, True, dx=dyv[:, :H], dev=(xv[:, :H], dyv[:, :H]))     # over dy
    assert (dyv[:, H:] == 3.0).all()
    dyv[:, :H] = dy.cuda()
    _check_backward(a3po, x[:, :H], w, dy, True, dx=xv[:, :H], dev=(xv[:, :H], dyv[:, :H]))      # over x
    assert torch.equal(xv[:, H:].cpu(), x[:, H:])


def test_sums_accumulate_are_optional_and_cleared_by_empty_calls(a3po):
    x, w, _, g = _inputs(700, 96, torch.float32, torch.float32, seed=6)
    dy = torch.randn(700, 96, generator=g)
    _, mean, rstd, _ = _forward(x, w, None, 1e-6, True)
    d = lambda t: t.float().cuda()
    whole = a3po.norm_bwd(d(dy), d(x), d(w), d(rstd), mean=d(mean), want_dbias=True)
    dw, db = torch.full((96,), 5.0, device="cuda"), torch.full((96,), 5.0, device="cuda")
    for i, (lo, hi) in enumerate([(0, 300), (300, 300), (300, 700)]):
        part = a3po.norm_bwd(d(dy[lo:hi]), d(x[lo:hi]), d(w), d(rstd[lo:hi]), mean=d(mean[lo:hi]), dweight=dw, dbias=db,
                             accumulate=i > 0)
        assert torch.equal(part["dx"], whole["dx"][lo:hi])
    bar = 256 * U * (dy.abs() * 5).sum(0).cuda()
    assert ((dw - whole["dweight"]).abs() <= bar).all() and ((db - whole["dbias"]).abs() <= bar).all()
    only = a3po.norm_bwd(d(dy), d(x), d(w), d(rstd), mean=d(mean), want_dweight=False, want_dbias=True)
    assert only["dweight"] is None and torch.equal(only["dbias"], whole["dbias"])
    none = a3po.norm_bwd(d(dy), d(x), d(w), d(rstd), mean=d(mean), want_dweight=False)
    assert none["workspace"] is None and torch.equal(none["dx"], whole["dx"])
    e = torch.empty((0, 96), device="cuda")
    empty = a3po.norm_bwd(e, e, d(w), e[:, 0].contiguous(), mean=e[:, 0].contiguous(), dweight=dw, dbias=db)
    assert empty["dx"].shape == (0, 96) and not dw.any() and not db.any()
    assert a3po.norm_fwd(e, d(w))[0].shape == (0, 96)


def test_on_another_stream(a3po):
    x, w, b, _ = _inputs(64, 1024, torch.bfloat16, torch.bfloat16, seed=7)
    xg, wg, bg = x.cuda(), w.cuda(), b.cuda()
    want = a3po.norm_fwd(xg, wg, bg)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = a3po.norm_fwd(xg, wg, bg)[0]
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("f32", "bf16")])
def test_backward_in_place_takes_the_sums_from_partial_ones(a3po, H, xt, yt):
    """dx over x: the sums cannot be taken from x and dy a second time."""
    x, w, _, g = _inputs(7, H, DT[xt], DT[xt], seed=H + 2)
    dy = torch.randn(7, H, generator=g).to(DT[yt])
    xg = x.cuda()
    out = _check_backward(a3po, x, w, dy, True, dx=xg, dev=(xg, dy.cuda()))
    assert out["workspace"] is not None


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 192, 193, 255, 256, 257, 511, 1023, 1024, 1025])
@pytest.mark.parametrize("H,xt", [(96, "f32"), (97, "bf16"), (3, "bf16"), (1001, "f32"), (1536, "bf16")])
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
def test_sums_over_few_rows_in_one_launch(a3po, T, H, xt, layer):
    x, w, _, g = _inputs(T, H, DT[xt], DT[xt], seed=T + H)
    dy = torch.randn(T, H, generator=g).to(DT[xt])
    out = _check_backward(a3po, x, w, dy, layer)
    assert (out["workspace"] is None) == (T <= a3po.A3PO_NORM_ONE_LAUNCH_ROWS)
    again = _check_backward(a3po, x, w, dy, layer)
    assert torch.equal(out["dweight"], again["dweight"])


def test_where_the_sums_need_a_workspace(a3po):
    x = torch.randn(1024, 3074, device="cuda")       # (beyond A3PO_NORM_ONE_LAUNCH_ELEMENTS)
    rstd = torch.ones(1024, device="cuda")
    assert x.numel() > a3po.A3PO_NORM_ONE_LAUNCH_ELEMENTS
    many = a3po.norm_bwd(x, x, None, rstd, kind=a3po.A3PO_NORM_RMS)
    few = a3po.norm_bwd(x[:512], x[:512], None, rstd[:512], kind=a3po.A3PO_NORM_RMS)
    assert many["workspace"] is not None and few["workspace"] is None
    rest = a3po.norm_bwd(x[512:], x[512:], None, rstd[512:], kind=a3po.A3PO_NORM_RMS, dweight=few["dweight"], accumulate=True)
    bar = 128 * U * (x.double() ** 2).sum(0)
    assert ((rest["dweight"].double() - (x.double() ** 2).sum(0)).abs() <= bar).all()
    assert ((many["dweight"].double() - (x.double() ** 2).sum(0)).abs() <= bar).all()
    y = x[:8].clone()                                # dx over x: refused before anything runs
    rc = a3po.lib().a3po_norm_bwd(x.data_ptr(), 0, 3074, y.data_ptr(), 0, 8, 3074, 3074, None, 0, None, rstd.data_ptr(), 1,
                                  y.data_ptr(), 3074, many["dweight"].data_ptr(), None, 0, None, 0, None)
    assert rc < 0 and "workspace" in a3po.binding.strerror(rc)


@pytest.mark.parametrize("T,in_place", [(64, False), (64, True), (3000, False)])
def test_both_passes_on_another_stream_and_in_a_graph(a3po, T, in_place):
    """One launch and two (dx over dy, many rows)."""
    H = 520
    x, w, b, g = _inputs(T, H, torch.bfloat16, torch.float32, seed=23)
    x, w, b, dy = x.cuda(), w.cuda(), b.cuda(), torch.randn(T, H, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(a3po.workspace_bytes(T, 0, H, which=a3po.A3PO_WS_NORM_BWD), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")

    def step(y, dx, dw, db, ws=None):
        _, mean, rstd = a3po.norm_fwd(x, w, b, out=y)
        if in_place:
            dx.copy_(dy)
        a3po.norm_bwd(dx if in_place else dy, x, w, rstd, mean=mean, want_dbias=True, dx=dx, dweight=dw, dbias=db, workspace=ws)
        return y, dx, dw, db

    fresh = lambda: step(torch.empty_like(x), torch.empty_like(x), torch.empty_like(dw), torch.empty_like(db))
    got, want = (y, dx, dw, db), fresh()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(*got, ws)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*got, ws)
    for i in range(3):
        x.copy_(torch.randn(T, H, generator=g))
        dy.copy_(torch.randn(T, H, generator=g))
        want = fresh()
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), i
