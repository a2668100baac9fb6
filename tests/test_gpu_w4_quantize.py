"""a3po_w4_quantize against its definition.

Scales are the difference of exact extremes times an fp32 constant: three roundings (the difference's, the constant 1 / 15's own,
the product's), each at most 2^-24 of the value, with their products below 3.01 * 2^-24; and 2^-8 more in bfloat16.  With the scale that
came out, codes and zero points are fp32 operations that float32 arithmetic of IEEE gives as well, rounded alike: equal.  What a
code stands for is within half a scale of the weight (and 2^-20 of it for the two products' rounding, up to 16 steps of 2^-24), a
whole one where the zero point's rounding or bfloat16's moved the range's ends."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def check(a3po, w, group, scale_dtype, zeros):
    N, H = w.shape
    codes, scales, zero = a3po.w4_quantize(w, group, scale_dtype, zeros)
    codes, s = codes.cpu(), scales.float().cpu()
    x = w.float().cpu().reshape(N, H // group, group)
    hi, lo = x.amax(2), x.amin(2)
    ref = (hi.clamp(min=0).double() - lo.clamp(max=0).double()) / 15 if zeros else torch.maximum(hi.double() / 7, lo.double() / -8)
    assert ((s.double() - ref).abs() <= (3.01 * 2.0 ** -24 + (2.0 ** -8 if scale_dtype == torch.bfloat16 else 0)) * ref + 2.0 ** -149).all()
    inverse = torch.where(s >= 2.0 ** -126, 1.0 / s, torch.zeros(()))
    want_zero = torch.round(-lo.clamp(max=0) * inverse).clamp(0, 15) if zeros else torch.full_like(s, 8.0)
    if zeros:
        assert torch.equal(zero.cpu().float(), want_zero)
    want = (torch.round(x * inverse[..., None]) + want_zero[..., None]).clamp(0, 15).to(torch.uint8).view(N, H)
    got = torch.stack((codes & 15, codes >> 4), 2).view(N, H)
    assert torch.equal(got, want)
    value = (got.view(N, -1, group).double() - want_zero[..., None].double()) * s[..., None].double()
    slack = 1.0 if zeros or scale_dtype == torch.bfloat16 else 0.5
    assert ((value - x.double()).abs() <= (slack + 2.0 ** -20) * s[..., None].double() + 2.0 ** -126 * 8).all()
    return codes, scales, zero


@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("st", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("N,groups", [(1, 1), (3, 5), (257, 7), (1000, 12)])
def test_every_form(a3po, N, groups, zeros, group, st, wt):
    g = torch.Generator().manual_seed(N + group)
    w = (0.02 * torch.randn(N, groups * group, generator=g) + 0.003).to(DT[wt])
    check(a3po, w.cuda(), group, DT[st], zeros)


@pytest.mark.parametrize("zeros", [False, True])
def test_groups_of_one_sign_of_nothing_and_of_extremes(a3po, zeros):
    w = torch.randn(12, 256, generator=torch.Generator().manual_seed(1))
    w[0], w[1], w[2], w[3] = 0, w[1].abs() + 1, -w[2].abs() - 1, 5.0
    w[4], w[5], w[6], w[7] = -5.0, w[5] * 1e-39, w[6] * 1e30, w[7] * 1e-30
    w[8, ::2], w[9], w[10, 1:] = 0, 1e-45, 0
    check(a3po, w.cuda(), 64, torch.float32, zeros)


@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (5, 1)])
def test_strides_and_unaligned_rows(a3po, pad, shift, wt):
    N, H = 37, 384
    buf = torch.full((N * (H + pad) + shift,), 1e4, dtype=DT[wt], device="cuda")
    w = buf[shift:].view(N, H + pad)[:, :H]
    w.copy_(torch.randn(N, H, generator=torch.Generator().manual_seed(4)))
    check(a3po, w, 128, torch.float32, True)


@pytest.mark.parametrize("zeros", [False, True])
def test_products_with_the_layout_are_those_of_its_values(a3po, zeros):
    """w4_linear on the codes, against 64-bit products with the values they stand for: fp32 sums of 512 products, 512 * 2^-24 of
    the sum of magnitudes at the most."""
    g = torch.Generator().manual_seed(5)
    w, x = 0.05 * torch.randn(300, 512, generator=g), torch.randn(3, 512, generator=g).bfloat16()
    codes, scales, zero = check(a3po, w.cuda(), 64, torch.float32, zeros)
    out = a3po.w4_linear(x.cuda(), codes.cuda(), scales, zero, group=64, out_dtype=torch.float32).cpu().double()
    q = torch.stack((codes & 15, codes >> 4), 2).view(300, -1, 64).double()
    q = (q - (zero.cpu().double()[..., None] if zeros else 8.0)) * scales.cpu().double()[..., None]
    q = q.view(300, 512)
    assert ((out - x.double() @ q.t()).abs() <= 512 * 2.0 ** -24 * (x.double().abs() @ q.abs().t())).all()


def test_on_another_stream_and_in_a_graph_and_empty(a3po):
    w = torch.randn(200, 256, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a = a3po.w4_quantize(w, 32, zeros=True)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b = a3po.w4_quantize(w, 32, zeros=True)
    for i in range(3):
        graph.replay()
        want = a3po.w4_quantize(w, 32, zeros=True)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, b))
        if i == 0:
            assert all(torch.equal(x, y) for x, y in zip(want, a))
        w.mul_(1.5)
    assert a3po.w4_quantize(torch.empty(0, 64, device="cuda"), 64)[0].shape == (0, 32)
