"""a3po_w4_linear against the product with the dequantised weight in 64 bits.

Products of a bfloat16 and a code are exact; what is rounded is the fp32 sum.  A group's accumulator starts at
-(16 + zero) sum x and adds (16 + code) x: at most 62 sum |x| in magnitude and some 32 roundings of 2^-24 of it, so an element
is off by at most 2^-24 * 32 * 62 * sum_k scale |x|.  Roundings are random: over many elements the relative 2-norm of the
errors is held to 4e-6 as well (estimated 6e-7).  Outputs in bfloat16 lie between the
rounded ends of the bar."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def _weight(N, H, group, zeros, st, g):
    q = torch.randint(0, 16, (N, H), generator=g, dtype=torch.uint8)
    scales = (0.01 * (0.2 + torch.rand(N, H // group, generator=g))).to(st)
    z = torch.randint(0, 16, (N, H // group), generator=g, dtype=torch.uint8) if zeros else None
    w = q.double() - (z.double().repeat_interleave(group, 1) if zeros else 8.0)
    s = scales.double().repeat_interleave(group, 1)
    return q[:, 0::2] | (q[:, 1::2] << 4), scales, z, w * s, s


def _check(a3po, T, N, H, group, zeros=False, st=torch.bfloat16, ot=torch.float32, seed=0, x=None, xg=None, out=None):
    g = torch.Generator().manual_seed(seed)
    codes, scales, z, w, s = _weight(N, H, group, zeros, st, g)
    if x is None:
        x = torch.randn(T, H, generator=g).to(torch.bfloat16)
    got = a3po.w4_linear(x.cuda() if xg is None else xg, codes.cuda(), scales.cuda(), zeros=None if z is None else z.cuda(),
                         group=group, out=out, out_dtype=ot)
    torch.cuda.synchronize()
    assert got.dtype == ot and got.shape == (T, N)
    ref = x.double() @ w.t()
    err = (got.cpu().double() - ref).abs()
    bar = U * 32 * 62 * (x.double().abs() @ s.t())
    assert (got.cpu() >= (ref - bar).to(ot)).all() and (got.cpu() <= (ref + bar).to(ot)).all()
    if ot == torch.float32 and T * N >= 256:
        assert err.norm() <= 4e-6 * ref.norm(), float(err.norm() / ref.norm())
    return got


@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 130])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_numbers_of_tokens(a3po, T, group, zeros):
    _check(a3po, T, 300, 1536, group, zeros, seed=T)


@pytest.mark.parametrize("H", [32, 64, 96, 128, 160, 224, 256, 288, 384, 896, 1056, 2080, 4128])
@pytest.mark.parametrize("T", [1, 20, 50])
@pytest.mark.parametrize("st", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("zeros", [False, True])
def test_lengths_that_end_inside_a_unit(a3po, H, T, st, zeros):
    for group in (32, 64, 128):
        if H % group == 0:
            _check(a3po, T, 77, H, group, zeros, st, seed=H)


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 63, 64, 127, 128, 129, 255, 257, 2000, 5003])
@pytest.mark.parametrize("T", [1, 17, 40])
@pytest.mark.parametrize("ot", [torch.float32, torch.bfloat16])
def test_numbers_of_rows(a3po, N, T, ot):
    _check(a3po, T, N, 256, 64, True, ot=ot, seed=N)


def test_many_rows(a3po):
    _check(a3po, 4, 70001, 128, 128, seed=3)
    _check(a3po, 40, 40001, 160, 32, True, torch.float32, seed=4)


def test_strided_unaligned_hidden_states_and_outputs(a3po):
    g = torch.Generator().manual_seed(5)
    for T in (3, 18, 61):
        x = torch.randn(T, 256, generator=g).to(torch.bfloat16)
        xg = torch.zeros(T * 267 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, 267)
        xg[:, :256] = x.cuda()
        out = torch.full((T, 103), 7.0, device="cuda")
        _check(a3po, T, 100, 256, 128, seed=T, x=x, xg=xg[:, :256], out=out[:, :100])
        assert (out[:, 100:] == 7.0).all()


def test_every_code_and_zero_point_is_the_value_it_stands_for(a3po):
    """One-hot hidden states read the weight itself, exactly: a code times a power of two."""
    H, N = 128, 16 * 16
    codes = torch.arange(N, dtype=torch.uint8)[:, None].expand(N, H // 2)      # every pair of codes
    zeros = (torch.arange(N, dtype=torch.uint8) % 16)[:, None].expand(N, 4)
    x = torch.zeros(64, H, dtype=torch.bfloat16)
    x[torch.arange(64), torch.arange(64) * 2 + torch.arange(64) % 2] = 1.0
    got = a3po.w4_linear(x.cuda(), codes.contiguous().cuda(), torch.full((N, 4), 0.5).cuda(), zeros=zeros.contiguous().cuda(),
                         group=32, out_dtype=torch.float32).cpu()
    n = torch.arange(N)
    for t in range(64):
        assert torch.equal(got[t], ((n >> 4 if t % 2 else n & 15) - n % 16).float() * 0.5), t


def test_zero_hidden_states_large_scales_and_empty_calls(a3po):
    g = torch.Generator().manual_seed(6)
    codes, scales, _, _, _ = _weight(40, 256, 64, False, torch.float32, g)
    x = torch.zeros(5, 256, dtype=torch.bfloat16, device="cuda")
    assert not a3po.w4_linear(x, codes.cuda(), (scales * 1e30).cuda(), group=64).any()
    assert a3po.w4_linear(x[:0], codes.cuda(), scales.cuda(), group=64).shape == (0, 40)


def test_on_another_stream_and_in_a_graph(a3po):
    g = torch.Generator().manual_seed(7)
    codes, scales, _, _, _ = _weight(1000, 512, 128, False, torch.bfloat16, g)
    codes, scales = codes.cuda(), scales.cuda()
    x = torch.randn(4, 512, generator=g).to(torch.bfloat16).cuda()
    out = torch.empty(4, 1000, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a3po.w4_linear(x, codes, scales, out=out)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a3po.w4_linear(x, codes, scales, out=out)
    for i in range(3):
        x.copy_(torch.randn(4, 512, generator=g).to(torch.bfloat16))
        want = a3po.w4_linear(x, codes, scales, out_dtype=torch.float32)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("T,H", [(16, 4224), (16, 4608), (9, 4480), (8, 8192), (3, 8192), (1, 8320), (4, 16384), (32, 2048), (32, 2176), (20, 1664),
                                 (17, 256), (1, 256), (1, 128), (5, 384), (12, 3968), (64, 4096), (65, 2432)])
@pytest.mark.parametrize("group,zeros,st", [(128, False, torch.bfloat16), (64, True, torch.float32), (32, True, torch.float32),
                                            (32, False, torch.bfloat16), (32, False, torch.float32), (64, False, torch.float32)])
def test_hidden_values_resident_and_streamed(a3po, T, H, group, zeros, st):
    """Every split of a row over wavefronts, runs that move down to end with the row, hidden values too many for LDS."""
    for N in (5, 530):
        _check(a3po, T, N, H, group, zeros, st, seed=T + H)


@pytest.mark.parametrize("zeros", [False, True])
def test_more_sets_than_compute_units(a3po, zeros):
    """Workgroups take several sets of rows each, the last of them not all."""
    for T, N, H in ((2, 33333, 256), (16, 20011, 512), (30, 9001, 768), (5, 12345, 384)):
        _check(a3po, T, N, H, 128, zeros, seed=N)


def test_refuses_arrays_that_are_not_the_weight_s_shape(a3po):
    """As many elements as it takes, in another shape: a transposed array would scale every group by another one's value."""
    T, N, H, group = 3, 96, 256, 64
    g = torch.Generator().manual_seed(8)
    codes, scales, z, _, _ = _weight(N, H, group, True, torch.float32, g)
    good = dict(x=torch.zeros(T, H, dtype=torch.bfloat16), codes=codes, scales=scales, zeros=z)
    call = lambda **kw: a3po.w4_linear(**{k: v.cuda() for k, v in {**good, **kw}.items()}, group=group)
    assert call().shape == (T, N)
    for name in ("codes", "scales", "zeros"):
        t = good[name]
        wrong = [t.t().contiguous(), t.flatten(), t[:-1], t[:, :-1].contiguous(), t.t().contiguous().cuda().t(), t.short()]
        if name == "codes":    # (its first length is the number of rows: the others' then do not fit)
            wrong = [t.flatten(), t[:, :-1].contiguous(), t.t().contiguous().cuda().t(), t.short()]
            with pytest.raises(AssertionError, match="codes: need"):
                call(codes=t.t().contiguous())
        for w in wrong:
            with pytest.raises((AssertionError, TypeError), match=name):
                call(**{name: w})


# ---- digits: hidden values of one sign, of all sizes --------------------------------------------------------------------


def _relative_error(a3po, x, codes, scales, zeros, group):
    half = codes[:, 0::2] | (codes[:, 1::2] << 4)
    got = a3po.w4_linear(x.cuda(), half.cuda(), scales.cuda(), zeros=None if zeros is None else zeros.cuda(), group=group,
                         out_dtype=torch.float32).cpu().double()
    zero = 8.0 if zeros is None else zeros.double().repeat_interleave(group, 1)
    w = (codes.double() - zero) * scales.double().repeat_interleave(group, 1)
    ref = x.double() @ w.t()
    return float((got - ref).norm() / ref.norm())


@pytest.mark.parametrize("T", [1, 16, 24, 50])
@pytest.mark.parametrize("group,zeros", [(128, False), (128, True), (64, True), (32, True), (32, False)])
@pytest.mark.parametrize("kind", ["zero mean", "around 1", "positive", "outliers"])
def test_errors_are_those_of_a_product_in_fp32_whatever_the_hidden_values_signs(a3po, T, group, zeros, kind):
    """Weights around zero against hidden values that are not: the sums of codes times hidden values are many times what the
    weights' differing signs leave.  With exact operands the errors are roundings of partial sums, each 2^-24 / sqrt(3) of one:
    the sum over groups grows to the result in H / group steps, sqrt(H / (2 group)) times that, up to 2.7e-7 here; a
    group's own sum, 1 / sqrt(H / group) of the result, is rounded up to 32 times in each of them, 2e-7: 3.4e-7
    together, and held to three times that."""
    H, N = 4096, 300
    g = torch.Generator().manual_seed(T + group)
    codes = (2.5 * torch.randn(N, H, generator=g) + 8.5).clamp(0, 15.99).to(torch.uint8)
    scales = 0.01 * (0.5 + torch.rand(N, H // group, generator=g))
    z = torch.randint(7, 10, (N, H // group), generator=g, dtype=torch.uint8) if zeros else None
    x = torch.randn(T, H, generator=g)
    if kind == "around 1":
        x = 1.0 + 0.5 * x
    elif kind == "positive":
        x = x.abs()
    elif kind == "outliers":
        x[:, ::97] *= 300.0
    assert _relative_error(a3po, x.bfloat16(), codes, scales, z, group) <= 1e-6


@pytest.mark.parametrize("T,H", [(3, 512), (16, 1024), (20, 1024), (40, 1056)])
def test_powers_of_two_pass_through_exactly(a3po, T, H):
    """Tokens times powers of two, each its own, from the least to the largest that bfloat16 holds: the same products."""
    g = torch.Generator().manual_seed(T)
    codes, scales, z, _, _ = _weight(70, H, 32, True, torch.float32, g)
    call = lambda x: a3po.w4_linear(x.cuda(), codes.cuda(), scales.cuda(), zeros=z.cuda(), group=32, out_dtype=torch.float32)
    x = torch.randn(T, H, generator=g).clamp(-3, 3).bfloat16()
    x[x.abs() < 2.0 ** -6] = 0.25             # (nothing falls below the least normal value on the way down)
    want = call(x).cpu().double()
    up = torch.linspace(-118, 120, T).round()
    got = call((x.double() * 2.0 ** up[:, None].double()).bfloat16()).cpu().double()
    scaled = want * 2.0 ** up[:, None].double()
    fine = (scaled.abs() < 3e38) & (scaled.abs() > 2e-38)
    assert fine.float().mean() > 0.8 and torch.equal(got[fine], scaled[fine])


@pytest.mark.parametrize("T,H", [(2, 512), (16, 1024), (30, 1024), (50, 1056)])
@pytest.mark.parametrize("below", [10, 20, 32])
def test_small_hidden_values_beside_a_large_one_keep_their_digits(a3po, T, H, below):
    """A hidden value 2^below times the others that every row multiplies with nothing (its code is the zero point): what is
    left is the others' product, of values with all of bfloat16's digits."""
    g = torch.Generator().manual_seed(below)
    N, group = 60, 32
    codes = torch.randint(0, 16, (N, H), generator=g, dtype=torch.uint8)
    z = torch.randint(0, 16, (N, H // group), generator=g, dtype=torch.uint8)
    scales = 0.01 * (0.5 + torch.rand(N, H // group, generator=g))
    at = torch.arange(0, H, group * 3)
    codes[:, at] = z[:, at // group]
    x = ((1.0 + torch.rand(T, H, generator=g)) * 2.0 ** -below).bfloat16()
    x[:, at] = 1.5
    assert _relative_error(a3po, x, codes, scales, z, group) <= 1e-6


@pytest.mark.parametrize("T,H", [(4, 512), (18, 1024), (40, 1056)])
def test_infinite_and_nan_hidden_values_stay_in_their_tokens(a3po, T, H):
    g = torch.Generator().manual_seed(9)
    codes, scales, z, w, _ = _weight(50, H, 32, True, torch.bfloat16, g)
    x = torch.randn(T, H, generator=g).bfloat16()
    want = a3po.w4_linear(x.cuda(), (codes).cuda(), scales.cuda(), zeros=z.cuda(), group=32, out_dtype=torch.float32).cpu()
    x[1, 5], x[3, H - 1] = float("nan"), float("inf")
    got = a3po.w4_linear(x.cuda(), (codes).cuda(), scales.cuda(), zeros=z.cuda(), group=32, out_dtype=torch.float32).cpu()
    rest = [t for t in range(T) if t not in (1, 3)]
    assert torch.equal(got[rest], want[rest]) and got[1].isnan().all() and not got[3].isfinite().any()


# ---- several sets, several tiles a workgroup ----------------------------------------------------------------------------

# T, N, H, group, zeros, fp32 scales.  With 256 compute units: more than two sets of rows a workgroup, an odd number for some and
# an even one for others; two, three and four units a wavefront; one and two blocks of tokens.
MANY_SETS = [(2, 200003, 256, 128, False, False), (16, 140003, 256, 32, True, False), (1, 200003, 384, 64, True, True),
             (16, 140003, 384, 32, False, True), (2, 200003, 512, 128, False, False), (16, 140003, 512, 64, True, False),
             (20, 200003, 256, 64, False, True), (32, 140003, 384, 32, True, False), (17, 200003, 512, 128, True, True),
             (5, 90001, 1536, 128, False, False), (12, 66001, 896, 32, True, False)]
# streamed: more than two rounds of 256 rows a workgroup and a ragged end; scales of one block of 64 bytes a row and of many
MANY_TILES = [(3, 140003, 160, 32, True, False), (20, 140003, 160, 32, True, True), (40, 200003, 160, 32, False, False),
              (50, 140003, 160, 32, True, False), (64, 140003, 384, 128, True, False), (50, 140003, 1056, 32, True, True),
              (40, 140003, 1088, 64, False, True), (130, 140003, 288, 32, True, False), (9, 140003, 4352, 128, False, False),
              (20, 140003, 2176, 128, True, True)]


@pytest.mark.parametrize("T,N,H,group,zeros,f32", MANY_SETS + MANY_TILES)
def test_more_rows_than_one_round_of_compute_units(a3po, T, N, H, group, zeros, f32):
    """Products are exact; what is rounded are the sums, no more often than a group has terms and a row groups, and the scaling."""
    g = torch.Generator(device="cuda").manual_seed(T + H)
    q = torch.randint(0, 16, (N, H), device="cuda", generator=g, dtype=torch.uint8)
    scales = 0.01 * (0.2 + torch.rand(N, H // group, device="cuda", generator=g))
    scales = scales if f32 else scales.bfloat16()
    z = torch.randint(0, 16, (N, H // group), device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    x = (0.5 + torch.randn(T, H, device="cuda", generator=g)).bfloat16()
    got = a3po.w4_linear(x, q[:, 0::2] | (q[:, 1::2] << 4), scales, zeros=z, group=group, out_dtype=torch.float32)
    w = q.double()
    w -= z.double().repeat_interleave(group, 1) if zeros else 8.0
    w *= scales.double().repeat_interleave(group, 1)
    ref = x.double() @ w.t().contiguous()
    err = (got.double() - ref).abs()
    bar = U * (group + H // group + 4) * (x.double().abs() @ w.abs_().t().contiguous())
    assert (err <= bar).all() and float(err.norm()) <= 1e-6 * float(ref.norm())
