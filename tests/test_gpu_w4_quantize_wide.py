"""a3po_w4_quantize on finite weights whose range is no fp32 number: between them lie up to 6.8e38."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_w4_quantize import DT, a3po  # noqa: E402, F401


@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("st", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_weights_up_to_the_types_largest(a3po, zeros, group, st, wt):  # noqa: F811
    """Scales are the range's fifteenth (the extremes' seventh or eighth) to four roundings and the type's; what codes stand for is within a
    scale of the weight and its own roundings (2^-8 of the largest in bfloat16: the scale's, times codes)."""
    big = torch.finfo(DT[wt]).max
    w = torch.randn(6, 2 * group, generator=torch.Generator().manual_seed(group)).clamp(-1, 1)
    w[0, 0], w[0, 1], w[1, 3], w[1, 7], w[2, 5], w[3, 6] = 1, -1, 1, -0.25, 1, -1
    w = (w.double() * big).to(DT[wt])
    w[4], w[5] = big, -big
    assert w.isfinite().all()
    codes, scales, zero = a3po.w4_quantize(w.cuda(), group, DT[st], zeros)
    x, s = w.double().view(6, 2, group), scales.cpu().double()
    hi, lo = x.amax(2), x.amin(2)
    ref = (hi.clamp(min=0) - lo.clamp(max=0)) / 15 if zeros else torch.maximum(hi / 7, lo / -8)
    bar = 4 * 2.0 ** -24 + (2.0 ** -8 if st == "bf16" else 0)
    assert ((s - ref).abs() <= bar * ref).all()
    c = codes.cpu()
    q = torch.stack((c & 15, c >> 4), 2).view(6, 2, group).double()
    value = (q - (zero.cpu().double()[..., None] if zeros else 8.0)) * s[..., None]
    assert ((value - x).abs() <= (1 + 16 * bar) * s[..., None]).all()
