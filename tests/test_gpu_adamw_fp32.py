"""AdamW's states are those of plain fp32 arithmetic, every product and every sum rounded once, so any other program that
keeps to the formulas gets the same bits: with bfloat16 gradients and beta1 = 0.9, 9 m + g lies on so coarse a grid that the new
mean often is a tie of two float8 numbers or exactly a power of two, and a product that enters its sum unrounded decides those otherwise."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_adamw import DT, a3po, make, state_of  # noqa: E402, F401

BETA1, BETA2 = 0.9, 0.999


def expected(m, v, g, factor=None):
    """fp32 on the CPU, an operation at a time; factor: a float32 tensor of one element."""
    g = g.float()
    if factor is not None:
        g = g * factor
    return BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g


def e4m3_blocks(x):
    """Bytes and exponents of exp_avg's format: the largest of 32 values between 2^7 and 2^8 of its unit, to nearest."""
    n = x.numel()
    top = torch.nn.functional.pad(x, (0, -n % 32)).view(-1, 32).abs().amax(1).view(torch.int32) >> 23
    scale = (top - 7).clamp(min=1)
    up = ((254 - scale) << 23).view(torch.float32).repeat_interleave(32)[:n]
    return (x * up).to(torch.float8_e4m3fn).view(torch.uint8), scale.to(torch.uint8)


@pytest.mark.parametrize("clip", [False, True])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 33, 70001])
def test_states_in_32_bits(a3po, n, param, grad, clip):  # noqa: F811
    x = make(n, 17 + n, param, grad)
    p, g, m, v = (x[k].cuda() for k in "pgmv")
    norm = a3po.grad_norm([g]) if clip else None
    factor = None if norm is None else torch.clamp(torch.tensor([0.3]) / (norm.cpu() + 1e-6), max=1.0)  # (a number over a tensor is two roundings)
    a3po.adamw_step([p], [g], [m], [v], step=7, lr=1e-3, beta1=BETA1, beta2=BETA2, norm=norm, max_norm=0.3, seed=7)
    rm, rv = expected(x["m"], x["v"], x["g"], factor)
    assert torch.equal(m.cpu(), rm) and torch.equal(v.cpu(), rv)


@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_bytes_of_8_bit_means(a3po, param, grad):  # noqa: F811
    n = 200001
    x = make(n, 29, param, grad)
    p, g = x["p"].cuda(), x["g"].cuda()
    m, v, scales = state_of(a3po, x, 8)
    old = [a3po.adamw_state_values(t, s).cpu() for t, s in zip((m, v), scales)]
    a3po.adamw_step([p], [g], [m], [v], scales=[scales], step=7, lr=1e-3, beta1=BETA1, beta2=BETA2, seed=7)
    want, exponents = e4m3_blocks(expected(*old, x["g"])[0])
    assert torch.equal(scales[0].cpu(), exponents)
    assert torch.equal(m.cpu().view(torch.uint8), want)
