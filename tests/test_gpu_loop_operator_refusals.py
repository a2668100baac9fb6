"""What the binding of the operators that close the loop refuses before a call: types, shapes, strides and lengths of tensors that
the library sees as pointers.  Tensors are on the GPU and all but one is right, so that the check that is meant fails."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operator_refusals import a3po, refuses, zeros  # noqa: E402, F401

T, V, H = 6, 100, 64
I32 = dict(dtype=torch.int32)
U8 = dict(dtype=torch.uint8)


@pytest.mark.parametrize("change,message", [
    (dict(logits=lambda: zeros(T, V).half()), "logits must be float32"), (dict(logits=lambda: zeros(V, T).t()), "logits must be a row"),
    (dict(logits=lambda: zeros(T)), "logits must be a row"), (dict(V=lambda: V + 1), "logits: need"), (dict(V=lambda: 0), "a3po_sample"),
    (dict(uniform=lambda: zeros(T - 1)), "uniform: need"), (dict(uniform=lambda: zeros(T).double()), "uniform: need"),
    (dict(uniform=lambda: zeros(T).cpu()), "uniform: need"), (dict(uniform=lambda: zeros(2 * T)[::2]), "uniform: need"),
    (dict(top_k=lambda: zeros(T)), "top_k: need"), (dict(top_k=lambda: zeros(T, dtype=torch.int64)), "top_k: need"),
    *[({name: f}, f"{name}: need") for name in ("temperature", "top_p", "min_p") for f in (lambda: zeros(T + 1), lambda: zeros(T).bfloat16())]])
def test_sample(a3po, change, message):  # noqa: F811
    one = torch.ones(T, device="cuda")
    args = dict(logits=zeros(T, V), uniform=zeros(T), temperature=one, top_k=zeros(T, **I32), top_p=one, min_p=zeros(T))
    a3po.sample(**args)
    refuses(lambda: a3po.sample(**{**args, **{k: f() for k, f in change.items()}}), message, (AssertionError, TypeError, ValueError, a3po.A3poError))


@pytest.mark.parametrize("change,message", [
    (dict(grads=lambda: [zeros(5), zeros(5).bfloat16()]), "grads.1.: need"), (dict(grads=lambda: [zeros(5).half()]), "grads must be"),
    (dict(grads=lambda: [zeros(5).cpu()]), "current device"), (dict(grads=lambda: [zeros(10)[::2]]), "grads.0.: need"), (dict(out=lambda: zeros(2)), "out: need")])
def test_grad_norm(a3po, change, message):  # noqa: F811
    args = dict(grads=[zeros(5), zeros(3)], out=zeros(1))
    a3po.grad_norm(**args)
    refuses(lambda: a3po.grad_norm(**{**args, **{k: f() for k, f in change.items()}}), message)


n = 70
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("change,message", [
    (dict(params=lambda: [zeros(n).half()]), "params must be"), (dict(params=lambda: [zeros(2 * n)[::2]]), "params.0.: need"), (dict(grads=lambda: [zeros(n + 1)]), "grads.0.: need"),
    (dict(grads=lambda: []), "grads: need one"), (dict(exp_avgs=lambda: [zeros(n - 1)]), "exp_avgs.0.: need"), (dict(exp_avgs=lambda: [zeros(n).double()]), "exp_avgs.0.: need"),
    (dict(exp_avg_sqs=lambda: [zeros(n).cpu()]), "current device"), (dict(exp_avg_sqs=lambda: []), "exp_avg_sqs: need one"), (dict(copies=lambda: [zeros(n)]), "copies.0.: need"),
    (dict(copies=lambda: []), "copies: need one"), (dict(grads=lambda: [1.0]), "grads|dtype"), (dict(exp_avgs=lambda: [None]), "exp_avgs|NoneType"), (dict(norm=lambda: zeros(2)), "norm: need"), (dict(step=lambda: zeros(1)), "step: need"),
    (dict(lr=lambda: zeros(1).double()), "lr: need"), (dict(scales=lambda: []), "scales: need one|exp_avgs.0.: need"),
    (dict(scales=lambda: [(zeros(2, **U8), zeros(3, **U8))]), "scales.0.: need|exp_avgs.0.: need"), (dict(scales=lambda: [(zeros(3, **U8), zeros(3))]), "scales.0.: need|exp_avgs.0.: need")])
def test_adamw_step(a3po, change, message, bits):  # noqa: F811
    p = zeros(n)
    m, v, scales = a3po.adamw_state(p, bits)
    args = dict(params=[p], grads=[zeros(n)], exp_avgs=[m], exp_avg_sqs=[v], scales=None if scales is None else [scales], copies=[zeros(n).bfloat16()],
                norm=zeros(1), step=1, lr=0.1)
    a3po.adamw_step(**args)
    refuses(lambda: a3po.adamw_step(**{**args, **{k: f() for k, f in change.items()}}), message, (AssertionError, TypeError, ValueError, AttributeError))


@pytest.mark.parametrize("change,message", [
    (dict(weight=lambda: zeros(V, H).half()), "weight must be float32"), (dict(weight=lambda: zeros(H, V).t()), "weight must be a row"), (dict(group=lambda: 48), "group must be"),
    (dict(group=lambda: 128), "group must be"), (dict(scale_dtype=lambda: torch.float16), "scales must be")])
def test_w4_quantize(a3po, change, message):  # noqa: F811
    args = dict(weight=zeros(V, H), group=32)
    a3po.w4_quantize(**args)
    refuses(lambda: a3po.w4_quantize(**{**args, **{k: f() for k, f in change.items()}}), message)
