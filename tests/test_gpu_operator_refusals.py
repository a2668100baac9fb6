"""What the binding of the operators around the log-probs refuses before a call: types, shapes, strides and lengths of tensors
that the library sees as pointers.  Tensors are on the GPU and all but one is right, so that the check that is meant fails."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def a3po():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_06547_amd as lib
    lib.lib()
    return lib


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def refuses(call, message, error=(AssertionError, TypeError, ValueError)):
    with pytest.raises(error, match=message):
        call()


T, H, V = 6, 64, 100


@pytest.mark.parametrize("change,message", [
    (dict(x=lambda: zeros(T)), "x must be a row-major"), (dict(x=lambda: zeros(T, H).half()), "x must be float32"), (dict(x=lambda: zeros(H, T).t()), "x must be a row"),
    (dict(x=lambda: zeros(T, H).cpu()), "x must be a row"), (dict(x=lambda: zeros(T, H, 1)), "x must be a row"),
    (dict(weight=lambda: zeros(H - 1)), "weight: need"), (dict(weight=lambda: zeros(2 * H)[::2]), "weight: need"), (dict(weight=lambda: zeros(H).half(), bias=lambda: None), "weight must be"),
    (dict(weight=lambda: zeros(H).cpu()), "weight: need"), (dict(bias=lambda: zeros(H + 1)), "bias: need"), (dict(bias=lambda: zeros(H).bfloat16()), "one dtype"),
    (dict(out=lambda: zeros(T, H + 1)), "out: need shape"), (dict(out=lambda: zeros(T - 1, H)), "out: need shape"), (dict(out=lambda: zeros(H, T).t()), "out must be a row")])
def test_norm_fwd(a3po, change, message):
    args = dict(x=zeros(T, H), weight=zeros(H), bias=zeros(H))
    a3po.norm_fwd(**args)
    refuses(lambda: a3po.norm_fwd(**{**args, **{k: f() for k, f in change.items()}}), message)


@pytest.mark.parametrize("change,message", [
    (dict(dy=lambda: zeros(T, H).half()), "dy must be float32"), (dict(x=lambda: zeros(T, H - 1)), "x: need shape"), (dict(x=lambda: zeros(H, T).t()), "x must be a row"),
    (dict(weight=lambda: zeros(H + 1)), "weight: need"), (dict(rstd=lambda: zeros(T + 1)), "rstd: need"), (dict(rstd=lambda: zeros(T).double()), "rstd: need"),
    (dict(mean=lambda: zeros(T - 1)), "mean: need"), (dict(mean=lambda: zeros(2 * T)[::2]), "mean: need"), (dict(dx=lambda: zeros(T, H).bfloat16()), "dx must have x's dtype"),
    (dict(dx=lambda: zeros(T, H - 1)), "dx: need shape"), (dict(dweight=lambda: zeros(H - 1)), "dweight: need"), (dict(dbias=lambda: zeros(H).bfloat16()), "dbias: need"),
    (dict(accumulate=lambda: True), "accumulate needs")])
def test_norm_bwd(a3po, change, message):
    args = dict(dy=zeros(T, H), x=zeros(T, H), weight=zeros(H), rstd=zeros(T), mean=zeros(T), want_dbias=True)
    a3po.norm_bwd(**args)
    refuses(lambda: a3po.norm_bwd(**{**args, **{k: f() for k, f in change.items()}}), message)


I32 = dict(dtype=torch.int32)
I64 = dict(dtype=torch.int64)
ADJUSTMENTS = [
    (dict(history=lambda: zeros(50, **I64)), "history: need"), (dict(history=lambda: zeros(100, **I32)[::2]), "history: need"), (dict(hist_start=lambda: zeros(T, **I32)), "hist_start: need"),
    (dict(hist_start=lambda: zeros(T + 1, **I64)), "hist_start: need"), (dict(hist_start=lambda: None), "history needs"), (dict(hist_len=lambda: None), "history needs"),
    (dict(hist_len=lambda: zeros(T, **I64)), "hist_len: need"), (dict(prompt_len=lambda: zeros(T - 1, **I32)), "prompt_len: need"),
    *[({name: f}, f"{name}: need") for name in ("repetition", "frequency", "presence", "temperature")
      for f in (lambda: zeros(T - 1), lambda: zeros(T).double(), lambda: zeros(T).cpu())],
    (dict(bias=lambda: zeros(V - 1)), "bias: need"), (dict(bias=lambda: zeros(V).bfloat16()), "bias: need"), (dict(bias=lambda: zeros(T - 1, V)), "bias: need one row"),
    (dict(bias=lambda: zeros(V, T).t()), "bias: need"), (dict(allowed=lambda: zeros(3, **I32)), "allowed: need"), (dict(allowed=lambda: zeros(4, **I64)), "allowed: need"),
    (dict(allowed=lambda: zeros(T + 1, 4, **I32)), "allowed: need one row")]


def adjustments():
    one = torch.ones(T, device="cuda")
    return dict(history=zeros(50, **I32), hist_start=zeros(T, **I64), hist_len=zeros(T, **I32), prompt_len=zeros(T, **I32), repetition=one,
                frequency=one, presence=one, temperature=one, bias=zeros(V), allowed=zeros(T, 4, **I32))


@pytest.mark.parametrize("change,message", ADJUSTMENTS + [
    (dict(logits=lambda: zeros(T, V).half()), "logits must be float32"), (dict(logits=lambda: zeros(V, T).t()), "logits must be a row"),
    (dict(chosen=lambda: zeros(T, **I64)), "chosen: need"), (dict(chosen=lambda: zeros(T + 1, **I32)), "chosen: need"),
    (dict(out=lambda: zeros(T, V - 1)), "out: need"), (dict(out=lambda: zeros(T + 1, V)), "out: need"), (dict(out=lambda: zeros(T, V).half()), "out must be float32")])
def test_adjust_logits(a3po, change, message):
    args = dict(logits=zeros(T, V), chosen=zeros(T, **I32), **adjustments())
    a3po.adjust_logits(**args)
    refuses(lambda: a3po.adjust_logits(**{**args, **{k: f() for k, f in change.items()}}), message)


@pytest.mark.parametrize("change,message", ADJUSTMENTS + [
    (dict(dout=lambda: zeros(T, V).half()), "logits must be float32"), (dict(logits=lambda: zeros(T - 1, V)), "logits: need"), (dict(logits=lambda: zeros(T, V - 1)), "logits: need"),
    (dict(dlogits=lambda: zeros(T, V - 1)), "dlogits: need"), (dict(dlogits=lambda: zeros(T, V).bfloat16()), "dlogits must have logits' dtype")])
def test_adjust_logits_bwd(a3po, change, message):
    args = dict(dout=zeros(T, V), logits=zeros(T, V), **adjustments())
    a3po.adjust_logits_bwd(**args)
    refuses(lambda: a3po.adjust_logits_bwd(**{**args, **{k: f() for k, f in change.items()}}), message)


@pytest.mark.parametrize("change,message", [
    (dict(x=lambda: zeros(T, H)), "x must be bfloat16"), (dict(x=lambda: zeros(H, T).bfloat16().t()), "x must be a row"), (dict(group=lambda: 48), "group must be"),
    (dict(group=lambda: 128), "group must be"), (dict(scales=lambda: zeros(V, 2).half()), "scales must be"), (dict(scales=lambda: zeros(V, 4)), "scales: need"),
    (dict(codes=lambda: zeros(V, H, dtype=torch.uint8)), "codes: need"), (dict(zeros=lambda: zeros(V, 2, **I32)), "zeros: need"), (dict(out=lambda: zeros(T, V - 1)), "out: need shape"),
    (dict(out=lambda: zeros(T, V).half()), "out must be float32")])
def test_w4_linear(a3po, change, message):
    args = dict(x=zeros(T, H).bfloat16(), codes=zeros(V, H // 2, dtype=torch.uint8), scales=zeros(V, 2), zeros=zeros(V, 2, dtype=torch.uint8), group=32)
    a3po.w4_linear(**args)
    refuses(lambda: a3po.w4_linear(**{**args, **{k: f() for k, f in change.items()}}), message)
