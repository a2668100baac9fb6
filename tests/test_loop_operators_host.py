"""Refusals and host-side sizes of the operators that close the loop (drawn tokens, optimizer step, 4-bit layout); no GPU needed:
every call here returns at validation, before any device pointer is used."""
import ctypes
import os

import pytest

from test_operators_host import P, caller

NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_2512_06547_amd as a3po
    if not os.path.exists(a3po.lib_path()):
        from paper_2512_06547_amd import build
        build.build(force=True)
    return a3po.lib()


def test_sample_refuses(lib):
    from paper_2512_06547_amd.binding import Sampling
    policy = lambda **kw: ctypes.byref(Sampling(**{"uniform": 0x1000, **kw}))
    need = lib.a3po_workspace_bytes(6, 4, 100, 0)
    # logits, dt, T, V, ld, policy, token, logp, logp_full, kept, allowed, allowed_ld, workspace, bytes, stream
    call = caller(lib.a3po_sample, [P(), 0, 4, 100, 100, policy(), P(), P(), P(), P(), P(), 4, P(0x10000), max(need, 1) - 1, None])
    if need:
        assert call() == -5 and call(a12=None, a13=1 << 30) == -5 and call(a12=P(0x10010), a13=need) == -4
    assert call(a2=0) == 0 and call(a2=0, a0=None, a5=None, a6=None) == 0
    assert call(a1=2) == -3 and call(a1=-1) == -3
    assert call(a2=-1) == -2 and call(a2=(1 << 40) + 1) == -2 and call(a3=0) == -2 and call(a3=1 << 31, a4=1 << 31) == -2
    assert call(a4=99) == -2 and call(a4=(1 << 40) + 1) == -2 and call(a11=3) == -2 and call(a11=(1 << 40) + 1) == -2
    assert call(a0=None) == -1 and call(a5=None) == -1 and call(a6=None) == -1 and call(a5=policy(uniform=0)) == -1
    assert call(a0=P(0x1002)) == -4
    for at in (6, 7, 8, 9, 10):
        assert call(**{f"a{at}": P(0x1002)}) == -4
    for name in ("uniform", "temperature", "top_k", "top_p", "min_p"):
        assert call(a5=policy(**{name: 0x1002})) == -4


def test_sample_workspaces_take_any_size(lib):
    for T in (-1, 0, 1, 300, 1 << 20, 1 << 50):
        for V in (-1, 0, 1, 151936, 1 << 40):
            assert lib.a3po_workspace_bytes(6, T, V, 0) % 256 == 0
    assert lib.a3po_workspace_bytes(6, 64, 151936, 0) < 64 << 20


def test_grad_norm_refuses(lib):
    def arrays(n, at=0x1000, size=100):
        return (ctypes.c_void_p * n)(*[at] * n), (ctypes.c_int64 * n)(*[size] * n)
    g, s = arrays(3)
    need = lib.a3po_workspace_bytes(7, 3, 0, 0)
    assert need > 0 and lib.a3po_workspace_bytes(7, 0, 0, 0) == 0 and lib.a3po_workspace_bytes(7, -5, 0, 0) == 0
    assert lib.a3po_workspace_bytes(7, 201, 0, 0) == 2 * need and lib.a3po_workspace_bytes(7, 1 << 50, 0, 0) == 0
    # grads, sizes, count, dt, scale, norm, workspace, bytes, stream
    call = caller(lib.a3po_grad_norm, [g, s, 3, 0, 1.0, P(), P(0x10000), need - 1, None])
    assert call() == -5 and call(a6=None, a7=1 << 20) == -5 and call(a6=P(0x10010), a7=need) == -4
    assert call(a3=2) == -3 and call(a2=-1) == -2 and call(a2=(1 << 24) + 1) == -2 and call(a4=NAN) == -7
    assert call(a5=None) == -1 and call(a0=None) == -1 and call(a1=None) == -1 and call(a5=P(0x1002)) == -4
    assert call(a0=arrays(3, 0x1002)[0]) == -4 and call(a0=arrays(3, 0)[0]) == -1
    assert call(a1=arrays(3, size=-1)[1]) == -2 and call(a1=arrays(3, size=(1 << 40) + 1)[1]) == -2


def test_adamw_step_refuses(lib):
    from paper_2512_06547_amd.binding import AdamwOptions, AdamwTensor
    good = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1, max_norm=1.0)
    options = lambda **kw: ctypes.byref(AdamwOptions(**{**good, **kw}))
    tensor = dict(param=0x1000, grad=0x1000, exp_avg=0x1000, exp_avg_sq=0x1000, exp_avg_scale=0x1000, exp_avg_sq_scale=0x1000, copy=0x1000, n=8)
    table = lambda **kw: (AdamwTensor * 2)(AdamwTensor(**tensor), AdamwTensor(**{**tensor, **kw}))
    # tensors, count, param_dt, grad_dt, state_format, options, stream
    call = caller(lib.a3po_adamw_step, [table(), 2, 0, 0, 0, options(), None])
    assert call(a1=0) == 0 and call(a1=0, a0=None) == 0 and call(a0=(AdamwTensor * 2)()) == 0  # nothing to do
    assert call(a2=2) == -3 and call(a3=-1) == -3 and call(a4=2) == -7 and call(a1=-1) == -2 and call(a1=(1 << 24) + 1) == -2
    assert call(a0=None) == -1 and call(a5=None) == -1
    for name, values in dict(lr=(-1e-3, NAN), beta1=(1.0, -0.1, NAN), beta2=(1.0, -0.1, NAN), eps=(-1e-9, NAN), weight_decay=(-1.0, NAN), step=(0, -1)).items():
        for v in values:
            assert call(a5=options(**{name: v})) == -7, name
    for v in (0.0, -1.0, NAN):
        assert call(a5=options(norm=0x1000, max_norm=v)) == -7
    assert call(a5=options(lr_dev=0x1002)) == -4 and call(a5=options(step_dev=0x1004)) == -4 and call(a5=options(norm=0x1002)) == -4
    assert call(a0=table(n=-1)) == -2 and call(a0=table(n=(1 << 40) + 1)) == -2
    for name in ("param", "grad", "exp_avg", "exp_avg_sq"):
        assert call(a0=table(**{name: 0})) == -1 and call(a0=table(**{name: 0x1002})) == -4
    assert call(a0=table(copy=0x1001)) == -4 and call(a0=table(param=0x1001), a2=1) == -4 and call(a0=table(grad=0x1001), a3=1) == -4
    assert call(a0=table(exp_avg_scale=0), a4=1) == -1 and call(a0=table(exp_avg_sq_scale=0), a4=1) == -1


def test_adamw_step_refuses_a_parameter_listed_twice(lib):
    from paper_2512_06547_amd.binding import AdamwOptions, AdamwTensor
    options = AdamwOptions(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1)
    row = lambda at, n=8: AdamwTensor(param=at, grad=0x1000, exp_avg=0x2000 + at, exp_avg_sq=0x3000 + at, n=n)
    for rows in ([0x1000, 0x1000], [0x5000, 0x1000, 0x3000, 0x1000]):
        table = (AdamwTensor * len(rows))(*map(row, rows))
        assert lib.a3po_adamw_step(table, len(rows), 0, 0, 0, ctypes.byref(options), None) == -7
    # (tensors without elements have no address of their own)
    empty = (AdamwTensor * 2)(row(0x1000, 0), row(0x1000, 0))
    assert lib.a3po_adamw_step(empty, 2, 0, 0, 0, ctypes.byref(options), None) == 0


def test_w4_quantize_refuses(lib):
    # weight, dt, N, H, ld, group, codes, scales, scale_dt, zeros, stream
    call = caller(lib.a3po_w4_quantize, [P(), 0, 4, 256, 256, 64, P(), P(), 0, P(), None])
    assert call(a2=0) == 0 and call(a2=0, a0=None, a6=None) == 0
    assert call(a1=2) == -3 and call(a8=2) == -3 and call(a5=48) == -2 and call(a5=256) == -2
    assert call(a2=-1) == -2 and call(a2=1 << 31) == -2 and call(a3=0) == -2 and call(a3=96) == -2 and call(a3=(1 << 20) + 64, a4=1 << 21) == -2
    assert call(a4=255) == -2 and call(a4=(1 << 40) + 1) == -2
    assert call(a0=None) == -1 and call(a6=None) == -1 and call(a7=None) == -1
    assert call(a0=P(0x1002)) == -4 and call(a0=P(0x1001), a1=1) == -4 and call(a6=P(0x1008)) == -4 and call(a7=P(0x1002)) == -4


def test_structs_are_as_the_header_lays_them_out(tmp_path):
    import subprocess
    from paper_2512_06547_amd import binding as B
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = dict(a3po_sampling=B.Sampling, a3po_adamw_tensor=B.AdamwTensor, a3po_adamw_options=B.AdamwOptions)
    lines = []
    for name, mirror in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {field}));' for field, _ in mirror._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "a3po.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for mirror in structs.values():
        want.append(ctypes.sizeof(mirror))
        want += [getattr(mirror, field).offset for field, _ in mirror._fields_]
    assert out == want


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    import paper_2512_06547_amd as a3po
    z = torch.zeros(4, 64)
    for call in (lambda: a3po.sample(z, torch.zeros(4)), lambda: a3po.grad_norm([z]), lambda: a3po.w4_quantize(z, 64),
                 lambda: a3po.adamw_step([z], [z], [z], [z], step=1, lr=0.1)):
        with pytest.raises((AssertionError, ValueError)):
            call()
    with pytest.raises(ValueError):
        a3po.adamw_state(z, 16)
