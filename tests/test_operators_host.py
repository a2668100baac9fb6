"""Refusals and host-side plans of the operators around the log-probs (norm, adjusted logits, 4-bit head); no GPU needed:
every call here returns at validation, before any device pointer is used."""
import ctypes
import os

import pytest

from test_launch_plans import run_on_host


@pytest.fixture(scope="module")
def lib():
    import paper_2512_06547_amd as a3po
    if not os.path.exists(a3po.lib_path()):
        from paper_2512_06547_amd import build
        build.build(force=True)
    return a3po.lib()


P = lambda a=0x1000: ctypes.c_void_p(a)


def caller(fn, base):
    def call(**kw):
        args = list(base)
        for k, v in kw.items():
            args[int(k[1:])] = v
        return fn(*args)
    return call


def test_norm_fwd_refuses(lib):
    # x, x_dt, T, H, ldx, weight, bias, param_dt, eps, kind, y, y_dt, ldy, mean, rstd, stream
    call = caller(lib.a3po_norm_fwd, [P(), 1, 4, 64, 64, P(), P(), 1, 1e-6, 0, P(), 1, 64, P(), P(), None])
    assert call(a2=0) == 0 and call(a2=0, a0=None, a10=None) == 0
    for at in (1, 7, 11):
        assert call(**{f"a{at}": 2}) == -3 and call(**{f"a{at}": -1}) == -3
    assert call(a2=-1) == -2 and call(a2=(1 << 40) + 1) == -2
    assert call(a3=0) == -2 and call(a3=16385, a4=20000, a12=20000) == -2
    assert call(a4=63) == -2 and call(a12=63) == -2 and call(a4=(1 << 40) + 1) == -2
    assert call(a8=-1e-6) == -7 and call(a8=float("nan")) == -7 and call(a9=2) == -7
    assert call(a9=1) == -7 and call(a9=1, a6=None) == -7          # the RMS form has no bias and no mean
    assert call(a0=None) == -1 and call(a10=None) == -1
    for at in (0, 5, 6, 10):
        assert call(**{f"a{at}": P(0x1001)}) == -4
    assert call(a0=P(0x1002), a1=0) == -4 and call(a10=P(0x1002), a11=0) == -4


def test_norm_bwd_refuses(lib):
    # dy, y_dt, lddy, x, x_dt, T, H, ldx, weight, param_dt, mean, rstd, kind, dx, lddx, dweight, dbias, accumulate, ws, bytes, stream
    need = lib.a3po_workspace_bytes(3, 4, 0, 64)
    call = caller(lib.a3po_norm_bwd, [P(), 1, 64, P(), 1, 4, 64, 64, P(), 1, P(), P(), 0, P(), 64, P(), P(), 0, P(0x10000), need - 1,
                                      None])
    assert call() == -5 and call(a18=None, a19=1 << 30) == -5 and call(a18=P(0x10010), a19=need) == -4
    assert call(a1=2) == -3 and call(a4=2) == -3 and call(a9=2) == -3
    assert call(a5=-1) == -2 and call(a6=0) == -2 and call(a6=16385) == -2
    assert call(a2=63) == -2 and call(a7=63) == -2 and call(a14=63) == -2
    assert call(a12=2) == -7 and call(a17=2) == -7 and call(a12=1) == -7   # no dbias in the RMS form
    assert call(a0=None) == -1 and call(a3=None) == -1 and call(a10=None) == -1 and call(a11=None) == -1 and call(a13=None) == -1
    assert call(a13=P(0x1001)) == -4 and call(a8=P(0x1001)) == -4
    assert call(a5=0, a15=None, a16=None, a18=None, a19=0) == 0            # nothing to do


def test_adjust_logits_refuses(lib):
    from paper_2512_06547_amd.binding import LogitAdjustments
    need = lib.a3po_workspace_bytes(4, 4, 100, 0)
    # logits, dt, T, V, ld, adj, chosen, out, out_dt, ld_out, lse, logp, ws, bytes, stream
    call = caller(lib.a3po_adjust_logits, [P(), 1, 4, 100, 100, None, P(), P(), 0, 100, P(), P(), P(0x10000), need - 1, None])
    assert call() == -5 and call(a12=None, a13=1 << 30) == -5 and call(a12=P(0x10010), a13=need) == -4
    assert call(a1=2) == -3 and call(a8=2) == -3
    assert call(a2=-1) == -2 and call(a3=0) == -2 and call(a4=99) == -2 and call(a9=99) == -2 and call(a3=1 << 31, a4=1 << 31) == -2
    assert call(a0=None) == -1 and call(a6=None) == -1                     # log-probs need chosen tokens
    assert call(a7=None, a10=None, a11=None) == -1                         # no output at all
    assert call(a0=P(0x1001)) == -4 and call(a7=P(0x1002)) == -4
    assert call(a2=0) == 0
    adj = lambda **kw: ctypes.byref(LogitAdjustments(**kw))
    assert call(a5=adj(history=0x1000, history_tokens=-1, hist_start=0x1000, hist_len=0x1000)) == -2
    assert call(a5=adj(history=0x1000, history_tokens=5, hist_len=0x1000)) == -1
    assert call(a5=adj(history=0x1000, history_tokens=5, hist_start=0x1000)) == -1
    assert call(a5=adj(bias=0x1000, bias_ld=99)) == -2 and call(a5=adj(bias=0x1002)) == -4
    assert call(a5=adj(allowed=0x1000, allowed_ld=3)) == -2 and call(a5=adj(allowed=0x1000, allowed_ld=4)) == -5
    assert call(a5=adj(history=0x1000, history_tokens=5, hist_start=0x1004, hist_len=0x1000)) == -4
    for name in ("repetition", "frequency", "presence", "temperature"):
        assert call(a5=adj(**{name: 0x1002})) == -4


def test_adjust_logits_bwd_refuses(lib):
    from paper_2512_06547_amd.binding import LogitAdjustments
    hist = lambda **kw: ctypes.byref(LogitAdjustments(history=0x1000, history_tokens=5, hist_start=0x1000, hist_len=0x1000, **kw))
    # dout, out_dt, ld_out, logits, dt, T, V, ld, adj, dlogits, ld_d, stream
    call = caller(lib.a3po_adjust_logits_bwd, [P(), 0, 100, P(), 1, 4, 100, 100, hist(repetition=0x1000), P(), 100, None])
    assert call(a1=2) == -3 and call(a4=2) == -3
    assert call(a2=99) == -2 and call(a7=99) == -2 and call(a10=99) == -2 and call(a5=-1) == -2 and call(a6=0) == -2
    assert call(a0=None) == -1 and call(a9=None) == -1 and call(a3=None) == -1
    assert call(a0=P(0x1002)) == -4 and call(a3=P(0x1001)) == -4 and call(a9=P(0x1001)) == -4
    assert call(a5=0, a3=None) == 0


def test_w4_linear_refuses(lib):
    # x, T, H, ldx, codes, scales, scale_dt, zeros, group, N, out, out_dt, ld_out, workspace, bytes, stream
    need = lib.a3po_workspace_bytes(5, 40, 0, 256)
    call = caller(lib.a3po_w4_linear, [P(), 40, 256, 256, P(), P(), 1, P(), 64, 100, P(), 0, 100, P(0x10000), need - 1, None])
    assert call() == -5 and call(a13=None, a14=1 << 30) == -5 and call(a13=P(0x10010), a14=need) == -4
    assert lib.a3po_workspace_bytes(5, 16, 0, 4096) == 0 and need % 256 == 0 and need > 40 * 256 * 2
    assert call(a6=2) == -3 and call(a11=2) == -3
    for group in (0, 16, 48, 256, -64):
        assert call(a8=group) == -2
    assert call(a2=0) == -2 and call(a2=224) == -2 and call(a2=(1 << 20) + 64, a3=1 << 21) == -2   # H: a multiple of the group
    assert call(a1=-1) == -2 and call(a1=65535 * 64 + 1) == -2 and call(a9=0) == -2 and call(a9=1 << 31, a12=1 << 31) == -2
    assert call(a3=255) == -2 and call(a12=99) == -2
    assert call(a0=None) == -1 and call(a4=None) == -1 and call(a5=None) == -1 and call(a10=None) == -1
    assert call(a0=P(0x1001)) == -4 and call(a4=P(0x1008)) == -4 and call(a5=P(0x1001)) == -4 and call(a10=P(0x1002)) == -4
    assert call(a1=0, a0=None, a4=None) == 0


def test_workspaces_grow_with_their_calls_and_take_any_size(lib):
    ws = lib.a3po_workspace_bytes
    for which in (3, 4, 5):
        sizes = [ws(which, T, 151936, 4096) for T in (-1, 0, 1, 7, 100, 10000, 65536)]
        assert all(s % 256 == 0 and (s > 0 or which == 5) for s in sizes) and (which == 4 or sizes == sorted(sizes))
    assert ws(3, 5, 0, -1) > 0 and ws(3, 5, 0, 1 << 40) > 0 and ws(4, 5, -1, 0) > 0


def test_binding_refuses_what_the_library_cannot_see():
    """Types and shapes of tensors (CPU tensors are refused before anything else is asked of them)."""
    torch = pytest.importorskip("torch")
    import paper_2512_06547_amd as a3po
    x = torch.zeros(4, 64)
    for call in (lambda: a3po.norm_fwd(x), lambda: a3po.norm_bwd(x, x, None, x[:, 0]), lambda: a3po.adjust_logits(x),
                 lambda: a3po.adjust_logits_bwd(x), lambda: a3po.w4_linear(x, x, x),
                 lambda: a3po.w4_linear(x.bfloat16(), x, x)):
        with pytest.raises((AssertionError, TypeError)):
            call()


def test_norm_plan_holds_every_row(tmp_path):
    """Every width has a kernel that holds its whole vectors, with no more than half of the lanes' vectors idle beyond the
    narrowest one, and the workspace holds every workgroup's share."""
    source = tmp_path / "norm.cpp"
    source.write_text('''#include <cstdio>
#include "a3po_common.h"
#include "a3po_launch.h"
using namespace a3po;
int main()
{
    for (int bytes : {2, 4})
        for (int64_t T : {1, 3, 5, 256, 257, 511, 513, 4096, 100000})
            for (int64_t k = 2; k <= 2 * kNormMaxH + 1; ++k) {
                const int64_t H = k / 2;
                const bool back = k % 2;
                const NormPlan p = norm_plan(T, H, bytes, back);
                const int64_t full = H / (16 / bytes), room = (int64_t)p.lanes * p.vectors, b = norm_bwd_blocks(T, H, bytes);
                const int v = p.vectors;
                bool known = false;
                if (p.lanes == 64) known = v == 1 || v == 2 || v == 3 || (v == 4 && (bytes == 4 || back)) || (v == 6 && bytes == 4);
                if (p.lanes == 256) known = v >= 1 && v <= 4;
                if (p.lanes == 512) known = v == 4 || (v == 3 && bytes == 2) || ((v == 6 || v == 8) && bytes == 4);
                if (!known || full > room || (v > 1 && full * 2 <= room - p.lanes) || b < 1 || b > T ||
                    (size_t)b * 8 * H > norm_bwd_workspace_bytes(T, H))
                    return std::printf("T %lld H %lld\\n", (long long)T, (long long)H), 1;
            }
    std::printf("ok\\n");
}
''')
    assert run_on_host(str(source), tmp_path) == "ok\n"


def test_adjust_plan_covers_every_row_within_lds(tmp_path):
    source = tmp_path / "adjust.cpp"
    source.write_text('''#include <cstdio>
#include "a3po_common.h"
#include "a3po_launch.h"
using namespace a3po;
int main()
{
    for (int bytes : {2, 4, -2, -4})  // (negative: the backward pass, without a workspace)
        for (int64_t T : {1, 2, 5, 64, 300, 1023, 1024, 5000, 1 << 24})
            for (int64_t V = 1; V < 0x7FFFFFFF; V += V < 70000 ? 1 : 1 + V / 9) {
                const AdjustPlan p = adjust_plan(T, V, bytes < 0 ? -bytes : bytes, bytes < 0);
                const int64_t parts = (int64_t)1 << p.shift;
                const bool ok = p.part % 512 == 0 && p.part > 0 && p.part <= kAdjustMaxPart && parts * p.part >= V &&
                                (parts == 1 || V > parts * 512 / 2) &&
                                (bytes < 0 || adjust_partials_offset(T) + (size_t)T * parts * 8 <= adjust_workspace_bytes(T, V));
                if (!ok) return std::printf("T %lld V %lld\\n", (long long)T, (long long)V), 1;
            }
    std::printf("ok\\n");
}
''')
    assert run_on_host(str(source), tmp_path) == "ok\n"


def test_w4_linear_asks_for_a_workspace_where_its_kernel_uses_one(lib):
    # x, T, H, ldx, codes, scales, scale_dt, zeros, group, N, out, out_dtype, ld_out, workspace, bytes, stream
    call = caller(lib.a3po_w4_linear, [P(), 1, 256, 1 << 20, P(), P(), 1, P(), 32, 100, P(0x1001), 0, 100, None, 0, None])
    ws = lib.a3po_workspace_bytes
    no_ws = [(1, 256), (8, 6144), (16, 4096), (17, 1920), (32, 1024), (32, 256), (20, 1664)]
    for T, H in no_ws:
        assert ws(5, T, 0, H) == 0, (T, H)
    for T, H in [(1, 128), (1, 8192), (9, 4224), (17, 2048), (32, 2176), (33, 256), (64, 4096), (5, 160)]:
        assert ws(5, T, 0, H) > 0, (T, H)
    # out of place, out is refused before the workspace; in place, only a missing workspace is
    for T, H in no_ws:
        assert call(a1=T, a2=H) == -4
    assert call(a1=17, a2=2048, a10=P(), a8=128) == -5 and call(a1=9, a2=4224, a10=P(), a8=64, a6=0) == -5
    assert call(a1=4, a2=8192, a10=P(), a8=32, a6=0) == -5


def test_w4_plans_fit_their_kernels(tmp_path):
    """A call has a resident plan exactly where it needs no workspace; the plan's units, rows and LDS are what its kernels are
    there for; tiles of the streaming kernel hold every row once; the workspace holds what its first kernels write."""
    source = tmp_path / "w4.cpp"
    source.write_text('''#include <cstdio>
#include "a3po_common.h"
#include "a3po_launch.h"
using namespace a3po;
int main()
{
    for (int cus : {256, 304, 80})
        for (int64_t N : {1, 15, 16, 17, 530, 4096, 65535, 65536, 131073, 151936, 1 << 22}) {
            const W4Tiles t = w4_tiles(N, cus);
            const int64_t rows = t.wide * 256ll + t.narrow * 128ll;
            const bool tight = t.narrow ? rows - 128 < N : rows - 256 < N;
            if (rows < N || !tight || t.blocks < 1 || t.blocks > cus || (t.narrow > t.blocks && t.blocks < cus))
                return std::printf("tiles of %lld rows\\n", (long long)N), 1;
            for (int64_t T = 1; T <= 40; ++T)
                for (int64_t H = 32; H <= 9000; H += 32)
                    for (int group : {32, 64, 128})
                        for (bool f32 : {false, true}) {
                            if (H % group) continue;
                            const W4Plan p = w4_plan(T, H, N, group, f32, cus);
                            const bool resident = w4_resident(T, H, group, f32);
                            bool ok = (p.units != 0) == resident && (w4_workspace_bytes(T, H) != 0 || resident);
                            if (p.units) {
                                const int64_t a_row = 1 << p.wk_shift, rows_a_set = 16 * (16 >> p.wk_shift);
                                ok = ok && p.units >= 2 && p.units <= (group == 32 && f32 ? 3 : 4) && p.units <= H / 128 &&
                                     p.units * a_row >= H / 128 && p.lds <= kW4MaxLds && (H << p.tp_shift) <= 8 * 8 * 1024 && (1 << p.tp_shift) >= T &&
                                     p.blocks16 * 16 >= (1 << p.tp_shift) && p.sets * rows_a_set >= N &&
                                     (p.sets - 1) * rows_a_set < N && p.blocks >= 1 && p.blocks <= p.sets && p.blocks <= cus &&
                                     (p.blocks == cus || p.blocks == p.sets);
                            }
                            if (!ok) return std::printf("T %lld H %lld N %lld\\n", (long long)T, (long long)H, (long long)N), 1;
                        }
        }
    for (int64_t T = 1; T < 5000; ++T)
        for (int64_t H : {32, 160, 4096, 4128, 1 << 20}) {
            const size_t have = w4_workspace_bytes(T, H);
            if (!have) continue;
            const int64_t readings = (T + 63) / 64, even = (T + readings - 1) / readings;
            const int64_t a_pass = even <= 16 ? 16 : even <= 32 ? 32 : even <= 48 ? 48 : 64, tokens = (T + a_pass - 1) / a_pass * a_pass;
            const size_t need = (size_t)tokens / 16 * ((H + 511) / 512 * 4) * kW4UnitBytes + tokens * 4 + 2 * kW4ShortBytes;
            if (have < need || have % 256) return std::printf("T %lld H %lld\\n", (long long)T, (long long)H), 1;
        }
    std::printf("ok\\n");
}
''')
    assert run_on_host(str(source), tmp_path) == "ok\n"


def test_adjusted_rows_numbers_and_lists_fit_lds(tmp_path):
    '''What a part keeps in LDS beside the kernel's own 100 bytes, and the threads that number its blocks of 512 entries.  Every
    plan that a call can get: parts of the forward pass end at 262,144 entries, those of the backward pass at 65,536.'''
    source = tmp_path / "lds.cpp"
    source.write_text('''#include <cstdio>
#include "a3po_common.h"
#include "a3po_launch.h"
using namespace a3po;
int main()
{
    int widest[2] = {0, 0}, small_list = 0, half_numbers = 0, few_threads = 0;
    for (int bytes : {2, 4})
        for (bool backward : {false, true})
            for (int64_t T : {1, 2, 64, 300, 600, 1023, 1024, 1030, 5000, 1 << 22})
                for (int64_t V = 1; V < 0x7FFFFFFF; V += V < 600000 ? 1 + V / 4096 : 1 + V / 9)
                    for (bool written : {false, true}) {
                        const AdjustPlan p = adjust_plan(T, V, bytes, backward);
                        const int threads = backward ? kAdjustThreads : adjust_threads(T, p, written);
                        const bool known = threads == kAdjustThreads || (!backward && threads == kAdjustThreads / 2);
                        if (!known || adjust_lds(p.part, threads, backward) > 64 * 1024 - 128 || (!backward && p.part / 512 > threads))
                            return std::printf("T %lld V %lld part %d\\n", (long long)T, (long long)V, p.part), 1;
                        if (p.part > widest[backward]) widest[backward] = p.part;
                        small_list += !backward && adjust_listed(p.part, threads) * (threads / kWave) == 1024;
                        half_numbers += !backward && adjust_numbers(p.part) == 1024;
                        few_threads += threads < kAdjustThreads;
                    }
    std::printf("%d %d %d %d %d\\n", widest[0], widest[1], small_list > 0, half_numbers > 0, few_threads > 0);
}
''')
    assert run_on_host(str(source), tmp_path) == f"{1 << 18} {1 << 16} 1 1 1\n"


def test_the_cases_of_many_rows_take_several_sets_and_tiles_a_workgroup(tmp_path):
    """What the GPU tests' sizes are there for, with the compute units of an MI355X."""
    pytest.importorskip("torch")
    from test_gpu_w4 import MANY_SETS, MANY_TILES
    source = tmp_path / "many.cpp"
    rows = lambda cases: ", ".join(f"{{{T}, {N}, {H}, {group}, {int(f32)}}}" for T, N, H, group, _, f32 in cases)
    source.write_text(f'''#include <cstdio>
#include "a3po_common.h"
#include "a3po_launch.h"
using namespace a3po;
int main()
{{
    const int sets[][5] = {{{rows(MANY_SETS)}}}, tiles[][5] = {{{rows(MANY_TILES)}}};
    for (auto &c : sets) {{
        const W4Plan p = w4_plan(c[0], c[2], c[1], c[3], c[4], 256);
        if (p.sets <= 2 * p.blocks || p.sets % p.blocks == 0) return std::printf("T %d N %d H %d\\n", c[0], c[1], c[2]), 1;
        std::printf("%d%d ", p.units, p.blocks16);
    }}
    for (auto &c : tiles) {{
        const W4Tiles t = w4_tiles(c[1], 256);
        if (w4_plan(c[0], c[2], c[1], c[3], c[4], 256).units || t.wide < 2 * t.blocks || t.narrow == 0)
            return std::printf("T %d N %d H %d\\n", c[0], c[1], c[2]), 1;
    }}
    std::printf("ok\\n");
}}
''')
    kinds = run_on_host(str(source), tmp_path).split()
    assert kinds.pop() == "ok" and {"21", "31", "41", "22", "32", "42"} <= set(kinds), kinds
