"""What the entry points of head norms with rotary positions, projections, the gated block and AdamW refuse, at the C ABI,
before any GPU call; and what the binding refuses."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_02091_amd import dflare as dfl
from product_shapes import WAYS

INV, UNS, OK = dfl.ERR_INVALID_ARG, dfl.ERR_UNSUPPORTED, dfl.OK
INF, NAN = float("inf"), float("nan")
FAR = [(i + 1) << 40 for i in range(20)]  # addresses far from one another


def refused(call, size, written, fine=()):
    """Every written tensor on the first and on the last bytes of every other one; `fine` names the pairs that may be one."""
    at = dict(zip(size, FAR))
    for w in written:
        for o in size:
            if o == w:
                continue
            step = 16 if size[o] >= 32 else 4
            assert call(**{**at, w: at[o] + size[o] - step}) == INV, (w, o, "end")
            assert call(**{**at, w: at[o] - size[w] + 16 if size[w] >= 32 else at[o]}) == INV, (w, o, "start")
            if (w, o) not in fine:
                assert call(**{**at, w: at[o]}) == INV, (w, o)


# ---- head norms with rotary positions ----

def qk(n=1, rows=4, B=1, hd=64, rot=64, dtype=dfl.BF16, layout=0, scale=1.0, eps=1e-6, pos=FAR[0], freq=FAR[1], x=FAR[2], y=FAR[3],
       gain=FAR[4], heads=2, strides=(128, 64, 128, 64), tab=True):
    t = (dfl.dflare_qk_tensor * 2)(*[dfl.dflare_qk_tensor(x, y, gain, *strides, heads)] * 2)
    return dfl.lib().dflare_qk_norm_rope_fwd(t if tab else None, n, pos, freq, rows, B, hd, rot, dtype, layout, scale, eps, None)


QK_BAD = [
    (dict(n=0), INV), (dict(n=3), INV), (dict(tab=False), INV), (dict(rows=-1), INV), (dict(B=0), INV), (dict(hd=1), INV), (dict(rot=0), INV),
    (dict(rot=63), INV), (dict(rot=66), INV), (dict(dtype=2), INV), (dict(layout=2), INV), (dict(scale=NAN), INV), (dict(scale=INF), INV),
    (dict(eps=-1.0), INV), (dict(eps=NAN), INV), (dict(eps=INF), INV), (dict(freq=None), INV), (dict(freq=FAR[1] + 4), INV),
    (dict(pos=FAR[0] + 2), INV), (dict(x=None), INV), (dict(x=FAR[2] + 1), INV), (dict(gain=FAR[4] + 1), INV), (dict(heads=-1), INV),
    (dict(hd=514, rot=64), UNS), (dict(heads=1 << 15), UNS)]


@pytest.mark.parametrize("kw,code", QK_BAD + [
    (dict(y=None), INV), (dict(y=FAR[3] + 1), INV), (dict(y=FAR[3] + 2, dtype=dfl.F32), INV), (dict(y=FAR[2], strides=(128, 64, 256, 64)), INV),
    (dict(n=2), INV), (dict(strides=(128, 64, 0, 64)), INV), (dict(strides=(128, 64, 128, 63)), INV), (dict(y=FAR[2] + 2), INV),
    (dict(y=FAR[0] + 4), INV), (dict(y=FAR[1] + 240), INV), (dict(y=FAR[4] + 126), INV), (dict(gain=FAR[3] + 1000), INV),
    (dict(rows=0, x=None, y=None), OK), (dict(heads=0, x=None, y=None), OK)])
def test_qk_norm_rope_refuses(kw, code):
    assert qk(**kw) == code


def qk_bwd(n=1, rows=4, B=1, hd=64, rot=64, dtype=dfl.BF16, layout=0, scale=1.0, eps=1e-6, pos=FAR[0], freq=FAR[1], x=FAR[2], dy=FAR[3],
           dx=FAR[4], gain=FAR[5], dgain=FAR[6], work=FAR[7], ws=1 << 30, heads=2, strides=(128, 64) * 3, tab=True):
    t = (dfl.dflare_qk_grad * 2)(*[dfl.dflare_qk_grad(x, dy, dx, gain, dgain, *strides, heads)] * 2)
    return dfl.lib().dflare_qk_norm_rope_bwd(t if tab else None, n, pos, freq, rows, B, hd, rot, dtype, layout, scale, eps, work, ws, None)


@pytest.mark.parametrize("kw,code", [(k, c) for k, c in QK_BAD if "gain" not in k] + [
    (dict(gain=FAR[5] + 1), INV), (dict(dgain=FAR[6] + 2), INV), (dict(dx=None), INV), (dict(dy=None), INV), (dict(dy=FAR[3] + 1), INV),
    (dict(work=None), INV), (dict(work=FAR[7] + 8), INV), (dict(ws=16), INV), (dict(n=2), INV),
    (dict(dx=FAR[2], strides=(128, 64, 128, 64, 256, 64)), INV), (dict(dx=FAR[3], strides=(128, 64, 128, 64, 256, 64)), INV),
    (dict(strides=(128, 64, 128, 64, 64, 64)), INV)])
def test_qk_norm_rope_bwd_refuses(kw, code):
    assert qk_bwd(**kw) == code


def test_qk_norm_rope_bwd_refuses_every_overlap():
    ws = dfl.lib().dflare_qk_norm_rope_bwd_workspace(4, 64, 1)
    size = dict(pos=16, freq=256, x=1024, dy=1024, dx=1024, gain=128, dgain=256, work=ws)
    refused(qk_bwd, size, ("dx", "dgain", "work"), fine={("dx", "x"), ("dx", "dy")})


def test_qk_norm_rope_workspace():
    ws = dfl.lib().dflare_qk_norm_rope_bwd_workspace
    assert ws(-1, 64, 1) == ws(4, 1, 1) == ws(4, 513, 1) == ws(4, 64, 0) == ws(4, 64, 3) == 0
    assert 0 < ws(1, 64, 1) <= ws(100, 64, 1) <= ws(100, 128, 1) <= ws(100, 128, 2) <= ws(1 << 20, 128, 2)


# ---- projections and the gated block ----

def lin(rows=40, N=136, K=64, act=0, x=FAR[0], w=FAR[1], bias=FAR[2], res=FAR[3], y=FAR[4], z=FAR[5], work=FAR[6], ws=1 << 40):
    return dfl.lib().dflare_linear_fwd(x, w, bias, res, rows, N, K, act, y, z, work, ws, None)


def lin_bwd(rows=40, N=136, K=64, act=2, dy=FAR[0], x=FAR[1], w=FAR[2], z=FAR[3], dx=FAR[4], dw=FAR[5], db=FAR[6], work=FAR[7], ws=1 << 40):
    return dfl.lib().dflare_linear_bwd(dy, x, w, z, rows, N, K, act, dx, dw, db, work, ws, None)


def gate(rows=40, H=64, F=136, act=2, x=FAR[0], wg=FAR[1], wu=FAR[2], h=FAR[3], g=FAR[4], u=FAR[5], work=FAR[6], ws=1 << 40):
    return dfl.lib().dflare_gated_fwd(x, wg, wu, rows, H, F, act, h, g, u, work, ws, None)


def gate_bwd(rows=40, H=64, F=136, act=2, dh=FAR[0], x=FAR[1], g=FAR[2], u=FAR[3], wg=FAR[4], wu=FAR[5], dx=FAR[6], dwg=FAR[7], dwu=FAR[8],
             work=FAR[9], ws=1 << 40):
    return dfl.lib().dflare_gated_bwd(dh, x, g, u, wg, wu, rows, H, F, act, dx, dwg, dwu, work, ws, None)


XB, WB, YB = 40 * 64 * 2, 136 * 64 * 2, 40 * 136 * 2


@pytest.mark.parametrize("call,wide,deep", [(lin, "N", "K"), (lin_bwd, "N", "K"), (gate, "F", "H"), (gate_bwd, "F", "H")])
def test_products_refuse_sizes(call, wide, deep):
    for kw, code in ((dict(rows=-1), INV), ({wide: 0}, INV), ({deep: 0}, INV), ({deep: -8}, INV), (dict(act=5), INV), (dict(act=-1), INV),
                     ({wide: 132}, UNS), ({deep: 60}, UNS), ({wide: (1 << 18) + 8}, UNS), ({deep: (1 << 18) + 8}, UNS),
                     (dict(rows=(1 << 22) + 1), UNS), ({"rows": 1 << 22, wide: 1 << 18}, UNS), ({wide: 1 << 18, deep: 1 << 18}, UNS),
                     (dict(ws=64), INV), (dict(work=None), INV), (dict(work=FAR[9] + 8), INV)):
        assert call(**kw) == code, kw


@pytest.mark.parametrize("call,needed", [
    (lin, ("x", "w", "y")), (lin_bwd, ("dy", "x", "w", "z")), (gate, ("x", "wg", "wu", "h", "g", "u")),
    (gate_bwd, ("dh", "x", "g", "u", "wg", "wu", "dwg", "dwu"))])
def test_products_refuse_what_is_missing_or_misplaced(call, needed):
    for k in needed:
        assert call(**{k: None}) == INV, k
        assert call(**{k: (1 << 45) + 8}) == INV, k


def test_products_refuse_every_overlap():
    L = dfl.lib()
    refused(lin, dict(x=XB, w=WB, bias=272, res=YB, y=YB, z=YB, work=L.dflare_linear_fwd_workspace(40, 136, 64)), ("y", "z", "work"),
            fine={("y", "res")})
    refused(lin_bwd, dict(dy=YB, x=XB, w=WB, z=YB, dx=XB, dw=WB, db=272, work=L.dflare_linear_bwd_workspace(40, 136, 64, 2, 1, 1, 1)),
            ("dx", "dw", "db", "work"))
    refused(gate, dict(x=XB, wg=WB, wu=WB, h=YB, g=YB, u=YB, work=L.dflare_gated_fwd_workspace(40, 64, 136)), ("h", "g", "u", "work"))
    refused(gate_bwd, dict(dh=YB, x=XB, g=YB, u=YB, wg=WB, wu=WB, dx=XB, dwg=WB, dwu=WB, work=L.dflare_gated_bwd_workspace(40, 64, 136, 1, 1)),
            ("dx", "dwg", "dwu", "work"))


def test_workspaces_of_products_grow_with_every_size():
    L = dfl.lib()
    rng = np.random.default_rng(3)
    calls = [L.dflare_linear_fwd_workspace, L.dflare_gated_fwd_workspace] + [
        (lambda *s, k=k: L.dflare_linear_bwd_workspace(*s, *k)) for k in ((0, 1, 1, 0), (2, 1, 1, 1), (2, 0, 1, 0), (1, 1, 0, 1))] + [
        (lambda *s, k=k: L.dflare_gated_bwd_workspace(*s, *k)) for k in ((1, 1), (0, 1), (1, 0))]
    for f in calls:
        assert f(-1, 8, 8) == f(4, 12, 8) == f(4, 8, 12) == f(4, 0, 8) == 0
        assert f(0, 8, 8) > 0
    for _ in range(2000):
        big = [int(2 ** rng.uniform(0, 14))] + [8 * int(2 ** rng.uniform(0, 11)) for _ in range(2)]
        small = [int(rng.integers(1, big[0] + 1))] + [8 * int(rng.integers(1, v // 8 + 1)) for v in big[1:]]
        for f in calls:
            assert 0 < f(*small) <= f(*big)


def test_workspace_of_a_bias_gradient_grows_across_its_chunks():
    """The rows are cut into fewer chunks where columns take more work-groups; the space does not shrink there."""
    f = dfl.lib().dflare_linear_bwd_workspace
    for rows in (1, 5, 1000, 8192, 1 << 20):
        last = 0
        for N in (8, 2040, 2048, 2056, 4096, 4104, 12288, 12296, 65536, 65544, 1 << 18):
            now = f(rows, N, 64, 0, 0, 0, 1)
            if now == 0:  # about 2^35 values
                break
            assert now >= last
            last = now
            chunks = max(1, min(-(-rows // 4), 2048 // -(-N // 2048)))
            assert now >= chunks * N * 4


# ---- AdamW ----

ADAM = dict(p=FAR[0], g=FAR[1], w=FAR[2], m=FAR[3], v=FAR[4], ms=FAR[5], vs=FAR[6])


def adam(n=1, tab=True, opt=True, values=600, pt=dfl.BF16, gt=dfl.BF16, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.1, step=1, lrd=None, stepd=None,
         sumsq=None, max_norm=1.0, bits=8, **at):
    a = {**ADAM, **at}
    t = dfl.dflare_adamw_tensor(a["p"], a["g"], a["w"], a["m"], a["v"], a["ms"], a["vs"], values, pt, gt)
    o = dfl.dflare_adamw_options(lr, b1, b2, eps, wd, step, lrd, stepd, sumsq, max_norm, bits)
    return dfl.lib().dflare_adamw((dfl.dflare_adamw_tensor * 2)(t, t) if tab else None, n, ctypes.byref(o) if opt else None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(opt=False), INV), (dict(n=-1), INV), (dict(tab=False), INV), (dict(n=2), INV), (dict(values=-1), INV), (dict(values=(1 << 36) + 1), UNS),
    (dict(pt=2), INV), (dict(gt=-1), INV), (dict(pt=dfl.F32), INV), (dict(lr=-1.0), INV), (dict(lr=NAN), INV), (dict(lr=INF), INV),
    (dict(b1=1.0), INV), (dict(b1=-0.1), INV), (dict(b2=1.0), INV), (dict(b2=NAN), INV), (dict(eps=0.0), INV), (dict(eps=1e-60), INV), (dict(eps=1e-39), INV),
    (dict(eps=INF), INV), (dict(wd=-1.0), INV), (dict(wd=INF), INV), (dict(step=0), INV), (dict(bits=16), INV), (dict(bits=0), INV),
    (dict(sumsq=FAR[8], max_norm=-1.0), INV), (dict(sumsq=FAR[8], max_norm=NAN), INV), (dict(sumsq=FAR[8] + 4), INV), (dict(lrd=FAR[8] + 4), INV),
    (dict(stepd=FAR[8] + 4), INV), (dict(p=None), INV), (dict(g=None), INV), (dict(m=None), INV), (dict(v=None), INV), (dict(ms=None), INV),
    (dict(vs=None), INV), (dict(p=FAR[0] + 1), INV), (dict(g=FAR[1] + 2, gt=dfl.F32), INV), (dict(w=FAR[2] + 2), INV), (dict(ms=FAR[5] + 2), INV),
    (dict(bits=32, m=FAR[3] + 2), INV), (dict(bits=32, v=FAR[4] + 1), INV)])
def test_adamw_refuses(kw, code):
    assert adam(**kw) == code


def test_adamw_refuses_every_overlap():
    size = dict(p=1200, g=1200, w=2400, m=600, v=600, ms=12, vs=12, sumsq=8, lrd=8, stepd=8)
    for bits in (8, 32):
        s = size if bits == 8 else {**size, "m": 2400, "v": 2400}
        at = dict(zip(s, FAR))
        for a in s:
            for b in s:
                if a == b or not {a, b} & {"p", "w", "m", "v", "ms", "vs"} or (bits == 32 and {a, b} & {"ms", "vs"}):
                    continue
                assert adam(**{**at, a: at[b]}, bits=bits) == INV, (a, b, bits)
                assert adam(**{**at, a: at[b] + s[b] // 8 * 8 - (8 if s[b] % 8 == 0 else 0)}, bits=bits) == INV, (a, b, bits)


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused is launched")
def test_tensors_that_lie_apart_are_not_refused():
    """Calls in place, and tensors that follow each other without a byte between them, reach the launch."""
    L, launched = dfl.lib(), dfl.ERR_HIP

    def packed(size):
        at, out = FAR[0], {}
        for k, n in size.items():
            out[k], at = at, at + n
        return out
    assert lin(**packed(dict(x=XB, w=WB, bias=272, res=YB, y=YB, z=YB, work=L.dflare_linear_fwd_workspace(40, 136, 64)))) == launched
    assert lin(y=FAR[3]) == launched and lin(bias=None, res=None, z=None) == launched and lin(rows=0, x=None, y=None) == OK
    assert lin_bwd(**packed(dict(dy=YB, x=XB, w=WB, z=YB, dx=XB, dw=WB, db=272, work=L.dflare_linear_bwd_workspace(40, 136, 64, 2, 1, 1, 1)))) == launched
    # what a call does not read may be written
    assert lin_bwd(act=0, z=None) == launched and lin_bwd(dx=None, dw=FAR[2]) == launched and lin_bwd(dw=None, dx=FAR[1]) == launched
    assert gate(**packed(dict(x=XB, wg=WB, wu=WB, h=YB, g=YB, u=YB, work=L.dflare_gated_fwd_workspace(40, 64, 136)))) == launched
    assert gate_bwd(**packed(dict(dh=YB, x=XB, g=YB, u=YB, wg=WB, wu=WB, dx=XB, dwg=WB, dwu=WB,
                                  work=L.dflare_gated_bwd_workspace(40, 64, 136, 1, 1)))) == launched
    assert qk(y=FAR[2]) == launched and qk(gain=None, pos=None) == launched
    assert qk_bwd(dx=FAR[2]) == launched and qk_bwd(dx=FAR[3]) == launched and qk_bwd(gain=None, dgain=None) == launched
    size = dict(p=1200, g=1200, w=2400, m=600, v=600, ms=12, vs=12, sumsq=8, lrd=8, stepd=8)
    assert adam(**packed(size)) == launched and adam(values=0, p=None, g=None, m=None, v=None) == launched


# ---- the binding ----

def test_binding_refuses_what_is_not_on_a_device():
    t, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 8, dtype=torch.bfloat16)
    for call in (lambda: dfl.linear_fwd(t, w), lambda: dfl.linear_bwd(t, t, w), lambda: dfl.gated_fwd(t, w, w),
                 lambda: dfl.gated_bwd(t, t, t, t, w, w), lambda: dfl.qk_norm_rope_fwd(t.view(4, 1, 8), None, t),
                 lambda: dfl.qk_norm_rope_bwd(t.view(4, 1, 8), t.view(4, 1, 8), None, t), lambda: dfl.linear_fwd(None, None),
                 lambda: dfl.adamw([t], [t], [t], [t], 1, 0.1)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        dfl.adamw([t], [], [t], [t], 1, 0.1)
    with pytest.raises(ValueError):
        dfl.adamw_state([t], 16)
    assert dfl.adamw([], [], [], [], 1, 0.1) is None
    m, v, ms, vs = dfl.adamw_state([torch.zeros(3, 100), torch.zeros(0)], 8)
    assert m[0].shape == (3, 100) and m[0].dtype == torch.float8_e4m3fn and ms[0].shape == (2,) and vs[1].shape == (0,)


def plans(kind, rows, N, K, act=2, dx=1, dw=1, dbias=1):
    """(forward, backward) plan of a projection or the gated block."""
    L, fwd, bwd = dfl.lib(), dfl.dflare_product_plan(), dfl.dflare_product_plan()
    rc = (L.dflare_linear_plan(rows, N, K, act, dx, dw, dbias, fwd, bwd) if kind == "linear" else
          L.dflare_gated_plan(rows, K, N, dx, dw, fwd, bwd))
    assert rc == OK
    return fwd, bwd


def test_workspace_of_a_call_is_what_its_plan_takes():
    L = dfl.lib()
    # none for what has no parts: few rows, and more values than parts may have
    for rows, N, K in ((1, 4096, 4096), (16, 12288, 4096), (32, 6144, 2560), (8192, 12288, 4096)):
        assert plans("linear", rows, N, K)[0].workspace == plans("gated", rows, N, K)[0].workspace == 256
    assert L.dflare_linear_fwd_workspace(32, 6144, 2560) == L.dflare_gated_fwd_workspace(16, 4096, 12288) == 256
    assert plans("gated", 8192, 12288, 4096)[1].workspace == 2 * 8192 * 12288 * 2  # (dgate and dup)
    rng = np.random.default_rng(5)
    for _ in range(3000):
        rows, N, K = int(2 ** rng.uniform(0, 14)), 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        act, dx, dw, dbias = (int(v) for v in (rng.integers(0, 2) * 2, *rng.integers(0, 2, 3)))
        up = lambda n: -(-n // 256) * 256  # noqa: E731
        for kind, n2 in (("linear", 1), ("gated", 2)):
            f, b = plans(kind, rows, N, K, act, dx, dw, dbias)
            assert f.workspace == max(256, up(rows * N * n2 * f.parts * 4) if f.parts > 1 else 0) and f.parts_w == 1
            d = n2 if n2 == 2 or act else 0
            sums = max(1, min(-(-rows // 4), 2048 // -(-N // 2048))) * N * 4 if n2 == 1 and dbias else 0
            assert b.workspace == max(256, d * up(rows * N * 2) + up(sums) + (up(rows * K * b.parts * 4) if b.parts > 1 else 0) + (
                up(n2 * N * K * b.parts_w * 4) if b.parts_w > 1 else 0))
            assert (dx or b.parts == 1) and (dw or b.parts_w == 1)
            most = ((L.dflare_linear_fwd_workspace(rows, N, K), L.dflare_linear_bwd_workspace(rows, N, K, act, dx, dw, dbias)) if n2 == 1 else
                    (L.dflare_gated_fwd_workspace(rows, K, N), L.dflare_gated_bwd_workspace(rows, K, N, dx, dw)))
            assert f.workspace <= most[0] and b.workspace <= most[1]


def test_plans_of_sizes_that_are_refused():
    L, p = dfl.lib(), dfl.dflare_product_plan()
    for kw, code in ((dict(rows=-1), INV), (dict(N=0), INV), (dict(N=12), UNS), (dict(K=12), UNS), (dict(N=1 << 18, K=1 << 18), UNS)):
        a = {**dict(rows=40, N=136, K=64), **kw}
        assert L.dflare_linear_plan(a["rows"], a["N"], a["K"], 0, 1, 1, 1, p, p) == L.dflare_gated_plan(a["rows"], a["K"], a["N"], 1, 1, p, p) == code
    assert L.dflare_linear_plan(40, 136, 64, 5, 1, 1, 1, p, p) == INV
    assert L.dflare_linear_plan(40, 136, 64, 0, 1, 1, 1, None, None) == L.dflare_gated_plan(40, 64, 136, 1, 1, None, None) == OK


def test_products_refuse_a_byte_less_than_their_plan():
    for rows, N, K in ((40, 136, 64), (64, 1032, 2056), (1000, 72, 4096)):
        (lf, lb), (gf, gb) = plans("linear", rows, N, K), plans("gated", rows, N, K)
        far = [(i + 1) << 44 for i in range(10)]
        for k, ws in enumerate((lf, lb, gf, gb)):
            call = (lambda n: lin(rows, N, K, 2, *far[:7], n), lambda n: lin_bwd(rows, N, K, 2, *far[:8], n),
                    lambda n: gate(rows, K, N, 2, *far[:7], n), lambda n: gate_bwd(rows, K, N, 2, *far[:10], n))[k]
            assert call(ws.workspace - 1) == INV, (rows, N, K, k)
            if not torch.cuda.is_available():
                assert call(ws.workspace) == dfl.ERR_HIP, (rows, N, K, k)


@pytest.mark.parametrize("kind,rows,N,K,fwd,bwd", WAYS)
def test_products_take_the_ways_that_are_tested(kind, rows, N, K, fwd, bwd):
    f, b = plans(kind, rows, N, K)
    assert (f.tiles, f.parts > 1) == fwd and (b.tiles, b.parts > 1, b.parts_w > 1) == bwd


def test_every_way_of_a_product_is_among_the_tested_ones():
    """Of sizes over the whole range none takes another kernel, or the same one in parts where only its whole is tested."""
    rng = np.random.default_rng(11)
    ways = {(kind, *w) for kind, _, _, _, fwd, bwd in WAYS for w in (fwd, bwd)}
    # (a gradient that is not cut beside one that is takes what it takes beside one that is not)
    halves = {(kind, t, k, cut) for kind, t, *cuts in ways if len(cuts) == 2 for k, cut in enumerate(cuts)}
    for _ in range(4000):
        rows, N, K = int(2 ** rng.uniform(0, 14)), 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        for kind in ("linear", "gated"):
            f, b = plans(kind, rows, N, K)
            assert (f.tiles == dfl.TILES_NONE) == (rows <= 32)
            assert rows <= 32 or (kind, f.tiles, f.parts > 1) in ways, (kind, rows, N, K)
            assert {(kind, b.tiles, 0, b.parts > 1), (kind, b.tiles, 1, b.parts_w > 1)} <= halves, (kind, rows, N, K)
