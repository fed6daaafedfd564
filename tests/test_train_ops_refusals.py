"""What the entry points of the training step's operators refuse, at the C ABI, before any GPU call; and the
frequencies of the rotary embedding, which are computed on the host."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2606_02091_amd import dflare as dfl

P = 0x1000  # an aligned address that no refused call reads
INV, UNS, OK = dfl.ERR_INVALID_ARG, dfl.ERR_UNSUPPORTED, dfl.OK
INF, NAN = float("inf"), float("nan")


def lce(rows=32, V=100, H=64, B=4, gamma=4.5, ws=1 << 40, hidden=P, head=16 * P, labels=P, loss=P, ce=P, dh=32 * P,
        dw=48 * P, work=64 * P):
    return dfl.lib().dflare_linear_ce(hidden, head, labels, rows, V, H, B, gamma, loss, ce, dh, dw, work, ws, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), INV), (dict(rows=-4), INV), (dict(V=0), INV), (dict(H=0), INV), (dict(B=0), INV), (dict(rows=33), INV),
    (dict(gamma=0.0), INV), (dict(gamma=-1.0), INV), (dict(gamma=NAN), INV), (dict(gamma=INF), INV), (dict(ws=64), INV),
    (dict(hidden=None), INV), (dict(head=None), INV), (dict(labels=None), INV), (dict(loss=None), INV), (dict(ce=None), INV),
    (dict(work=None), INV), (dict(hidden=P + 8), INV), (dict(head=P + 2), INV), (dict(dh=32 * P + 4), INV), (dict(dw=48 * P + 8), INV),
    (dict(work=P + 8), INV), (dict(dh=P), INV), (dict(dw=16 * P), INV), (dict(dw=P + 16), INV), (dict(dh=48 * P + 32), INV),
    (dict(dh=16 * P + 12784), INV), (dict(H=60), UNS), (dict(H=16392), UNS), (dict(rows=(1 << 22) + 4), UNS),
    (dict(rows=1 << 22, V=1 << 20), UNS)])
def test_linear_ce_refuses(kw, code):
    assert lce(**kw) == code


def test_linear_ce_workspace():
    ws = dfl.lib().dflare_linear_ce_workspace
    assert ws(0, 10, 8, 0, 0) == 0 and ws(8, 10, 12, 0, 0) == 0 and ws(8, 0, 8, 0, 0) == 0
    # without logits: below a quarter of rows x V floats, and more where more is asked for
    a, b, c = ws(8192, 151936, 4096, 0, 0), ws(8192, 151936, 4096, 1, 0), ws(8192, 151936, 4096, 1, 1)
    assert 0 < a < b <= c < 8192 * 151936 * 4 // 4
    # one workspace for the largest call serves the smaller ones
    last = (0, 0, 0)
    for rows, V, H in ((32, 500, 64), (300, 500, 64), (300, 40000, 64), (300, 40000, 1000), (2000, 40000, 1000),
                       (2000, 200000, 1000), (2000, 200000, 4096), (9000, 200000, 4096)):
        now = tuple(ws(rows, V, H, *k) for k in ((0, 0), (1, 0), (1, 1)))
        assert all(x <= y for x, y in zip(last, now))
        last = now
    need = ws(32, 100, 64, 1, 1)
    assert lce(ws=need - 1) == INV


def test_linear_ce_workspace_does_not_grow_with_rows_times_words():
    """Past the sizes at which a piece has its full room, twice the rows and twice the words need twice as much at most, and the words
    alone some bytes each (the flags of pieces); one call's workspace serves every smaller call."""
    ws = dfl.lib().dflare_linear_ce_workspace
    for k in ((0, 0), (1, 0), (0, 1), (1, 1)):
        for rows, V, H in ((8192, 151936, 4096), (65536, 100000, 64), (1 << 18, 50000, 1024), (1 << 19, 100000, 64), (1 << 20, 40000, 8)):
            one, words, both = ws(rows, V, H, *k), ws(rows, 2 * V, H, *k), ws(2 * rows, 2 * V, H, *k)
            assert 0 < one <= words <= both
            assert both <= 2 * one + (1 << 16), (rows, V, H, k)
            assert words - one <= V, (rows, V, H, k)
        # the rows themselves once (dhidden: and their sums), dz and the parts up to their room
        assert ws(1 << 20, 200000, 64, *k) <= (1 << 20) * 64 * (2 + 4 * k[0]) + (1 << 20) * 64 + (512 + 128 + 128 + 32 << 20) + (1 << 20)
    rng = np.random.default_rng(3)
    for _ in range(3000):
        big = [int(2 ** rng.uniform(0, m)) for m in (22, 20)] + [8 * int(2 ** rng.uniform(0, 10))]
        small = [int(rng.integers(1, v + 1)) for v in big[:2]] + [8 * int(rng.integers(1, big[2] // 8 + 1))]
        for k in ((0, 0), (1, 0), (0, 1), (1, 1)):
            if ws(*big, *k):
                assert ws(*small, *k) <= ws(*big, *k), (small, big, k)


def rope(n=1, rows=4, B=1, hd=64, rot=64, dtype=dfl.BF16, layout=0, scale=1.0, pos=P, freq=P, x=P, y=2 * P, heads=2,
         strides=(128, 64, 128, 64), tab=True):
    t = (dfl.dflare_rope_tensor * 2)(*[dfl.dflare_rope_tensor(x, y, *strides, heads)] * 2)
    return dfl.lib().dflare_rope(t if tab else None, n, pos, freq, rows, B, hd, rot, dtype, layout, scale, 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), INV), (dict(n=3), INV), (dict(tab=False), INV), (dict(rows=-1), INV), (dict(B=0), INV), (dict(hd=1), INV),
    (dict(rot=0), INV), (dict(rot=63), INV), (dict(rot=66), INV), (dict(dtype=2), INV), (dict(dtype=-1), INV),
    (dict(layout=2), INV), (dict(scale=NAN), INV), (dict(scale=INF), INV), (dict(freq=None), INV), (dict(freq=P + 4), INV),
    (dict(pos=P + 2), INV), (dict(x=None), INV), (dict(y=None), INV), (dict(x=P + 1), INV), (dict(y=P + 2, dtype=dfl.F32), INV),
    (dict(heads=-1), INV), (dict(y=P, strides=(128, 64, 256, 64)), INV), (dict(hd=1026), UNS), (dict(heads=1 << 15), UNS),
    (dict(rows=0), OK), (dict(heads=0, x=None, y=None), OK)])
def test_rope_refuses(kw, code):
    assert rope(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(y=P + 2), dict(y=P + 1022), dict(y=P - 1022), dict(strides=(128, 64, 0, 64)), dict(strides=(128, 64, 128, 0)),
    dict(strides=(128, 64, 128, 63)), dict(strides=(128, 64, 127, 64)), dict(strides=(64, 256, 64, 255)),
    dict(y=P, strides=(0, 64, 0, 64)), dict(y=P, strides=(128, 0, 128, 0)), dict(n=2), dict(n=2, y=P),
    dict(x=P, y=P + 128, strides=(192, 64, 192, 64)), dict(strides=(128, 64, -128, 63))])
def test_rope_refuses_outputs_that_meet(kw):
    """Rows or heads of y on each other, y beside x itself on a part of it, both tensors the same."""
    assert rope(**kw) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused is launched")
def test_rope_refuses_every_overlap():
    """Against the sets of bytes, over small strides and offsets; and layouts that are not to be refused."""
    rng = np.random.default_rng(5)

    def call(sides, rows, hd):
        t = (dfl.dflare_rope_tensor * len(sides))(*[dfl.dflare_rope_tensor(P + 2 * x, P + 2 * y, *st, h) for x, y, st, h in sides])
        return dfl.lib().dflare_rope(t, len(sides), None, P, rows, 1, hd, 2, dfl.BF16, 0, 1.0, 0, None)

    def places(at, row, head, rows, heads, hd):
        return (at + row * np.arange(rows)[:, None, None] + head * np.arange(heads)[:, None] + np.arange(hd)).ravel()

    met = refused = 0
    for _ in range(6000):
        rows, hd, heads = int(rng.integers(1, 4)), int(rng.integers(2, 5)), rng.integers(1, 4, 2)
        same = rng.integers(-24, 25, 4)
        sides = []
        for k in range(int(rng.integers(1, 3))):
            st = same if rng.random() < 0.7 else rng.integers(-24, 25, 4)
            x, y = (int(v) for v in rng.integers(0, 120, 2))
            if rng.random() < 0.5:
                st, y = np.concatenate([st[:2], st[:2]]), x
            sides.append((x, y, [int(v) for v in st], int(heads[k])))
        bad = False
        written = [places(y, *st[2:], rows, h, hd) for x, y, st, h in sides]
        read = [places(x, *st[:2], rows, h, hd) for x, y, st, h in sides]
        for k, w in enumerate(written):
            bad |= len(set(w)) < len(w)
            for j in range(len(sides)):
                bad |= j != k and bool(set(w) & set(written[j]))
                bad |= (j != k or sides[k][0] != sides[k][1]) and bool(set(w) & set(read[j]))
        rc = call(sides, rows, hd)
        met += bad
        refused += rc == INV
        assert rc == INV if bad else rc in (INV, dfl.ERR_HIP)
    assert met > 1000 and refused < 6000
    n = 5 * 8
    fine = [[(0, 0, (n, 8) * 2, 3), (24, 24, (n, 8) * 2, 1)],          # queries and keys of one buffer, in place
            [(0, 24, (n, 8) * 2, 2)],                                  # from one part of a buffer to another
            [(0, 0, (8, 64) * 2, 3), (192, 192, (8, 64) * 2, 2)],      # heads first
            [(0, 0, (48, 24) * 2, 2), (8, 8, (48, 24) * 2, 2)],        # query, key and value of a head side by side
            [(0, 500, (0, 8, 24, 8), 3)], [(0, 500, (8, 0, 24, 8), 3)]]  # broadcast inputs
    for sides in fine:
        assert call(sides, 4, 8) == dfl.ERR_HIP, sides


def norm_fwd(rows=4, H=64, dtype=dfl.BF16, kind=0, eps=1e-6, x=P, res=None, gain=P, bias=None, sum_=None, y=P, mean=P, rstd=P):
    return dfl.lib().dflare_norm_fwd(x, res, gain, bias, rows, H, dtype, kind, eps, sum_, y, mean, rstd, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INV), (dict(H=0), INV), (dict(dtype=7), INV), (dict(kind=2), INV), (dict(eps=-1.0), INV), (dict(eps=NAN), INV),
    (dict(eps=INF), INV), (dict(bias=P), INV), (dict(x=None), INV), (dict(y=None), INV), (dict(rstd=None), INV),
    (dict(kind=1, mean=None), INV), (dict(res=P), INV), (dict(x=P + 1), INV), (dict(gain=P + 2, dtype=dfl.F32), INV),
    (dict(H=16385), UNS), (dict(rows=0, x=None, y=None, rstd=None), OK)])
def test_norm_fwd_refuses(kw, code):
    assert norm_fwd(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(y=P + 128), dict(y=P - 2), dict(y=64 * P, gain=64 * P + 510), dict(kind=1, y=64 * P, bias=64 * P, gain=None),
    dict(gain=None, res=2 * P, sum_=P, y=P), dict(gain=None, res=2 * P, sum_=8 * P, y=8 * P + 510), dict(gain=None, res=2 * P, sum_=2 * P + 2),
    dict(res=2 * P, sum_=8 * P, gain=8 * P, y=4 * P)])
def test_norm_fwd_refuses_outputs_that_meet(kw):
    assert norm_fwd(**kw) == INV


def norm_bwd(rows=4, H=64, dtype=dfl.BF16, kind=0, dy=P, h=P, gain=P, mean=P, rstd=P, dsum=None, dx=P, dgain=P, dbias=None,
             work=P, ws=1 << 30):
    return dfl.lib().dflare_norm_bwd(dy, h, gain, mean, rstd, dsum, rows, H, dtype, kind, dx, dgain, dbias, work, ws, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INV), (dict(H=0), INV), (dict(dtype=2), INV), (dict(kind=-1), INV), (dict(dy=None), INV), (dict(h=None), INV),
    (dict(rstd=None), INV), (dict(kind=1, mean=None), INV), (dict(dx=None), INV), (dict(dgain=None), INV), (dict(dbias=P), INV),
    (dict(work=None), INV), (dict(work=P + 4), INV), (dict(ws=100), INV), (dict(dsum=P + 1), INV), (dict(H=20000), UNS)])
def test_norm_bwd_refuses(kw, code):
    assert norm_bwd(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(dx=P + 2, gain=None), dict(dx=9 * P + 510, dy=9 * P, gain=None), dict(dx=9 * P - 510, dsum=9 * P, gain=None), dict(gain=P + 256)])
def test_norm_bwd_refuses_dx_that_meets_an_input(kw):
    assert norm_bwd(**kw) == INV


def tensors(*items):
    return (dfl.dflare_grad_tensor * max(1, len(items)))(*[dfl.dflare_grad_tensor(*t) for t in items])


def grad_norm(items, n=None, sumsq=P, work=P, ws=1 << 30, tab=True):
    return dfl.lib().dflare_grad_norm(tensors(*items) if tab else None, len(items) if n is None else n, sumsq, None, work, ws, None)


def clip(items, n=None, sumsq=P, max_norm=1.0):
    return dfl.lib().dflare_clip_grads(tensors(*items), len(items) if n is None else n, sumsq, max_norm, None)


GOOD = (P, None, 64, dfl.F32)


@pytest.mark.parametrize("items,kw,code", [
    ([GOOD], dict(n=-1), INV), ([GOOD], dict(tab=False), INV), ([GOOD], dict(sumsq=None), INV), ([GOOD], dict(sumsq=P + 4), INV),
    ([GOOD], dict(work=None), INV), ([GOOD], dict(work=P + 4), INV), ([GOOD], dict(ws=100), INV), ([(None, None, 1, 0)], {}, INV),
    ([(P + 2, None, 1, 0)], {}, INV), ([(P + 1, None, 1, 1)], {}, INV), ([(P, None, -1, 0)], {}, INV), ([(P, None, 1, 2)], {}, INV),
    ([(P, None, (1 << 36) + 1, 0)], {}, UNS)])
def test_grad_norm_refuses(items, kw, code):
    assert grad_norm(items, **kw) == code


@pytest.mark.parametrize("items,kw,code", [
    ([GOOD], dict(sumsq=None), INV), ([GOOD], dict(max_norm=-1.0), INV), ([GOOD], dict(max_norm=NAN), INV), ([GOOD, GOOD], {}, INV),
    ([GOOD, (P + 252, None, 4, 0)], {}, INV), ([(P, 2 * P, 64, 0), (2 * P + 8, None, 4, 0)], {}, INV),
    ([(P, 2 * P, 64, 0), (3 * P, 2 * P, 4, 0)], {}, INV), ([(P, P + 4, 64, 0)], {}, INV), ([(P, 2 * P + 2, 64, 0)], {}, INV)])
def test_clip_refuses(items, kw, code):
    assert clip(items, **kw) == code


def test_binding_refuses_lists_that_are_no_gradients():
    t = torch.zeros(4)
    with pytest.raises(TypeError):
        dfl.grad_norm([t])  # not on a device
    with pytest.raises(TypeError):
        dfl.grad_norm([t.double()])
    with pytest.raises(TypeError):
        dfl.grad_norm([None])
    with pytest.raises(ValueError):
        dfl.grad_norm([])
    with pytest.raises(ValueError):
        dfl.clip_grads([t], t, 1.0, out=[])
    for call in (lambda: dfl.rope(t, t), lambda: dfl.norm_fwd(t), lambda: dfl.norm_bwd(t, t, None, None, t),
                 lambda: dfl.linear_ce(t, t, t, 1, 1.0)):
        with pytest.raises(TypeError):
            call()


def test_binding_refuses_numbers_beyond_32_bits():
    assert dfl._i32(2 ** 31 - 1, "n") == 2 ** 31 - 1
    for n in (2 ** 31, -2 ** 31 - 1, 2 ** 40):
        with pytest.raises(ValueError):
            dfl._i32(n, "n")


def freqs(d, base, method=0, factor=1.0, length=0.0):
    f, s = np.zeros(max(d // 2, 1)), ctypes.c_float()
    rc = dfl.lib().dflare_rope_frequencies(d, base, method, factor, length, f.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                           ctypes.byref(s))
    return rc, f, s.value


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (-2, 1e4), (64, 0.0), (64, -1.0), (64, NAN), (64, INF), (64, 1e4, 4), (64, 1e4, -1),
                                  (64, 1e4, 1, 0.5), (64, 1e4, 2, NAN), (64, 1e4, 3, INF, 100.0), (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, NAN)])
def test_frequencies_refuse(args):
    assert freqs(*args)[0] == INV


@pytest.mark.parametrize("d,base", [(2, 1e4), (64, 1e4), (128, 1e6)])
def test_frequencies(d, base):
    m = np.arange(d // 2)
    plain = base ** (-2.0 * m / d)
    rc, f, s = freqs(d, base)
    assert rc == OK and s == 1.0 and np.allclose(f, plain, rtol=1e-14)
    assert np.allclose(freqs(d, base, dfl.ROPE_LINEAR, 4.0)[1], plain / 4, rtol=1e-14)
    rc, f, s = freqs(d, base, dfl.ROPE_NTK, 4.0)
    assert rc == OK and s == 1.0 and f[0] == 1.0
    if d > 2:  # the slowest pair is stretched by the whole factor
        assert np.isclose(f[-1], plain[-1] / 4, rtol=1e-12)
    rc, f, s = freqs(d, base, dfl.ROPE_YARN, 8.0, 4096.0)
    assert rc == OK and np.isclose(s, 0.1 * math.log(8.0) + 1, rtol=1e-6)
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(f[turns >= 32], plain[turns >= 32], rtol=1e-14)
    assert np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert np.all((f[mid] < plain[mid]) & (f[mid] > plain[mid] / 8))


FAR = {k: (i + 1) << 32 for i, k in enumerate("abcdefghijkl")}  # addresses far from one another


@pytest.mark.parametrize("lead", [1, 2, 3])
def test_numbers_off_their_alignment_are_refused(lead):
    """Labels, losses, statistics and gradients of gains, in fp32 and int32, at addresses that are no multiple of 4."""
    a = FAR
    kw = dict(hidden=a["a"], head=a["b"], labels=a["c"], loss=a["d"], ce=a["e"], dh=a["f"], dw=a["g"], work=a["h"])
    for k in ("labels", "loss", "ce"):
        assert lce(**{**kw, k: kw[k] + lead}) == INV, k
    kw = dict(x=a["a"], gain=a["b"], y=a["c"], mean=a["d"], rstd=a["e"], kind=dfl.NORM_LAYER)
    for k in ("mean", "rstd"):
        assert norm_fwd(**{**kw, k: kw[k] + lead}) == INV, k
    kw = dict(dy=a["a"], h=a["b"], gain=a["c"], mean=a["d"], rstd=a["e"], dx=a["f"], dgain=a["g"], dbias=a["h"], work=a["i"], kind=dfl.NORM_LAYER)
    for k in ("mean", "rstd", "dgain", "dbias"):
        assert norm_bwd(**{**kw, k: kw[k] + lead}) == INV, k
    assert dfl.lib().dflare_grad_norm(tensors((a["a"], None, 64, dfl.F32)), 1, a["b"], a["c"] + lead, a["d"], 1 << 30, None) == INV


def refused(call, kw, pairs):
    """Every pair (written, other, bytes of the other): the first bytes of what is written lie on the other's last ones."""
    for w, o, n in pairs:
        assert call(**{**kw, w: kw[o] + n - 16 if n >= 16 else kw[o]}) == INV, (w, o)


def test_linear_ce_refuses_every_output_on_another_tensor():
    a = FAR
    kw = dict(hidden=a["a"], head=a["b"], labels=a["c"], loss=a["d"], ce=a["e"], dh=a["f"], dw=a["g"], work=a["h"])
    size = dict(hidden=32 * 128, head=100 * 128, labels=128, loss=4, ce=128, dh=32 * 128, dw=100 * 128,
                work=dfl.lib().dflare_linear_ce_workspace(32, 100, 64, 1, 1) // 16 * 16)
    for w in ("loss", "ce", "dh", "dw", "work"):
        refused(lce, kw, [(w, o, size[o]) for o in size if o != w])


def test_norms_refuse_statistics_on_another_tensor():
    a = FAR
    kw = dict(x=a["a"], res=a["b"], gain=a["c"], bias=a["d"], sum_=a["e"], y=a["f"], mean=a["g"], rstd=a["h"], kind=dfl.NORM_LAYER)
    size = dict(x=512, res=512, gain=128, bias=128, sum_=512, y=512, mean=16, rstd=16)
    for w in ("mean", "rstd"):
        refused(norm_fwd, kw, [(w, o, size[o]) for o in size if o != w])
    kw = dict(dy=a["a"], h=a["b"], gain=a["c"], mean=a["d"], rstd=a["e"], dsum=a["f"], dx=a["g"], dgain=a["h"], dbias=a["i"],
              work=a["j"], kind=dfl.NORM_LAYER)
    size = dict(dy=512, h=512, gain=128, mean=16, rstd=16, dsum=512, dx=512, dgain=256, dbias=256,
                work=dfl.lib().dflare_norm_bwd_workspace(4, 64, dfl.NORM_LAYER))
    refused(norm_bwd, kw, [("work", o, size[o]) for o in size if o != "work"])
    refused(norm_bwd, kw, [("dx", o, size[o]) for o in ("mean", "rstd", "gain", "dgain", "dbias", "work")])
    refused(norm_bwd, kw, [("dgain", o, size[o]) for o in ("dx", "dbias", "work")])
    refused(norm_bwd, kw, [("dbias", o, size[o]) for o in ("dx", "dgain", "work")])


def test_rope_refuses_outputs_on_the_positions():
    y = FAR["b"]  # 4 rows of 128 elements, 2 bytes each
    for pos in (y, y + 4, y + 1020, y - 12):
        assert rope(x=FAR["a"], y=y, pos=pos, freq=FAR["c"]) == INV
        assert rope(x=FAR["a"], y=y, pos=pos, freq=FAR["c"], n=1, B=4 if pos != y - 12 else 1) == INV


def test_gradients_refuse_results_on_another_tensor():
    t, lib = tensors((FAR["a"], None, 64, dfl.F32), (FAR["b"], None, 64, dfl.F32)), dfl.lib()
    ws = lib.dflare_grad_norm_workspace(2)

    def norm(sumsq=FAR["c"], out=FAR["d"], work=FAR["e"]):
        return lib.dflare_grad_norm(t, 2, sumsq, out, work, ws, None)
    for at in (FAR["a"] + 248, FAR["b"]):
        assert norm(sumsq=at) == INV and norm(out=at) == INV and norm(work=at) == INV
    assert norm(sumsq=FAR["e"] + ws - 8) == INV and norm(out=FAR["e"]) == INV and norm(out=FAR["c"] + 4) == INV
    assert clip([(FAR["a"], None, 64, dfl.F32)], sumsq=FAR["a"] + 248) == INV
    assert clip([(FAR["a"], FAR["b"], 64, dfl.F32)], sumsq=FAR["b"]) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused is launched")
def test_tensors_that_lie_apart_are_not_refused():
    """Calls in place, and tensors that follow each other without a byte between them, reach the launch."""
    a, launched = FAR, dfl.ERR_HIP
    at, ptr = a["a"], {}
    sizes = dict(hidden=32 * 128, head=100 * 128, work=dfl.lib().dflare_linear_ce_workspace(32, 100, 64, 1, 1), dh=32 * 128, dw=100 * 128,
                 labels=128, ce=128, loss=4)
    for k, n in sizes.items():
        ptr[k], at = at, at + n
    assert lce(**ptr) == launched
    assert norm_fwd(x=a["a"], res=a["b"], gain=a["c"], sum_=a["a"], y=a["b"], rstd=a["a"] + 512, mean=a["a"]) == launched  # (no mean is written)
    assert norm_fwd(x=a["a"], gain=a["c"], y=a["a"], mean=a["b"], rstd=a["b"] + 16, kind=dfl.NORM_LAYER) == launched
    for over in ("a", "b", "f"):
        assert norm_bwd(dy=a["a"], h=a["b"], dsum=a["f"], gain=a["c"], mean=a["d"], rstd=a["e"], dx=a[over], dgain=a["h"], dbias=a["h"] + 256,
                        work=a["h"] + 512, kind=dfl.NORM_LAYER) == launched
    assert rope(x=a["a"], y=a["a"], pos=a["a"] + 1024, freq=a["c"]) == launched
    ws = dfl.lib().dflare_grad_norm_workspace(1)
    assert dfl.lib().dflare_grad_norm(tensors((a["a"], None, 64, dfl.F32)), 1, a["a"] + 256, a["a"] + 264, a["b"], ws, None) == launched
    assert clip([(a["a"], None, 64, dfl.F32)], sumsq=a["a"] + 256) == launched
    assert clip([(None, None, 0, dfl.F32), (a["a"], a["b"], 64, dfl.F32)], sumsq=a["b"] + 256) == launched


def test_binding_refuses_numbers_that_are_cut():
    """A dimension beyond 32 bits would reach the library as another one, with room for the first; a broken number as a whole one."""
    for d in (2 ** 31, 2 ** 32 + 64, -2 ** 32 + 64, 64.5):
        with pytest.raises(ValueError):
            dfl.rope_frequencies(d, 1e4, device="cpu")
    with pytest.raises(ValueError):
        dfl.rope_frequencies(64, 1e4, 2 ** 32, device="cpu")
    with pytest.raises(ValueError):
        dfl._i32(4.5, "B")
    assert dfl._i32(16.0, "B") == 16 and dfl.rope_frequencies(64, 1e4, device="cpu")[0].shape == (32,)
