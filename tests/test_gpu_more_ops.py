"""The operators that complete a draft layer's training step against their formulas in 64 bits: head norms with rotary
positions, projections and the gated feed-forward block with their epilogues, and AdamW.

Bounds count roundings: a stored bf16 value is off by at most half a step (2^-8 of it, or half the smallest number), a sum of n
fp32 terms by n 2^-24 of the terms' magnitudes (twice that on the matrix cores, which may truncate); where a bound has another
part it is said there.
"""
import math

import pytest
import torch

from paper_2606_02091_amd import dflare as dfl
from product_shapes import WAYS

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

BF, F32, F8, F64 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float64
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}  # half a step, relative
U = 2.0 ** -24
# An activation or its derivative, formed through exp2: the exponent, below 2^7 where the result is not 0, is rounded by 2^-18 twice and
# its power by as much of itself; the other steps are some units of 2^-24.
REL = 2.0 ** -16
ACTS = dict(none=dfl.ACT_NONE, relu=dfl.ACT_RELU, silu=dfl.ACT_SILU, gelu=dfl.ACT_GELU, gelu_tanh=dfl.ACT_GELU_TANH)


def randn(shape, dtype=BF, seed=0, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def within(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((got.double() - want).abs().max()), float(bound.max()))


def same(a, b):
    return all((x is None and y is None) or torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


# ---- head norms with rotary positions ----

def turned(u, pos, freq, half, scale, inverse=False):
    """(scale R(+-p) u, the sizes of the terms)."""
    rot = 2 * freq.numel()
    th = pos.double()[:, None] * freq.double()
    c, s = torch.cos(th)[:, None] * scale, torch.sin(th)[:, None] * scale * (-1 if inverse else 1)
    a, b = (u[..., :rot // 2], u[..., rot // 2:rot]) if half else (u[..., 0:rot:2], u[..., 1:rot:2])
    p, q, n = a * c - b * s, b * c + a * s, (a.abs() + b.abs()) * abs(scale)
    y, size = u.clone(), u.abs()
    if half:
        y[..., :rot // 2], y[..., rot // 2:rot] = p, q
        size[..., :rot // 2] = size[..., rot // 2:rot] = n
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, q
        size[..., 0:rot:2] = size[..., 1:rot:2] = n
    return y, size


def qk_check(x, gain, pos, freq, half, scale, eps, y, dy, dx, dgain):
    t, hd = x.dtype, x.shape[-1]
    g = torch.ones(hd, dtype=F64, device="cuda") if gain is None else gain.double()
    u = x.double()
    rstd = ((u * u).mean(-1, keepdim=True) + eps).rsqrt()
    n = u * rstd
    # the norm: a sum of hd squares, division, root (hd + 8 units of rstd at most); the products; the turn as of a rotary
    # position (cosine and sine within a few units)
    k = (hd + 32) * U
    want, size = turned(n * g, pos, freq, half, scale)
    within(y, want, 1.01 * (HALF[t] * want.abs() + k * size) + 1e-38, "y")
    if dy is None:
        return
    d, size = turned(dy.double(), pos, freq, half, scale, inverse=True)
    e, esize = d * g, size * g.abs()
    m = (e * n).mean(-1, keepdim=True)
    want = rstd * (e - n * m)
    msize = (esize * n.abs()).mean(-1, keepdim=True)
    within(dx, want, 1.01 * (HALF[t] * want.abs() + 2 * k * rstd * (esize + n.abs() * msize)) + 1e-38, "dx")
    if gain is None:
        assert dgain is None
    else:
        terms = size * n.abs()
        # added in lanes, waves, groups and their list: no chain is longer than the terms
        chain = min(terms.shape[0] * terms.shape[1], 4096) + 64
        within(dgain, (d * n).sum((0, 1)), (k + chain * U) * terms.sum((0, 1)) + 1e-38, "dgain")


# (rows, B, query heads, key heads, head, rotated): one token, blocks, long sequences; parts that fit no wide access; odd heads,
# heads of two, the largest; more lanes than items and the other way round
@pytest.mark.parametrize("rows,B,nq,nk,hd,rot", [
    (1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (33, 16, 8, 2, 128, 128), (257, 257, 5, 1, 64, 32), (1500, 1, 4, 4, 96, 96),
    (70, 3, 3, 0, 80, 36), (9, 2, 7, 2, 5, 4), (6, 6, 2, 1, 512, 512), (5, 4, 33, 3, 256, 64), (2100, 16, 2, 1, 64, 64),
    (3, 1, 1, 2, 511, 2), (40, 8, 3, 1, 512, 16)])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_qk_norm_rope(rows, B, nq, nk, hd, rot, half, dtype):
    print(f"[more ops] qk {(rows, B, nq, nk, hd, rot, half, dtype)}", flush=True)
    layout = dfl.ROPE_HALF if half else dfl.ROPE_INTERLEAVED
    heads = [n for n in (nq, nk) if n]
    xs = tuple(randn((rows, n, hd), dtype, seed=n, std=2.0) for n in heads)
    dys = tuple(randn((rows, n, hd), dtype, seed=50 + n) for n in heads)
    gains = tuple(randn((hd,), dtype, seed=90 + n, std=0.3, mean=1.0) for n in heads)
    freq, _ = dfl.rope_frequencies(rot, 1e4)
    g = torch.Generator(device="cuda").manual_seed(rows)
    starts = torch.randint(-50, 1_000_000, (-(-rows // B),), generator=g, device="cuda", dtype=torch.int32)
    pos = starts.repeat_interleave(B)[:rows].long() + torch.arange(rows, device="cuda") % B
    kw = dict(B=B, layout=layout, scale=1.25, eps=1e-5)
    outs = dfl.qk_norm_rope_fwd(xs, gains, freq, starts, **kw)
    dxs, dgains = dfl.qk_norm_rope_bwd(dys, xs, gains, freq, starts, **kw)
    for i in range(len(heads)):
        qk_check(xs[i], gains[i], pos, freq, half, 1.25, 1e-5, outs[i], dys[i], dxs[i], dgains[i])
    again = dfl.qk_norm_rope_bwd(dys, xs, gains, freq, starts, **kw)
    assert same(dxs + dgains, again[0] + again[1])
    # one tensor, without a gain, rows at their own index
    y = dfl.qk_norm_rope_fwd(xs[0], None, freq, layout=layout)
    dx, dgain = dfl.qk_norm_rope_bwd(dys[0], xs[0], None, freq, layout=layout)
    qk_check(xs[0], None, torch.arange(rows, device="cuda"), freq, half, 1.0, 1e-6, y, dys[0], dx, dgain)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_qk_norm_rope_views_and_in_place(dtype):
    """Heads inside a joint projection's rows, at offsets of every alignment; only the heads are written."""
    freq, _ = dfl.rope_frequencies(64, 1e6)
    rows, nq, nk, hd = 37, 6, 2, 64
    pos = torch.arange(rows, device="cuda", dtype=torch.int32) * 3
    gains = tuple(randn((hd,), dtype, seed=k, mean=1.0, std=0.2) for k in range(2))
    for lead in (0, 1, 8, 13):
        buf, dbuf = (randn((rows, lead + (nq + 2 * nk) * hd + 5), dtype, seed=lead + k) for k in range(2))
        keep = buf.clone()

        def heads(b):
            return (b[:, lead:lead + nq * hd].view(rows, nq, hd), b[:, lead + nq * hd:lead + (nq + nk) * hd].view(rows, nk, hd))
        (q, k), (dq, dk) = heads(buf), heads(dbuf)
        kt = k.transpose(0, 1).contiguous().transpose(0, 1)  # head-major memory
        out = dfl.qk_norm_rope_fwd((q, kt), gains, freq, pos)
        back = dfl.qk_norm_rope_bwd((dq, dk), (q, kt), gains, freq, pos)
        for i, (x, d) in enumerate(((q, dq), (k, dk))):
            qk_check(x, gains[i], pos.long(), freq, True, 1.0, 1e-6, out[i], d, back[0][i], back[1][i])
        assert torch.equal(buf, keep)
        dfl.qk_norm_rope_fwd((q, k), gains, freq, pos, out=(q, k))
        assert torch.equal(q, out[0]) and torch.equal(k, out[1])
        buf[:, lead:lead + (nq + nk) * hd] = keep[:, lead:lead + (nq + nk) * hd]
        assert torch.equal(buf, keep)


def qk_bwd_raw(x, dy, dx, gain, dgain, freq, rows, ws):
    t = dfl.dflare_qk_grad(x.data_ptr(), dy.data_ptr(), dx.data_ptr(), gain.data_ptr(), dgain.data_ptr(), *x.stride()[:2],
                           *dy.stride()[:2], *dx.stride()[:2], x.shape[1])
    code = dfl.F32 if x.dtype == F32 else dfl.BF16
    return dfl.lib().dflare_qk_norm_rope_bwd((dfl.dflare_qk_grad * 1)(t), 1, None, freq.data_ptr(), rows, 1, x.shape[2], 2 * freq.numel(),
                                             code, 0, 1.0, 1e-6, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("over", ["x", "dy"])
def test_qk_norm_rope_gradient_in_place(over):
    freq, _ = dfl.rope_frequencies(128, 1e6)
    x, dy, gain = randn((100, 9, 128), seed=1), randn((100, 9, 128), seed=2), randn((128,), seed=3, mean=1.0)
    want, wg = dfl.qk_norm_rope_bwd(dy, x, gain, freq)
    t = dict(x=x.clone(), dy=dy.clone())
    dgain = torch.empty(128, device="cuda")
    ws = torch.empty(dfl.lib().dflare_qk_norm_rope_bwd_workspace(100, 128, 1), dtype=torch.uint8, device="cuda")
    assert qk_bwd_raw(t["x"], t["dy"], t[over], gain, dgain, freq, 100, ws) == dfl.OK
    assert torch.equal(t[over], want) and torch.equal(dgain, wg)


def test_qk_norm_rope_gradient_against_differences():
    freq, _ = dfl.rope_frequencies(32, 1e4)
    x, dy, gain = randn((20, 3, 48), F32, 1), randn((20, 3, 48), F32, 2), randn((48,), F32, 3, mean=1.0, std=0.3)
    pos = torch.arange(20, device="cuda")

    def f(u, g):
        n = u * ((u * u).mean(-1, keepdim=True) + 1e-6).rsqrt() * g
        return (turned(n, pos, freq, True, 1.0)[0] * dy.double()).sum()
    dx, dgain = dfl.qk_norm_rope_bwd(dy, x, gain, freq)
    h = 1e-5
    for seed in range(5):
        v, w = randn(x.shape, F64, 10 + seed), randn(gain.shape, F64, 20 + seed)
        num = (f(x.double() + h * v, gain.double()) - f(x.double() - h * v, gain.double())) / (2 * h)
        # differences: h^2 of third derivatives and 1e-16 / h of the sums, below 1e-8 of these; the kernel: 100 units a value
        assert abs(float(num - (dx.double() * v).sum())) <= 1e-6 * float((dx.double() * v).abs().sum()) + 1e-5
        num = (f(x.double(), gain.double() + h * w) - f(x.double(), gain.double() - h * w)) / (2 * h)
        assert abs(float(num - (dgain.double() * w).sum())) <= 1e-5 * float((dgain.double() * w).abs().sum()) + 1e-4


def test_qk_norm_rope_of_nothing_and_of_zeros():
    freq, _ = dfl.rope_frequencies(64, 1e6)
    gain = randn((64,), seed=1)
    none = torch.empty((0, 4, 64), dtype=BF, device="cuda")
    assert dfl.qk_norm_rope_fwd(none, gain, freq).shape == (0, 4, 64)
    dx, dgain = dfl.qk_norm_rope_bwd(none, none, gain, freq)
    assert dx.shape == none.shape and not dgain.any()
    empty = torch.empty((3, 0, 64), dtype=BF, device="cuda")
    x = randn((3, 2, 64), seed=2)
    dxs, dgains = dfl.qk_norm_rope_bwd((empty, x), (empty, x), (gain, gain), freq)
    assert not dgains[0].any() and dgains[1].any()
    zero = torch.zeros((3, 2, 64), dtype=BF, device="cuda")
    assert not dfl.qk_norm_rope_fwd(zero, gain, freq).any()
    dx, dgain = dfl.qk_norm_rope_bwd(x, zero, gain, freq)
    assert torch.isfinite(dx.float()).all() and not dgain.any()


def test_qk_norm_rope_of_a_head_whose_squares_are_hardly_there():
    """Without an eps the root mean square is a head's size, however small."""
    freq, _ = dfl.rope_frequencies(64, 1e4)
    x, dy, gain = randn((9, 3, 64), F32, 1) * 2.0 ** -66, randn((9, 3, 64), F32, 2), randn((64,), F32, 3, mean=1.0)
    y, (dx, dgain) = dfl.qk_norm_rope_fwd(x, gain, freq, eps=0.0), dfl.qk_norm_rope_bwd(dy, x, gain, freq, eps=0.0)
    pos = torch.arange(9, device="cuda")
    rstd = x.double().square().mean(-1, keepdim=True).rsqrt()
    n, g = x.double() * rstd, gain.double()
    want, size = turned(n * g, pos, freq, True, 1.0)
    # 64 sums and a product of numbers near 2^-132, each within 2^-150: 2^-19 of their mean at most, half of that of the root; and the
    # units of test_qk_norm_rope
    k = 2.0 ** -19 + (64 + 32) * U
    within(y, want, k * size, "y")
    d, ds = turned(dy.double(), pos, freq, True, 1.0, inverse=True)
    e = d * g
    mean, es = (e * n).mean(-1, keepdim=True), ds * g.abs()
    within(dx, rstd * (e - n * mean), 4 * k * rstd * (es + n.abs() * (es * n.abs()).mean(-1, keepdim=True)), "dx")
    within(dgain, (d * n).sum((0, 1)), 4 * k * (ds * n.abs()).sum((0, 1)), "dgain")


def test_qk_norm_rope_keeps_nan_in_its_head():
    freq, _ = dfl.rope_frequencies(64, 1e6)
    x, dy, gain = randn((30, 5, 64), seed=1), randn((30, 5, 64), seed=2), randn((64,), seed=3, mean=1.0)
    y, (dx, _) = dfl.qk_norm_rope_fwd(x, gain, freq), dfl.qk_norm_rope_bwd(dy, x, gain, freq)
    for bad in (float("nan"), float("inf")):
        u = x.clone()
        u[7, 3, 11] = bad
        y2, (dx2, _) = dfl.qk_norm_rope_fwd(u, gain, freq), dfl.qk_norm_rope_bwd(dy, u, gain, freq)
        for a, b in ((y, y2), (dx, dx2)):
            keep = torch.ones(a.shape[:2], dtype=torch.bool, device="cuda")
            keep[7, 3] = False
            assert torch.equal(a[keep], b[keep]) and torch.isnan(b[7, 3]).any()


def test_qk_norm_rope_of_more_rows_than_a_launch_takes():
    rows, hd = (1 << 21) + 3, 512  # a row per work-group
    x = torch.empty((rows, 1, hd), dtype=BF, device="cuda")
    x[:] = randn((1, 1, hd), seed=1)
    gain = randn((hd,), seed=2, mean=1.0)
    freq, _ = dfl.rope_frequencies(hd, 1e6)
    y = dfl.qk_norm_rope_fwd(x, gain, freq)
    at = torch.tensor([0, 1, 77, (1 << 21) - 1, 1 << 21, rows - 1], device="cuda")
    qk_check(x[at], gain, at, freq, True, 1.0, 1e-6, y[at], None, None, None)


# ---- projections and the gated block ----

def act64(name, z):
    """(value, derivative) in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp_min(0), (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if name == "gelu":
        p = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    a = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(a * (z + 0.044715 * z ** 3))
    return z * s, s + z * s * (1 - s) * a * (1 + 3 * 0.044715 * z * z)


LEAST = 2.0 ** -126  # of bf16 and fp32 above which numbers have all their digits


def products_check(d, ed, x, w, dx, dw, what):
    """dx = d w and dw = d^T x for a d within ed of d, added in fp32."""
    rows, N = d[0].shape
    K = x.shape[1]
    if dx is not None:
        want = sum(p @ q.double() for p, q in zip(d, w))
        err = sum((e + len(d) * N * 2 * U * p.abs()) @ q.double().abs() for p, e, q in zip(d, ed, w))
        within(dx, want, 1.01 * (err + HALF[BF] * want.abs()) + LEAST, what + " dx")
    if dw is not None:
        for p, e, g in zip(d, ed, dw):
            want = p.t() @ x.double()
            err = (e + rows * 2 * U * p.abs()).t() @ x.double().abs()
            within(g, want, 1.01 * (err + HALF[BF] * want.abs()) + LEAST, what + " dw")


def linear_check(x, w, bias, res, act, dy, y, z, dx, dw, dbias):
    K = x.shape[1]
    zw = x.double() @ w.double().t() + (0 if bias is None else bias.double())
    # (the bias is the first of the K + 1 terms)
    ez = 2 * (K + 1) * U * (x.double().abs() @ w.double().abs().t() + (0 if bias is None else bias.double().abs()))
    if z is not None:
        within(z, zw, 1.01 * (ez + HALF[BF] * zw.abs()) + LEAST, "z")
    a, _ = act64(act, zw)
    want = a + (0 if res is None else res.double())
    # (derivatives of the activations are below 1.13)
    within(y, want, 1.01 * (1.13 * ez + REL * a.abs() + U * want.abs() + HALF[BF] * want.abs()) + LEAST, "y")
    if dy is None:
        return
    d = dy.double()
    if act == "none":
        ed = exact = torch.zeros_like(d)
    else:
        dd = act64(act, z.double())[1]
        d = d * dd
        exact = REL * 2 * dy.double().abs()  # (value and derivative of z's sizes up to 1.13 and 1, before they are rounded)
        ed = exact + HALF[BF] * d.abs()
    products_check([d], [ed], x, [w], dx, None if dw is None else [dw], "linear")
    if dbias is not None:
        want = d.sum(0)
        within(dbias, want, 1.01 * ((exact + d.shape[0] * U * d.abs()).sum(0) + HALF[BF] * want.abs()) + LEAST, "dbias")


SHAPES = [(1, 8, 8), (1, 4096, 64), (3, 8, 72), (16, 264, 2560), (64, 128, 128), (65, 136, 120), (63, 520, 56), (129, 256, 64),
          (257, 264, 200), (300, 2880, 1000), (1000, 72, 4096), (513, 1032, 648), (2000, 8, 16), (17, 2048, 8), (31, 16, 9000)]


@pytest.mark.parametrize("rows,N,K", SHAPES)
def test_linear(rows, N, K):
    print(f"[more ops] linear {(rows, N, K)}", flush=True)
    x, w = randn((rows, K), seed=1), randn((N, K), seed=2, std=K ** -0.5)
    bias, res, dy = randn((N,), seed=3), randn((rows, N), seed=4), randn((rows, N), seed=5)
    for act, b, r in (("none", None, None), ("none", bias, res), ("silu", None, res), ("gelu", bias, None), ("gelu_tanh", bias, res),
                      ("relu", bias, None)):
        code = ACTS[act]
        y, z = dfl.linear_fwd(x, w, b, residual=r, act=code, save=True)
        dx, dw, dbias = dfl.linear_bwd(dy, x, w, z, act=code, need_dbias=True)
        linear_check(x, w, b, r, act, dy, y, z, dx, dw, dbias)
        y2, none = dfl.linear_fwd(x, w, b, residual=r, act=code)
        assert none is None and torch.equal(y, y2)
        assert same((dx, dw, dbias), dfl.linear_bwd(dy, x, w, z, act=code, need_dbias=True))
        if act in ("none", "gelu"):  # with fewer outputs each is within the same bounds
            for k in range(8):
                part = dfl.linear_bwd(dy, x, w, z, act=code, need_dx=k & 1 > 0, need_dw=k & 2 > 0, need_dbias=k & 4 > 0)
                assert [p is not None for p in part] == [k & 1 > 0, k & 2 > 0, k & 4 > 0]
                linear_check(x, w, b, r, act, dy, y, z, *part)


def gated_check(x, wg, wu, act, dh, h, gate, up, dx, dwg, dwu):
    H = x.shape[1]
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    eg, eu = (2 * H * U * (x.double().abs() @ t.double().abs().t()) for t in (wg, wu))
    a, _ = act64(act, g)
    want = a * u
    ea = 1.13 * eg + REL * a.abs()
    within(h, want, 1.01 * (ea * (u.abs() + eu) + eu * a.abs() + (U + HALF[BF]) * want.abs()) + LEAST, "h")
    if dh is None:
        return
    within(gate, g, 1.01 * (eg + HALF[BF] * g.abs()) + LEAST, "gate")
    within(up, u, 1.01 * (eu + HALF[BF] * u.abs()) + LEAST, "up")
    v, d = act64(act, gate.double())
    dg, du = dh.double() * up.double() * d, dh.double() * v
    exact = (2 * REL * (dh.double() * up.double()).abs(), REL * du.abs())
    ed = [e + HALF[BF] * t.abs() for e, t in zip(exact, (dg, du))]
    products_check([dg, du], ed, x, [wg, wu], dx, None if dwg is None else [dwg, dwu], "gated")


@pytest.mark.parametrize("rows,F,H", SHAPES)
def test_gated(rows, F, H):
    print(f"[more ops] gated {(rows, F, H)}", flush=True)
    x, wg, wu = randn((rows, H), seed=1), randn((F, H), seed=2, std=1.5 * H ** -0.5), randn((F, H), seed=3, std=H ** -0.5)
    dh = randn((rows, F), seed=4)
    for act in ACTS:
        code = ACTS[act]
        h, gate, up = dfl.gated_fwd(x, wg, wu, act=code, save=True)
        grads = dfl.gated_bwd(dh, x, gate, up, wg, wu, act=code)
        gated_check(x, wg, wu, act, dh, h, gate, up, *grads)
        h2, none, _ = dfl.gated_fwd(x, wg, wu, act=code)
        assert none is None and torch.equal(h, h2)
        assert same(grads, dfl.gated_bwd(dh, x, gate, up, wg, wu, act=code))
        part = dfl.gated_bwd(dh, x, gate, up, wg, wu, act=code, need_dw=False)
        assert part[1] is None and part[2] is None
        gated_check(x, wg, wu, act, dh, h, gate, up, part[0], None, None)
        part = dfl.gated_bwd(dh, x, gate, up, wg, wu, act=code, need_dx=False)
        assert part[0] is None
        gated_check(x, wg, wu, act, dh, h, gate, up, *part)


@pytest.mark.parametrize("kind", ["linear", "gated"])
def test_products_on_the_large_tile(kind):
    """Enough rows and columns that a product is not cut along k, with an end inside a tile on every side."""
    rows, N, K = 2049, 4104, 328
    x, w, w2 = randn((rows, K), seed=1), randn((N, K), seed=2, std=K ** -0.5), randn((N, K), seed=3, std=K ** -0.5)
    dy, res = randn((rows, N), seed=4), randn((rows, N), seed=5)
    if kind == "linear":
        y, z = dfl.linear_fwd(x, w, res[0].contiguous(), residual=res, act=dfl.ACT_SILU, save=True)
        linear_check(x, w, res[0], res, "silu", dy, y, z, *dfl.linear_bwd(dy, x, w, z, act=dfl.ACT_SILU, need_dbias=True))
    else:
        h, g, u = dfl.gated_fwd(x, w, w2, save=True)
        gated_check(x, w, w2, "silu", dy, h, g, u, *dfl.gated_bwd(dy, x, g, u, w, w2))


@pytest.mark.parametrize("rows,N,K", [(777, 5096, 136), (1003, 5120, 72), (300, 12040, 200), (4095, 2040, 1032), (2496, 2888, 328)])
def test_products_on_tiles_of_two_sizes(rows, N, K):
    """More small tiles than CUs and less than twice as many (a part of the rows on halves of them), and a gated block's large tile."""
    x, w, w2 = randn((rows, K), seed=1), randn((N, K), seed=2, std=K ** -0.5), randn((N, K), seed=3, std=K ** -0.5)
    dy, res = randn((rows, N), seed=4), randn((rows, N), seed=5)
    y, z = dfl.linear_fwd(x, w, res[0].contiguous(), residual=res, act=dfl.ACT_GELU, save=True)
    linear_check(x, w, res[0], res, "gelu", dy, y, z, *dfl.linear_bwd(dy, x, w, z, act=dfl.ACT_GELU, need_dbias=True))
    half = N // 16 * 8
    for F in (half, N):
        u, v = w[:F].contiguous(), w2[:F].contiguous()
        dh = dy[:, :F].contiguous()
        h, gate, up = dfl.gated_fwd(x, u, v, act=dfl.ACT_SILU, save=True)
        gated_check(x, u, v, "silu", dh, h, gate, up, *dfl.gated_bwd(dh, x, gate, up, u, v, act=dfl.ACT_SILU))


@pytest.mark.parametrize("rows,N,K", [(1, 8, 8), (67, 200, 72), (300, 520, 136)])
def test_products_without_rows_and_values_beside_them(rows, N, K):
    """Inputs between NaN, outputs between values that stay: nothing past a tensor's end is read into a result or written."""
    lib, st = dfl.lib(), torch.cuda.current_stream().cuda_stream

    def between(n, fill, seed=None):
        b = torch.full((n + 1024,), fill, dtype=BF, device="cuda")
        if seed is not None:
            b[512:512 + n] = randn((n,), seed=seed)
        return b, b[512:512 + n]
    ins = {k: between(n, float("nan"), s) for s, (k, n) in enumerate(dict(
        x=rows * K, w=N * K, w2=N * K, bias=N, res=rows * N, dy=rows * N, z=rows * N, z2=rows * N).items())}
    p = {k: v[1].data_ptr() for k, v in ins.items()}
    outs = {k: between(n, 7.0) for k, n in dict(y=rows * N, zo=rows * N, zo2=rows * N, dx=rows * K, dw=N * K, dw2=N * K, db=N).items()}
    o = {k: v[1].data_ptr() for k, v in outs.items()}
    size = max(lib.dflare_linear_fwd_workspace(rows, N, K), lib.dflare_linear_bwd_workspace(rows, N, K, 2, 1, 1, 1),
               lib.dflare_gated_fwd_workspace(rows, K, N), lib.dflare_gated_bwd_workspace(rows, K, N, 1, 1))
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # (NaN as fp32 and as bf16)

    def clean(*names):
        for k in names:
            b, v = outs[k]
            n = v.numel()
            assert torch.isfinite(v.float()).all(), k
            assert (b[:512] == 7.0).all() and (b[512 + n:] == 7.0).all(), k
    assert lib.dflare_linear_fwd(p["x"], p["w"], p["bias"], p["res"], rows, N, K, 3, o["y"], o["zo"], ws.data_ptr(), size, st) == dfl.OK
    clean("y", "zo")
    assert lib.dflare_linear_bwd(p["dy"], p["x"], p["w"], p["z"], rows, N, K, 2, o["dx"], o["dw"], o["db"], ws.data_ptr(), size, st) == dfl.OK
    clean("dx", "dw", "db")
    ws.fill_(255)
    assert lib.dflare_gated_fwd(p["x"], p["w"], p["w2"], rows, K, N, 2, o["y"], o["zo"], o["zo2"], ws.data_ptr(), size, st) == dfl.OK
    clean("y", "zo", "zo2")
    assert lib.dflare_gated_bwd(p["dy"], p["x"], p["z"], p["z2"], p["w"], p["w2"], rows, K, N, 2, o["dx"], o["dw"], o["dw2"], ws.data_ptr(),
                                size, st) == dfl.OK
    clean("dx", "dw", "dw2")


def test_products_of_no_rows():
    x, w = torch.empty((0, 64), dtype=BF, device="cuda"), randn((136, 64))
    dy = torch.empty((0, 136), dtype=BF, device="cuda")
    y, z = dfl.linear_fwd(x, w, act=dfl.ACT_GELU, save=True)
    assert y.shape == z.shape == (0, 136)
    dx, dw, dbias = dfl.linear_bwd(dy, x, w, z, act=dfl.ACT_GELU, need_dbias=True)
    assert dx.shape == (0, 64) and dw.shape == w.shape and not dw.any() and not dbias.any()
    h, g, u = dfl.gated_fwd(x, w, w, save=True)
    dx, dg, du = dfl.gated_bwd(dy, x, g, u, w, w)
    assert h.shape == (0, 136) and not dg.any() and not du.any()


@pytest.mark.parametrize("rows", [5, 300])
def test_residual_in_place(rows):
    lib, st = dfl.lib(), torch.cuda.current_stream().cuda_stream
    N, K = 1000, 264
    x, w, res = randn((rows, K), seed=1), randn((N, K), seed=2, std=0.1), randn((rows, N), seed=3)
    want, _ = dfl.linear_fwd(x, w, residual=res)
    size = lib.dflare_linear_fwd_workspace(rows, N, K)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert lib.dflare_linear_fwd(x.data_ptr(), w.data_ptr(), None, res.data_ptr(), rows, N, K, 0, res.data_ptr(), None, ws.data_ptr(), size,
                                 st) == dfl.OK
    assert torch.equal(res, want)


@pytest.mark.parametrize("rows", [5, 200])
def test_products_keep_nan_and_infinities_where_they_belong(rows):
    N, K = 136, 200
    x, w, dy = randn((rows, K), seed=1), randn((N, K), seed=2, std=0.1), randn((rows, N), seed=3)
    y, z = dfl.linear_fwd(x, w, act=dfl.ACT_SILU, save=True)
    dx, dw, db = dfl.linear_bwd(dy, x, w, z, act=dfl.ACT_SILU, need_dbias=True)
    h, g, u = dfl.gated_fwd(x, w, w, save=True)
    for bad in (float("nan"), float("inf"), -float("inf")):
        x2 = x.clone()
        x2[3, 199] = bad
        y2, _ = dfl.linear_fwd(x2, w, act=dfl.ACT_SILU)
        h2, _, _ = dfl.gated_fwd(x2, w, w)
        keep = torch.arange(rows, device="cuda") != 3
        assert torch.equal(y2[keep], y[keep]) and torch.equal(h2[keep], h[keep])
        assert not torch.isfinite(h2[3].float()).all()
        d2 = dy.clone()
        d2[3, 135] = bad
        dx2, dw2, db2 = dfl.linear_bwd(d2, x, w, z, act=dfl.ACT_SILU, need_dbias=True)
        assert torch.equal(dx2[keep], dx[keep]) and torch.equal(dw2[:135], dw[:135]) and torch.equal(db2[:135], db[:135])
        assert not torch.isfinite(dw2[135].float()).any() and not torch.isfinite(db2[135].float())


@pytest.mark.parametrize("act", list(ACTS))
def test_activations_at_their_limits(act):
    """Infinite, huge and tiny pre-activations: a weight of ones passes them on one by one."""
    inf = float("inf")
    z = torch.tensor([0.0, -0.0, 1e-38, -1e-38, 1e-3, -1e-3, 3.0, -3.0, 9.0, -9.0, 40.0, -40.0, 90.0, -90.0, 200.0, -200.0, 1e20, -1e20,
                      3e38, -3e38, inf, -inf, float("nan"), 1.0], device="cuda").to(BF)
    n = z.numel()
    x = torch.zeros((n, 8), dtype=BF, device="cuda")
    x[:, 0] = z
    w = torch.zeros((8, 8), dtype=BF, device="cuda")
    w[:, 0] = 1.0
    x[z.isinf() | z.isnan(), 1:] = 0.0
    y, zs = dfl.linear_fwd(x, w, act=ACTS[act], save=True)
    assert torch.equal(zs[:, 0].float().nan_to_num(1.5), z.float().nan_to_num(1.5))
    dy = torch.ones((n, 8), dtype=BF, device="cuda")
    eye = torch.eye(8, dtype=BF, device="cuda")
    zin = z[:, None].expand(n, 8).contiguous()
    dx, _, _ = dfl.linear_bwd(dy, x, eye, zin, act=ACTS[act])
    lim = z.double().clamp(-1e4, 1e4)  # where all of them have reached their limits
    v, d = act64(act, lim)
    v = torch.where(z.double() > 1e4, z.double(), v)
    v = torch.where(z.double() < -1e4, z.double() if act == "none" else torch.zeros_like(v), v)
    if act != "none":  # (whose derivative is 1 anywhere)
        d = torch.where(z.isnan(), z.double(), d)
    for got, want in ((y[:, 0], v), (dx[:, 0], d)):
        got, fine, inf = got.double(), torch.isfinite(want), torch.isinf(want)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[inf], want[inf])
        within(got[fine], want[fine], ((HALF[BF] + REL) * want.abs() + REL * 1e-2 + LEAST)[fine], act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated_gradient_against_differences(act):
    """The formula in 64 bits, moved along random directions."""
    rows, F, H = 40, 72, 64
    x, wg, wu, dh = randn((rows, H), seed=1), randn((F, H), seed=2, std=0.2), randn((F, H), seed=3, std=0.2), randn((rows, F), seed=4)
    _, gate, up = dfl.gated_fwd(x, wg, wu, act=ACTS[act], save=True)
    grads = dfl.gated_bwd(dh, x, gate, up, wg, wu, act=ACTS[act])

    def f(a, b, c):
        return (act64(act, a @ b.t())[0] * (a @ c.t()) * dh.double()).sum()
    at = [t.double() for t in (x, wg, wu)]
    h = 1e-6
    for k in range(3):
        for seed in range(3):
            v = randn(at[k].shape, F64, 30 + seed)
            hi, lo = ([t + (s * h * v if i == k else 0) for i, t in enumerate(at)] for s in (1, -1))
            num = (f(*hi) - f(*lo)) / (2 * h)
            got = (grads[k].double() * v).sum()
            # a gradient: pre-activations stored in bf16, gradients as operands and as results, each off by 2^-8 at most and
            # at random; in a sum of thousands of terms, five times their root mean square
            noise = 4 * HALF[BF] * float((grads[k].double() * v).square().sum().sqrt()) * math.sqrt(H + F)
            assert abs(float(num - got)) <= noise, (k, float(num), float(got), noise)


# ---- AdamW ----

def state_of(sizes, types, bits, masters, seed=0, fresh=False):
    ps = [randn((n,), t, seed + i, std=0.1) for i, (n, t) in enumerate(zip(sizes, types))]
    m, v, ms, vs = dfl.adamw_state(ps, bits)
    if not fresh:
        for i, n in enumerate(sizes):
            a, b = randn((n,), F32, seed + 100 + i, std=0.3), randn((n,), F32, seed + 200 + i).square()
            if bits == 32:
                m[i].copy_(a)
                v[i].copy_(b)
            else:
                for q, s, t in ((m[i], ms[i], a), (v[i], vs[i], b.sqrt())):
                    pad = torch.nn.functional.pad(t, (0, -n % 256)).view(-1, 256)
                    s.copy_(pad.abs().amax(1) / 448)
                    q.copy_((pad / s[:, None]).view(-1)[:n].to(F8))
    w = [p.float() + randn(p.shape, F32, seed + 300 + i, std=1e-4) if masters and p.dtype == BF else None for i, p in enumerate(ps)]
    return ps, m, v, ms, vs, w


def spread(s, n):
    return s.double().repeat_interleave(256)[:n]


def adamw_check(before, after, grads, step, lr, b1, b2, eps, wd, factor, bits):
    for i, g in enumerate(grads):
        p, m, v, ms, vs, w = (None if t is None or t[i] is None else t[i] for t in before)
        P, M, V, MS, VS, W = (None if t is None or t[i] is None else t[i] for t in after)
        n = p.numel()
        if n == 0:
            continue
        g = g.double() * factor
        m, v = (m.double(), v.double()) if bits == 32 else (m.double() * spread(ms, n), (v.double() * spread(vs, n)) ** 2)
        mw, vw = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        # numbers of the formula in fp32: each product, sum and constant within a unit of its terms
        em, ev = 6 * U * (b1 * m.abs() + (1 - b1) * g.abs()) + 1e-44, 8 * U * vw + 1e-44
        old = (p if w is None else w).double()
        den = (vw / (1 - b2 ** step)).sqrt() + eps
        upd = lr / (1 - b1 ** step) * mw / den
        want = old * (1 - lr * wd) - upd
        rel = 16 * U + 0.5 * ev / vw.clamp_min(1e-300) * (vw > 0)
        ew = 4 * U * (old.abs() + upd.abs()) + upd.abs() * rel + lr / (1 - b1 ** step) * em / den
        if W is not None:
            within(W, want, 1.01 * (ew + U * want.abs()) + 1e-44, "master")
            assert torch.equal(P, W.to(BF))
        else:
            within(P, want, 1.01 * (ew + HALF[p.dtype] * want.abs()) + 1e-40, "param")
        if bits == 32:
            within(M, mw, 1.01 * em, "m")
            within(V, vw, 1.01 * ev, "v")
            continue
        for Q, S, t, e in ((M, MS, mw, em), (V, VS, vw.sqrt(), vw.sqrt() * 8 * U + 1e-22)):
            pad = torch.nn.functional.pad(t, (0, -n % 256)).view(-1, 256).abs().amax(1) / 448
            within(S, pad.clamp_min(2.0 ** -96), 16 * U * pad + 1e-40, "scale")
            s = spread(S, n)
            # half a step: 2^-4 of a number, or of its distance from zero 2^-10 below 2^-6; a root above zero at least 2^-9
            step8 = torch.maximum(t.abs() * 2.0 ** -4, s * 2.0 ** -10)
            if Q is V:
                step8 = torch.where(t > 0, torch.maximum(step8, s * 2.0 ** -9), step8)
                assert ((Q.float() > 0) == (t > 1e-22)).all()
            within(Q.double() * s, t, 1.001 * step8 + 16 * U * t.abs() + 2 * e, "8-bit state")


SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 0, 70001, 5000]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("masters", [True, False])
@pytest.mark.parametrize("clip", [None, 0.5, 1e9])
def test_adamw(bits, masters, clip):
    print(f"[more ops] adamw {bits} {masters} {clip}", flush=True)
    types = [BF if i % 2 else F32 for i in range(len(SIZES))]
    gtypes = [BF if i % 3 else F32 for i in range(len(SIZES))]
    state = state_of(SIZES, types, bits, masters)
    kw = dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    for step in (5, 6, 7):
        grads = [randn((n,), t, 400 + 20 * step + i) for i, (n, t) in enumerate(zip(SIZES, gtypes))]
        before = tuple(None if t is None else [None if x is None else x.clone() for x in t] for t in state)
        factor, sumsq = 1.0, None
        if clip is not None:
            norm, sumsq = dfl.grad_norm(grads)
            factor = min(1.0, clip / float(sumsq.sqrt()))
        ps, m, v, ms, vs, w = state
        keep = [g.clone() for g in grads]
        dfl.adamw(ps, grads, m, v, step, 1e-2, masters=w, m_scales=ms, v_scales=vs, sumsq=sumsq,
                  max_norm=float("inf") if clip is None else clip, **kw)
        assert same(grads, keep)
        adamw_check(before, state, grads, step, 1e-2, 0.9, 0.95, 1e-8, 0.1, factor, bits)


def test_adamw_8_bit_states_are_the_formula_s_bit_by_bit():
    """Each operation in fp32 by itself, as tensors' operations are: the same numbers and scales, also after several steps."""
    n = 1 << 20
    ps, m, v, ms, vs, _ = state_of([n], [F32], 8, False, seed=3)
    M, V, MS, VS = (t[0].clone() for t in (m, v, ms, vs))
    b1, b2 = 0.9, 0.999
    for step in range(1, 5):
        g = randn((n,), BF, 70 + step, std=1.0)
        _, sumsq = dfl.grad_norm([g])
        dfl.adamw(ps, [g], m, v, step, 1e-3, beta1=b1, beta2=b2, m_scales=ms, v_scales=vs, sumsq=sumsq, max_norm=1.0)
        f = (1.0 / sumsq.sqrt()).float()
        x = g.float() * f
        a = b1 * (M.float().view(-1, 256) * MS[:, None]).view(-1) + (1.0 - b1) * x
        r = (V.float().view(-1, 256) * VS[:, None]).view(-1)
        r = (b2 * (r * r) + (1.0 - b2) * (x * x)).sqrt()
        for t, q, s, got_q, got_s in ((a, M, MS, m[0], ms[0]), (r, V, VS, v[0], vs[0])):
            t = t.view(-1, 256)
            s.copy_((t.abs().amax(1) * torch.tensor(1.0 / 448.0, dtype=F32, device="cuda")).clamp_min(2.0 ** -96))
            k = t / s[:, None]
            if q is V:
                k = torch.where(t > 0, k.clamp_min(2.0 ** -9), k)
            q.copy_(k.view(-1).to(F8))
            assert torch.equal(got_s, s) and same([got_q], [q]), step


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 1e-30])
def test_adamw_of_gradients_whose_squares_are_hardly_there(bits, eps):
    """Second moments down to the smallest number in fp32, whose root is no special case of the formula."""
    b1, b2, lr, n = 0.9, 0.95, 1e-3, 700
    for mag in (1e-26, 1e-20, 1e-19, 1e-18, 1e-17, 1e-16, 1e-14, 1e-10, 1e10, 1e17):
        p = torch.zeros(n, dtype=F32, device="cuda")
        (m,), (v,), ms, vs = dfl.adamw_state([p], bits)
        ms, vs = (ms or [None])[0], (vs or [None])[0]
        for step in (1, 2, 3):
            g = (randn((n,), F32, step).sign() * (0.5 + randn((n,), F32, 9 + step).abs().clamp_max(2.0))) * mag
            value = [t.double() if bits == 32 else t.double() * spread(s, n) for t, s in ((m, ms), (v, vs))]
            mw, vw = b1 * value[0] + (1 - b1) * g.double(), b2 * (value[1] if bits == 32 else value[1] ** 2) + (1 - b2) * g.double() ** 2
            # the products and their sum within units of their terms, and each within half of the smallest number besides
            em, ev = 6 * U * (b1 * value[0].abs() + (1 - b1) * g.double().abs()) + 2.0 ** -147, 8 * U * vw + 2.0 ** -147
            root, old = vw.sqrt(), p.double()
            er = torch.where(vw > 2 * ev, ev / root.clamp_min(1e-200), (vw + ev).sqrt())
            den = root / math.sqrt(1 - b2 ** step) + eps
            low = (root - er).clamp_min(0) / math.sqrt(1 - b2 ** step) + eps
            k = lr / (1 - b1 ** step)
            dfl.adamw([p], [g], [m], [v], step, lr, beta1=b1, beta2=b2, eps=eps, weight_decay=0.0, m_scales=None if ms is None else [ms],
                      v_scales=None if vs is None else [vs])
            bound = k * (mw.abs() + em) / low * (1 + 16 * U) - k * mw.abs() / den + 4 * U * old.abs() + 2.0 ** -147
            within(p, old - k * mw / den, 1.01 * bound, f"parameter at {mag}")
            if bits == 32:
                within(m, mw, 1.01 * em, "m")
                within(v, vw, 1.01 * ev, "v")
            else:
                for q, s, t, e in ((m, ms, mw, em), (v, vs, root, er)):
                    # half a step of e4m3 with its scale's own rounding, and a root above zero at least the smallest number
                    within(q.double() * spread(s, n), t, 1.01 * (2.0 ** -4 * (t.abs() + e) + 2.0 ** -9 * spread(s, n) + e), "8-bit state")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_the_first_step(bits):
    """Zero states; gradients of zero; the first step moves a value by lr against its gradient's sign."""
    state = state_of([600], [F32], bits, False, fresh=True)
    ps, m, v, ms, vs, _ = state
    p0 = ps[0].clone()
    g = randn((600,), F32, 7)
    g[100:200] = 0
    before = tuple(None if t is None else [None if x is None else x.clone() for x in t] for t in state)
    dfl.adamw(ps, [g], m, v, 1, 0.01, weight_decay=0.0, m_scales=ms, v_scales=vs)
    adamw_check(before, state, [g], 1, 0.01, 0.9, 0.999, 1e-8, 0.0, 1.0, bits)
    within(p0.double() - ps[0].double(), 0.01 * g.double().sign(), 1e-5, "lr sign")
    assert torch.equal(ps[0][100:200], p0[100:200])


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_many_tensors_and_views(bits):
    """More tensors than a launch's table holds, side by side at offsets of every alignment; what lies between stays."""
    n = [(37 * i) % 611 + 1 for i in range(230)]
    flat = {k: torch.full((sum(n) + 3 * len(n),), 5.0, dtype=t, device="cuda") for k, t in
            dict(p=BF, g=BF, w=F32).items()}
    at, places = 1, []
    for k in n:
        places.append(at)
        at += k + 3
    views = {k: [b[a:a + s] for a, s in zip(places, n)] for k, b in flat.items()}
    for i, (p, g, w) in enumerate(zip(views["p"], views["g"], views["w"])):
        w.copy_(randn(w.shape, F32, i))
        p.copy_(w)
        g.copy_(randn(g.shape, BF, 1000 + i))
    m, v, ms, vs = dfl.adamw_state(views["p"], bits)
    before = ([t.clone() for t in views["p"]], [t.clone() for t in m], [t.clone() for t in v],
              ms and [t.clone() for t in ms], vs and [t.clone() for t in vs], [t.clone() for t in views["w"]])
    gaps = torch.ones(flat["p"].numel(), dtype=torch.bool, device="cuda")
    for a, s in zip(places, n):
        gaps[a:a + s] = False
    dfl.adamw(views["p"], views["g"], m, v, 3, 1e-2, masters=views["w"], m_scales=ms, v_scales=vs)
    adamw_check(before, (views["p"], m, v, ms, vs, views["w"]), views["g"], 3, 1e-2, 0.9, 0.999, 1e-8, 0.01, 1.0, bits)
    assert all((b[gaps] == 5.0).all() for b in flat.values())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_adamw_leaves_out_a_step_that_is_not_finite(bits, bad):
    state = state_of([3000, 10], [BF, F32], bits, True)
    grads = [randn((3000,), BF, 1), randn((10,), F32, 2)]
    grads[0][77] = bad
    _, sumsq = dfl.grad_norm(grads)
    before = [[None if x is None else x.clone() for x in t] for t in state if t is not None]
    ps, m, v, ms, vs, w = state
    dfl.adamw(ps, grads, m, v, 2, 1e-2, masters=w, m_scales=ms, v_scales=vs, sumsq=sumsq, max_norm=1.0)
    for a, b in zip(before, [t for t in state if t is not None]):
        assert same(a, b)
    # without a sum of squares it touches its value, or its 256 values of the states
    dfl.adamw(ps, grads, m, v, 2, 1e-2, masters=w, m_scales=ms, v_scales=vs)
    keep = torch.ones(3000, dtype=torch.bool, device="cuda")
    keep[77] = False
    assert torch.isfinite(w[0][keep]).all() and not torch.isfinite(m[0].float()[77] * (1 if ms is None else ms[0][0]))
    assert torch.isfinite(m[0].float()[256:]).all()


def test_adamw_agrees_with_clipping_first():
    a, b = (state_of([5000, 300], [F32, F32], 32, False) for _ in range(2))
    grads = [randn((5000,), F32, 1), randn((300,), F32, 2)]
    _, sumsq = dfl.grad_norm(grads)
    dfl.adamw(a[0], grads, a[1], a[2], 9, 1e-3, sumsq=sumsq, max_norm=0.25)
    dfl.clip_grads(grads, sumsq, 0.25)
    dfl.adamw(b[0], grads, b[1], b[2], 9, 1e-3)
    assert all(same(x, y) for x, y in zip(a[:3], b[:3]))


def test_adamw_8_bit_states_follow_32_bit_ones():
    """200 steps of a noisy quadratic: both reach the neighbourhood of its minimum, at the same pace."""
    target = randn((4096,), F32, 1)
    gaps = []
    for bits in (32, 8):
        p = [torch.zeros(4096, device="cuda")]
        m, v, ms, vs = dfl.adamw_state(p, bits)
        for step in range(1, 201):
            g = [p[0] - target + randn((4096,), F32, 1000 + step, std=0.3)]
            dfl.adamw(p, g, m, v, step, 0.03, beta2=0.95, weight_decay=0.0, m_scales=ms, v_scales=vs)
        gaps.append(float((p[0] - target).square().mean().sqrt()))
    assert gaps[1] <= 2 * gaps[0]


# ---- streams, graphs, a whole step ----

def operators(seed=0):
    """Each call with inputs of its own, as functions without arguments that give their outputs."""
    rows, H, F = 48, 256, 520
    freq, _ = dfl.rope_frequencies(64, 1e6)
    pos = torch.arange(3, device="cuda", dtype=torch.int32) * 50
    xs, dys = (tuple(randn((rows, n, 64), seed=seed + s + n) for n in (4, 2)) for s in (1, 11))
    gains = tuple(randn((64,), seed=seed + 20 + k, mean=1.0) for k in range(2))
    x, wg, wu, wd = randn((rows, H), seed=seed + 30), *(randn(s, seed=seed + 31 + k, std=0.1) for k, s in
                                                        enumerate(((F, H), (F, H), (H, F))))
    dy, res, bias = randn((rows, H), seed=seed + 40), randn((rows, H), seed=seed + 41), randn((H,), seed=seed + 42)

    def qk():
        return dfl.qk_norm_rope_fwd(xs, gains, freq, pos, B=16) + sum(dfl.qk_norm_rope_bwd(dys, xs, gains, freq, pos, B=16), ())

    def block():
        h, g, u = dfl.gated_fwd(x, wg, wu, save=True)
        y, z = dfl.linear_fwd(h, wd, bias, residual=res, act=dfl.ACT_GELU, save=True)
        dh, dwd, db = dfl.linear_bwd(dy, h, wd, z, act=dfl.ACT_GELU, need_dbias=True)
        return (h, g, u, y, z, dh, dwd, db, *dfl.gated_bwd(dh, x, g, u, wg, wu))
    return [qk, block], (xs[0], x, dy)


def test_on_another_stream():
    calls, _ = operators()
    want = [f() for f in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [f() for f in calls]
    torch.cuda.current_stream().wait_stream(side)
    assert all(same(a, b) for a, b in zip(got, want))
    x, w = randn((20, 64)), randn((72, 64))
    y, _ = dfl.linear_fwd(x, w, stream=side)
    side.synchronize()
    assert torch.equal(y, dfl.linear_fwd(x, w)[0])


def test_captured_and_replayed():
    """Replays on changed inputs, with the program's own work between them."""
    calls, inputs = operators()
    for f in calls:
        f()  # (workspaces)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [f() for f in calls]
    for turn in range(4):
        for k, t in enumerate(inputs):
            t.copy_(randn(t.shape, seed=100 * turn + k))
        graph.replay()
        want = [f() for f in calls]
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(outs, want)), turn


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_captured_goes_on_counting(bits):
    a, b = (state_of([5000, 300, 77], [BF, F32, BF], bits, True, fresh=True) for _ in range(2))
    grads = [randn((n,), BF, 60 + n) for n in (5000, 300, 77)]
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-2, dtype=F64, device="cuda")

    def go(s, step, lr):
        _, sumsq = dfl.grad_norm(grads)
        dfl.adamw(s[0], grads, s[1], s[2], step, lr, masters=s[5], m_scales=s[3], v_scales=s[4], sumsq=sumsq, max_norm=1.0)
    go(a, step, lr)
    go(b, 1, 1e-2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        go(a, step, lr)
    for k in range(2, 6):
        for i, g in enumerate(grads):
            g.copy_(randn(g.shape, BF, 1000 * k + i))
        lr.fill_(1e-2 / k)
        graph.replay()
        go(b, k, 1e-2 / k)
        torch.cuda.synchronize()
        assert all(same(x, y) for x, y in zip(a, b) if x is not None), k


def test_a_training_step_of_a_draft_layer():
    """All of a layer's operators together, as a step runs them, against autograd in 64 bits; then the parameters' update."""
    n_blocks, B, T, H, F, V, nq, nk, hd = 6, 8, 40, 128, 264, 300, 4, 2, 64
    rows, gamma = n_blocks * B, 4.5
    g = torch.Generator(device="cuda").manual_seed(1)
    names = ["norm1", "wqkv", "bqkv", "gq", "gk", "wo", "norm2", "wg", "wu", "wd", "norm3", "head"]
    shapes = [(H,), ((nq + 2 * nk) * hd, H), ((nq + 2 * nk) * hd,), (hd,), (hd,), (H, nq * hd), (H,), (F, H), (F, H), (H, F), (H,), (V, H)]
    P = {k: randn(s, seed=i, std=0.15 if len(s) == 2 else 0.2, mean=1.0 if len(s) == 1 and k != "bqkv" else 0.0)
         for i, (k, s) in enumerate(zip(names, shapes))}
    x = randn((rows, H), seed=50)
    kc, vc = randn((T, nk, hd), seed=51), randn((T, nk, hd), seed=52)
    anchors = torch.randint(0, T + 1, (n_blocks,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    freq, _ = dfl.rope_frequencies(hd, 1e4)

    # forward
    n1, _, _, r1 = dfl.norm_fwd(x, P["norm1"])
    qkv, _ = dfl.linear_fwd(n1, P["wqkv"], P["bqkv"])
    cut = qkv.view(rows, nq + 2 * nk, hd).split([nq, nk, nk], 1)
    q, k = dfl.qk_norm_rope_fwd(cut[:2], (P["gq"], P["gk"]), freq, anchors, B=B)
    v = cut[2].contiguous()
    att, lse = dfl.anchor_attention_fwd(q, kc, vc, k, v, anchors, B)
    att16 = att.to(BF).view(rows, nq * hd)
    h1, _ = dfl.linear_fwd(att16, P["wo"], residual=x)
    n2, _, _, r2 = dfl.norm_fwd(h1, P["norm2"])
    act, gate, up = dfl.gated_fwd(n2, P["wg"], P["wu"], save=True)
    h2, _ = dfl.linear_fwd(act, P["wd"], residual=h1)
    n3, _, _, r3 = dfl.norm_fwd(h2, P["norm3"])
    loss, _, dn3, dhead = dfl.linear_ce(n3, P["head"], labels, B, gamma, need_dhead=True)
    # backward
    G = {"head": dhead}
    dh2, G["norm3"], _ = dfl.norm_bwd(dn3, h2, P["norm3"], None, r3)
    dact, G["wd"], _ = dfl.linear_bwd(dh2, act, P["wd"])
    dn2, G["wg"], G["wu"] = dfl.gated_bwd(dact, n2, gate, up, P["wg"], P["wu"])
    dh1, G["norm2"], _ = dfl.norm_bwd(dn2, h1, P["norm2"], None, r2, dsum=dh2)
    datt, G["wo"], _ = dfl.linear_bwd(dh1, att16, P["wo"])
    dq, _, _, dk, dv = dfl.anchor_attention_bwd(q, kc, vc, k, v, anchors, B, att, lse, datt.float().view(rows, nq, hd))
    dqkv = torch.empty_like(qkv)
    d3 = dqkv.view(rows, nq + 2 * nk, hd).split([nq, nk, nk], 1)
    dxs, (G["gq"], G["gk"]) = dfl.qk_norm_rope_bwd((dq.to(BF), dk.to(BF)), cut[:2], (P["gq"], P["gk"]), freq, anchors, B=B)
    for to, t in zip(d3, (*dxs, dv.to(BF))):
        to.copy_(t)
    dn1, G["wqkv"], G["bqkv"] = dfl.linear_bwd(dqkv, n1, P["wqkv"], need_dbias=True)
    dx, G["norm1"], _ = dfl.norm_bwd(dn1, x, P["norm1"], None, r1, dsum=dh1)

    # the same in 64 bits
    W = {k: t.double().requires_grad_() for k, t in P.items()}
    x64 = x.double().requires_grad_()

    def rms(u, w):
        return u * (u.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w
    pos = anchors.repeat_interleave(B).long() + torch.arange(rows, device="cuda") % B
    th = pos.double()[:, None] * freq
    cs, sn = torch.cos(th)[:, None], torch.sin(th)[:, None]

    def rot(u):
        a, b = u.chunk(2, -1)
        return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)
    parts = (rms(x64, W["norm1"]) @ W["wqkv"].t() + W["bqkv"]).view(rows, nq + 2 * nk, hd).split([nq, nk, nk], 1)
    q6, k6, v6 = rot(rms(parts[0], W["gq"])), rot(rms(parts[1], W["gk"])), parts[2]
    seen = torch.arange(T, device="cuda")[None] < anchors.repeat_interleave(B)[:, None]
    own = torch.arange(rows, device="cuda")[None] // B == torch.arange(rows, device="cuda")[:, None] // B
    mask = torch.cat([seen, own], 1)
    outs = []
    for i in range(nq):
        kk, vv = torch.cat([kc[:, i // 2].double(), k6[:, i // 2]]), torch.cat([vc[:, i // 2].double(), v6[:, i // 2]])
        s = (q6[:, i] @ kk.t() / math.sqrt(hd)).masked_fill(~mask, -math.inf)
        outs.append(torch.softmax(s, -1) @ vv)
    a1 = x64 + torch.cat(outs, 1) @ W["wo"].t()
    m2 = rms(a1, W["norm2"])
    a2 = a1 + (torch.nn.functional.silu(m2 @ W["wg"].t()) * (m2 @ W["wu"].t())) @ W["wd"].t()
    z = rms(a2, W["norm3"]) @ W["head"].t()
    b = torch.arange(rows, device="cuda") % B
    w = torch.where(b > 0, torch.exp(-(b - 1).double() / gamma), 0.0)
    want = (w * torch.nn.functional.cross_entropy(z, labels.long(), reduction="none")).sum() / w.sum()
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 1e-2 * float(want.detach())
    # Some 30 tensors on the way are rounded to bf16, each by 2^-8 at most and about a third of that at root mean square; what they do
    # to a gradient adds up as their squares do, each passed on by a factor about one.
    for k in names:
        rel = float((G[k].double() - W[k].grad).norm() / W[k].grad.norm())
        assert rel <= math.sqrt(30) * HALF[BF], (k, rel)
    assert float((dx.double() - x64.grad).norm() / x64.grad.norm()) <= math.sqrt(30) * HALF[BF]

    # the update
    params, grads = [P[k] for k in names], [G[k] for k in names]
    for bits in (32, 8):
        ps = [p.clone() for p in params]
        masters = [p.float() for p in ps]
        m, v, ms, vs = dfl.adamw_state(ps, bits)
        _, sumsq = dfl.grad_norm(grads)
        before = ([p.clone() for p in ps], [t.clone() for t in m], [t.clone() for t in v], ms and [t.clone() for t in ms],
                  vs and [t.clone() for t in vs], [t.clone() for t in masters])
        dfl.adamw(ps, grads, m, v, 1, 1e-3, masters=masters, m_scales=ms, v_scales=vs, sumsq=sumsq, max_norm=1.0)
        flat = [t.view(-1) for t in grads]
        adamw_check([t and [x.view(-1) for x in t] for t in before], [t and [x.view(-1) for x in t] for t in (ps, m, v, ms, vs, masters)],
                    flat, 1, 1e-3, 0.9, 0.999, 1e-8, 0.01, min(1.0, 1.0 / float(sumsq.sqrt())), bits)


def test_adamw_of_tensors_that_lie_far_apart():
    """Parameters and masters in turn with tensors that have none; addresses in any order, also where gigabytes lie between."""
    big = torch.empty(3 << 30, dtype=torch.uint8, device="cuda")
    spots = [torch.empty(0)] * 3
    for i, at in enumerate(((3 << 30) - (1 << 20), 1 << 30, 0)):
        spots[i] = big[at:at + 4000].view(F32)
    ps = [spots[0], randn((500,), BF, 1), spots[1], randn((600,), BF, 2), spots[2]]
    for i, p in enumerate(ps):
        p.copy_(randn(p.shape, F32, 10 + i))
    masters = [None, ps[1].float(), None, ps[3].float(), None]
    grads = [randn(p.shape, BF, 20 + i) for i, p in enumerate(ps)]
    m, v, _, _ = dfl.adamw_state(ps)
    before = ([p.clone() for p in ps], [t.clone() for t in m], [t.clone() for t in v], None, None,
              [None if t is None else t.clone() for t in masters])
    dfl.adamw(ps, grads, m, v, 2, 1e-2, masters=masters)
    adamw_check(before, (ps, m, v, None, None, masters), grads, 2, 1e-2, 0.9, 0.999, 1e-8, 0.01, 1.0, 32)


def test_binding_refuses_tensors_that_do_not_fit():
    x, w = randn((8, 64)), randn((72, 64))
    dy, z = randn((8, 72)), randn((8, 72))
    for f in (lambda: dfl.linear_fwd(x, randn((72, 56))), lambda: dfl.linear_fwd(x, w, randn((64,))), lambda: dfl.linear_fwd(x, w, residual=x),
              lambda: dfl.linear_fwd(x.t(), w), lambda: dfl.linear_bwd(x, x, w), lambda: dfl.gated_fwd(x, w, randn((64, 64))),
              lambda: dfl.gated_bwd(dy, x, z, x, w, w), lambda: dfl.qk_norm_rope_fwd(x.view(8, 1, 64), randn((32,)), torch.zeros(32, dtype=F64, device="cuda")),
              lambda: dfl.qk_norm_rope_fwd((x.view(8, 1, 64),), (None, None), torch.zeros(32, dtype=F64, device="cuda")),
              lambda: dfl.linear_fwd(x.view(2, 4, 64), w)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: dfl.linear_fwd(x.float(), w.float()), lambda: dfl.linear_fwd(x, w.float()), lambda: dfl.linear_bwd(None, x, w),
              lambda: dfl.gated_bwd(dy, x, None, z, w, w), lambda: dfl.linear_fwd(x, w, act="silu"),
              lambda: dfl.qk_norm_rope_fwd(x.view(8, 1, 64), None, torch.zeros(32, device="cuda")),
              lambda: dfl.adamw([x], [x], [x], [x], 1, 0.1), lambda: dfl.adamw([x], [x], [x.float()], [x.float()], 1.5, 0.1)):
        with pytest.raises(TypeError):
            f()
    for f, status in ((lambda: dfl.linear_fwd(x, w, act=9), dfl.ERR_INVALID_ARG), (lambda: dfl.linear_bwd(dy, x, w, act=dfl.ACT_SILU), dfl.ERR_INVALID_ARG),
                      (lambda: dfl.linear_fwd(randn((4, 60)), randn((8, 60))), dfl.ERR_UNSUPPORTED),
                      (lambda: dfl.linear_fwd(randn((520,))[4:516].view(8, 64), w), dfl.ERR_INVALID_ARG),
                      (lambda: dfl.adamw([x], [x], [x.float()], [x.float()], 0, 0.1), dfl.ERR_INVALID_ARG)):
        with pytest.raises(dfl.DFlareError) as e:
            f()
        assert e.value.status == status
    m, v, ms, vs = dfl.adamw_state([x], 8)
    for f in (lambda: dfl.adamw([x], [x], m, v, 1, 0.1, m_scales=[ms[0][:1]], v_scales=vs),
              lambda: dfl.adamw([x], [x, x], m, v, 1, 0.1, m_scales=ms, v_scales=vs), lambda: dfl.adamw([x], [dy], m, v, 1, 0.1, m_scales=ms, v_scales=vs),
              lambda: dfl.adamw([x], [x], [x.float()], [x.float()], 1, 0.1, m_scales=ms, v_scales=vs)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(dfl.DFlareError):  # 8-bit moments without scales
        dfl.adamw([x], [x], m, v, 1, 0.1)


def test_two_graphs_in_turn():
    """Two captured graphs of the same calls on other inputs, replayed in turn with eager calls between."""
    made = []
    for seed in (0, 500):
        calls, inputs = operators(seed)
        for f in calls:
            f()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = [f() for f in calls]
        made.append((calls, inputs, graph, outs))
    for turn in range(3):
        for k, (calls, inputs, graph, outs) in enumerate(made):
            inputs[1].copy_(randn(inputs[1].shape, seed=turn * 10 + k))
            graph.replay()
        for calls, inputs, graph, outs in made:
            want = [f() for f in calls]
            torch.cuda.synchronize()
            assert all(same(a, b) for a, b in zip(outs, want))


def test_calls_of_two_streams_at_once():
    """Each call has a workspace of its own."""
    calls, _ = operators()
    more, _ = operators(900)
    want, want2 = [f() for f in calls], [f() for f in more]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b):
        s.wait_stream(torch.cuda.current_stream())
    got = {}
    for turn in range(5):
        with torch.cuda.stream(a):
            got[0] = [f() for f in calls]
        with torch.cuda.stream(b):
            got[1] = [f() for f in more]
    torch.cuda.synchronize()
    assert all(same(x, y) for x, y in zip(got[0], want)) and all(same(x, y) for x, y in zip(got[1], want2))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_qk_norm_rope_of_small_and_large_heads_without_an_eps(dtype, eps):
    """Heads of one call from 2^-55 to 2^58 at root mean square: the squares' sums are inside fp32 for all of them."""
    freq, _ = dfl.rope_frequencies(64, 1e4)
    size = torch.tensor([2.0 ** k for k in (-55, -48, -20, 0, 30, 52, 53, 58)], device="cuda")[:, None]
    x, dy = (randn((9, 8, 64), F32, 1) * size).to(dtype), randn((9, 8, 64), dtype, 2)
    gain = randn((64,), dtype, 3, mean=1.0, std=0.3)
    kw = dict(layout=dfl.ROPE_HALF, eps=eps)
    y, (dx, dgain) = dfl.qk_norm_rope_fwd(x, gain, freq, **kw), dfl.qk_norm_rope_bwd(dy, x, gain, freq, **kw)
    qk_check(x, gain, torch.arange(9, device="cuda"), freq, True, 1.0, eps, y, dy, dx, dgain)


@pytest.mark.parametrize("masters", [True, False])
@pytest.mark.parametrize("lr,decay", [(1e-6, 0.1), (1e-6, 0.01)])
def test_adamw_decay_of_small_rates_adds_up(masters, lr, decay):
    """lr weight_decay of 1e-7 and 1e-8, next to and below fp32's steps under 1: what 64 steps take off a million values at the mean."""
    n, steps, b1, b2 = 1 << 20, 64, 0.9, 0.95
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(n, device="cuda").uniform_(1.1, 1.9, generator=g)
    p = w.to(BF) if masters else w
    m, v = randn((n,), F32, 2), torch.empty(n, device="cuda").uniform_(0.5, 1.5, generator=g)
    want, mw, vw = w.double(), m.double(), v.double()
    for step in range(50, 50 + steps):
        x = randn((n,), F32, step)
        dfl.adamw([p], [x], [m], [v], step, lr, beta1=b1, beta2=b2, weight_decay=decay, masters=[w] if masters else None)
        mw = b1 * mw + (1 - b1) * x.double()
        vw = b2 * vw + (1 - b2) * x.double() ** 2
        want = want * (1 - lr * decay) - lr / (1 - b1 ** step) * mw / ((vw / (1 - b2 ** step)).sqrt() + 1e-8)
    # A step rounds each value to half of 2^-23 at most, the update (several times that, another one for each value) deciding the
    # side: 2^-23 / sqrt(12) at root mean square, which n values times `steps` bring down to 2.7e-10 at the mean; 30 of these.  Errors
    # of the update itself are 2^-22 of 1e-6 a step.
    off = float((w.double() - want).mean())
    assert abs(off) <= 30 * 2.0 ** -23 / math.sqrt(12) * math.sqrt(steps / n) + steps * 2.0 ** -22 * lr, off
    assert not masters or torch.equal(p, w.to(BF))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_decay_of_what_is_no_number(bits):
    """Infinite and undefined parameters stay what they are, beside others that are not touched by it."""
    p = randn((300,), F32, 1)
    p[5], p[6], p[7] = float("inf"), -float("inf"), float("nan")
    q = p.clone()
    q[5:8] = 1.0
    x = randn((300,), F32, 2)
    for t in (p, q):
        m, v, ms, vs = dfl.adamw_state([t], bits)
        dfl.adamw([t], [x], m, v, 1, 1e-2, weight_decay=0.1, m_scales=ms, v_scales=vs)
    assert p[5] == float("inf") and p[6] == -float("inf") and p[7].isnan()
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[5:8] = False
    assert torch.equal(p[keep], q[keep])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_adamw_8_bit_states_of_gradients_that_are_not_finite(bad):
    """The 256 values that share a scale with such a one are what the formula gives; the others are what they are without it."""
    n, at = 1000, 300
    state, clean = (state_of([n], [F32], 8, False, seed=3) for _ in range(2))
    M, V, MS, VS = (state[k][0].clone() for k in (1, 2, 3, 4))
    g = randn((n,), F32, 9)
    dfl.adamw(clean[0], [g], clean[1], clean[2], 4, 1e-3, m_scales=clean[3], v_scales=clean[4])
    g[at] = bad
    dfl.adamw(state[0], [g], state[1], state[2], 4, 1e-3, m_scales=state[3], v_scales=state[4])
    pad = lambda t: torch.nn.functional.pad(t, (0, -n % 256)).view(-1, 256)  # noqa: E731
    a = 0.9 * (pad(M.float()) * MS[:, None]) + (1.0 - 0.9) * pad(g)
    r = (pad(V.float()) * VS[:, None])
    r = (0.999 * (r * r) + (1.0 - 0.999) * (pad(g) * pad(g))).sqrt()
    for t, q, s, q0, s0, root in ((a, state[1][0], state[3][0], clean[1][0], clean[3][0], False),
                                  (r, state[2][0], state[4][0], clean[2][0], clean[4][0], True)):
        scale = (t.abs().amax(1) * torch.tensor(1.0 / 448.0, dtype=F32, device="cuda")).clamp_min(2.0 ** -96)
        k = t / scale[:, None]
        if root:
            k = torch.where(t > 0, k.clamp_min(2.0 ** -9), k)
        want, got = k.to(F8).float() * scale[:, None], pad(q.float()) * s[:, None]
        assert torch.equal(s.nan_to_num(1.25, 2.5, -2.5), scale.nan_to_num(1.25, 2.5, -2.5))
        assert torch.equal(got[1].nan_to_num(1.25, 2.5, -2.5), want[1].nan_to_num(1.25, 2.5, -2.5)) and not torch.isfinite(got[1]).any()
        others = torch.arange(n, device="cuda") // 256 != at // 256
        assert torch.equal(q.view(torch.uint8)[others], q0.view(torch.uint8)[others]) and torch.equal(s[[0, 2, 3]], s0[[0, 2, 3]])
    keep = torch.arange(n, device="cuda") != at
    assert torch.equal(state[0][0][keep], clean[0][0][keep])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("step,lr", [(0, 1e-2), (-3, 1e-2), (2, float("nan")), (2, -1e-2), (2, float("inf")), (0, None), (None, -1e-2)])
def test_adamw_leaves_out_a_step_whose_number_or_rate_is_none(bits, step, lr):
    """On the device, where the call cannot refuse them; the next step, with others in their place, is taken."""
    state = state_of([3000, 10, 300], [BF, F32, BF], bits, True)
    ps, m, v, ms, vs, w = state
    grads = [randn((n,), BF, 1 + n) for n in (3000, 10, 300)]
    before = [[None if x is None else x.clone() for x in t] for t in state if t is not None]
    at = torch.full((1,), 2 if step is None else step, dtype=torch.int64, device="cuda") if step is not None else 2
    rate = torch.full((1,), lr, dtype=F64, device="cuda") if lr is not None else 1e-2
    dfl.adamw(ps, grads, m, v, at, rate, masters=w, m_scales=ms, v_scales=vs)
    for a, b in zip(before, [t for t in state if t is not None]):
        assert same(a, b)
    if step is not None:
        at.fill_(2)
    if lr is not None:
        rate.fill_(1e-2)
    other = [None if t is None else [None if x is None else x.clone() for x in t] for t in state]
    dfl.adamw(ps, grads, m, v, at, rate, masters=w, m_scales=ms, v_scales=vs)
    dfl.adamw(other[0], grads, other[1], other[2], 2, 1e-2, masters=other[5], m_scales=other[3], v_scales=other[4])
    assert all(same(a, b) for a, b in zip(state, other) if a is not None) and not same(state[0], before[0])


@pytest.mark.parametrize("rows,N,K", [(5, 264, 520), (63, 264, 2056), (300, 520, 2056), (1000, 72, 4096)])
def test_products_stay_inside_the_workspace_of_their_plan(rows, N, K):
    """A workspace of just the plan's bytes between others that stay; the results do not hang on what lay in it."""
    lib, st = dfl.lib(), torch.cuda.current_stream().cuda_stream
    x, w, u, dy = randn((rows, K), seed=1), randn((N, K), seed=2, std=K ** -0.5), randn((N, K), seed=3, std=K ** -0.5), randn((rows, N), seed=4)
    y, z = dfl.linear_fwd(x, w, act=dfl.ACT_SILU, save=True)
    h, gate, up = dfl.gated_fwd(x, w, u, save=True)
    want = [(y,), dfl.linear_bwd(dy, x, w, z, act=dfl.ACT_SILU, need_dbias=True), (h,), dfl.gated_bwd(dy, x, gate, up, w, u)]
    plan = [dfl.dflare_product_plan() for _ in range(4)]
    assert lib.dflare_linear_plan(rows, N, K, 2, 1, 1, 1, plan[0], plan[1]) == lib.dflare_gated_plan(rows, K, N, 1, 1, plan[2], plan[3]) == dfl.OK
    for k, p in enumerate(plan):
        n = p.workspace
        buf = torch.full((n + 8192,), 255, dtype=torch.uint8, device="cuda")  # (NaN as fp32 and as bf16)
        ws, got = buf.data_ptr() + 4096, [torch.empty_like(t) for t in want[k]]
        o = [t.data_ptr() for t in got]
        rc = (lambda: lib.dflare_linear_fwd(x.data_ptr(), w.data_ptr(), None, None, rows, N, K, 2, o[0], None, ws, n, st),
              lambda: lib.dflare_linear_bwd(dy.data_ptr(), x.data_ptr(), w.data_ptr(), z.data_ptr(), rows, N, K, 2, *o, ws, n, st),
              lambda: lib.dflare_gated_fwd(x.data_ptr(), w.data_ptr(), u.data_ptr(), rows, K, N, 2, o[0], None, None, ws, n, st),
              lambda: lib.dflare_gated_bwd(dy.data_ptr(), x.data_ptr(), gate.data_ptr(), up.data_ptr(), w.data_ptr(), u.data_ptr(), rows, K, N,
                                           2, *o, ws, n, st))[k]()
        assert rc == dfl.OK and same(got, want[k]), k
        assert (buf[:4096] == 255).all() and (buf[4096 + n:] == 255).all(), k


@pytest.mark.parametrize("kind,rows,N,K,fwd,bwd", WAYS)
def test_products_on_each_of_their_ways(kind, rows, N, K, fwd, bwd):
    """Every tile, whole and in parts, with each epilogue; and both gradients beside one of them alone."""
    print(f"[more ops] {kind} {(rows, N, K, fwd, bwd)}", flush=True)
    x, w, dy = randn((rows, K), seed=1), randn((N, K), seed=2, std=K ** -0.5), randn((rows, N), seed=4)
    if kind == "linear":
        res, bias = randn((rows, N), seed=5), randn((N,), seed=6)
        for act, b, r, save in (("none", None, None, False), ("none", bias, None, True), ("none", None, res, False), ("silu", bias, None, True),
                                ("gelu", None, res, True)):
            code = ACTS[act]
            y, z = dfl.linear_fwd(x, w, b, residual=r, act=code, save=save)
            grads = dfl.linear_bwd(dy, x, w, z, act=code, need_dbias=b is not None)
            linear_check(x, w, b, r, act, dy, y, z, *grads)
            for part in ((True, False), (False, True)):
                one = dfl.linear_bwd(dy, x, w, z, act=code, need_dx=part[0], need_dw=part[1])
                linear_check(x, w, b, r, act, dy, y, z, *one)
        return
    u = randn((N, K), seed=3, std=K ** -0.5)
    for act, save in (("silu", True), ("none", True), ("gelu_tanh", False)):
        h, gate, up = dfl.gated_fwd(x, w, u, act=ACTS[act], save=save)
        if not save:
            gated_check(x, w, u, act, None, h, gate, up, None, None, None)
            continue
        gated_check(x, w, u, act, dy, h, gate, up, *dfl.gated_bwd(dy, x, gate, up, w, u, act=ACTS[act]))
        for part in ((True, False), (False, True)):
            one = dfl.gated_bwd(dy, x, gate, up, w, u, act=ACTS[act], need_dx=part[0], need_dw=part[1])
            gated_check(x, w, u, act, dy, h, gate, up, *one)


@pytest.mark.parametrize("half", [True, False])
def test_qk_norm_rope_of_work_groups_that_take_many_rows(half):
    """Each work-group walks a part of the heads with many fills of its table: distinct rows, checked around the ends of the parts of
    any number of work-groups up to those of a launch, and the gains' gradients over all of them."""
    rows, hd, B = 70_001, 512, 7
    x, dy = randn((rows, 1, hd), seed=1), randn((rows, 1, hd), seed=2)
    gain = randn((hd,), seed=3, mean=1.0, std=0.3)
    freq, _ = dfl.rope_frequencies(hd, 1e6)
    g = torch.Generator(device="cuda").manual_seed(4)
    starts = torch.randint(0, 100_000, (-(-rows // B),), generator=g, device="cuda", dtype=torch.int32)
    kw = dict(B=B, layout=dfl.ROPE_HALF if half else dfl.ROPE_INTERLEAVED)
    y, (dx, dgain) = dfl.qk_norm_rope_fwd(x, gain, freq, starts, **kw), dfl.qk_norm_rope_bwd(dy, x, gain, freq, starts, **kw)
    pos = starts.repeat_interleave(B)[:rows].long() + torch.arange(rows, device="cuda") % B
    for first in range(0, rows, 10_000):  # (all rows, some at a time)
        at = slice(first, min(first + 10_000, rows))
        u = x[at].double()
        n = u * (u.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        want, size = turned(n * gain.double(), pos[at], freq, half, 1.0)
        k = (hd + 32) * U
        within(y[at], want, 1.01 * (HALF[BF] * want.abs() + k * size) + 1e-38, "y")
        d, size = turned(dy[at].double(), pos[at], freq, half, 1.0, inverse=True)
        part, terms = (d * n).sum((0, 1)), (size * n.abs()).sum((0, 1))
        total, sizes = (part, terms) if first == 0 else (total + part, sizes + terms)
        e, es = d * gain.double(), size * gain.double().abs()
        rstd = (u.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        want = rstd * (e - n * (e * n).mean(-1, keepdim=True))
        err = es + n.abs() * (es * n.abs()).mean(-1, keepdim=True)
        within(dx[at], want, 1.01 * (HALF[BF] * want.abs() + 2 * k * rstd * err) + 1e-38, "dx")
    # (no chain of additions is longer than 4,160 of them: see qk_check)
    within(dgain, total, ((hd + 32) * U + 4160 * U) * sizes + 1e-38, "dgain")
