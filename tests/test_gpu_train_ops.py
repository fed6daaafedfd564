"""The operators of a draft layer's training step against their formulas in 64 bits: the LM head with
the weighted cross-entropy, rotary positions, norms, and the gradients' norm and clipping.

Bounds count roundings: a stored bf16 value is off by at most half a step (2^-8 of it), a sum of n fp32
terms by n 2^-24 of the terms' magnitudes; where a bound has another part it is said there.
"""
import math

import numpy as np
import pytest
import torch

from paper_2606_02091_amd import dflare as dfl

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}  # half a step, relative
U = 2.0 ** -24


def randn(shape, dtype=BF, seed=0, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def within(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((got.double() - want).abs().max()), float(bound.max()))


# ---- LM head with the weighted cross-entropy ----

def lce_inputs(n, B, V, H, seed=0, ignored=0.1, lean=None, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    head = randn((V, H), seed=seed, std=0.02)
    y = torch.randint(0, V, (n * B,), generator=g, device="cuda", dtype=torch.int32)
    u = torch.rand((n * B, 1), generator=g, device="cuda") * (1000.0 / H if lean is None else lean)
    h = ((randn((n * B, H), F32, seed + 2) + u / 0.02 * head[y.long()].float()) * scale).to(BF)
    drop = torch.rand(n * B, generator=g, device="cuda")
    y[drop < ignored] = -1
    y[(drop >= ignored) & (drop < 1.5 * ignored)] = V  # past the vocabulary: no loss either
    return h, head, y


def lce_check(h, head, y, B, gamma, got):
    """Every output against the formula, with the bounds of the kernels' roundings."""
    loss, ce, dh, dw = got
    rows, H = h.shape
    V = head.shape[0]
    b = torch.arange(rows, device="cuda") % B
    on = (b > 0) & (y >= 0) & (y < V)
    w = torch.where(on, torch.exp(-(b - 1).double() / gamma), 0.0)
    c = w / w.sum().clamp_min(1e-300)
    h64, w64 = torch.where(on[:, None], h.double(), 0.0), head.double()
    z = h64 @ w64.t()
    lab = torch.where(on, y, 0).long()[:, None]
    lse = torch.logsumexp(z, 1, keepdim=True)
    want_ce = torch.where(on, (lse - z.gather(1, lab))[:, 0], 0.0)
    # a logit: H products of bf16 values, exact, added in fp32 (twice the bound of rounded sums: the matrix cores may
    # truncate); its scaling by log2 e and the exponent's own rounding are relative to the logits' size
    tz = float(2 * H * U * (h64.abs() @ w64.abs().t()).max() + 8 * U * z.abs().max())
    within(ce, want_ce, 2 * tz + 32 * U * (1 + want_ce.abs()), "row_ce")
    assert abs(float(loss) - float((c * want_ce).sum())) <= 2 * tz + 40 * U * (1 + float(want_ce.abs().max()))
    dz = (z - lse).exp()
    dz.scatter_add_(1, lab, torch.full_like(lab, -1, dtype=torch.float64))
    dz *= c[:, None]
    # dz: the relative error of p, at the label the error of p against the difference p - 1, and half a bf16 step
    rel = 2 * tz + 32 * U
    edz = dz.abs() * (rel + HALF[BF]) + torch.zeros_like(dz).scatter_(1, lab, (c * rel)[:, None])
    if dh is not None:
        want = dz @ w64
        within(dh, want, 1.01 * ((edz + V * 2 * U * dz.abs()) @ w64.abs() + HALF[BF] * want.abs()) + 1e-37, "dhidden")
        assert not dh[~on].any()
    if dw is not None:
        want = dz.t() @ h64  # (from one piece of the vocabulary dz's scale is on the rows of h, rounded as well)
        edz = edz + (HALF[BF] + rows * 2 * U) * dz.abs()
        within(dw, want, 1.01 * (edz.t() @ h64.abs() + HALF[BF] * want.abs()) + 1e-37, "dhead")


# (blocks, B, V, H): one word, one row; widths below, at and past a stage of 64; vocabularies around a tile of 256; 255,
# 256 and 257 rows with a loss at ignored = 0; 4,096 x 70,000 and 128 x 1,100,000: two pieces of the vocabulary,
# on either tile
@pytest.mark.parametrize("n,B,V,H,ignored", [
    (1, 2, 1, 8, 0), (1, 2, 2, 8, 0), (2, 2, 255, 64, 0), (3, 5, 256, 72, 0.1), (7, 3, 257, 56, 0.1),
    (17, 16, 1000, 512, 0), (128, 3, 515, 128, 0), (257, 2, 300, 200, 0), (23, 9, 32003, 264, 0.1),
    (40, 16, 5000, 2880, 0.5), (1, 700, 2049, 1024, 0.2), (256, 16, 70000, 64, 0.05), (5, 13, 3001, 4096, 0.1),
    (1, 128, 1100000, 8, 0.1), (1, 300, 1500, 640, 0)])
def test_linear_ce(n, B, V, H, ignored):
    print(f"[train ops] linear ce {(n, B, V, H)}", flush=True)
    h, head, y = lce_inputs(n, B, V, H, seed=n + V, ignored=ignored)
    gamma = 4.5
    got = dfl.linear_ce(h, head, y, B, gamma, need_dhidden=True, need_dhead=True)
    lce_check(h, head, y, B, gamma, got)
    # the same call gives the same bits; with fewer outputs each is within the same bounds
    again = dfl.linear_ce(h, head, y, B, gamma, need_dhidden=True, need_dhead=True)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    for dh, dw in ((False, False), (True, False), (False, True)):
        part = dfl.linear_ce(h, head, y, B, gamma, need_dhidden=dh, need_dhead=dw)
        assert (part[2] is not None, part[3] is not None) == (dh, dw)
        lce_check(h, head, y, B, gamma, part)


@pytest.mark.parametrize("lean,scale,gamma", [(0.0, 1e-3, 7.0), (3.0, 1.0, 1e9), (20.0, 4.0, 0.3), (-20.0, 4.0, 4.0)])
def test_linear_ce_flat_and_peaked_rows(lean, scale, gamma):
    """Uniform rows, rows whose label takes all, and rows whose label is hopeless (cross-entropies of hundreds)."""
    print(f"[train ops] linear ce lean {lean} scale {scale}", flush=True)
    h, head, y = lce_inputs(30, 11, 3333, 192, seed=3, lean=lean, scale=scale)
    for dw in (False, True):
        lce_check(h, head, y, 11, gamma, dfl.linear_ce(h, head, y, 11, gamma, need_dhead=dw))


def test_linear_ce_far_outlier_words():
    """Words whose logits exceed all others of their row by hundreds, first, in the middle and last."""
    h, head, y = lce_inputs(20, 4, 2100, 64, seed=5, lean=0.0)
    h[:, 0] = 100.0
    head[:, 0] = torch.linspace(-1.0, 1.0, 2100, device="cuda").to(BF)
    for words in ((0,), (1024,), (2099,), (0, 700, 2099)):
        w = head.clone()
        for k, v in enumerate(words):
            w[v, 0] = 4.0 + 3.0 * k
        for dw in (False, True):
            lce_check(h, w, y, 4, 4.5, dfl.linear_ce(h, w, y, 4, 4.5, need_dhead=dw))


def test_linear_ce_outlier_words_of_two_pieces():
    """Rows whose largest logit rises by hundreds within a piece and again in the next one, and rows that stay."""
    h, head, y = lce_inputs(256, 16, 70000, 64, seed=6, lean=0.0)
    h[:, 0] = torch.where(torch.arange(4096, device="cuda") % 3 == 0, 100.0, 0.0).to(BF)
    for words in ((69999,), (5, 69000), (30000, 34000, 40000), (35071, 35072)):
        w = head.clone()
        for k, v in enumerate(words):
            w[v, 0] = 4.0 + 3.0 * k
        lce_check(h, w, y, 16, 4.5, dfl.linear_ce(h, w, y, 16, 4.5))


def test_linear_ce_rows_without_a_loss_may_hold_anything():
    B = 8
    h, head, y = lce_inputs(40, B, 700, 128, seed=8, ignored=0.3)
    off = (torch.arange(h.shape[0], device="cuda") % B == 0) | (y < 0) | (y >= 700)
    want = dfl.linear_ce(h, head, y, B, 4.5, need_dhead=True)
    h[off] = float("nan")
    got = dfl.linear_ce(h, head, y, B, 4.5, need_dhead=True)
    assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_linear_ce_without_any_loss():
    h, head, y = lce_inputs(20, 4, 300, 64, seed=9)
    y.fill_(-1)
    for hh, yy, B in ((h, y, 4), (h, lce_inputs(20, 4, 300, 64, seed=9)[2], 1)):
        loss, ce, dh, dw = dfl.linear_ce(hh, head, yy, B, 4.5, need_dhead=True)
        assert float(loss) == 0 and not ce.any() and not dh.any() and not dw.any()


def test_linear_ce_agrees_with_weighted_ce():
    """The call on logits that the framework has besides: the same loss on the same rows."""
    h, head, y = lce_inputs(9, 16, 4001, 256, seed=11)
    loss, ce, _, _ = dfl.linear_ce(h, head, y, 16, 4.5)
    z = (h.double() @ head.double().t()).float()
    loss2, ce2, _ = dfl.weighted_ce(z, y, 16, 4.5)
    assert abs(float(loss) - float(loss2)) <= 1e-5 * float(loss2)
    assert float((ce - ce2).abs().max()) <= 1e-4


# ---- rotary positions ----

def rope_want(x, pos, freq, rot, half, scale, inverse):
    th = pos.double()[:, None] * freq.double()
    c, s = torch.cos(th)[:, None] * scale, torch.sin(th)[:, None] * scale * (-1 if inverse else 1)
    u = x.double()
    a, b = (u[..., :rot // 2], u[..., rot // 2:rot]) if half else (u[..., 0:rot:2], u[..., 1:rot:2])
    p, q = a * c - b * s, b * c + a * s
    y, size = u.clone(), u.abs()
    if half:
        y[..., :rot // 2], y[..., rot // 2:rot] = p, q
        size[..., :rot // 2] = size[..., rot // 2:rot] = a.abs() + b.abs()
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, q
        size[..., 0:rot:2] = size[..., 1:rot:2] = a.abs() + b.abs()
    return y, size * scale


def rope_check(got, x, pos, freq, rot, half, scale=1.0, inverse=False):
    want, size = rope_want(x, pos, freq, rot, half, scale, inverse)
    # the turn in fp32 (2 pi 2^-25) and cosine and sine within a few units, the two products and their sum
    within(got, want, HALF[x.dtype] * want.abs() + 16 * U * size, "rope")
    if rot < x.shape[-1]:
        assert torch.equal(got[..., rot:], x[..., rot:])


# (rows, B, query heads, key heads, head, rotated): one token, blocks, a whole sequence; rotated parts that end inside an
# access; odd heads and heads of two
@pytest.mark.parametrize("rows,B,nq,nk,hd,rot", [
    (1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (33, 16, 8, 2, 128, 128), (257, 257, 5, 1, 64, 32), (2500, 1, 4, 4, 96, 96),
    (70, 3, 3, 0, 80, 36), (9, 2, 7, 2, 5, 4), (6, 6, 2, 1, 1024, 1024), (5, 4, 65, 3, 256, 64), (4100, 16, 2, 1, 64, 64)])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope(rows, B, nq, nk, hd, rot, half, dtype):
    print(f"[train ops] rope {(rows, B, nq, nk, hd, rot, half, dtype)}", flush=True)
    layout = dfl.ROPE_HALF if half else dfl.ROPE_INTERLEAVED
    xs = tuple(randn((rows, n, hd), dtype, seed=n) for n in (nq, nk) if n)
    freq, _ = dfl.rope_frequencies(rot, 1e4)
    g = torch.Generator(device="cuda").manual_seed(rows)
    starts = torch.randint(-50, 1_000_000, (-(-rows // B),), generator=g, device="cuda", dtype=torch.int32)
    pos = starts.repeat_interleave(B)[:rows].long() + torch.arange(rows, device="cuda") % B
    outs = dfl.rope(xs, freq, starts, B=B, layout=layout, scale=1.25)
    for x, y in zip(xs, outs):
        rope_check(y, x, pos, freq, rot, half, 1.25)
    backs = dfl.rope(xs, freq, starts, B=B, layout=layout, scale=1.25, inverse=True)
    for x, y in zip(xs, backs):
        rope_check(y, x, pos, freq, rot, half, 1.25, inverse=True)
    plain = dfl.rope(xs[0], freq, layout=layout)  # one tensor, rows at their own index
    rope_check(plain, xs[0], torch.arange(rows, device="cuda"), freq, rot, half)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_views_and_in_place(dtype):
    """Heads inside wider rows (a joint projection), at offsets of every alignment; only the heads are written."""
    freq, _ = dfl.rope_frequencies(64, 1e6)
    rows, nq, nk, hd = 37, 6, 2, 64
    pos = torch.arange(rows, device="cuda", dtype=torch.int32) * 3
    for lead in (0, 1, 8, 13):
        buf = randn((rows, lead + (nq + nk) * hd + 5), dtype, seed=lead)
        keep = buf.clone()
        q = buf[:, lead:lead + nq * hd].view(rows, nq, hd)
        k = buf[:, lead + nq * hd:lead + (nq + nk) * hd].unflatten(1, (nk, hd))
        k_heads = k.transpose(0, 1).contiguous().transpose(0, 1)  # head-major memory
        assert not k_heads.is_contiguous()
        out = dfl.rope((q, k_heads), freq, pos)
        for x, y in zip((q, k), out):
            rope_check(y, x, pos.long(), freq, 64, True)
        assert torch.equal(buf, keep)
        dfl.rope((q, k), freq, pos, out=(q, k))
        assert torch.equal(q, out[0]) and torch.equal(k, out[1])
        buf[:, lead:lead + (nq + nk) * hd] = keep[:, lead:lead + (nq + nk) * hd]
        assert torch.equal(buf, keep)


def test_rope_gradient_is_the_inverse():
    """<rope(x), dy> = <x, inverse(dy)>, which also checks it against the differences' definition (the map is linear)."""
    freq, scale = dfl.rope_frequencies(64, 1e6, dfl.ROPE_YARN, 8.0, 4096)
    x, dy = randn((50, 3, 64), F32, 1), randn((50, 3, 64), F32, 2)
    pos = torch.randint(0, 30000, (50,), device="cuda", dtype=torch.int32)
    a = (dfl.rope(x, freq, pos, scale=scale).double() * dy.double()).sum()
    b = (x.double() * dfl.rope(dy, freq, pos, scale=scale, inverse=True).double()).sum()
    assert abs(float(a - b)) <= 32 * U * scale * 2 * float((x.abs().double() * dy.abs().double()).sum())


def test_rope_of_more_rows_than_a_launch_takes():
    rows, hd = (1 << 21) + 3, 512  # a row per work-group
    x = torch.empty((rows, 1, hd), dtype=BF, device="cuda")
    x[:] = randn((1, 1, hd), seed=1)
    freq, _ = dfl.rope_frequencies(hd, 1e6)
    y = dfl.rope(x, freq)
    at = torch.tensor([0, 1, 77, (1 << 21) - 1, 1 << 21, rows - 1], device="cuda")
    rope_check(y[at], x[at], at, freq, hd, True)


def test_rope_of_no_rows():
    freq, _ = dfl.rope_frequencies(64, 1e6)
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    assert dfl.rope(torch.empty((0, 4, 64), dtype=BF, device="cuda"), freq, pos).shape == (0, 4, 64)
    assert dfl.rope(torch.empty((3, 0, 64), dtype=BF, device="cuda"), freq).shape == (3, 0, 64)


# ---- norms ----

def norm_check(x, r, gain, bias, dy, dsum, layer, eps=1e-6):
    kind = dfl.NORM_LAYER if layer else dfl.NORM_RMS
    rows, H = x.shape
    half = HALF[x.dtype]
    y, h, mean, rstd = dfl.norm_fwd(x, gain, bias, residual=r, kind=kind, eps=eps)
    if r is None:
        assert h is x
    else:
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    u = h.double()
    mu = u.mean(1, keepdim=True) if layer else torch.zeros((rows, 1), dtype=torch.float64, device="cuda")
    d = u - mu
    inv = ((d * d).mean(1, keepdim=True) + eps).rsqrt()
    # sums of a row: at most 64 terms in a thread, then 6 + 16 steps over threads, each 2^-24 of the magnitudes
    n = 90 * U
    emu = n * u.abs().mean(1, keepdim=True) if layer else torch.zeros_like(mu)
    einv = (2 * n + 4 * U) + 2 * inv * emu  # relative
    within(rstd, inv[:, 0], (einv * inv)[:, 0], "rstd")
    if layer:
        within(mean, mu[:, 0], emu[:, 0] + 1e-38, "mean")
    xh = d * inv
    exh = xh.abs() * (einv + 4 * U) + inv * (emu + U * (u.abs() + mu.abs()))
    g = torch.ones(H, dtype=torch.float64, device="cuda") if gain is None else gain.double()
    b = torch.zeros(H, dtype=torch.float64, device="cuda") if bias is None else bias.double()
    want = xh * g + b
    within(y, want, 1.01 * (half * want.abs() + exh * g.abs() + 4 * U * ((xh * g).abs() + b.abs())) + 1e-38, "y")
    dx, dgain, dbias = dfl.norm_bwd(dy, h, gain, mean, rstd, dsum=dsum, kind=kind)
    e = dy.double() * g
    s1 = e.mean(1, keepdim=True) if layer else 0.0
    s2 = (e * xh).mean(1, keepdim=True)
    es1 = n * e.abs().mean(1, keepdim=True) if layer else 0.0
    es2 = (n * (e * xh).abs() + e.abs() * exh).mean(1, keepdim=True)
    add = 0.0 if dsum is None else dsum.double()
    want = inv * (e - s1 - xh * s2) + add
    size = inv * (e.abs() + (s1.abs() if layer else 0.0) + (xh * s2).abs())
    err = (einv + 8 * U) * size + inv * (es1 + exh * s2.abs() + (xh.abs() + exh) * es2)
    within(dx, want, 1.01 * (half * want.abs() + err + 2 * U * (add.abs() if dsum is not None else 0.0)) + 1e-38, "dx")
    p = dy.double() * xh
    within(dgain, p.sum(0), ((rows + 40) * U * p.abs() + dy.double().abs() * exh).sum(0) + 1e-38, "dgain")
    if layer:
        within(dbias, dy.double().sum(0), ((rows + 40) * U * dy.double().abs()).sum(0) + 1e-38, "dbias")
    else:
        assert dbias is None
    again = dfl.norm_bwd(dy, h, gain, mean, rstd, dsum=dsum, kind=kind)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)


# one row, one value; widths around every form's end in 16-byte accesses and single values; more rows than work-groups
@pytest.mark.parametrize("rows,H", [(1, 1), (3, 7), (5, 64), (17, 513), (2, 1024), (9, 1025), (33, 2560), (6, 2881), (4, 4096),
                                    (3, 4104), (5, 4097), (2, 8192), (3, 8200), (2, 16384), (2, 16383), (2100, 128), (1500, 520)])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm(rows, H, layer, dtype):
    print(f"[train ops] norm {(rows, H, layer, dtype)}", flush=True)
    x, r = randn((rows, H), dtype, 1, 2.0, 0.5), randn((rows, H), dtype, 2)
    gain, bias = randn((H,), dtype, 3, 0.1, 1.0), randn((H,), dtype, 4) if layer else None
    dy, dsum = randn((rows, H), dtype, 5), randn((rows, H), dtype, 6)
    norm_check(x, r, gain, bias, dy, dsum, layer)
    norm_check(x, None, None, None, dy, None, layer)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_unaligned_rows(dtype):
    """Tensors that start on no 16-byte boundary."""
    def shifted(t):
        buf = torch.empty(t.numel() + 3, dtype=t.dtype, device="cuda")
        buf[3:] = t.flatten()
        return buf[3:].view(t.shape)
    x, r, dy, dsum = (shifted(randn((20, 512), dtype, k)) for k in range(4))
    norm_check(x, r, shifted(randn((512,), dtype, 5)), None, dy, dsum, False)


def test_norm_large_means_and_zero_rows():
    x = randn((40, 1000), F32, 1, 1.0, 300.0)  # the variance is a small difference if formed from squares
    norm_check(x, None, None, None, randn((40, 1000), F32, 2), None, True)
    x[3] = 0
    x[5] = 7.0
    y, _, mean, rstd = dfl.norm_fwd(x, kind=dfl.NORM_LAYER)
    assert not y[3].any() and float(rstd[3]) == pytest.approx(1e3) and float(mean[5]) == 7.0 and not y[5].any()
    y, _, _, rstd = dfl.norm_fwd(x)
    assert not y[3].any() and float(rstd[3]) == pytest.approx(1e3)


def test_norm_of_no_rows():
    x = torch.empty((0, 64), dtype=BF, device="cuda")
    y, h, mean, rstd = dfl.norm_fwd(x, kind=dfl.NORM_LAYER)
    assert y.shape == (0, 64) and rstd.shape == (0,)
    dx, dgain, dbias = dfl.norm_bwd(x, h, None, mean, rstd, kind=dfl.NORM_LAYER)
    assert dx.shape == (0, 64) and not dgain.any() and not dbias.any()


def test_norm_of_more_rows_than_a_launch_takes():
    rows = (1 << 24) + 5  # of one value: rms 1 up to its rounding, so y is the sign
    x = randn((rows, 1), BF, 3)
    x[x == 0] = 1.0
    x[:7] = x[-7:] = torch.tensor([2.0, -2.0, 1.0, -1.0, 0.5, -0.5, 4.0], device="cuda").to(BF)[:, None]
    y, _, _, rstd = dfl.norm_fwd(x, eps=0.0)
    assert torch.equal(y, torch.sign(x)) and float(rstd[-7]) == 0.5 and float(rstd[-1]) == 0.25
    dx, dgain, _ = dfl.norm_bwd(y, x, None, None, rstd)
    assert not dx[-7:].any() and abs(float(dgain) - rows) <= 512 * U * rows


def test_norm_gradients_against_differences():
    """Central differences of the 64-bit formula's loss, along random directions of every input."""
    for layer in (False, True):
        x, gain, bias, dy = randn((6, 96), F32, 1), randn((96,), F32, 2, 0.1, 1.0), randn((96,), F32, 3), randn((6, 96), F32, 4)
        kind = dfl.NORM_LAYER if layer else dfl.NORM_RMS
        _, h, mean, rstd = dfl.norm_fwd(x, gain, bias if layer else None, kind=kind)
        grads = dfl.norm_bwd(dy, h, gain, mean, rstd, kind=kind)

        def loss(x, gain, bias):
            d = x - x.mean(1, keepdim=True) if layer else x
            return ((d * ((d * d).mean(1, keepdim=True) + 1e-6).rsqrt() * gain + (bias if layer else 0)) * dy.double()).sum()
        args = [x.double(), gain.double(), bias.double()]
        for k, g in enumerate(grads):
            if g is None:
                continue
            v = randn(args[k].shape, F32, 10 + k).double()
            up, dn = list(args), list(args)
            up[k], dn[k] = args[k] + 1e-4 * v, args[k] - 1e-4 * v
            # third differences: about (1e-4)^2 of the loss's scale
            assert abs(float((loss(*up) - loss(*dn)) / 2e-4 - (g.double() * v).sum())) <= 1e-5 * float((g.abs() * v.abs()).sum())


# ---- gradients' norm and clipping ----

def grads_of(sizes, seed=0, std=1.0, pad=0):
    """Tensors of alternating type, `pad` elements apart in one buffer of each type."""
    out = []
    for k, dtype in ((0, BF), (1, F32)):
        mine = sizes[k::2]
        buf = randn((sum(mine) + pad * len(mine) + 1,), dtype, seed + k, std)
        at = pad
        for s in mine:
            out.append(buf[at:at + s])
            at += s + pad
    return out


def clip_check(grads, max_norm, **kw):
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    before = [g.clone() for g in grads]
    norm, sumsq = dfl.grad_norm(grads)
    assert abs(float(norm) - want) <= 2 * U * want and abs(math.sqrt(float(sumsq)) - want) <= 1e-12 * want
    coef = max_norm / want if want > max_norm else 1.0
    out = [torch.full_like(g, 9.0) for g in grads]
    dfl.clip_grads(grads, sumsq, max_norm, out=out)
    dfl.clip_grads(grads, sumsq, max_norm)
    for b, g, o in zip(before, grads, out):
        assert torch.equal(g, o)
        if coef == 1.0:
            assert torch.equal(g, b)
        else:
            # (below the normal range half a step is absolute: 2^-134 in bf16, 2^-150 in fp32, the range starting at 2^-126)
            least = 2.0 ** -126 * HALF[g.dtype]
            within(g, b.double() * coef, (HALF[g.dtype] + 3 * U) * b.double().abs() * coef + least, "clip")


@pytest.mark.parametrize("sizes,pad", [
    ([1], 0), ([0], 0), ([0, 0, 5], 0), ([7, 8, 9, 15, 16, 17], 1), ([16384, 8192, 16385, 8193, 100000, 70001], 0),
    ([3, 40000, 1, 32769], 3), (list(range(0, 500)), 1), ([1000003], 5)])
@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0, float("inf")])
def test_grad_norm_and_clip(sizes, pad, max_norm):
    print(f"[train ops] clip {len(sizes)} tensors, max {max_norm}", flush=True)
    clip_check(grads_of(sizes, pad=pad), max_norm)


@pytest.mark.parametrize("std", [1e-30, 1e25])
def test_grad_norm_of_tiny_and_huge_values(std):
    """Squares beyond fp32's range in both directions."""
    clip_check(grads_of([5000, 6000, 77], std=std), 1e-3 * std)


def test_grad_clip_into_tensors_of_other_alignment():
    g = grads_of([5001, 3003], pad=1)
    _, sumsq = dfl.grad_norm(g)
    buf = [torch.zeros(t.numel() + 9, dtype=t.dtype, device="cuda") for t in g]
    for lead in range(9):
        out = [b[lead:lead + t.numel()] for b, t in zip(buf, g)]
        for b in buf:
            b.zero_()
        dfl.clip_grads(g, sumsq, 1.0, out=out)
        ref = [torch.empty_like(t) for t in g]
        dfl.clip_grads(g, sumsq, 1.0, out=ref)
        assert all(torch.equal(o, r) for o, r in zip(out, ref))
        assert all(not b[:lead].any() and not b[lead + t.numel():].any() for b, t in zip(buf, g))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_grad_clip_leaves_gradients_that_are_not_finite(bad):
    g = grads_of([300, 301])
    g[1][7] = bad
    before = [t.clone() for t in g]
    norm, sumsq = dfl.grad_norm(g)
    assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(bad)
    out = [torch.empty_like(t) for t in g]
    dfl.clip_grads(g, sumsq, 1.0, out=out)
    dfl.clip_grads(g, sumsq, 1.0)
    for t, b, o in zip(g, before, out):
        assert torch.equal(t.nan_to_num(5.0), b.nan_to_num(5.0)) and torch.equal(o.nan_to_num(5.0), b.nan_to_num(5.0))


def test_grad_clip_refuses_overlapping_tensors():
    t = randn((100,), F32)
    _, sumsq = dfl.grad_norm([t, t])  # only read: allowed
    for grads, out in (([t, t], None), ([t[:60], t[59:]], None), ([t[:50], t[50:]], [t[50:], t[:50]]),
                       ([t], [t[:]]), ([t[:50]], [t[1:51]])):
        if out is not None and out[0].data_ptr() == grads[0].data_ptr():
            dfl.clip_grads(grads, sumsq, 1.0, out=out)  # in place, said twice
            continue
        with pytest.raises(dfl.DFlareError) as ei:
            dfl.clip_grads(grads, sumsq, 1.0, out=out)
        assert ei.value.status == dfl.ERR_INVALID_ARG


# ---- streams and graphs ----

def one_of_each():
    """(call, its outputs as a list) of every operator, on inputs of its own."""
    h, head, y = lce_inputs(30, 8, 1500, 264, seed=1)
    q, k = randn((77, 8, 64), seed=2), randn((77, 2, 64), seed=3)
    freq, _ = dfl.rope_frequencies(64, 1e6)
    pos = torch.arange(77, device="cuda", dtype=torch.int32)
    x, r, gain, dy = randn((60, 512), seed=4), randn((60, 512), seed=5), randn((512,), seed=6), randn((60, 512), seed=7)
    g = grads_of([999, 5000, 3, 70000], seed=8)
    out = [torch.empty_like(t) for t in g]

    def norm():
        y, hh, mean, rstd = dfl.norm_fwd(x, gain, residual=r)
        return [y, hh, rstd, *dfl.norm_bwd(dy, hh, gain, mean, rstd)[:2]]

    def clip():
        n, s = dfl.grad_norm(g)
        dfl.clip_grads(g, s, 1.0, out=out)
        return [n, s, *out]
    inputs = [h, q, k, x, r, dy, *g]
    return inputs, [lambda: list(dfl.linear_ce(h, head, y, 8, 4.5, need_dhead=True)), lambda: list(dfl.rope((q, k), freq, pos)),
                    norm, clip]


def test_every_operator_in_a_graph():
    """Captured calls replayed on changed inputs, with eager work between the replays."""
    inputs, calls = one_of_each()
    for call in calls:
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = [call() for call in calls]
    for k in range(3):
        for t in inputs:
            t.mul_(-0.75 if k == 1 else 0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in outs] for outs in kept]
        want = [[t.clone() for t in call()] for call in calls]
        torch.cuda.synchronize()
        for outs, refs in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(outs, refs)), k


def test_every_operator_on_a_side_stream():
    _, calls = one_of_each()
    want = [[t.clone() for t in call()] for call in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [[t.clone() for t in call()] for call in calls]
    x = randn((60, 512), seed=4)
    torch.cuda.synchronize()
    y = dfl.norm_fwd(x, stream=side)[0]  # the stream as an argument
    z = dfl.norm_fwd(x, stream=side.cuda_stream)[0]
    side.synchronize()
    for outs, refs in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(outs, refs))
    ref = dfl.norm_fwd(x)[0]
    assert torch.equal(y, ref) and torch.equal(z, ref)


# ---- together: the training step of one draft layer ----

def test_training_step_of_a_layer():
    """Residual norm, rotary positions, anchor attention, final norm, LM head with its loss, and back to the gradients,
    their norm and clipping, as a program strings them together; against 64-bit autograd."""
    n, B, T, nq, nkv, hd, V = 6, 8, 50, 4, 2, 64, 700
    H, M = nq * hd, n * B
    w = {k: randn(s, seed=40 + i, std=0.05) for i, (k, s) in enumerate(
        {"q": (H, H), "k": (nkv * hd, H), "v": (nkv * hd, H), "o": (H, H), "head": (V, H)}.items())}
    gains = {k: randn((H,), seed=50 + i, std=0.1, mean=1.0) for i, k in enumerate(("attn", "final"))}
    x, r = randn((M, H), seed=60), randn((M, H), seed=61)
    kc, vc = randn((T, nkv, hd), seed=62), randn((T, nkv, hd), seed=63)
    g = torch.Generator(device="cuda").manual_seed(5)
    anchors = torch.randint(1, T - B, (n,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    y[3] = -1
    freq, _ = dfl.rope_frequencies(hd, 1e6)

    def mm(a, b):  # a b^T, products outside the framework: fp32 sums, rounded to bf16
        return (a.float() @ b.float().t()).to(BF)

    # forward
    kc_r = dfl.rope(kc, freq)  # context row r at position r
    a1, h1, _, rs1 = dfl.norm_fwd(x, gains["attn"], residual=r)
    q, k, v = (mm(a1, w[m]).view(M, -1, hd) for m in ("q", "k", "v"))
    qr, kr = dfl.rope((q, k), freq, anchors, B=B)
    o, lse = dfl.anchor_attention_fwd(qr, kc_r, vc, kr, v, anchors, B)
    a2, h2, _, rs2 = dfl.norm_fwd(mm(o.view(M, H), w["o"]), gains["final"], residual=h1)
    loss, ce, da2, dhead = dfl.linear_ce(a2, w["head"], y, B, 4.5, need_dhead=True)
    # backward
    dh2, dfinal, _ = dfl.norm_bwd(da2, h2, gains["final"], None, rs2)
    do = (dh2.float() @ w["o"].float()).view(M, nq, hd).contiguous()
    dwo = (dh2.float().t() @ o.view(M, H)).to(BF)
    dq, dkc, dvc, dkb, dvb = dfl.anchor_attention_bwd(qr, kc_r, vc, kr, v, anchors, B, o, lse, do)
    dq, dkb = dfl.rope((dq, dkb), freq, anchors, B=B, inverse=True)
    dkc = dfl.rope(dkc, freq, inverse=True)
    da1 = sum(t.reshape(M, -1) @ w[m].float() for t, m in ((dq, "q"), (dkb, "k"), (dvb, "v"))).to(BF)
    dw = {m: (t.reshape(M, -1).t() @ a1.float()).to(BF) for t, m in ((dq, "q"), (dkb, "k"), (dvb, "v"))}
    dh1, dattn, _ = dfl.norm_bwd(da1, h1, gains["attn"], None, rs1, dsum=dh2)
    got = {"x": dh1, "kc": dkc, "vc": dvc, "attn": dattn, "final": dfinal, "o": dwo, "head": dhead, **dw}

    # the same in 64 bits
    p = {k: t.double().requires_grad_() for k, t in {**w, **gains, "x": x, "kc": kc, "vc": vc}.items()}

    def rms(t, gain):
        return t * (t * t).mean(-1, keepdim=True).add(1e-6).rsqrt() * gain

    def rope64(t, pos):
        th = pos.double()[:, None] * freq
        c, s = torch.cos(th)[:, None], torch.sin(th)[:, None]
        a, b = t[..., :hd // 2], t[..., hd // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    pos = anchors.repeat_interleave(B).long() + torch.arange(M, device="cuda") % B
    h = p["x"] + r.double()
    a = rms(h, p["attn"])
    Q, K, W = ((a @ p[m].t()).view(M, -1, hd) for m in ("q", "k", "v"))
    Q, K, KC = rope64(Q, pos), rope64(K, pos), rope64(p["kc"], torch.arange(T, device="cuda"))
    rows = []
    for i in range(n):
        s = slice(i * B, (i + 1) * B)
        keys, vals = torch.cat([KC[:int(anchors[i])], K[s]]), torch.cat([p["vc"][:int(anchors[i])], W[s]])
        heads = [torch.softmax(Q[s, j] @ keys[:, j // (nq // nkv)].t() / math.sqrt(hd), -1) @ vals[:, j // (nq // nkv)]
                 for j in range(nq)]
        rows.append(torch.cat(heads, -1))
    z = rms(h + torch.cat(rows) @ p["o"].t(), p["final"]) @ p["head"].t()
    b = torch.arange(M, device="cuda") % B
    wt = torch.where((b > 0) & (y >= 0), torch.exp(-(b - 1).double() / 4.5), 0.0)
    want = (wt * torch.nn.functional.cross_entropy(z, y.clamp_min(0).long(), reduction="none")).sum() / wt.sum()
    want.backward()
    want = want.detach()
    # about ten bf16 roundings lie between input and loss or gradient, each at most 2^-8 of the values they fall on and
    # independent of one another: sqrt(10) 2^-8 = 1.2% in the 2-norm
    assert abs(float(loss) - float(want)) <= 0.012 * float(want)
    for k, t in got.items():
        ref = p[k].grad
        assert float((t.double().view(ref.shape) - ref).norm()) <= 0.012 * float(ref.norm()), k
    grads = list(got.values())
    norm, sumsq = dfl.grad_norm(grads)
    total = math.sqrt(sum(float(p[k].grad.norm()) ** 2 for k in got))
    assert abs(float(norm) - total) <= 0.012 * total
    dfl.clip_grads(grads, sumsq, 0.1 * total)
    assert abs(float(dfl.grad_norm(grads)[0]) - 0.1 * total) <= 0.012 * 0.1 * total


def test_binding_refuses_tensors_that_do_not_fit():
    """Every one is refused on the host, before a launch."""
    x, gain, f32 = randn((6, 64)), randn((64,)), randn((6, 64), F32)
    rstd = torch.ones(6, device="cuda")
    for args, why in (((x[0],), ValueError), ((x.t(),), ValueError), ((x.double(),), TypeError), ((x, gain[:63]), ValueError),
                      ((x, gain.float()), TypeError), ((x, None, gain[:32]), ValueError), ((x, gain, None, f32), TypeError),
                      ((x, gain, None, x[:5]), ValueError), ((x, gain.cpu()), TypeError), ((x, gain, None, None, 2 ** 40), ValueError),
                      ((x, gain, None, None, 7), dfl.DFlareError), ((x, gain, None, None, "rms"), TypeError)):
        with pytest.raises(why):
            dfl.norm_fwd(*args)
    for args, why in (((x[:5], x, gain, None, rstd), ValueError), ((x, x, gain, None, rstd[:5]), ValueError),
                      ((x, x, gain, None, rstd.double()), TypeError), ((f32, x, gain, None, rstd), TypeError),
                      ((x, x, gain, None, rstd, x[:, :32].contiguous()), ValueError), ((x, x, gain, None, None), dfl.DFlareError),
                      ((None, x, gain, None, rstd), dfl.DFlareError), ((x, x, gain, None, rstd, None, dfl.NORM_LAYER), dfl.DFlareError)):
        with pytest.raises(why):
            dfl.norm_bwd(*args)
    q, k, pos = randn((6, 4, 16)), randn((6, 2, 16)), torch.zeros(6, dtype=torch.int32, device="cuda")
    freq, _ = dfl.rope_frequencies(16, 1e4)
    wide, _ = dfl.rope_frequencies(32, 1e4)
    for args, kw, why in (((q[0], freq), {}, ValueError), (((q, k[:5]), freq), {}, ValueError), (((q, k.float()), freq), {}, ValueError),
                          ((q.transpose(1, 2), freq), {}, ValueError), ((q, freq.float()), {}, TypeError), ((q, None), {}, TypeError),
                          ((q, wide), {}, dfl.DFlareError), ((q, freq, pos.long()), {}, TypeError), ((q, freq, pos[:5]), {}, ValueError),
                          ((q, freq, pos, 2), {}, ValueError), ((q, freq, None, 0), {}, ValueError), (((q, k, q), freq), {}, ValueError),
                          (((), freq), {}, ValueError), ((q, freq), {"out": (q, k)}, ValueError), ((q, freq), {"out": k}, ValueError),
                          ((q, freq), {"out": q.float()}, ValueError), ((q, freq), {"layout": 5}, dfl.DFlareError)):
        with pytest.raises(why):
            dfl.rope(*args, **kw)
    t = randn((100,), F32)
    _, sumsq = dfl.grad_norm([t])
    for args, why in ((([t, t.double()], sumsq, 1.0), TypeError), (([t.view(10, 10).t()], sumsq, 1.0), ValueError),
                      (([t], sumsq.float(), 1.0), TypeError), (([t], sumsq.expand(2), 1.0), ValueError), (([t], None, 1.0), TypeError),
                      (([t], sumsq, 1.0, []), ValueError), (([t], sumsq, 1.0, [t[:50]]), ValueError), (([t], sumsq, 1.0, [t.bfloat16()]), ValueError),
                      (([t], sumsq, "all"), TypeError), (([t.cpu()], sumsq, 1.0), TypeError)):
        with pytest.raises(why):
            dfl.clip_grads(*args)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = dfl.norm_fwd(x, gain)[0]
    side.synchronize()
    got = dfl.norm_fwd(x, gain, stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want)  # a refusal leaves nothing behind


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_of_views_of_one_buffer(dtype):
    """In place on queries and keys of one buffer, in three layouts; of broadcast rows and heads; the values beside
    them stay; outputs that meet are refused."""
    rows, nq, hd = 37, 6, 32
    freq, _ = dfl.rope_frequencies(hd, 1e4)

    def views():
        flat = randn((rows, nq + 4, hd), dtype, seed=3)
        yield flat, flat[:, :nq], flat[:, nq:nq + 2], flat[:, nq + 2:]
        first = randn((nq + 4, rows, hd), dtype, seed=4)
        yield first, first[:nq].transpose(0, 1), first[nq:nq + 2].transpose(0, 1), first[nq + 2:]
        group = randn((rows, nq, 3, hd), dtype, seed=5)
        yield group, group[:, :, 0], group[:, :, 1], group[:, :, 2]
    for buf, q, k, v in views():
        want = dfl.rope((q.contiguous(), k.contiguous()), freq)
        kept = v.clone()
        got = dfl.rope((q, k), freq, out=(q, k))
        assert got[0] is q and got[1] is k
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, kept)
        for bad in (((q, q), (q, q)), ((q, k), (q, q[:, :k.shape[1]])), ((k,), (k[:1].expand(rows, -1, -1),))):
            with pytest.raises((ValueError, dfl.DFlareError)):
                dfl.rope(bad[0], freq, out=bad[1])
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    one = randn((1, 1, hd), dtype, seed=6).expand(rows, nq, hd)
    assert torch.equal(dfl.rope(one, freq), dfl.rope(one.contiguous(), freq))
    with pytest.raises(dfl.DFlareError):
        dfl.rope(one, freq, out=one)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H", [1, 2, 3, 4, 5, 7, 8, 9, 15, 255, 257, 511, 513, 1023, 1025, 2047, 2049, 4095, 4097, 6047, 8191, 8193, 16381])
def test_norm_rows_off_the_boundaries(H, dtype):
    print(f"[train ops] norm off the boundaries {(H, dtype)}", flush=True)
    for layer in (False, True):
        x, r, dy, dsum = (randn((37, H), dtype, seed) for seed in range(4))
        norm_check(x, r, randn((H,), dtype, 4), randn((H,), dtype, 5) if layer else None, dy, dsum, layer)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H", [5, 64, 513, 1030, 2881, 6047])
def test_norm_in_place_off_the_boundaries(H, dtype):
    """Tensors that start at any element, y and sum over the inputs and dx over each of its own; what lies around them stays."""
    rows, code = 41, dfl._dtype(torch.empty(0, dtype=dtype))
    lib, st = dfl.lib(), torch.cuda.current_stream().cuda_stream
    x, r, dy, dsum = (randn((rows, H), dtype, seed) for seed in range(4))
    gain, bias = randn((H,), dtype, 4), randn((H,), dtype, 5)
    ws = torch.empty(lib.dflare_norm_bwd_workspace(rows, H, 1), dtype=torch.uint8, device="cuda")

    def put(t, lead):
        buf = torch.full((t.numel() + lead + 9,), 7.0, dtype=dtype, device="cuda")
        buf[lead:lead + t.numel()] = t.reshape(-1)
        return buf, buf[lead:lead + t.numel()].view(t.shape)

    for kind in (dfl.NORM_RMS, dfl.NORM_LAYER):
        layer = kind == dfl.NORM_LAYER
        # (one operand at an odd place has the same kernel take the others wherever they are: the same bits)
        odd = [put(t, 1)[1] for t in (x, gain)]
        y, h, mean, rstd = dfl.norm_fwd(odd[0], odd[1], bias if layer else None, residual=r, kind=kind)
        dx, dgain, dbias = dfl.norm_bwd(dy, h, odd[1], mean, rstd, dsum=dsum, kind=kind)
        for lead in (0, 1, 3, 6):
            (bx, vx), (br, vr), (bg, vg), (bb, vb) = put(x, lead), put(r, lead + 1), put(gain, 1), put(bias, 1)
            m, s = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
            # sum over x, y over the residual
            assert lib.dflare_norm_fwd(vx.data_ptr(), vr.data_ptr(), vg.data_ptr(), vb.data_ptr() if layer else None, rows, H, code, kind,
                                       1e-6, vx.data_ptr(), vr.data_ptr(), m.data_ptr(), s.data_ptr(), st) == dfl.OK
            torch.cuda.synchronize()
            assert torch.equal(vx, h) and torch.equal(vr, y) and torch.equal(s, rstd) and (not layer or torch.equal(m, mean))
            assert bx[:lead].eq(7).all() and br[:lead + 1].eq(7).all() and bx[-9:].eq(7).all() and br[-9:].eq(7).all()
            for over in range(3):
                (b0, v0), (b1, v1), (b2, v2) = put(dy, lead), put(h, lead), put(dsum, lead)
                to, g = (v0, v1, v2)[over], torch.zeros(H, device="cuda")
                assert lib.dflare_norm_bwd(v0.data_ptr(), v1.data_ptr(), vg.data_ptr(), m.data_ptr() if layer else None, s.data_ptr(),
                                           v2.data_ptr(), rows, H, code, kind, to.data_ptr(), g.data_ptr(), None, ws.data_ptr(),
                                           ws.numel(), st) == dfl.OK
                torch.cuda.synchronize()
                assert torch.equal(to, dx) and torch.equal(g, dgain)
                for k, (b, v, t) in enumerate(((b0, v0, dy), (b1, v1, h), (b2, v2, dsum))):
                    assert b[:lead].eq(7).all() and b[-9:].eq(7).all() and (k == over or torch.equal(v, t))


# rows with a loss around 64 (n (B - 1) of them at most), on which the products' tile depends; the vocabulary in two pieces
@pytest.mark.parametrize("n,B,V,H", [(1, 64, 3000, 320), (1, 65, 3000, 320), (1, 66, 3000, 320), (13, 6, 40001, 72), (16, 5, 129, 2880),
                                     (1, 2, 70001, 1000), (1, 33, 12800, 4096), (1, 50, 1100000, 8), (32, 3, 127, 8)])
def test_linear_ce_of_few_rows(n, B, V, H):
    print(f"[train ops] linear ce of few rows {(n, B, V, H)}", flush=True)
    h, head, y = lce_inputs(n, B, V, H, seed=21, ignored=0.0)
    for dh, dw in ((False, False), (True, False), (False, True), (True, True)):
        got = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
        lce_check(h, head, y, B, 4.5, got)
        again = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
        assert all(u is v or torch.equal(u, v) for u, v in zip(got, again))


@pytest.mark.parametrize("n,B,V,H", [(100, 16, 3001, 264), (64, 17, 1000, 72), (65, 17, 1000, 72)])
def test_linear_ce_of_one_piece_and_many_rows(n, B, V, H):
    """Around 1,024 rows with a loss; plain, and with words that take a reference of their own."""
    h, head, y = lce_inputs(n, B, V, H, seed=31, ignored=0.0)
    for dh, dw in ((False, False), (True, False), (True, True)):
        lce_check(h, head, y, B, 4.5, dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw))
    h, head, y = lce_inputs(n, B, V, H, seed=32, lean=0.0)
    h[:, 0] = torch.where(torch.arange(n * B, device="cuda") % 3 == 0, 100.0, 0.0).to(BF)
    head[V // 3, 0], head[V - 1, 0] = 3.0, 5.0
    for dw in (False, True):
        lce_check(h, head, y, B, 4.5, dfl.linear_ce(h, head, y, B, 4.5, need_dhead=dw))


@pytest.mark.parametrize("n,B,V,H,ignored", [(200, 16, 300, 264, 0.0), (200, 16, 300, 264, 0.6), (512, 16, 1000, 1024, 0.0), (300, 9, 1, 8, 0.0),
                                             (64, 33, 777, 520, 0.3), (130, 16, 4000, 72, 0.0)])
def test_linear_ce_of_few_words_and_many_rows(n, B, V, H, ignored):
    """Many rows of every label: dhead's rows are split into parts."""
    print(f"[train ops] linear ce of few words {(n, B, V, H)}", flush=True)
    h, head, y = lce_inputs(n, B, V, H, seed=41, ignored=ignored)
    for dh in (False, True):
        got = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=True)
        lce_check(h, head, y, B, 4.5, got)
        again = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=True)
        assert all(u is v or torch.equal(u, v) for u, v in zip(got, again))


# ---- rows whose label takes all ----

def peaked_inputs(n, B, V, H, low, high, seed):
    """Label logits of low to high, those of the other words around zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    head = randn((V, H), seed=seed, std=0.02)
    y = torch.randint(0, V, (n * B,), generator=g, device="cuda", dtype=torch.int32)
    size = torch.empty((n * B, 1), device="cuda").uniform_(low, high, generator=g)
    word = head[y.long()].float()
    return (word * size / (word * word).sum(1, keepdim=True)).to(BF), head, y


def peaked_check(h, head, y, B, gamma, got):
    """As lce_check, but the error of 1 - p is relative to 1 - p and not to 1: cross-entropies and gradients far below 2^-24
    have correct digits too."""
    loss, ce, dh, dw = got
    rows, H = h.shape
    V = head.shape[0]
    b = torch.arange(rows, device="cuda") % B
    w = torch.where(b > 0, torch.exp(-(b - 1).double() / gamma), 0.0)
    c = (w / w.sum())[:, None]
    h64, w64, lab = torch.where(b[:, None] > 0, h.double(), 0.0), head.double(), y.long()[:, None]
    z = h64 @ w64.t()
    tz = float(2 * H * U * (h64.abs() @ w64.abs().t()).max() + 8 * U * z.abs().max())  # as in lce_check
    d = (z - z.gather(1, lab)).scatter_(1, lab, float("-inf"))
    del z
    rest = torch.logsumexp(d, 1, keepdim=True)  # log of (1 - p) / p
    total = torch.nn.functional.softplus(rest, threshold=700.0)
    want_ce = torch.where(b > 0, torch.log1p(rest.exp())[:, 0], 0.0)
    # sums of exponentials and their logarithm: a few units each, of values whose exponents are off by 2 tz
    rel = math.expm1(2 * tz) + 64 * U
    assert bool((ce >= 0).all())
    within(ce, want_ce, rel * want_ce + 1e-44, "row_ce")
    assert abs(float(loss) - float((c[:, 0] * want_ce).sum())) <= (rel + 2 * U) * float((c[:, 0] * want_ce).sum())
    dz = (d - total).exp_()
    del d
    dz.scatter_(1, lab, -(rest - total).exp())
    dz *= c
    edz = dz.abs() * (rel + HALF[BF]) + (V * 2 * U) * dz.abs()
    if dh is not None:
        want = dz @ w64
        within(dh, want, 1.01 * (edz @ w64.abs() + HALF[BF] * want.abs()) + 1e-37, "dhidden")
    if dw is not None:
        want = dz.t() @ h64
        edz += (HALF[BF] + rows * 2 * U) * dz.abs()
        within(dw, want, 1.01 * (edz.t() @ h64.abs() + HALF[BF] * want.abs()) + 1e-37, "dhead")


# one piece of the vocabulary, and two
@pytest.mark.parametrize("n,B,V,H,low,high", [(30, 11, 3333, 192, 25.0, 60.0), (5, 9, 700, 64, 30.0, 80.0), (256, 16, 70000, 64, 60.0, 75.0),
                                              (8, 5, 1, 64, 20.0, 40.0)])
def test_linear_ce_of_rows_whose_label_takes_all(n, B, V, H, low, high):
    print(f"[train ops] linear ce of peaked rows {(n, B, V, H)}", flush=True)
    h, head, y = peaked_inputs(n, B, V, H, low, high, seed=V)
    for dh, dw in ((False, False), (True, False), (False, True), (True, True)):
        peaked_check(h, head, y, B, 4.5, dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw))


@pytest.mark.parametrize("n,B,V,H", [(12, 16, 4099, 64), (256, 16, 70000, 64)])
def test_linear_ce_moved_references_round_nothing_again(n, B, V, H):
    """The label 20 or 60 powers of two below all other words: the others' gradients are the same sums, which in the second
    case are written against references that move.  Both differ by the rounding of exponents of about 20 (2^-20 of a
    value, which turns one value in 4,000 to the next bf16, so 2^-13.5 of a sum, and one output in 60 to its next one: 2^-10.8
    of the 2-norm at most); a second rounding of every value would add 2^-9.3 to each sum, 2^-9 with the outputs'."""
    g = torch.Generator(device="cuda").manual_seed(V)
    head = randn((V, H), seed=1, std=0.05)
    y = torch.randint(0, 40, (n * B,), generator=g, device="cuda", dtype=torch.int32)  # the first 40 words are the labels
    h = randn((n * B, H), seed=2, std=1.0 if V < 10000 else 0.05)  # (a sum of many words is mostly their common part otherwise)
    h[:, 0] = 16.0
    head[:, 0] = 0.0
    head[:40, 1:] = 0.0
    outs = []
    for below in (20.0, 60.0):
        head[:40, 0] = -below * math.log(2.0) / 16.0
        outs.append(dfl.linear_ce(h, head, y, B, 4.5)[2][:, 1:].double())
    on = torch.arange(n * B, device="cuda") % B > 0
    assert outs[0][on].abs().max() > 0
    assert float((outs[0] - outs[1]).norm()) <= 2.0 ** -10 * float(outs[0].norm())


@pytest.mark.parametrize("lean", [1.0, 40.0])
def test_linear_ce_of_many_pieces(lean):
    """Many rows of which few carry a loss, a vocabulary in 17 pieces (and, without gradients, in pieces of its parts' room): as the
    rows with a loss by themselves.  Then with words that move the references in some of the pieces."""
    B, V, H, m = 16, 1100000, 8, 128
    h, head, y = lce_inputs(256, B, V, H, seed=61, lean=lean)
    y[m:] = -1
    for words in ((), (7,), (40000, 300000, 1099999)):
        w = head.clone()
        for k, v in enumerate(words):
            w[v, 0] = 4.0 + 3.0 * k
            h[::3, 0] = 100.0
        for dh, dw in ((False, False), (True, False), (True, True)):
            loss, ce, gh, gw = dfl.linear_ce(h, w, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
            assert not ce[m:].any() and (gh is None or not gh[m:].any())
            lce_check(h[:m], w, y[:m], B, 4.5, (loss, ce[:m], None if gh is None else gh[:m], gw))


# ---- no word and no row of a product is lost ----

def near_in_norm(got, want, err, what):
    """Roundings that are independent of one another: the 2-norm of the difference against that of the values' errors `err`
    (elementwise, root mean square)."""
    off, most = float((got.double() - want).norm()), float(err.norm())
    assert off <= 1.1 * most, (what, off, most)


def sparse_inputs(rows, B, targets, V, H, seed):
    """Row r's probability is all on word targets[k] for the k-th row with a loss, its label another word; the last word of
    a stage, a part or a piece that is lost then changes dhidden of its row and dhead of its word by all of them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    head = torch.where(torch.rand((V, H), generator=g, device="cuda") < 0.5, 0.5, -0.5).to(BF)
    b = torch.arange(rows, device="cuda") % B
    on = torch.nonzero(b > 0)[:, 0]
    t = torch.full((rows,), -1, device="cuda")
    t[on] = targets[torch.arange(on.numel(), device="cuda") % targets.numel()]
    y = torch.where(b > 0, (t + V // 2) % V, 0).to(torch.int32)
    h = torch.where(t[:, None] >= 0, head[t.clamp_min(0)].float(), 0.0) * (600.0 / H)
    return h.to(BF), head, y


# targets: the first and the last word of every stage of 64 words, as many as there are rows, from a start that moves; on each of
# the tiles, with one piece of the vocabulary and two
@pytest.mark.parametrize("n,B,V,H,calls", [(23, 9, 32003, 264, 6), (5, 13, 3001, 512, 2), (40, 16, 5000, 328, 1), (256, 16, 70000, 256, 1),
                                           (1, 128, 1100000, 64, 3), (9, 8, 12801, 1024, 4), (200, 16, 300, 264, 1), (260, 16, 20011, 520, 1)])
def test_linear_ce_keeps_every_word_and_row(n, B, V, H, calls):
    ends = torch.arange(V, device="cuda")
    ends = ends[(ends % 64 == 0) | (ends % 64 == 63) | (ends == V - 1)]
    rows, m = n * B, n * (B - 1)
    for k in range(calls):
        print(f"[train ops] linear ce keeps words and rows {(n, B, V, H, k)}", flush=True)
        # the last words in every call, the others in turn (where they are too many: evenly spread)
        mine = torch.cat([ends[-4:], ends[(torch.arange(max(m - 4, 1), device="cuda") * max(1, ends.numel() // (m * calls)) + k * (m - 4)) % ends.numel()]])
        h, head, y = sparse_inputs(rows, B, mine, V, H, seed=k)
        for dw in (False, True):
            lce_check(h, head, y, B, 9.0, dfl.linear_ce(h, head, y, B, 9.0, need_dhead=dw))


@pytest.mark.parametrize("n,B,V,H,ignored", [(23, 9, 32003, 264, 0.1), (5, 13, 3001, 4096, 0.1), (256, 16, 70000, 64, 0.05), (17, 16, 1000, 512, 0.0),
                                             (512, 16, 1000, 1024, 0.0), (13, 6, 40001, 72, 0.0)])
def test_linear_ce_gradients_in_the_norm(n, B, V, H, ignored):
    """A rounding to bf16 is off by 2^-8 / sqrt(3) of the value in the root mean square, at most.  dhidden: those of dz and of the result;
    dhead: those of dz, of the scaled rows and of the result; the labels' terms are not rounded on the way."""
    h, head, y = lce_inputs(n, B, V, H, seed=51, ignored=ignored, lean=100.0 / H)
    _, _, dh, dw = dfl.linear_ce(h, head, y, B, 4.5, need_dhead=True)
    only = dfl.linear_ce(h, head, y, B, 4.5)[2]
    b = torch.arange(n * B, device="cuda") % B
    on = (b > 0) & (y >= 0) & (y < V)
    w = torch.where(on, torch.exp(-(b - 1).double() / 4.5), 0.0)
    h64, w64, lab = torch.where(on[:, None], h.double(), 0.0), head.double(), torch.where(on, y, 0).long()[:, None]
    dz = torch.softmax(h64 @ w64.t(), 1) * (w / w.sum())[:, None]
    square = (dz * dz).scatter_(1, lab, 0.0)
    dz.scatter_add_(1, lab, -(w / w.sum())[:, None])
    want, want_w = dz @ w64, dz.t() @ h64
    half = HALF[BF] / math.sqrt(3.0)
    for got in (dh, only):
        near_in_norm(got, want, half * (want * want + square @ (w64 * w64)).sqrt(), "dhidden")
    near_in_norm(dw, want_w, half * (want_w * want_w + 2 * (square.t() @ (h64 * h64))).sqrt(), "dhead")


@pytest.mark.parametrize("V,ignored", [(300, 0.3), (5000, 0.0)])
def test_linear_ce_of_large_rows_and_one_piece(V, ignored):
    """Gathered rows of more than 32 MB take dhead's scale where they lie."""
    n, B, H = 512, 16, 2568
    print(f"[train ops] linear ce of large rows {(n, B, V, H)}", flush=True)
    h, head, y = lce_inputs(n, B, V, H, seed=71, ignored=ignored)
    for dh in (False, True):
        got = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=True)
        lce_check(h, head, y, B, 4.5, got)
        again = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=True)
        assert all(u is v or torch.equal(u, v) for u, v in zip(got, again))


# ---- values that are not finite ----

@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_linear_ce_of_values_that_are_not_finite(bad):
    """NaN and infinities, in a row that takes part or in a word, on both forms of the call: the loss and the rows that they
    reach are NaN or infinite; the other rows' cross-entropies are as without them where a row holds them."""
    B = 8
    h, head, y = lce_inputs(40, B, 700, 128, seed=8, ignored=0.3)
    on = (torch.arange(h.shape[0], device="cuda") % B > 0) & (y >= 0) & (y < 700)
    row = int(torch.nonzero(on)[5])
    for dh, dw in ((False, False), (True, False), (False, True), (True, True)):
        clean = dfl.linear_ce(h, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
        x = h.clone()
        x[row, 17] = bad
        loss, ce, gh, gw = dfl.linear_ce(x, head, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
        rest = torch.arange(h.shape[0], device="cuda") != row
        assert not math.isfinite(float(loss)) and not math.isfinite(float(ce[row])) and torch.equal(ce[rest], clean[1][rest])
        if dh:
            assert gh[row].isnan().all() and torch.equal(gh[rest], clean[2][rest])
        if dw:  # every word has a share of the row
            assert not gw[:, 17].isfinite().any()
        w = head.clone()
        w[333, 5] = bad
        loss, ce, gh, gw = dfl.linear_ce(h, w, y, B, 4.5, need_dhidden=dh, need_dhead=dw)
        # the word's logit is NaN, or infinite with the sign of bad h: +inf and NaN reach the row's sum
        z = h[:, 5].float() * bad
        hit = on & ~(z == -float("inf"))
        assert not math.isfinite(float(loss)) and not ce[hit].isfinite().any() and torch.equal(ce[~on], torch.zeros_like(ce[~on]))
        if dh:
            assert not gh[on][:, 5].isfinite().any()
            assert not gh[hit].isfinite().any()


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_of_values_that_are_not_finite(layer, dtype):
    """A row with NaN is NaN, one with an infinity what the formula gives (RMSNorm: zeros beside the infinity); the other rows
    and their gradients are as without them, dgain and dbias are NaN where such a row reaches them."""
    kind = dfl.NORM_LAYER if layer else dfl.NORM_RMS
    x, dy = randn((12, 1000), dtype, 1), randn((12, 1000), dtype, 2)
    clean = dfl.norm_fwd(x, kind=kind)
    back = dfl.norm_bwd(dy, clean[1], None, clean[2], clean[3], kind=kind)
    bad = x.clone()
    bad[3, 7], bad[8, 999] = float("nan"), float("inf")
    y, h, mean, rstd = dfl.norm_fwd(bad, kind=kind)
    dx, dgain, _ = dfl.norm_bwd(dy, h, None, mean, rstd, kind=kind)
    rest = torch.tensor([k for k in range(12) if k not in (3, 8)], device="cuda")
    assert torch.equal(y[rest], clean[0][rest]) and torch.equal(rstd[rest], clean[3][rest]) and torch.equal(dx[rest], back[0][rest])
    assert y[3].isnan().all() and rstd[3].isnan() and dx[3].isnan().all() and y[8, 999].isnan()
    if layer:
        assert y[8].isnan().all() and dx[8].isnan().all()
    else:
        assert not y[8, :999].any() and rstd[8] == 0
    assert dgain.isnan().all()


@pytest.mark.parametrize("std,max_norm", [(1e37, 1.0), (5e36, 1e-20), (1e-20, 1e-42)])
def test_grad_clip_by_factors_below_the_normal_range(std, max_norm):
    """Finite gradients whose norm is beyond fp32 (the fp32 norm is infinite, the sum of squares is not), and bounds so small that
    max_norm / norm is below its normal range: the clipped values keep their digits."""
    grads = grads_of([5000, 6001, 77], std=std)
    _, sumsq = dfl.grad_norm(grads)
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert abs(math.sqrt(float(sumsq)) - want) <= 1e-12 * want
    coef = float(np.float32(max_norm)) / want
    out = [torch.empty_like(g) for g in grads]
    dfl.clip_grads(grads, sumsq, max_norm, out=out)
    for g, o in zip(grads, out):  # (bounds as in clip_check)
        least = 2.0 ** -126 * HALF[g.dtype]
        within(o, g.double() * coef, (HALF[g.dtype] + 3 * U) * g.double().abs() * coef + least, "clip")
    dfl.clip_grads(grads, sumsq, max_norm)
    assert all(torch.equal(g, o) for g, o in zip(grads, out))


@pytest.mark.parametrize("n,B,first,gamma", [(3, 700, 400, 2.0), (40, 4, 2, 0.01), (2, 1024, 900, 4.5), (300, 8, 7, 0.06), (40, 4, 1, 0.01)])
def test_linear_ce_of_late_positions(n, B, first, gamma):
    """The first positions of every block have no target, so that all weights lie below fp32: only their ratios count."""
    h, head, y = lce_inputs(n, B, 300, 64, seed=81, ignored=0.1)
    y[torch.arange(n * B, device="cuda") % B < first] = -1
    for dh, dw in ((False, False), (True, False), (True, True)):
        lce_check(h, head, y, B, gamma, dfl.linear_ce(h, head, y, B, gamma, need_dhidden=dh, need_dhead=dw))
