"""Operators of a draft layer's training step, around the anchor attention: cases, inputs, plain
forms and 64-bit results.

* ``lce``: the LM head with the position-weighted cross-entropy and its gradients, without logits
  in memory;
* ``rope``: rotary positions of queries and keys, forward and backward;
* ``norm``: RMSNorm and LayerNorm with a residual sum, forward and backward;
* ``clip``: the global norm of many gradient tensors, and their clipping.

The plain forms compute in 32 bits (angles and long sums in 64) with elementary tensor operations.
"""
import math

import torch

own = False

GAMMA = 4.5
EPS = 1e-6


def listed():
    return [
        # the training benchmark's 512 blocks of 16 positions against the 151,936-word head, which is frozen
        dict(name="lce_train", kind="lce", n_blocks=512, block=16, vocab=151936, hidden=4096, grads="hidden",
             ignored=0.05),
        # the largest vocabulary with a head that is trained too, few blocks, many positions without a target
        dict(name="lce_head", kind="lce", n_blocks=65, block=16, vocab=201088, hidden=2880, grads="both", ignored=0.3),
        # a small odd vocabulary and ragged blocks: launches and latency
        dict(name="lce_small", kind="lce", n_blocks=23, block=9, vocab=32003, hidden=264, grads="both", ignored=0.1),
        # queries and block keys of 512 anchored blocks, in one call
        dict(name="rope_blocks", kind="rope", rows=8192, block=16, n_q=32, n_kv=8, hd=128, rot=128, layout="half",
             dtype="bf16", inverse=False, method="none", factor=1.0, far=4096),
        # the gradient through a stretched context: interleaved pairs, half of each head, far positions, fp32
        dict(name="rope_far_grad", kind="rope", rows=4001, block=4001, n_q=16, n_kv=0, hd=128, rot=64,
             layout="interleaved", dtype="f32", inverse=True, method="yarn", factor=8.0, far=1000000),
        # one token of each of 32 sequences, 64-wide heads
        dict(name="rope_token", kind="rope", rows=32, block=1, n_q=64, n_kv=8, hd=64, rot=64, layout="half",
             dtype="bf16", inverse=False, method="linear", factor=4.0, far=8192),
        # the norm before a projection with the residual sum, 512 blocks, forward and backward
        dict(name="norm_train", kind="norm", rows=8192, hidden=4096, norm="rms", dtype="bf16", residual=True,
             backward=True),
        # LayerNorm in fp32 over odd rows
        dict(name="norm_layer_odd", kind="norm", rows=777, hidden=2881, norm="layer", dtype="f32", residual=False,
             backward=True),
        # the norm of one drafted block
        dict(name="norm_block", kind="norm", rows=16, hidden=2560, norm="rms", dtype="bf16", residual=True,
             backward=False),
        # the gradients of eight draft layers (Qwen3-8B shape), matrices in bf16 and norm gains in fp32
        dict(name="clip_layers", kind="clip", tensors=104, small=4096, large=50331648, max_norm=1.0),
        # many small ragged tensors: table and latency
        dict(name="clip_ragged", kind="clip", tensors=301, small=1, large=70001, max_norm=0.5),
    ]


def _log_int(rng, lo, hi):
    """Uniform over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lce", "lce", "rope", "norm", "clip"])
    if kind == "lce":
        grads = rng.choice(["none", "hidden", "hidden", "both"])
        V = rng.choice([151936, 201088, _log_int(rng, 1000, 200000)])
        H = rng.choice([4096, 2880, 2560, 8 * _log_int(rng, 8, 512)])
        block = rng.choice([16, rng.randint(2, 16)])
        most = 4.0 * 8192 * 151936 * 4096 / ({"none": 2, "hidden": 4, "both": 6}[grads] * V * H)
        most = min(8192, most, 1.2e9 / V)
        return dict(kind=kind, n_blocks=max(1, int(_log_int(rng, 16, most) / block)), block=block, vocab=V, hidden=H,
                    grads=grads, ignored=round(rng.uniform(0.0, 0.5), 2))
    if kind == "rope":
        hd = rng.choice([64, 128, 128, 96, 256])
        return dict(kind=kind, rows=_log_int(rng, 1, 8192), block=rng.choice([1, 16, rng.randint(2, 300)]),
                    n_q=rng.choice([8, 16, 32, 40, rng.randint(1, 40)]), n_kv=rng.choice([0, 8, rng.randint(1, 8)]),
                    hd=hd, rot=rng.choice([hd, hd, hd // 2]), layout=rng.choice(["half", "interleaved"]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), inverse=rng.random() < 0.4,
                    method=rng.choice(["none", "linear", "ntk", "yarn"]), factor=rng.choice([2.0, 4.0, 8.0]),
                    far=_log_int(rng, 10, 1000000))
    if kind == "norm":
        return dict(kind=kind, rows=_log_int(rng, 1, 8192), hidden=rng.choice([4096, 2880, 2560, 128, _log_int(rng, 30, 8192)]),
                    norm=rng.choice(["rms", "rms", "layer"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    residual=rng.random() < 0.5, backward=rng.random() < 0.6)
    large = _log_int(rng, 1000, 50000000)
    return dict(kind=kind, tensors=_log_int(rng, 1, max(2, min(400, int(6e9 / large)))), small=_log_int(rng, 1, 999),
                large=large, max_norm=round(math.exp(rng.uniform(-2.0, 2.0)), 3))


# ---- inputs ---------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(1000 * seed + salt)


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(shape, dtype, g, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def _lce_inputs(case, seed):
    """Head N(0, 0.02); each hidden row is N(0, 1) plus a share of its label's head row, so that the
    probability of the label runs from that of any other word to nearly one."""
    g = _gen(seed, 1)
    rows, V, H = case["n_blocks"] * case["block"], case["vocab"], case["hidden"]
    head = _normal((V, H), torch.bfloat16, g, 0.02)
    y = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lean = torch.rand((rows, 1), generator=g, device="cuda") * (1000.0 / H)
    h = (_normal((rows, H), torch.float32, g) + lean / 0.02 * head[y.long()].float()).to(torch.bfloat16)
    y[torch.rand(rows, generator=g, device="cuda") < case["ignored"]] = -1
    return h, head, y


def _frequencies(case):
    """(inverse frequencies, fp64 [rot / 2], factor on cos and sin)."""
    d, f, base = case["rot"], case["factor"], 1e6
    m = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    if case["method"] == "ntk" and d > 2:
        base *= f ** (d / (d - 2))
    freq = base ** (-2.0 * m / d)
    if case["method"] == "linear":
        freq = freq / f
    if case["method"] == "yarn":
        turns = case["far"] / f * freq / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return freq * (keep + (1.0 - keep) / f), 0.1 * math.log(f) + 1.0
    return freq, 1.0


def _rope_inputs(case, seed):
    g = _gen(seed, 2)
    rows, t = case["rows"], _TYPES[case["dtype"]]
    xs = [_normal((rows, n, case["hd"]), t, g) for n in (case["n_q"], case["n_kv"]) if n > 0]
    n_blocks = -(-rows // case["block"])
    pos = torch.randint(0, max(case["far"] - case["block"], 0) + 1, (n_blocks,), generator=g, device="cuda",
                        dtype=torch.int32)
    return xs, pos


def _norm_inputs(case, seed):
    g = _gen(seed, 3)
    shape, t = (case["rows"], case["hidden"]), _TYPES[case["dtype"]]
    x = _normal(shape, t, g, 2.0, 0.3)
    r = _normal(shape, t, g) if case["residual"] else None
    gain = _normal(shape[1:], t, g, 0.02, 1.0)
    bias = _normal(shape[1:], t, g, 0.02) if case["norm"] == "layer" else None
    dy = _normal(shape, t, g) if case["backward"] else None
    dsum = _normal(shape, t, g) if case["backward"] and case["residual"] else None
    return x, r, gain, bias, dy, dsum


def _clip_sizes(case):
    """Sizes spread over the logarithm of [small, large], none of them at random: (bf16 ones, fp32 ones)."""
    n, lo, hi = case["tensors"], math.log(case["small"]), math.log(case["large"])
    if case["small"] == 4096:  # layers: 13 tensors each, matrices of the draft layer, then its gains
        layer = [4096 * 4096] * 2 + [1024 * 4096] * 4 + [12288 * 4096] * 3
        return layer * (n // 13), [4096] * (4 * (n // 13))
    sizes = [int(round(math.exp(lo + (hi - lo) * (((7 * i + 3) % n) + 0.5) / n))) for i in range(n)]
    return sizes[0::2], sizes[1::2]


class _Grads:
    """Gradients as a program keeps them: tensors side by side in one buffer of each type."""

    def __init__(self, case, seed):
        g = _gen(seed, 4)
        self.max_norm = case["max_norm"]
        sizes = _clip_sizes(case)
        std = 3.0 * case["max_norm"] / math.sqrt(sum(map(sum, sizes)))
        self.flat = [_normal((sum(s),), t, g, std) for s, t in zip(sizes, (torch.bfloat16, torch.float32))]
        self.out_flat = [torch.empty_like(x) for x in self.flat]
        self.grads = [v for x, s in zip(self.flat, sizes) for v in x.split(s)]
        self.out = [v for x, s in zip(self.out_flat, sizes) for v in x.split(s)]


def prepare(case, seed):
    kind = case["kind"]
    if kind == "lce":
        return kind, case, _lce_inputs(case, seed)
    if kind == "rope":
        return kind, case, (*_rope_inputs(case, seed), *_frequencies(case))
    if kind == "norm":
        return kind, case, _norm_inputs(case, seed)
    return kind, case, _Grads(case, seed)


# ---- one pass ---------------------------------------------------------------------------------

def run(state):
    kind, case, x = state
    return {"lce": _lce, "rope": _rope, "norm": _norm, "clip": _clip}[kind](case, x)


def _lce(case, x):
    h, head, y = x
    B, grads = case["block"], case["grads"]
    if own:
        from paper_2606_02091_amd import dflare as dfl
        loss, ce, dh, dhead = dfl.linear_ce(h, head, y, B, GAMMA, need_dhidden=grads != "none",
                                            need_dhead=grads == "both")
        return [loss, ce] + [t for t in (dh, dhead) if t is not None]
    rows = h.shape[0]
    r = torch.arange(rows, device=h.device)
    b = r % B
    on = (b > 0) & (y >= 0)
    w = torch.exp(-(b - 1).float() / GAMMA) * on
    c = w / w.double().sum().clamp_min(1e-300)
    label = y.clamp_min(0).long()
    hf, wf = h.float(), head.float()
    z = hf @ wf.t()
    z -= z.amax(1, keepdim=True)
    zy = z[r, label]
    p = z.exp_()
    s = p.sum(1, keepdim=True)
    ce = torch.where(on, torch.log(s[:, 0]) - zy, 0.0)
    outs = [(c * ce.double()).sum().float().view(1), ce]
    if grads != "none":
        dz = p.mul_((c / s[:, 0]).float()[:, None])
        dz[r, label] -= c.float()
        outs.append((dz @ wf).to(h.dtype))
        if grads == "both":
            outs.append((dz.t() @ hf).to(head.dtype))
    return outs


def _rope(case, x):
    xs, pos, freq, scale = x
    if own:
        from paper_2606_02091_amd import dflare as dfl
        layout = dfl.ROPE_HALF if case["layout"] == "half" else dfl.ROPE_INTERLEAVED
        return list(dfl.rope(tuple(xs), freq, pos, B=case["block"], layout=layout, scale=scale,
                             inverse=case["inverse"]))
    B, rot = case["block"], case["rot"]
    r = torch.arange(case["rows"], device=pos.device)
    th = (pos[r // B].double() + r % B)[:, None] * freq
    if case["inverse"]:
        th = -th
    c, s = (torch.cos(th) * scale).float()[:, None], (torch.sin(th) * scale).float()[:, None]
    half = case["layout"] == "half"
    outs = []
    for t in xs:
        u = t[..., :rot].float()
        a, b = (u[..., :rot // 2], u[..., rot // 2:]) if half else (u[..., 0::2], u[..., 1::2])
        pair = (a * c - b * s, b * c + a * s)
        u = torch.cat(pair, -1) if half else torch.stack(pair, -1).flatten(-2)
        outs.append(torch.cat([u.to(t.dtype), t[..., rot:]], -1))
    return outs


def _norm(case, x):
    x, r, gain, bias, dy, dsum = x
    layer = case["norm"] == "layer"
    if own:
        from paper_2606_02091_amd import dflare as dfl
        kind = dfl.NORM_LAYER if layer else dfl.NORM_RMS
        y, h, mean, rstd = dfl.norm_fwd(x, gain, bias, residual=r, kind=kind, eps=EPS)
        outs = [y, rstd] + ([h] if r is not None else []) + ([mean] if layer else [])
        if dy is not None:
            dx, dgain, dbias = dfl.norm_bwd(dy, h, gain, mean, rstd, dsum=dsum, kind=kind)
            outs += [dx, dgain] + ([dbias] if layer else [])
        return outs
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    u = h.float()
    if layer:
        mean = u.mean(1, keepdim=True)
        u = u - mean
    rstd = torch.rsqrt((u * u).mean(1, keepdim=True) + EPS)
    xh = u * rstd
    y = xh * gain.float()
    if layer:
        y = y + bias.float()
    outs = [y.to(x.dtype), rstd[:, 0]] + ([h] if r is not None else []) + ([mean[:, 0]] if layer else [])
    if dy is not None:
        d = dy.float()
        e = d * gain.float()
        dx = e - xh * (e * xh).mean(1, keepdim=True)
        if layer:
            dx = dx - e.mean(1, keepdim=True)
        dx = dx * rstd
        if dsum is not None:
            dx = dx + dsum.float()
        outs += [dx.to(x.dtype), (d * xh).double().sum(0).float()]
        if layer:
            outs.append(d.double().sum(0).float())
    return outs


def _clip(case, x):
    if own:
        from paper_2606_02091_amd import dflare as dfl
        norm, sumsq = dfl.grad_norm(x.grads)
        dfl.clip_grads(x.grads, sumsq, x.max_norm, out=x.out)
        return [norm, *x.out_flat]
    f = [t.float() for t in x.flat]
    norm = torch.sqrt((f[0] * f[0]).sum(dtype=torch.float64) + (f[1] * f[1]).sum(dtype=torch.float64))
    coef = torch.where(norm > x.max_norm, x.max_norm / norm, 1.0).float()
    x.out_flat[0].copy_(f[0] * coef)
    x.out_flat[1].copy_(f[1] * coef)
    return [norm.float().view(1), *x.out_flat]


# ---- work -----------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "lce":
        rows, V, H = case["n_blocks"] * case["block"], case["vocab"], case["hidden"]
        products = {"none": 1, "hidden": 2, "both": 3}[case["grads"]]
        moved = 2 * (rows + V) * H + 8 * rows
        moved += (2 * rows * H if products > 1 else 0) + (2 * V * H if products > 2 else 0)
        return {"bytes": moved, "flops": 2 * products * rows * V * H}
    if kind == "rope":
        n = case["rows"] * (case["n_q"] + case["n_kv"]) * case["hd"]
        return {"bytes": 2 * n * (2 if case["dtype"] == "bf16" else 4) + 4 * -(-case["rows"] // case["block"]),
                "flops": 3 * n}
    if kind == "norm":
        n, size = case["rows"] * case["hidden"], 2 if case["dtype"] == "bf16" else 4
        passes = 2 + 2 * case["residual"] + case["backward"] * (2 + case["residual"])
        return {"bytes": passes * n * size + 8 * case["rows"] + 16 * case["hidden"],
                "flops": (5 + 10 * case["backward"]) * n}
    a, b = map(sum, _clip_sizes(case))
    return {"bytes": 2 * (2 * a + 4 * b), "flops": 3 * (a + b)}


# ---- 64-bit results ---------------------------------------------------------------------------

def _exact_lce(case, seed):
    h, head, y = _lce_inputs(case, seed)
    rows, V = h.shape[0], head.shape[0]
    w64 = head.double()
    b = torch.arange(rows, device="cuda") % case["block"]
    on = (b >= 1) & (y >= 0)
    w = torch.where(on, torch.exp((1.0 - b.double()) / GAMMA), 0.0)
    c = w / max(float(w.sum()), 1e-300)
    ce = torch.zeros(rows, dtype=torch.float64, device="cuda")
    dh = torch.empty(h.shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w64) if case["grads"] == "both" else None
    step = max(1, int(2e8 / V))
    for s in range(0, rows, step):
        x = h[s:s + step].double()
        z = x @ w64.t()
        i, lab = torch.arange(z.shape[0], device="cuda"), y[s:s + step].clamp_min(0).long()
        lse = torch.logsumexp(z, 1)
        ce[s:s + step] = torch.where(on[s:s + step], lse - z[i, lab], 0.0)
        if case["grads"] == "none":
            continue
        dz = torch.exp(z - lse[:, None])
        dz[i, lab] -= 1.0
        dz *= c[s:s + step, None]
        dh[s:s + step] = dz @ w64
        if dw is not None:
            dw += dz.t() @ x
    outs = [(c * ce).sum().view(1), ce]
    return outs + ([dh] if case["grads"] != "none" else []) + ([dw] if dw is not None else [])


def _exact_rope(case, seed):
    xs, pos = _rope_inputs(case, seed)
    freq, scale = _frequencies(case)
    rot, B = case["rot"], case["block"]
    at = torch.tensor([k % B for k in range(case["rows"])], device="cuda") \
        + pos.long().repeat_interleave(B)[:case["rows"]]
    turn = torch.polar(torch.full_like(freq, scale).expand(case["rows"], -1), at.double()[:, None] * freq)[:, None]
    if case["inverse"]:
        turn = turn.conj()
    outs = []
    for t in xs:
        u = t.double()
        v = u.clone()
        pairs = u[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" \
            else u[..., :rot].unflatten(-1, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        v[..., :rot] = z.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else z.flatten(-2)
        outs.append(v)
    return outs


def _exact_norm(case, seed):
    x, r, gain, bias, dy, dsum = _norm_inputs(case, seed)
    layer = case["norm"] == "layer"
    total = x.double() if r is None else x.double() + r.double()
    h = total if r is None else total.to(x.dtype).double()  # the norm is that of the stored sum
    mu = h.sum(1, keepdim=True) / h.shape[1] if layer else torch.zeros_like(h[:, :1])
    dev = h - mu
    var = dev.square().sum(1, keepdim=True) / h.shape[1]
    inv = 1.0 / torch.sqrt(var + EPS)
    n = dev * inv
    y = n * gain.double() + (bias.double() if layer else 0.0)
    outs = [y, inv.squeeze(1)] + ([total] if r is not None else []) + ([mu.squeeze(1)] if layer else [])
    if dy is not None:
        d = dy.double()
        dn = d * gain.double()
        # the derivative of dev * inv: through dev, and through the variance
        dvar = (dn * dev).sum(1, keepdim=True) * (-0.5) * inv ** 3
        ddev = dn * inv + dvar * 2.0 * dev / h.shape[1]
        dx = ddev - (ddev.sum(1, keepdim=True) / h.shape[1] if layer else 0.0)
        outs += [dx + (0.0 if dsum is None else dsum.double()), (d * n).sum(0)]
        if layer:
            outs.append(d.sum(0))
    return outs


def _exact_clip(case, seed):
    x = _Grads(case, seed)
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in x.flat))
    factor = min(1.0, x.max_norm / norm) if norm else 1.0
    return [torch.tensor([norm], dtype=torch.float64, device="cuda"), *[t.double() * factor for t in x.flat]]


def exact(case, seed):
    with torch.no_grad():
        return {"lce": _exact_lce, "rope": _exact_rope, "norm": _exact_norm, "clip": _exact_clip}[case["kind"]](
            case, seed)
