"""Measured operators around the blocks of a fine-tuning step on packed rows.

Beside its products and its attention, such a step passes every row through

  dropout  dropout from a counter-based generator: the mask is never stored, the backward
           is the same call on the gradient
  norm     the boundary of two sublayers in one pass: norm of the branch, dropout, gate and
           scales, residual add, norm for the next sublayer; its backward with the gradients
           of gains, shifts and gate
  loss     the head's product with softmax cross entropy over the whole vocabulary and its
           gradients, without keeping the logits; without gradients it scores tokens

Where `own` is false, `run` computes them with elementary torch operations.
"""

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # one image's rows (16 x 16 patches and the class token): launch latency
        dict(op="dropout", name="drop_image", rows=257, cols=1280, spare=0, p=0.1, dtype="bf16"),
        # the hidden rows of the widest MLP in training
        dict(op="dropout", name="drop_mlp", rows=8192, cols=16384, spare=0, p=0.1, dtype="bf16"),
        # fp32 gradients, odd rows inside a wider buffer
        dict(op="dropout", name="drop_f32_odd", rows=20011, cols=1021, spare=3, p=0.35, dtype="fp32"),
        # a single token between two sublayers
        dict(op="norm", name="norm_token", rows=1, d=4096, stream="fp32", pre="rms", post="", shift=False, gate=False,
             alpha=1.0, beta=1.0, p=0.0, back=False),
        # backward of images' rows: layer norm, a gate for each channel, dropout, a residual stream in 16 bits
        dict(op="norm", name="norm_image_bwd", rows=16448, d=1280, stream="bf16", pre="layer", post="", shift=True, gate=True,
             alpha=1.0, beta=1.0, p=0.1, back=True),
        # text rows of the widest model, norms before and after the sublayer
        dict(op="norm", name="norm_text", rows=16384, d=4096, stream="fp32", pre="rms", post="rms", shift=False, gate=False,
             alpha=1.0, beta=0.5, p=0.1, back=False),
        # everything at once, backward
        dict(op="norm", name="norm_text_bwd", rows=16384, d=4096, stream="fp32", pre="layer", post="layer", shift=True,
             gate=True, alpha=0.9, beta=0.5, p=0.1, back=True),
        # the smallest task of a sweep
        dict(op="loss", name="loss_tiny", rows=64, d=64, vocab=512, pad=0, bias=False, ignored=0.0, weights=False, train=True),
        # the next token of eight sequences scored
        dict(op="loss", name="loss_score", rows=8, d=1024, vocab=50257, pad=0, bias=False, ignored=0.0, weights=False, train=False),
        # a small model on full rows of text, a vocabulary of odd size
        dict(op="loss", name="loss_text", rows=8192, d=768, vocab=50257, pad=0, bias=False, ignored=0.0, weights=False, train=True),
        # answers behind prompts that are not learned, weighted rows, a vocabulary filled up with entries that never win
        dict(op="loss", name="loss_answers", rows=8161, d=1024, vocab=50304, pad=47, bias=True, ignored=0.55, weights=True, train=True),
        # the widest model
        dict(op="loss", name="loss_wide", rows=4096, d=4096, vocab=50400, pad=0, bias=True, ignored=0.0, weights=False, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["dropout", "norm", "norm", "loss", "loss"])
    if op == "dropout":
        cols = _log_int(rng, 1, 16384)
        if rng.random() < 0.6:
            cols = 8 * max(1, cols // 8)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        return dict(op="dropout", rows=_log_int(rng, 1, min(65536, (1 << 26 if dtype == "bf16" else 1 << 25) // cols)), cols=cols,
                    spare=rng.choice([0, 0, 1, 8, 64]), p=rng.choice([0.0, 0.05, 0.1, 0.5, round(rng.random(), 3)]), dtype=dtype)
    if op == "norm":
        d = _log_int(rng, 16, 8192)
        if rng.random() < 0.8:
            d = 8 * max(1, d // 8)
        post = rng.choice(["", "rms", "layer"])
        return dict(op="norm", rows=_log_int(rng, 1, min(32768, (1 << 26) // d)), d=d, stream=rng.choice(["fp32", "bf16"]),
                    pre=rng.choice(["rms", "layer", "rms", "layer", ""]), post=post, shift=rng.random() < 0.5, gate=rng.random() < 0.5,
                    alpha=rng.choice([1.0, 1.0, 0.7]), beta=rng.choice([1.0, 0.25]), p=rng.choice([0.0, 0.1, 0.3]), back=rng.random() < 0.6)
    d = 8 * _log_int(rng, 4, 512)
    vocab = _log_int(rng, 2, 65000)
    rows = _log_int(rng, 1, min(16384, (1 << 39) // (d * vocab), (1 << 29) // vocab))
    return dict(op="loss", rows=rows, d=d, vocab=vocab, pad=rng.choice([0, 0, vocab // 40]), bias=rng.random() < 0.5,
                ignored=rng.choice([0.0, 0.0, 0.3, round(rng.random(), 2)]), weights=rng.random() < 0.4, train=rng.random() < 0.75)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _counter(case, seed):
    """The generator's key and the step that it is at, as a training loop keeps them."""
    return dict(key=0x9E3779B97F4A7C15 * (seed + 1) % (1 << 64), step=torch.tensor([seed % 1000 + (3 << 32)], dtype=torch.int64, device=DEV))


def prepare(case, seed):
    return {"dropout": _prepare_dropout, "norm": _prepare_norm, "loss": _prepare_loss}[case["op"]](case, seed)


def _prepare_dropout(case, seed):
    g = _gen(seed)
    dt, R, C, W = _dtype(case["dtype"]), case["rows"], case["cols"], case["cols"] + case["spare"]
    return dict(case=case, x=_randn(g, R, W).to(dt)[:, :C], y=torch.zeros(R, W, device=DEV, dtype=dt)[:, :C], **_counter(case, seed))


def _prepare_norm(case, seed):
    g = _gen(seed)
    T, d, dt = case["rows"], case["d"], _dtype(case["stream"])
    gain = lambda: 1 + 0.2 * _randn(g, d)  # noqa: E731
    s = dict(case=case, f=_randn(g, T, d).to(torch.bfloat16), **_counter(case, seed))
    s["gate"] = 0.5 * _randn(g, d) if case["gate"] else None
    for n in ("pre", "post"):
        s["g_" + n] = gain() if case[n] else None
        s["b_" + n] = 0.1 * _randn(g, d) if case[n] == "layer" and case["shift"] else None
    s["stats"] = torch.zeros(4, T, device=DEV)
    # a stream of several blocks: channels of different sizes, a mean of its own in each row
    stream = (2 * _randn(g, T, d) * torch.exp(0.5 * _randn(g, d)) + 0.3 * _randn(g, T, 1)).to(dt)
    if not case["back"]:
        s.update(x=stream, y=torch.zeros_like(stream), h=torch.zeros(T, d, device=DEV, dtype=torch.bfloat16) if case["pre"] else None)
        return s
    # the backward finds what the forward kept: its sum, the branch, and the norms' statistics
    s.update(y=stream, dy=(1e-3 * _randn(g, T, d)).to(dt), dx=torch.zeros_like(stream), df=torch.zeros_like(s["f"]),
             dh=(1e-3 * _randn(g, T, d)).to(torch.bfloat16) if case["pre"] else None)
    for i, (n, a) in enumerate((("post", s["f"]), ("pre", s["y"]))):
        if case[n]:
            mean, rstd, _ = _stats(a.double(), case[n])
            s["stats"][2 * i], s["stats"][2 * i + 1] = mean[:, 0].float(), rstd[:, 0].float()
    grads = dict(dgate=case["gate"], dg_pre=case["pre"], db_pre=s["b_pre"] is not None, dg_post=case["post"],
                 db_post=s["b_post"] is not None)
    s["grads"] = {n: torch.zeros(d, device=DEV) for n, on in grads.items() if on}
    return s


def _labelled(case):
    return case["rows"] - int(case["rows"] * case["ignored"])


def _prepare_loss(case, seed):
    g = _gen(seed)
    N, d, V, bf = case["rows"], case["d"], case["vocab"], torch.bfloat16
    w = _randn(g, V, d) / math.sqrt(d)
    # tokens are as frequent as words: the n-th most frequent one about n times as rare as the first
    live = V - case["pad"]
    labels = (torch.exp(torch.rand(N, device=DEV, generator=g) * math.log(live + 1)) - 1).long().clamp(0, live - 1)
    labels = torch.randperm(live, device=DEV, generator=g)[labels]
    # rows that see their token coming, more or less clearly
    x = 1.5 * _randn(g, N, d) + w[labels] * (16 * torch.rand(N, 1, device=DEV, generator=g) ** 2)
    n = N - _labelled(case)
    for i in range(8):  # prompts: the first rows of each of eight sequences
        labels[i * N // 8:i * N // 8 + (i + 1) * n // 8 - i * n // 8] = -1
    s = dict(case=case, x=x.to(bf), w=w.to(bf), labels=labels.to(torch.int32), loss=torch.zeros(N, device=DEV), lse=torch.zeros(N, device=DEV),
             inv_n=torch.zeros(1, device=DEV), bias=None, weight=None, dx=None, dw=None, db=None)
    if case["bias"]:
        s["bias"] = 0.5 * _randn(g, V)
        s["bias"][live:] = -math.inf
    if case["weights"]:
        s["weight"] = torch.rand(N, device=DEV, generator=g) / N
    if case["train"]:
        s.update(dx=torch.zeros_like(s["x"]), dw=torch.zeros_like(s["w"]), db=torch.zeros(V, device=DEV, dtype=bf) if case["bias"] else None)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return {"dropout": _run_dropout, "norm": _run_norm, "loss": _run_loss}[s["case"]["op"]](s)


def _mul(a, b):
    """High and low 32 bits of a b, of int64 tensors that hold 32 bits and a number of 32 bits."""
    lo, hi = a * (b & 0xFFFF), a * (b >> 16)
    lo, hi = (lo & 0xFFFF) + ((hi + (lo >> 16) & 0xFFFF) << 16), hi + (lo >> 16) >> 16
    return hi, lo


def _kept(rows, cols, p, key, step):
    """(mask [rows, cols], factor) of dropout: Philox4x32-10 of (column / 8, row, step), 16 bits of it for each column."""
    t = round(65536 * p)
    k0, k1, step = key & 0xFFFFFFFF, key >> 32, step[0]
    c = [torch.arange(-(-cols // 8), device=DEV)[None, :], torch.arange(rows, device=DEV)[:, None], step & 0xFFFFFFFF, step >> 32]
    for _ in range(10):
        h0, l0 = _mul(c[0], 0xD2511F53)
        h1, l1 = _mul(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    r = torch.stack([x for word in c for x in (word & 0xFFFF, word >> 16)], -1).reshape(rows, -1)[:, :cols]
    return r >= t, 65536 / (65536 - t) if t < 65536 else 0.0


def _run_dropout(s):
    c = s["case"]
    if own:
        from paper_2309_01226_amd import ops
        return ops.dropout(s["x"], c["p"], s["key"], step=s["step"], out=s["y"])
    keep, up = _kept(c["rows"], c["cols"], c["p"], s["key"], s["step"])
    s["y"].copy_(torch.where(keep, s["x"].float() * up, 0.0))
    return s["y"]


def _stats(a, kind):
    """Mean (0 for rms) and reciprocal deviation of every row, and the rows normalised by them."""
    mean = a.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(a[:, :1])
    a = a - mean
    rstd = 1 / torch.sqrt((a * a).mean(1, keepdim=True) + EPS)
    return mean, rstd, a * rstd


def _shifted(a, gain, shift):
    return a * gain if shift is None else a * gain + shift


def _norm_back(g, xh, rstd, gain, kind):
    """Gradient of a norm's rows from the gradient g of its outcome."""
    a = g * gain
    b = a - xh * (a * xh).mean(1, keepdim=True)
    return rstd * (b - a.mean(1, keepdim=True) if kind == "layer" else b)


def _run_norm(s):
    c = s["case"]
    opts = dict(pre=c["pre"] or None, post=c["post"] or None, g_pre=s["g_pre"], b_pre=s["b_pre"], g_post=s["g_post"],
                b_post=s["b_post"], gate=s["gate"], alpha=c["alpha"], beta=c["beta"], eps=EPS, p=c["p"], seed=s["key"], step=s["step"])
    if own:
        from paper_2309_01226_amd import ops
        if not c["back"]:
            ops.residual_norm_fwd(s["x"], s["f"], s["y"], s["h"], s["stats"], c["d"], **opts)
            return s["y"], s["h"], s["stats"]
        ops.residual_norm_bwd(s["dy"], s["dh"], s["y"], s["f"], s["stats"], s["dx"], s["df"], c["d"], **s["grads"], **opts)
        return s["dx"], s["df"], s["grads"]
    m = 1.0
    if c["p"] > 0:
        keep, up = _kept(c["rows"], c["d"], c["p"], s["key"], s["step"])
        m = torch.where(keep, up, 0.0).float()
    m = m * c["beta"]
    f, st = s["f"].float(), s["stats"][:, :, None]
    gate = 1.0 if s["gate"] is None else s["gate"]
    if not c["back"]:
        u = f
        if c["post"]:
            st[0], st[1], u = _stats(f, c["post"])
            u = _shifted(u, s["g_post"], s["b_post"])
        s["y"].copy_(c["alpha"] * s["x"].float() + gate * m * u)
        if c["pre"]:
            st[2], st[3], h = _stats(s["y"].float(), c["pre"])
            s["h"].copy_(_shifted(h, s["g_pre"], s["b_pre"]))
        return s["y"], s["h"], s["stats"]
    t, grads = s["dy"].float(), s["grads"]
    if c["pre"]:
        yh, dh = (s["y"].float() - st[2]) * st[3], s["dh"].float()
        t = t + _norm_back(dh, yh, st[3], s["g_pre"], c["pre"])
        grads["dg_pre"].copy_((dh * yh).sum(0))
        if "db_pre" in grads:
            grads["db_pre"].copy_(dh.sum(0))
    s["dx"].copy_(c["alpha"] * t)
    u = fh = (f - st[0]) * st[1] if c["post"] else f
    if c["post"]:
        u = _shifted(fh, s["g_post"], s["b_post"])
    if c["gate"]:
        grads["dgate"].copy_((t * m * u).sum(0))
    du = t * m * gate
    if c["post"]:
        grads["dg_post"].copy_((du * fh).sum(0))
        if "db_post" in grads:
            grads["db_post"].copy_(du.sum(0))
        du = _norm_back(du, fh, st[1], s["g_post"], c["post"])
    s["df"].copy_(du)
    return s["dx"], s["df"], grads


def _run_loss(s):
    c = s["case"]
    if own:
        from paper_2309_01226_amd import ops
        ops.linear_cross_entropy(s["x"], s["w"], s["labels"], s["loss"], s["lse"], s["inv_n"], bias=s["bias"], row_weight=s["weight"],
                                 dx=s["dx"], dw=s["dw"], db=s["db"])
    else:
        x, w = s["x"].float(), s["w"].float()
        live = s["labels"] >= 0
        at = torch.where(live, s["labels"], 0).long()[:, None]
        z = x @ w.T
        if c["bias"]:
            z += s["bias"]
        top = z.amax(1, keepdim=True)
        label = z.gather(1, at) - top
        total = z.sub_(top).exp_().sum(1, keepdim=True)
        log = torch.log(total)
        s["lse"].copy_(torch.where(live, (top + log)[:, 0], 0.0))
        s["loss"].copy_(torch.where(live, (log - label)[:, 0], 0.0))
        s["inv_n"].copy_(1 / live.sum().clamp(min=1))
        if c["train"]:
            row = (s["inv_n"] if s["weight"] is None else s["weight"]) * live
            dz = z.mul_((row / total[:, 0])[:, None])
            dz.scatter_add_(1, at, -row[:, None])
            s["dx"].copy_(dz @ w)
            s["dw"].copy_(dz.T @ x)
            if c["bias"]:
                s["db"].copy_(dz.sum(0))
    return s["loss"], s["lse"], s["inv_n"], s["dx"], s["dw"], s["db"]


def work(case):
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * (2 if case["dtype"] == "bf16" else 4), "flops": 2 * n}
    if case["op"] == "norm":
        n, e, pre = case["rows"] * case["d"], 2 if case["stream"] == "bf16" else 4, bool(case["pre"])
        # sums of a gate or a norm behind the branch need the branch again
        branch = bool(case["gate"] or case["post"])
        moved = n * (2 * e + 2 + 2 * pre if not case["back"] else (2 + pre) * e + 2 * pre + 2 * branch + 2)
        return {"bytes": moved, "flops": n * (30 if case["back"] else 15)}
    # rows without a label need nothing but zeros in their gradient
    N, n, d, V, t = case["rows"], _labelled(case), case["d"], case["vocab"], case["train"]
    return {"bytes": 2 * (V * d * (1 + t) + n * d + t * N * d) + 12 * N + case["bias"] * (4 + 2 * t) * V, "flops": 2 * n * V * d * (3 if t else 1)}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "norm": _exact_norm, "loss": _exact_loss}[case["op"]](s, case)


def _factors(s, rows, cols, p):
    """[rows, cols] of 0 or 1 / (1 - p): the generator in halves of 32 bits, a column of eight at a time."""
    t = round(65536 * p)
    step = int(s["step"][0])
    out = torch.zeros(rows, cols, device=DEV, dtype=torch.float64)
    if t >= 65536:
        return out

    def times(a, m):
        """a m by its four products of 16 bits."""
        a0, a1, m0, m1 = a % 65536, a // 65536, m % 65536, m // 65536
        mid = a1 * m0 + a0 * m1 + a0 * m0 // 65536
        return a1 * m1 + mid // 65536, mid % 65536 * 65536 + a0 * m0 % 65536

    n = -(-cols // 8)
    a = torch.arange(n, device=DEV).repeat(rows)
    b = torch.repeat_interleave(torch.arange(rows, device=DEV), n)
    c, d = torch.full_like(a, step % (1 << 32)), torch.full_like(a, step // (1 << 32))
    for i in range(10):
        ka, kb = (s["key"] % (1 << 32) + i * 0x9E3779B9) % (1 << 32), (s["key"] // (1 << 32) + i * 0xBB67AE85) % (1 << 32)
        (p1, p0), (q1, q0) = times(a, 0xD2511F53), times(c, 0xCD9E8D57)
        a, b, c, d = torch.bitwise_xor(torch.bitwise_xor(q1, b), ka), q0, torch.bitwise_xor(torch.bitwise_xor(p1, d), kb), p0
    for e in range(8):
        word = (a, b, c, d)[e // 2]
        half = (word // 65536 if e % 2 else word % 65536).reshape(rows, n)
        at = out[:, e::8]
        at.copy_(torch.where(half < t, 0.0, 1 / (1 - t / 65536))[:, :at.shape[1]])
    return out


def _exact_dropout(s, case):
    return s["x"].double() * _factors(s, case["rows"], case["cols"], case["p"])


def _exact_norm(s, case):
    """Gradients by automatic differentiation, from the values that the backward is given."""
    T, d = case["rows"], case["d"]
    d64 = lambda t: None if t is None else t.double()  # noqa: E731
    leaf = lambda t: None if t is None else t.double().requires_grad_()  # noqa: E731

    def norm(a, kind, gain, shift):
        if not kind:
            return a, None, None
        mean = a.sum(1) / d if kind == "layer" else torch.zeros(T, device=DEV, dtype=torch.float64)
        var = (a - mean[:, None]).square().sum(1) / d
        rstd = (var + EPS) ** -0.5
        out = (a - mean[:, None]) * rstd[:, None] * gain
        return out if shift is None else out + shift, mean, rstd

    mask = _factors(s, T, d, case["p"]) if case["p"] else torch.ones(1, device=DEV, dtype=torch.float64)
    if not case["back"]:
        stats = torch.zeros(4, T, device=DEV, dtype=torch.float64)
        u, m, r = norm(s["f"].double(), case["post"], d64(s["g_post"]), d64(s["b_post"]))
        if case["post"]:
            stats[0], stats[1] = m, r
        y = case["alpha"] * s["x"].double() + case["beta"] * mask * (u if s["gate"] is None else u * s["gate"].double())
        h = None
        if case["pre"]:
            h, stats[2], stats[3] = norm(y.to(s["x"].dtype).double(), case["pre"], d64(s["g_pre"]), d64(s["b_pre"]))
        return y, h, stats
    y, f = leaf(s["y"]), leaf(s["f"])
    p = {n: leaf(s[n]) for n in ("gate", "g_pre", "b_pre", "g_post", "b_post")}
    t = s["dy"].double()
    h, _, _ = norm(y, case["pre"], p["g_pre"], p["b_pre"])
    names = [n for n in ("g_pre", "b_pre") if p[n] is not None]
    out = {}
    if case["pre"]:
        got = torch.autograd.grad(h, [y] + [p[n] for n in names], s["dh"].double())
        t = t + got[0]
        out.update({"d" + n: v for n, v in zip(names, got[1:])})
    u, _, _ = norm(f, case["post"], p["g_post"], p["b_post"])
    branch = case["beta"] * mask * (u if p["gate"] is None else u * p["gate"])
    names = [n for n in ("gate", "g_post", "b_post") if p[n] is not None]
    got = torch.autograd.grad(branch, [f] + [p[n] for n in names], t)
    out.update({"d" + n: v for n, v in zip(names, got[1:])})
    return case["alpha"] * t, got[0], {n: out[n] for n in s["grads"]}


def _exact_loss(s, case):
    """A few rows at a time."""
    N, d, V = case["rows"], case["d"], case["vocab"]
    w = s["w"].double()
    zero = lambda *shape: torch.zeros(*shape, device=DEV, dtype=torch.float64)  # noqa: E731
    lse, loss = zero(N), zero(N)
    rows = (s["labels"] >= 0).nonzero()[:, 0]
    inv = 1 / max(1, rows.numel())
    dx, dw, db = (zero(N, d), zero(V, d), zero(V)) if case["train"] else (None, None, None)
    for at in rows.split(1024):
        x, y = s["x"][at].double(), s["labels"][at].long()
        z = torch.mm(x, w.T)
        if case["bias"]:
            z = z + s["bias"].double()
        lse[at] = torch.logsumexp(z, 1)
        loss[at] = lse[at] - z[torch.arange(len(at), device=DEV), y]
        if case["train"]:
            weight = s["weight"][at].double() if case["weights"] else torch.full((len(at),), inv, device=DEV, dtype=torch.float64)
            g = torch.exp(z - lse[at][:, None])
            g[torch.arange(len(at), device=DEV), y] -= 1
            g = g * weight[:, None]
            dx[at] = torch.mm(g, w)
            dw += torch.mm(g.T, x)
            db += g.sum(0)
    return loss, lse, torch.tensor([inv], device=DEV, dtype=torch.float64), dx, dw, db if case["bias"] else None
