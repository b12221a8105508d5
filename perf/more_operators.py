"""Cases and plain forms of the operators around packed attention in a training
step: attention with a sliding window and sinks (forward and backward), the
norms of queries and keys with the rotation of their positions (forward and
backward), and the clipping of gradients by their global norm.

``run`` computes an operator in its plain form (elementary torch operations in
32 bits, rounded once at the end) or, where ``own`` is true, through the
framework's entry points.  ``exact`` restates the definitions in 64 bits.
"""
import math

import torch

own = False

# heads, key / value heads, head dimension: GPT-2 Small, a LLaMA ~1B layer
# (2048 wide) with 128- or 64-wide heads, Qwen3-1.7B, and generic layouts (one
# key / value head for all; groups of three; head dimensions that are no power
# of two)
LAYOUTS = [(12, 12, 64), (16, 16, 128), (32, 32, 64), (16, 8, 128), (8, 1, 128), (6, 2, 96), (5, 5, 80)]
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CLIP_EPS = 1e-6      # added to the norm in max_norm / (norm + eps)
NORM_EPS = 1e-6      # added to the mean square of a head's values


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _win(op, layout, dtype, tokens, lengths, window, sinks, **kw):
    h, hk, d = layout
    return dict(op=op, heads=h, kv_heads=hk, head_dim=d, dtype=dtype, tokens=tokens, window=window, sinks=sinks,
                lengths=",".join(str(n) for n in lengths), **kw)


def _rot(op, layout, dtype, weight, tokens, lengths, first, rotary, base, interleaved, **kw):
    h, hk, d = layout
    return dict(op=op, heads=h, kv_heads=hk, head_dim=d, dtype=dtype, weight=weight, tokens=tokens,
                lengths=",".join(str(n) for n in lengths), first=first, rotary=rotary, base=base,
                interleaved=interleaved, **kw)


def _clip(shapes, dtype, to, flat, limit, **kw):
    """shapes: rows x cols, each with a count.  to: "same" or "bf16", the type of
    the clipped copies, or "place" (nothing is copied, and nothing changes where
    the norm is below the limit).  limit: max_norm as a part of about the norm
    that the inputs have.  flat: the gradients are slices of one buffer."""
    return dict(op="clip", shapes=",".join("%dx%dx%d" % s for s in shapes), dtype=dtype, to=to, flat=flat, limit=limit, **kw)


def listed():
    packed = [4096, 2500, 1, 700, 64, 129, 511]
    return [
        # a forward pass over a handful of short GPT-2 sequences: launch latency
        _win("win_fwd", (12, 12, 64), "bf16", 96, [1, 17, 46, 32], 16, 2, name="win_fwd_gpt2_short"),
        # one packed Qwen3-1.7B micro-batch of documents of very different
        # lengths, a local layer, with a tail of the buffer left unused
        _win("win_fwd", (16, 8, 128), "bf16", 8192, packed, 1024, 4, name="win_fwd_qwen3_packed"),
        # one long document at Qwen3-1.7B's layout, a long window
        _win("win_fwd", (16, 8, 128), "bf16", 32768, [32768], 4096, 4, name="win_fwd_qwen3_long"),
        # gradients in full precision of a short GPT-2 batch (a gradient check,
        # or a model trained without autocast)
        _win("win_bwd", (12, 12, 64), "f32", 1000, [640, 359, 1], 100, 3, name="win_bwd_gpt2_f32"),
        # GPT-2 Small's training shape, a local layer without sinks
        _win("win_bwd", (12, 12, 64), "bf16", 8192, [1024] * 8, 256, 0, name="win_bwd_gpt2_8x1024"),
        # the backward pass of the long document
        _win("win_bwd", (16, 8, 128), "bf16", 32768, [32768], 4096, 4, name="win_bwd_qwen3_long"),
        # a few tokens in fp32, pairs of neighbours, part of an odd head dimension
        _rot("rot_fwd", (6, 2, 96), "f32", "f32", 37, [20, 17], 0, 24, 10000.0, True, name="rot_fwd_small_f32"),
        # a Qwen3-1.7B micro-batch: one packed buffer of documents
        _rot("rot_fwd", (16, 8, 128), "bf16", "bf16", 16384, [8192, 5000, 3192], 0, 128, 1e6, False, name="rot_fwd_qwen3"),
        # a short ragged batch of a LLaMA ~1B layer's heads, fp32 weights
        _rot("rot_bwd", (32, 32, 64), "bf16", "f32", 333, [200, 132, 1], 0, 64, 10000.0, False, name="rot_bwd_llama_ragged"),
        # the micro-batch's backward pass
        _rot("rot_bwd", (16, 8, 128), "bf16", "bf16", 16384, [8192, 5000, 3192], 0, 128, 1e6, False, name="rot_bwd_qwen3"),
        # the parameters of a small language model (two blocks of width 256),
        # fp32, clipped copies of gradients that lie in one bucket
        _clip([(1, 512, 256), (2, 256, 256), (4, 704, 256), (2, 256, 704), (5, 1, 256), (1, 333, 1)], "f32", "same", True,
              0.5, name="clip_small_f32"),
        # the hidden matrices of eight LLaMA ~1B layers: gradients summed in
        # fp32 over several micro-batches, handed to the optimizer in bf16
        _clip([(32, 2048, 2048), (16, 2048, 5504), (8, 5504, 2048)], "f32", "bf16", False, 0.5, name="clip_llama_8_layers"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cut(rng, total, most):
    """total in up to `most` lengths."""
    n = rng.randint(1, min(most, total))
    cuts = sorted(rng.sample(range(1, total), n - 1)) if n > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def draw(rng):
    op = rng.choice(["win_fwd", "win_bwd", "win_fwd", "win_bwd", "rot_fwd", "rot_bwd", "clip"])
    layout = rng.choice(LAYOUTS)
    if op.startswith("win"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        total = _log_int(rng, 16, 14000 if dtype == "bf16" else 2500)
        lengths = _cut(rng, total, 12)
        if rng.random() < 0.3:
            lengths.insert(rng.randrange(len(lengths) + 1), 0)     # a sequence without tokens
        return _win(op, layout, dtype, total + rng.choice([0, 0, rng.randint(1, 99)]), lengths,
                    _log_int(rng, 1, 8192), rng.choice([0, 1, 4, rng.randint(2, 300)]))
    if op.startswith("rot"):
        tokens = _log_int(rng, 1, 16384)
        d = layout[2]
        return _rot(op, layout, rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"]), tokens,
                    _cut(rng, tokens, 12), rng.choice([0, 0, rng.randint(1, 1000000)]),
                    rng.choice([d, d, d // 2, 2 * (d // 8)]), rng.choice([10000.0, 500000.0, 1e6]), rng.random() < 0.3)
    shapes, left = [], 1 << 26
    for _ in range(_log_int(rng, 1, 60)):
        rows, cols = _log_int(rng, 1, 4000), _log_int(rng, 1, 4000)
        if rows * cols <= left:
            shapes.append((1, rows, cols))
            left -= rows * cols
    to = rng.choice(["same", "bf16", "place"])
    return _clip(shapes or [(1, 7, 5)], rng.choice(["f32", "bf16", "mixed"]), to, rng.random() < 0.3,
                 4.0 if to == "place" else rng.choice([0.25, 0.5, 4.0]))


def _lengths(case):
    return [int(n) for n in case["lengths"].split(",")]


def _shapes(case):
    return [(r, c) for n, r, c in (map(int, s.split("x")) for s in case["shapes"].split(",")) for _ in range(n)]


def _clip_types(case):
    """The type of each gradient."""
    n = len(_shapes(case))
    return [("bf16", "f32")[i % 2] for i in range(n)] if case["dtype"] == "mixed" else [case["dtype"]] * n


def _pairs(case):
    w, s = case["window"], case["sinks"]
    total = 0
    for n in _lengths(case):
        m = min(n, w)                          # rows that see all before them
        total += m * (m + 1) // 2 + (n - m) * w
        out = n - m                            # rows with 1 .. n - w keys before the window
        full = max(0, out - s)
        total += (out - full) * (out - full + 1) // 2 + full * s
    return total


def work(case):
    """Inputs read once and outputs written once; products of the visible
    (query, key) pairs only."""
    if case["op"] == "clip":
        size = {"bf16": 2, "f32": 4}
        n = b = 0
        for (rows, cols), t in zip(_shapes(case), _clip_types(case)):
            n += rows * cols
            b += rows * cols * (size[t] + {"same": size[t], "bf16": 2, "place": 0}[case["to"]])
        return {"bytes": b, "flops": 3 * n}
    h, hk, d, t = case["heads"], case["kv_heads"], case["head_dim"], case["tokens"]
    e = 2 if case["dtype"] == "bf16" else 4
    q, kv, lse = t * h * d * e, t * hk * d * e, 4 * t * h
    if case["op"] == "win_fwd":                # Q, K, V in; O and the log-sum out; Q K^T, P V
        return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * d * h * _pairs(case)}
    if case["op"] == "win_bwd":                # Q, K, V, O, dO, log-sum in; dQ, dK, dV out; five products
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * d * h * _pairs(case)}
    n = t * (h + hk) * d
    weights = 2 * d * (2 if case["weight"] == "bf16" else 4)
    if case["op"] == "rot_fwd":                # q, k in, q, k out, positions, weights
        return {"bytes": 2 * n * e + 8 * t + weights, "flops": 7 * n}
    return {"bytes": 3 * n * e + 8 * t + 2 * weights, "flops": 16 * n}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _randn(seed, k, *shape):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + k)
    return torch.randn(*shape, generator=g, device="cuda")


def _pieces(case):
    """The attention in pieces: rows r0 .. r1 of the pack and the pack's rows
    that hold the keys they may see, with both counted from the sequence's
    first."""
    w, s = case["window"], case["sinks"]
    at = 0
    for n in _lengths(case):
        for i0 in range(0, n, 1024):
            i1 = min(n, i0 + 1024)
            j0 = max(0, i0 - w + 1)
            first = min(s, j0)                 # sinks before the window's first key
            yield at, i0, i1, first, j0
        at += n


def _seen(i, j, w, s):
    return (j[None, :] <= i[:, None]) & ((i[:, None] - j[None, :] < w) | (j[None, :] < s))


def _keys(x, at, first, j0, i1):
    x = x.float() if x.dtype != torch.float64 else x
    return torch.cat([x[at:at + first], x[at + j0:at + i1]]).transpose(0, 1)


def _scores(s, case, at, i0, i1, first, j0):
    """Masked scores [kv heads, group * rows, keys] of a piece, and its q, k."""
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    dev = s["q"].device
    q = s["q"][at + i0:at + i1].float().transpose(0, 1).reshape(hk, -1, d)
    k = _keys(s["k"], at, first, j0, i1)
    z = (q @ k.transpose(1, 2)).mul_(d ** -0.5).view(h, i1 - i0, -1)
    j = torch.cat([torch.arange(first, device=dev), torch.arange(j0, i1, device=dev)])
    z.masked_fill_(~_seen(torch.arange(i0, i1, device=dev), j, case["window"], case["sinks"]), -math.inf)
    return z, q, k


def _attention(s, case):
    """Output (32 bits) and log-sum."""
    h, hk, d, t = case["heads"], case["kv_heads"], case["head_dim"], case["tokens"]
    out = torch.zeros(t, h, d, device=s["q"].device)
    lse = torch.full((h, t), -math.inf, device=s["q"].device)
    for at, i0, i1, first, j0 in _pieces(case):
        z, _, _ = _scores(s, case, at, i0, i1, first, j0)
        m = z.amax(-1, keepdim=True)
        p = z.sub_(m).exp_()
        l = p.sum(-1, keepdim=True)
        o = p.view(hk, -1, p.shape[-1]) @ _keys(s["v"], at, first, j0, i1)
        out[at + i0:at + i1] = (o.view(h, i1 - i0, d) / l).transpose(0, 1)
        lse[:, at + i0:at + i1] = (m + torch.log(l)).squeeze(-1)
    return out, lse


def _positions(case):
    parts = [torch.arange(case["first"], case["first"] + n, device="cuda") for n in _lengths(case)]
    return torch.cat(parts)


def prepare(case, seed):
    s = dict(case)
    if case["op"] == "clip":
        shapes, types = _shapes(case), _clip_types(case)
        s["grads"], s["out"] = [], []
        buffers = {}
        if case["flat"]:
            # buckets, one for each type, with a word in front of the gradients
            for t in set(types):
                size = sum(r * c for (r, c), u in zip(shapes, types) if u == t)
                buffers[t] = [torch.empty(size + 1, dtype=DTYPES[t], device="cuda"), 1]
        for i, ((rows, cols), t) in enumerate(zip(shapes, types)):
            # layers differ in scale, rows too
            x = _randn(seed, 10 + i, rows, cols)
            x *= 10.0 ** (-3 - (i * 7) % 3) * torch.exp(0.5 * _randn(seed, 5000 + i, rows, 1))
            if case["flat"]:
                buf, at = buffers[t]
                g = buf[at:at + rows * cols].view(rows, cols)
                buffers[t][1] += rows * cols
                g.copy_(x)
            else:
                g = x.to(DTYPES[t])
            s["grads"].append(g)
            if case["to"] != "place":
                s["out"].append(torch.empty(rows, cols, dtype=DTYPES["bf16" if case["to"] == "bf16" else t], device="cuda"))
        # E exp(2 * 0.5 n) = exp(0.5) for each square
        size = sum(r * c * 10.0 ** (2 * (-3 - (i * 7) % 3)) for i, (r, c) in enumerate(shapes)) * math.exp(0.5)
        s["max_norm"] = case["limit"] * math.sqrt(size)
        return s
    dt = DTYPES[case["dtype"]]
    t, h, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    # queries, keys and values are slices of one projection's output; the heads
    # differ in scale, and so in how sharp their attention is
    x = _randn(seed, 1, t, h + 2 * hk, d)
    x[:, :h] *= torch.exp(0.7 * _randn(seed, 2, h))[None, :, None]
    x = x.to(dt)
    s["q"], s["k"], s["v"] = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    if case["op"].startswith("win"):
        if case["op"] == "win_bwd":
            out, s["lse"] = _attention(s, case)
            s["out"] = out.to(dt)
            s["dout"] = (_randn(seed, 3, t, h, d) * 0.01).to(dt)
        if own:
            from paper_2609_36692_gb300 import layers
            lengths = _lengths(case)
            s["plan"] = layers.PackedAttention(h, hk, d, max_tokens=t, max_seqs=len(lengths), dtype=dt,
                                               window=case["window"], sinks=case["sinks"])
            s["plan"].set_lengths(lengths)
        return s
    wt = DTYPES[case["weight"]]
    s["qw"], s["kw"] = ((1 + 0.2 * _randn(seed, k, d)).to(wt) for k in (4, 5))
    s["positions"] = _positions(case)
    if case["op"] == "rot_bwd":
        s["dq"] = (_randn(seed, 6, t, h, d) * 0.01).to(dt)
        s["dk"] = (_randn(seed, 7, t, hk, d) * 0.01).to(dt)
    if own:
        from paper_2609_36692_gb300 import layers
        s["plan"] = layers.QKNormRotary(h, hk, d, rotary_dim=case["rotary"], base=case["base"],
                                        interleaved=case["interleaved"], eps=NORM_EPS, dtype=dt)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_win_bwd(s):
    h, hk, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["tokens"]
    dev, dt, scale = s["q"].device, s["q"].dtype, d ** -0.5
    dq = torch.zeros(t, h, d, device=dev)
    dk, dv = torch.zeros(t, hk, d, device=dev), torch.zeros(t, hk, d, device=dev)
    for at, i0, i1, first, j0 in _pieces(s):
        rows = slice(at + i0, at + i1)
        z, q, k = _scores(s, s, at, i0, i1, first, j0)
        p = z.sub_(s["lse"][:, rows, None]).exp_().view(hk, -1, z.shape[-1])
        do = s["dout"][rows].float()
        delta = (do * s["out"][rows].float()).sum(-1).t().reshape(hk, -1, 1)
        do = do.transpose(0, 1).reshape(hk, -1, d)
        ds = (do @ _keys(s["v"], at, first, j0, i1).transpose(1, 2)).sub_(delta).mul_(p).mul_(scale)
        dq[rows] = (ds @ k).view(h, i1 - i0, d).transpose(0, 1)
        for to, g in ((dk, ds.transpose(1, 2) @ q), (dv, p.transpose(1, 2) @ do)):
            g = g.transpose(0, 1)
            to[at:at + first] += g[:first]
            to[at + j0:at + i1] += g[first:]
    return {"dq": dq.to(dt), "dk": dk.to(dt), "dv": dv.to(dt)}


def _angles(s):
    """cos and sin of the angles, [tokens, 1, rotary / 2]."""
    f = s["base"] ** (-torch.arange(0, s["rotary"], 2, device="cuda", dtype=torch.float64) / s["rotary"])
    a = s["positions"].double()[:, None, None] * f
    return torch.cos(a).float(), torch.sin(a).float()


def _turn(y, cos, sin, r, interleaved):
    """The first r dimensions of y, turned in pairs."""
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, y[..., r:]], -1)


def _plain_rot(s):
    cos, sin = _angles(s)
    dt, d, r, inter = s["q"].dtype, s["head_dim"], s["rotary"], s["interleaved"]
    got = {}
    for name, wn, gn in (("q", "qw", "dq"), ("k", "kw", "dk")):
        x, w = s[name].float(), s[wn].float()
        inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + NORM_EPS)
        if s["op"] == "rot_fwd":
            got[name] = _turn(x * inv * w, cos, sin, r, inter).to(dt)
            continue
        g = _turn(s[gn].float(), cos, -sin, r, inter)
        xh, u = x * inv, g * w
        got[gn] = (inv * (u - xh * (u * xh).mean(-1, keepdim=True))).to(dt)
        got["d" + wn] = (g * xh).sum((0, 1), dtype=torch.float64).to(s[wn].dtype)
    return got


def _plain_clip(s):
    norm = torch.sqrt(sum((g.float() ** 2).sum(dtype=torch.float64) for g in s["grads"]))
    c = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0).float()
    if s["to"] == "place":
        for g in s["grads"]:
            g.copy_(g.float() * c)
        return {"norm": norm.float(), "grads": s["grads"]}
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * c)
    return {"norm": norm.float(), "grads": s["out"]}


def _run_plain(s):
    if s["op"] == "win_fwd":
        out, lse = _attention(s, s)
        return {"out": out.to(s["q"].dtype), "lse": lse}
    if s["op"] == "win_bwd":
        return _plain_win_bwd(s)
    return _plain_clip(s) if s["op"] == "clip" else _plain_rot(s)


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    if s["op"] == "win_fwd":
        out, lse = s["plan"].forward(s["q"], s["k"], s["v"])
        return {"out": out, "lse": lse}
    if s["op"] == "win_bwd":
        dq, dk, dv = s["plan"].backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if s["op"] == "rot_fwd":
        q, k = s["plan"].forward(s["q"], s["k"], s["positions"], s["qw"], s["kw"])
        return {"q": q, "k": k}
    if s["op"] == "rot_bwd":
        dq, dk, dqw, dkw = s["plan"].backward(s["q"], s["k"], s["positions"], s["dq"], s["dk"], s["qw"], s["kw"])
        return {"dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw}
    from paper_2609_36692_gb300 import optim
    if s["to"] == "place":
        return {"norm": optim.clip_grads(s["grads"], s["max_norm"], eps=CLIP_EPS), "grads": s["grads"]}
    return {"norm": optim.clip_grads(s["grads"], s["max_norm"], eps=CLIP_EPS, out=s["out"]), "grads": s["out"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_win(s, forward):
    h, hk, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["tokens"]
    w, sinks = s["window"], s["sinks"]
    dev, f64, scale = s["q"].device, torch.float64, 1.0 / math.sqrt(d)
    zeros = lambda n: torch.zeros(t, n, d, dtype=f64, device=dev)  # noqa: E731
    out, dq, dk, dv = zeros(h), zeros(h), zeros(hk), zeros(hk)
    lse = torch.full((h, t), -math.inf, dtype=f64, device=dev)
    start = 0
    for n in _lengths(s):
        for r0 in range(0, n, 2048):
            r1 = min(n, r0 + 2048)
            rows = slice(start + r0, start + r1)
            lo = max(0, r0 - w + 1)
            key = torch.arange(r1, device=dev)
            key = key[(key >= lo) | (key < sinks)]
            row = torch.arange(r0, r1, device=dev)[:, None]
            hidden = (key > row) | ((key <= row - w) & (key >= sinks))
            at = key + start
            for head in range(h):
                kh = head // (h // hk)
                k, v, q = s["k"][at, kh].double(), s["v"][at, kh].double(), s["q"][rows, head].double()
                z = scale * torch.einsum("id,jd->ij", q, k)
                z[hidden] = -math.inf
                norm = torch.logsumexp(z, 1)
                p = torch.exp(z - norm[:, None])
                o = p @ v
                lse[head, rows], out[rows, head] = norm, o
                if forward:
                    continue
                g = s["dout"][rows, head].double()
                dz = p * (g @ v.T - (g * o).sum(1, keepdim=True))
                dq[rows, head] = scale * (dz @ k)
                dk[:, kh].index_add_(0, at, scale * (dz.T @ q))
                dv[:, kh].index_add_(0, at, p.T @ g)
        start += n
    return {"out": out, "lse": lse} if forward else {"dq": dq, "dk": dk, "dv": dv}


def _exact_rot(s):
    """By complex numbers: a pair (a, b) is a + i b, turned by exp(i angle)."""
    d, r = s["head_dim"], s["rotary"]
    i = torch.arange(r // 2, device="cuda")
    ia, ib = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + r // 2)
    speed = torch.exp(-math.log(s["base"]) * 2.0 * i.double() / r)
    angle = s["positions"].double()[:, None] * speed
    phase = torch.polar(torch.ones_like(angle), angle)[:, None, :]

    def turn(y, phase):
        c = torch.complex(y[..., ia], y[..., ib]) * phase
        y = y.clone()
        y[..., ia], y[..., ib] = c.real, c.imag
        return y

    got = {}
    for name, wn, gn in (("q", "qw", "dq"), ("k", "kw", "dk")):
        x, w = s[name].double(), s[wn].double()
        size = torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + NORM_EPS)
        if s["op"] == "rot_fwd":
            got[name] = turn(x / size * w, phase)
            continue
        g = turn(s[gn].double(), phase.conj())
        got["d" + wn] = torch.einsum("thd,thd->d", g, x / size)
        gw = g * w
        got[gn] = gw / size - x * (gw * x).sum(-1, keepdim=True) / (d * size ** 3)
    return got


def exact(case, seed):
    global own
    mine, own = own, False                 # inputs only: no plan of the framework's
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    if case["op"].startswith("win"):
        return _exact_win(s, case["op"] == "win_fwd")
    if case["op"].startswith("rot"):
        return _exact_rot(s)
    square = 0.0
    for g in s["grads"]:
        square = square + torch.linalg.vector_norm(g.double()) ** 2
    norm = torch.sqrt(square)
    factor = torch.minimum(torch.ones_like(norm), s["max_norm"] / (norm + CLIP_EPS))
    return {"norm": norm, "grads": [g.double() * factor for g in s["grads"]]}
