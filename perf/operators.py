"""Cases and plain forms of the training operators: packed causal attention
(forward and backward) and 8-bit activation checkpoints (pack / restore, a
linear layer's weight gradient taken from a checkpoint, and a gated activation
whose backward reads checkpoints).

``run`` computes an operator in its plain form (elementary torch operations in
32 bits, rounded once at the end) or, where ``own`` is true, through the
framework's entry points.  ``exact`` restates the definitions in 64 bits.
"""
import math

import torch

own = False

# heads, key / value heads, head dimension: GPT-2 Small, a LLaMA ~1B layer
# (2048 wide) with 128- or 64-wide heads, Qwen3-1.7B, and two generic layouts
# (one key / value head for all; a head dimension that fills no power of two)
LAYOUTS = [(12, 12, 64), (16, 16, 128), (32, 32, 64), (16, 8, 128), (8, 1, 128), (6, 2, 96), (5, 5, 80)]
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32   # elements that share one power-of-two step in a checkpoint


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _attn(op, layout, dtype, tokens, lengths, **kw):
    h, hk, d = layout
    return dict(op=op, heads=h, kv_heads=hk, head_dim=d, dtype=dtype, tokens=tokens,
                lengths=",".join(str(n) for n in lengths), **kw)


def listed():
    return [
        # a forward pass over a handful of short GPT-2 sequences: launch latency
        _attn("attn_fwd", (12, 12, 64), "bf16", 96, [1, 17, 46, 32], name="attn_fwd_gpt2_short"),
        # one packed Qwen3-1.7B micro-batch of documents of very different
        # lengths, with a tail of the buffer left unused
        _attn("attn_fwd", (16, 8, 128), "bf16", 8192, [4096, 2500, 1, 700, 64, 129, 511], name="attn_fwd_qwen3_packed"),
        # one long document at Qwen3-1.7B's layout
        _attn("attn_fwd", (16, 8, 128), "bf16", 16384, [16384], name="attn_fwd_qwen3_long"),
        # gradients in full precision of a short GPT-2 batch (a gradient check,
        # or a model trained without autocast)
        _attn("attn_bwd", (12, 12, 64), "f32", 1000, [640, 359, 1], name="attn_bwd_gpt2_f32"),
        # GPT-2 Small's training shape, eight sequences of 1024 tokens
        _attn("attn_bwd", (12, 12, 64), "bf16", 8192, [1024] * 8, name="attn_bwd_gpt2_8x1024"),
        # the backward pass of the long document
        _attn("attn_bwd", (16, 8, 128), "bf16", 16384, [16384], name="attn_bwd_qwen3_long"),
        # a few tokens' residual stream, an odd width, fp32
        dict(op="pack", tokens=37, features=1001, dtype="f32", name="pack_small_f32"),
        # the input of Qwen3-1.7B's down projection over a micro-batch
        dict(op="pack", tokens=16384, features=6144, dtype="bf16", name="pack_qwen3_down"),
        # GPT-2 Small's attention projection: a small matrix under a long sum,
        # its gradient kept in fp32
        dict(op="wgrad", tokens=8192, out_features=768, features=768, dtype="bf16", grad="f32", name="wgrad_gpt2_proj"),
        # Qwen3-1.7B's gate projection, a bf16 gradient as its optimizer takes it
        dict(op="wgrad", tokens=16384, out_features=6144, features=2048, dtype="bf16", grad="bf16", name="wgrad_qwen3_gate"),
        # a short ragged batch through the LLaMA ~1B gated MLP
        dict(op="swiglu", tokens=333, features=5504, dtype="bf16", name="swiglu_llama_ragged"),
        # a full Qwen3-1.7B micro-batch
        dict(op="swiglu", tokens=16384, features=6144, dtype="bf16", name="swiglu_qwen3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn_fwd", "attn_bwd", "attn_fwd", "attn_bwd", "pack", "wgrad", "swiglu"])
    if op.startswith("attn"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        total = _log_int(rng, 16, 12000 if dtype == "bf16" else 2500)
        n = rng.randint(1, min(12, total))
        cuts = sorted(rng.sample(range(1, total), n - 1)) if n > 1 else []
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        if rng.random() < 0.3:
            lengths.insert(rng.randrange(n + 1), 0)     # a sequence without tokens
        return _attn(op, rng.choice(LAYOUTS), dtype, total + rng.choice([0, 0, rng.randint(1, 99)]), lengths)
    if op == "wgrad":
        return dict(op=op, tokens=_log_int(rng, 1, 16384), out_features=8 * _log_int(rng, 8, 768),
                    features=_log_int(rng, 60, 2050), dtype="bf16", grad=rng.choice(["bf16", "f32"]))
    return dict(op=op, tokens=_log_int(rng, 1, 16384), features=_log_int(rng, 30, 6100),
                dtype=rng.choice(["bf16", "bf16", "f32"]))


def _lengths(case):
    return [int(n) for n in case["lengths"].split(",")]


def work(case):
    """Inputs read once and outputs written once; products of the visible
    (query, key) pairs only."""
    if case["op"].startswith("attn"):
        h, hk, d, t = case["heads"], case["kv_heads"], case["head_dim"], case["tokens"]
        e = 2 if case["dtype"] == "bf16" else 4
        pairs = sum(n * (n + 1) // 2 for n in _lengths(case))
        q, kv, lse = t * h * d * e, t * hk * d * e, 4 * t * h
        if case["op"] == "attn_fwd":       # Q, K, V in; O and the log-sum out; Q K^T, P V
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * d * h * pairs}
        # Q, K, V, O, dO, log-sum in; dQ, dK, dV out; Q K^T, dO V^T, P^T dO, dS^T Q, dS K
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * d * h * pairs}
    t, f = case["tokens"], case["features"]
    e = 2 if case["dtype"] == "bf16" else 4
    packed = t * f + t * -(-f // BLOCK)
    if case["op"] == "pack":               # values in, packed out; packed in, values out
        return {"bytes": 2 * t * f * e + 2 * packed, "flops": 4 * t * f}
    if case["op"] == "wgrad":
        n = case["out_features"]
        return {"bytes": t * n * e + packed + n * f * (2 if case["grad"] == "bf16" else 4), "flops": 2 * t * n * f}
    # forward: gate, up in, h and two checkpoints out; backward: checkpoints
    # and dh in, dgate and dup out
    return {"bytes": 6 * t * f * e + 4 * packed, "flops": 30 * t * f}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _randn(seed, k, *shape):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + k)
    return torch.randn(*shape, generator=g, device="cuda")


def _reference_rows(q, k, v, lengths, scale):
    """Output and log-sum of the attention, sequence by sequence and a block of
    rows at a time: what a forward pass left behind for the backward one."""
    t, h, d = q.shape
    g = h // k.shape[1]
    out = torch.zeros(t, h, d, device=q.device)
    lse = torch.full((h, t), -math.inf, device=q.device)
    at = 0
    for n in lengths:
        for i0 in range(at, at + n, 1024):
            i1 = min(at + n, i0 + 1024)
            qs = q[i0:i1].float().transpose(0, 1)
            ks = k[at:i1].float().transpose(0, 1).repeat_interleave(g, 0)
            vs = v[at:i1].float().transpose(0, 1).repeat_interleave(g, 0)
            s = qs @ ks.transpose(1, 2) * scale
            seen = torch.arange(at, i1, device=q.device)[None, :] <= torch.arange(i0, i1, device=q.device)[:, None]
            s = s.masked_fill(~seen, -math.inf)
            lse[:, i0:i1] = torch.logsumexp(s, -1)
            out[i0:i1] = (torch.exp(s - lse[:, i0:i1, None]) @ vs).transpose(0, 1)
        at += n
    return out, lse


def prepare(case, seed):
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    t = case["tokens"]
    if case["op"].startswith("attn"):
        h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
        # queries, keys and values are slices of one projection's output; the
        # heads differ in how sharp their attention is
        x = _randn(seed, 1, t, h + 2 * hk, d)
        x[:, :h] *= torch.exp(0.7 * _randn(seed, 2, h))[None, :, None]
        x = x.to(dt)
        s["q"], s["k"], s["v"] = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
        lengths = _lengths(case)
        s["seq"] = torch.repeat_interleave(torch.arange(len(lengths) + 1, device="cuda"),
                                           torch.tensor(lengths + [t - sum(lengths)], device="cuda"))
        s["n_seqs"] = len(lengths)
        if case["op"] == "attn_bwd":
            out, s["lse"] = _reference_rows(s["q"], s["k"], s["v"], lengths, d ** -0.5)
            s["out"] = out.to(dt)
            s["dout"] = (_randn(seed, 3, t, h, d) * 0.01).to(dt)
        if own:
            from paper_2609_36692_gb300 import layers
            s["plan"] = layers.PackedAttention(h, hk, d, max_tokens=t, max_seqs=len(lengths), dtype=dt)
            s["plan"].set_lengths(lengths)
        return s
    f = case["features"]
    # activations with a few loud channels
    loud = torch.exp(_randn(seed, 4, f))
    if case["op"] == "swiglu":
        s["gate"] = (_randn(seed, 5, t, f) * loud).to(dt)
        s["up"] = _randn(seed, 6, t, f).to(dt)
        s["dh"] = (_randn(seed, 7, t, f) * 0.01).to(dt)
        return s
    s["x"] = (_randn(seed, 8, t, f) * loud).to(dt)
    if case["op"] == "wgrad":
        s["dy"] = (_randn(seed, 9, t, case["out_features"]) * 0.01).to(dt)
        # the checkpoint that the forward pass kept
        if own:
            from paper_2609_36692_gb300 import layers
            s["ckpt"] = layers.ckpt_pack(s["x"])
        else:
            s["codes"], s["exponents"] = _pack(s["x"])
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _pack(x):
    """Whole numbers of at most 127 in absolute value, and for each block of 32
    elements of a row the exponent e of its step 2^e: the least e >= -126 with
    max |x| <= 127 * 2^e."""
    t, f = x.shape
    pad = -f % BLOCK
    xb = torch.nn.functional.pad(x.float(), (0, pad)).view(t, -1, BLOCK)
    m, ex = torch.frexp(xb.abs().amax(-1))
    e = (ex - 7 + (m * 128 > 127).int()).clamp(min=-126)
    return torch.round(xb * torch.exp2(-e.float())[..., None]).to(torch.int8), e


def _unpack(codes, e, f):
    t = codes.shape[0]
    return (codes.float() * torch.exp2(e.float())[..., None]).view(t, -1)[:, :f]


def _plain_attention(s):
    h, hk, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["tokens"]
    g, scale = h // hk, d ** -0.5
    q = s["q"].float().permute(1, 0, 2).reshape(hk, g * t, d)
    k = s["k"].float().permute(1, 0, 2)
    v = s["v"].float().permute(1, 0, 2)
    at = torch.arange(t, device=q.device)
    seen = (s["seq"][:, None] == s["seq"][None, :]) & (at[None, :] <= at[:, None]) & (s["seq"] < s["n_seqs"])[:, None]
    sc = (q @ k.transpose(1, 2)).mul_(scale).view(hk, g, t, t)
    sc.masked_fill_(~seen, -math.inf)
    if s["op"] == "attn_fwd":
        m = sc.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        p = sc.sub_(m).exp_()
        l = p.sum(-1, keepdim=True)
        o = (p.view(hk, g * t, t) @ v).view(hk, g, t, d) / torch.where(l > 0, l, torch.ones_like(l))
        lse = (m + torch.log(l)).view(h, t)
        return {"out": o.reshape(h, t, d).permute(1, 0, 2).to(s["q"].dtype).contiguous(), "lse": lse}
    do = s["dout"].float().permute(1, 0, 2).reshape(hk, g * t, d)
    lse = s["lse"].view(hk, g, t, 1)
    p = sc.sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_().view(hk, g * t, t)
    delta = (s["dout"].float() * s["out"].float()).sum(-1).t().reshape(hk, g * t, 1)
    dv = p.transpose(1, 2) @ do
    ds = (do @ v.transpose(1, 2)).sub_(delta).mul_(p).mul_(scale)
    dq = (ds @ k).view(h, t, d)
    dk = ds.transpose(1, 2) @ q
    dt = s["q"].dtype
    return {n: x.permute(1, 0, 2).to(dt).contiguous() for n, x in (("dq", dq), ("dk", dk), ("dv", dv))}


def _plain_swiglu(s):
    gate, up, dt, f = s["gate"], s["up"], s["gate"].dtype, s["features"]
    a, b = gate.float(), up.float()
    h = (a / (1 + torch.exp(-a)) * b).to(dt)
    a, b, dh = _unpack(*_pack(gate), f), _unpack(*_pack(up), f), s["dh"].float()
    sig = 1 / (1 + torch.exp(-a))
    return {"h": h, "dgate": (dh * b * sig * (1 + a * (1 - sig))).to(dt), "dup": (dh * a * sig).to(dt)}


def _run_plain(s):
    if s["op"].startswith("attn"):
        return _plain_attention(s)
    if s["op"] == "swiglu":
        return _plain_swiglu(s)
    if s["op"] == "pack":
        return _unpack(*_pack(s["x"]), s["features"]).to(s["x"].dtype)
    x = _unpack(s["codes"], s["exponents"], s["features"])
    return (s["dy"].float().t() @ x).to(DTYPES[s["grad"]])


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    from paper_2609_36692_gb300 import layers
    if s["op"] == "attn_fwd":
        out, lse = s["plan"].forward(s["q"], s["k"], s["v"])
        return {"out": out, "lse": lse}
    if s["op"] == "attn_bwd":
        dq, dk, dv = s["plan"].backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if s["op"] == "pack":
        return layers.ckpt_pack(s["x"]).restore()
    if s["op"] == "wgrad":
        return layers.ckpt_wgrad(s["dy"], s["ckpt"], dtype=DTYPES[s["grad"]])
    h, cg, cu = layers.ckpt_swiglu(s["gate"], s["up"])
    dgate, dup = layers.ckpt_swiglu_backward(cg, cu, s["dh"])
    return {"h": h, "dgate": dgate, "dup": dup}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_restore(x):
    t, f = x.shape
    y = torch.zeros(t, -(-f // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    y[:, :f] = x.double()
    y = y.view(t, -1, BLOCK)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -149) / 127.0))
    for _ in range(2):                     # log2's rounding: take the least e that holds
        e = torch.where(top > 127.0 * torch.exp2(e), e + 1, e)
        e = torch.where(top <= 127.0 * torch.exp2(e - 1), e - 1, e)
    step = torch.exp2(torch.clamp(e, min=-126.0))
    return (torch.round(y / step) * step).view(t, -1)[:, :f]


def _exact_attention(s, forward):
    h, hk, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["tokens"]
    dev, f64, scale = s["q"].device, torch.float64, 1.0 / math.sqrt(d)
    zeros = lambda n: torch.zeros(t, n, d, dtype=f64, device=dev)  # noqa: E731
    out, dq, dk, dv = zeros(h), zeros(h), zeros(hk), zeros(hk)
    lse = torch.full((h, t), -math.inf, dtype=f64, device=dev)
    start = 0
    for n in _lengths(s):
        for head in range(h):
            kh = head // (h // hk)
            k, v = s["k"][start:start + n, kh].double(), s["v"][start:start + n, kh].double()
            for r0 in range(0, n, 2048):
                r1 = min(n, r0 + 2048)
                rows = slice(start + r0, start + r1)
                q = s["q"][rows, head].double()
                z = scale * torch.einsum("id,jd->ij", q, k[:r1])
                late = torch.ones(r1 - r0, r1, dtype=torch.bool, device=dev).triu(r0 + 1)
                z[late] = -math.inf
                norm = torch.logsumexp(z, 1)
                p = torch.exp(z - norm[:, None])
                o = p @ v[:r1]
                lse[head, rows], out[rows, head] = norm, o
                if forward:
                    continue
                g = s["dout"][rows, head].double()
                dz = p * (g @ v[:r1].T - (g * o).sum(1, keepdim=True))
                dq[rows, head] = scale * (dz @ k[:r1])
                dk[start:start + r1, kh] += scale * (dz.T @ q)
                dv[start:start + r1, kh] += p.T @ g
        start += n
    return {"out": out, "lse": lse} if forward else {"dq": dq, "dk": dk, "dv": dv}


def exact(case, seed):
    global own
    mine, own = own, False                 # inputs only: no plan, no checkpoint of the framework's
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    if case["op"].startswith("attn"):
        return _exact_attention(s, case["op"] == "attn_fwd")
    if case["op"] == "pack":
        return _exact_restore(s["x"])
    if case["op"] == "wgrad":
        return s["dy"].double().T @ _exact_restore(s["x"])
    a, b = s["gate"].double(), s["up"].double()
    ra, rb, g = _exact_restore(s["gate"]), _exact_restore(s["up"]), s["dh"].double()
    sig = torch.sigmoid(ra)
    return {"h": a * torch.sigmoid(a) * b, "dgate": g * rb * (sig + ra * sig * (1 - sig)), "dup": g * ra * sig}
