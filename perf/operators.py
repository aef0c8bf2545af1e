"""Timing cases of the operators of a decoder's attention block with rotary positions and a sliding window, each through
the entry points of `paper_2505_05856_amd.binding`.

Kinds of case:
  rotary   queries and keys of a packed projection [T, (q_heads + 2 kv_heads) * dim]: every head's vector divided by its root
           mean square and multiplied by a gain (`norm`), its first `rot` elements turned by the token's position
           (op_qk_rotary_fwd); with `train` also the gradients of the projection and of the gains (op_qk_rotary_bwd)
  window   causal attention in which a query sees the `window` newest keys up to its own and the first `sinks` keys of its
           sequence; several query heads may share a key head, sequences may be shorter than the batch's length (`lens`)
           (op_window_attention_fwd); with `train` also the gradients of queries, keys and values (op_window_attention_bwd)

A case is a dict of plain values.  `own` chooses between the library's kernels and their plain form in torch.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rotary(name, **kw):
    case = {"kind": "rotary", "batch": 1, "seq": 512, "q_heads": 16, "kv_heads": 16, "dim": 64, "rot": 64, "interleaved": False,
            "norm": True, "far": False, "dtype": "bf16", "train": True}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _window(name, **kw):
    case = {"kind": "window", "batch": 1, "seq": 512, "q_heads": 16, "kv_heads": 16, "dim": 64, "window": 128, "sinks": 0,
            "lens": False, "dtype": "bf16", "train": True}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a handful of tokens in 32 bits, the size a program checks itself with: launches and latency
        _rotary("rotary_tiny", seq=5, q_heads=2, kv_heads=1, dtype="f32"),
        # GPT-2-XL width (25 heads of 64), half of each head turned, neighbouring elements paired, no norm
        _rotary("rotary_partial", batch=4, seq=1024, q_heads=25, kv_heads=25, rot=32, interleaved=True, norm=False),
        # tokens of packed documents far into a long context, frequencies stretched for it, a head dimension that is no
        # power of two; the forward pass alone, as a recomputed block runs it
        _rotary("rotary_far", seq=9001, q_heads=16, kv_heads=2, dim=80, rot=40, far=True, train=False),
        # the widest stage (32 heads of 128, sequence 2048, batch 8), four query heads a key head: memory traffic
        _rotary("rotary_wide", batch=8, seq=2048, q_heads=32, kv_heads=8, dim=128, rot=128),
        # a handful of tokens in 32 bits: launches and latency
        _window("window_tiny", seq=5, q_heads=2, kv_heads=1, window=3, sinks=1, dtype="f32"),
        # one short sequence: few workgroups, latency counts
        _window("window_short", seq=200, q_heads=8, kv_heads=2, dim=128, window=64, sinks=4),
        # a padded batch of sequences of no round length
        _window("window_ragged", batch=3, seq=709, q_heads=12, kv_heads=4, window=200, sinks=4, lens=True),
        # a layer of the encoder's width (16 heads of 64, sequence 512) in 32 bits
        _window("window_f32", batch=2, window=128, dtype="f32"),
        # GPT-2-XL width, the forward pass alone
        _window("window_forward", batch=4, seq=1024, q_heads=25, kv_heads=25, window=256, sinks=1, train=False),
        # a window longer than the sequence: ordinary causal attention with shared key heads
        _window("window_causal", batch=2, seq=1500, q_heads=16, kv_heads=4, dim=128, window=2048),
        # one device's heads of a long sequence
        _window("window_long", seq=16384, q_heads=4, kv_heads=1, dim=128, window=4096, sinks=4),
        # the widest stage: matrix products
        _window("window_wide", batch=8, seq=2048, q_heads=32, kv_heads=8, dim=128, window=512, sinks=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    group = rng.choice((1, 2, 4, 8))
    if rng.random() < 0.4:
        dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 256))
        kv = rng.randint(1, max(1, 32 // group))
        seq = _log(rng, 1, 16384)
        batch = rng.randint(1, max(1, min(8, 16384 // seq)))
        while batch * seq * kv * (group + 1) * dim > (80_000_000 if dtype == "bf16" else 40_000_000):   # (a drawn case stays below the widest listed one)
            seq = (seq + 1) // 2
        return _rotary(None, batch=batch, seq=seq, q_heads=kv * group, kv_heads=kv, dim=dim, rot=dim // rng.choice((1, 1, 2, 4)),
                       interleaved=rng.random() < 0.4, norm=rng.random() < 0.7, far=rng.random() < 0.3, dtype=dtype,
                       train=rng.random() < 0.7)
    dim = rng.choice((64, 128)) if dtype == "bf16" else rng.choice((32, 64, 80, 128))
    kv = rng.randint(1, max(1, 32 // group))
    seq = _log(rng, 1, 16384 if dtype == "bf16" else 2048)
    batch = rng.randint(1, 8)
    most = 500_000_000 if dtype == "bf16" else 40_000_000          # pairs of a query and a key
    while batch * kv * group * seq * seq > most:
        if batch > 1:
            batch -= 1
        elif kv > 1:
            kv -= 1
        else:
            seq = seq * 3 // 4
    window = _log(rng, 1, 2 * seq)
    # (a query that sees one key alone has no gradient of its logits: rounding is all there is to return)
    return _window(None, batch=batch, seq=seq, q_heads=kv * group, kv_heads=kv, dim=dim, window=window,
                   sinks=rng.choice((0, 1, 4, 16, 100)), lens=batch > 1 and rng.random() < 0.3, dtype=dtype,
                   train=min(seq, window) > 1 and rng.random() < 0.7)


# ------------------------------------------------------------------ inputs

def _lens(case):
    """Tokens of each sequence: with `lens` from the whole length down to none."""
    B, S = case["batch"], case["seq"]
    return [S * (B - 1 - b) // (B - 1) for b in range(B)] if case["lens"] and B > 1 else [S] * B


def prepare(case, seed):
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    T, nq, nk, dh = case["batch"] * case["seq"], case["q_heads"], case["kv_heads"], case["dim"]

    def normal(*shape, sd=1.0, mean=0.0):
        return torch.randn(shape, generator=gen, device=DEV).mul_(sd).add_(mean).to(dt)

    # the packed projection [Q | K | V] of a layer, and its gradient
    qkv, dqkv = normal(T, nq + 2 * nk, dh), torch.zeros(T, nq + 2 * nk, dh, device=DEV, dtype=dt)
    s = {"case": case}
    if case["kind"] == "rotary":
        s.update(q=qkv[:, :nq], k=qkv[:, nq:nq + nk], dq=dqkv[:, :nq], dk=dqkv[:, nq:nq + nk],
                 qg=normal(dh, sd=0.05, mean=1.0) if case["norm"] else None, kg=normal(dh, sd=0.05, mean=1.0) if case["norm"] else None,
                 dqo=normal(T, nq, dh), dko=normal(T, nk, dh), qo=torch.empty(T, nq, dh, device=DEV, dtype=dt),
                 ko=torch.empty(T, nk, dh, device=DEV, dtype=dt), pos=None, scale=1.0)
        s.update(dqg=torch.empty_like(s["qg"]) if case["norm"] else None, dkg=torch.empty_like(s["kg"]) if case["norm"] else None)
        half = case["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        if case["far"]:   # frequencies for a context 32 times as long: the slow ones divided by 32, the fast ones kept, a ramp between
            turns = 4096 * freq / (2 * math.pi)
            keep = ((turns - 1) / 31).clamp(0, 1)
            freq = freq * keep + freq / 32 * (1 - keep)
            s["scale"] = 0.1 * math.log(32) + 1
            start = torch.randint(0, 131072, (T,), generator=gen, device=DEV, dtype=torch.int32)
            doc = torch.arange(T, device=DEV, dtype=torch.int32) // 1000           # documents of 1000 tokens, each somewhere
            s["pos"] = start[doc.long()] + torch.arange(T, device=DEV, dtype=torch.int32) % 1000
        s["freq"] = freq.float().to(DEV)
        return s
    s.update(q=normal(T, nq, dh, sd=1.4), k=normal(T, nk, dh), v=qkv[:, nq + nk:], dv=dqkv[:, nq + nk:], do=normal(T, nq, dh),
             o=torch.empty(T, nq, dh, device=DEV, dtype=dt), dq=torch.empty(T, nq, dh, device=DEV, dtype=dt),
             dk=torch.empty(T, nk, dh, device=DEV, dtype=dt), lse=torch.empty(case["batch"], nq, case["seq"], device=DEV), lens=None)
    if case["lens"]:
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    if own:
        from paper_2505_05856_amd import binding as B
        if c["kind"] == "rotary":
            form = {"seq": c["seq"], "interleaved": c["interleaved"], "eps": EPS, "scale": s["scale"], "positions": s["pos"]}
            B.op_qk_rotary_fwd(s["q"], s["k"], s["qg"], s["kg"], s["freq"], s["qo"], s["ko"], **form)
            if not c["train"]:
                return {n: s[n] for n in ("qo", "ko")}
            if "ws" not in s:   # a program keeps its workspace
                s["ws"] = torch.empty(B.op_qk_rotary_workspace_bytes(s["q"].shape[0], c["q_heads"], c["kv_heads"], c["dim"]),
                                      dtype=torch.uint8, device=DEV)
            B.op_qk_rotary_bwd(s["dqo"], s["dko"], s["q"], s["k"], s["qg"], s["kg"], s["freq"], s["dq"], s["dk"], s["dqg"], s["dkg"],
                               s["ws"], **form)
            return {n: s[n] for n in ("qo", "ko", "dq", "dk", "dqg", "dkg")}
        B.op_window_attention_fwd(s["q"], s["k"], s["v"], c["seq"], c["window"], c["sinks"], s["o"], s["lse"], lens=s["lens"])
        if not c["train"]:
            return {n: s[n] for n in ("o", "lse")}
        if "ws" not in s:
            s["ws"] = torch.empty(B.op_window_attention_workspace_bytes(s["q"], s["k"], c["seq"], c["window"], c["sinks"]),
                                  dtype=torch.uint8, device=DEV)
        B.op_window_attention_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], c["seq"], c["window"], c["sinks"], s["dq"],
                                  s["dk"], s["dv"], s["ws"], lens=s["lens"])
        return {n: s[n] for n in ("o", "lse", "dq", "dk", "dv")}
    return _plain_rotary(s) if c["kind"] == "rotary" else _plain_window(s)


def _turn(x, cos, sin, rot, interleaved):
    """The first `rot` elements of every vector turned: (a, b) -> (a cos - b sin, b cos + a sin) for each pair."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_rotary(s):
    c, dt = s["case"], s["q"].dtype
    T, rot = c["batch"] * c["seq"], c["rot"]
    pos = torch.arange(T, device=DEV) % c["seq"] if s["pos"] is None else s["pos"]
    angle = pos.double()[:, None, None] * s["freq"].double()
    cos, sin = (angle.cos() * s["scale"]).float(), (angle.sin() * s["scale"]).float()

    def norm(x, g):
        x = x.float()
        if g is None:
            return x, x, None
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        return x * r * g.float(), x * r, r

    nq, xq, rq = norm(s["q"], s["qg"])
    nk, xk, rk = norm(s["k"], s["kg"])
    out = {"qo": _turn(nq, cos, sin, rot, c["interleaved"]).to(dt), "ko": _turn(nk, cos, sin, rot, c["interleaved"]).to(dt)}
    if not c["train"]:
        return out

    def back(dy, g, unit, r):
        dn = _turn(dy.float(), cos, -sin, rot, c["interleaved"])
        if g is None:
            return dn.to(dt), None
        du = dn * g.float()
        return ((du - unit * (du * unit).mean(-1, keepdim=True)) * r).to(dt), (dn * unit).sum((0, 1)).to(dt)

    out["dq"], out["dqg"] = back(s["dqo"], s["qg"], xq, rq)
    out["dk"], out["dkg"] = back(s["dko"], s["kg"], xk, rk)
    return out


def _plain_window(s):
    c, dt = s["case"], s["q"].dtype
    Bn, S, nq, nk, dh = c["batch"], c["seq"], c["q_heads"], c["kv_heads"], c["dim"]
    g, scale = nq // nk, 1 / math.sqrt(dh)
    heads = lambda x: x.float().view(Bn, S, nk, -1, dh).permute(0, 2, 3, 1, 4)   # noqa: E731  [batch, key head, query head of it, token, dim]
    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    i, j = torch.arange(S, device=DEV)[:, None], torch.arange(S, device=DEV)
    seen = (j <= i) & ((i - j < c["window"]) | (j < c["sinks"]))
    seen = seen.expand(Bn, S, S)
    if s["lens"] is not None:
        n = s["lens"].view(Bn, 1, 1)
        seen = seen & (i < n) & (j < n)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    l = p.sum(-1, keepdim=True)
    p.div_(torch.where(l > 0, l, torch.ones_like(l)))                             # a row that sees nothing: zeros
    o = torch.matmul(p, v)
    rows = lambda t: t.permute(0, 3, 1, 2, 4).reshape(Bn * S, -1, dh).to(dt)       # noqa: E731
    out = {"o": rows(o), "lse": (m + l.log()).view(Bn, nq, S)}
    if not c["train"]:
        return out
    do = heads(s["do"])
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    out["dq"] = rows(torch.matmul(ds, k))
    # a key head's gradient: the sum over its query heads
    out["dk"] = rows(torch.matmul(ds.transpose(-1, -2).reshape(Bn, nk, g, S, S), q).sum(2, keepdim=True))
    del ds
    out["dv"] = rows(torch.matmul(p.transpose(-1, -2).reshape(Bn, nk, g, S, S), do).sum(2, keepdim=True))
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    T, nq, nk, dh = case["batch"] * case["seq"], case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rotary":   # in and out; with the gradient the same again
        n = T * (nq + nk) * dh
        return {"bytes": (4 if case["train"] else 2) * n * e, "flops": (20 if case["train"] else 8) * n}

    def pairs(n):   # of a query and a key it sees: the window's, and the first keys that the window has left behind
        w = min(case["window"], n)
        left = n - w
        first = min(left, case["sinks"])
        return w * (w + 1) // 2 + left * w + first * (first + 1) // 2 + (left - first) * case["sinks"]

    read = sum(_lens(case))
    # q, k, v; o and the log-sum-exps
    moved = (nq + 2 * nk) * read * dh * e + nq * T * (dh * e + 4)
    if case["train"]:   # the gradient of o; dq, dk, dv
        moved += nq * read * dh * e + (nq + 2 * nk) * T * dh * e
    return {"bytes": moved, "flops": (14 if case["train"] else 4) * nq * dh * sum(map(pairs, _lens(case)))}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_rotary(s):
    c = s["case"]
    rot, T = c["rot"], c["batch"] * c["seq"]
    pos = s["pos"].double() if s["pos"] is not None else torch.arange(T, device=DEV).remainder(c["seq"]).double()
    spin = torch.polar(torch.full((T, 1, rot // 2), float(s["scale"]), dtype=torch.float64, device=DEV),
                       torch.outer(pos, s["freq"].double())[:, None])
    out = {}
    for name, gain in (("q", "qg"), ("k", "kg")):
        x = s[name].double().requires_grad_()
        g = None if s[gain] is None else s[gain].double().requires_grad_()
        n = x if g is None else x / (x.square().sum(-1, keepdim=True) / c["dim"] + EPS).sqrt() * g
        pairs = n[..., :rot].unflatten(-1, (rot // 2, 2)) if c["interleaved"] else n[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * spin)
        z = z if c["interleaved"] else z.transpose(-1, -2)
        y = torch.cat((z.flatten(-2), n[..., rot:]), -1)
        out[name + "o"] = y.detach()
        if c["train"]:
            grads = torch.autograd.grad(y, [x] if g is None else [x, g], s["d" + name + "o"].double())
            out["d" + name], out["d" + gain] = grads[0], None if g is None else grads[1]
    return out


def _exact_window(s):
    c = s["case"]
    Bn, S, nq, nk, dh = c["batch"], c["seq"], c["q_heads"], c["kv_heads"], c["dim"]
    shape = lambda n: (Bn, S, n, dh)   # noqa: E731
    zeros = lambda n: torch.zeros(shape(n), dtype=torch.float64, device=DEV)   # noqa: E731
    q, k, v, do = (s[n].double().reshape(shape(-1)) for n in ("q", "k", "v", "do"))
    out = {"o": zeros(nq), "lse": torch.full((Bn, nq, S), -math.inf, dtype=torch.float64, device=DEV)}
    if c["train"]:
        out.update(dq=zeros(nq), dk=zeros(nk), dv=zeros(nk))
    lens = [S] * Bn if s["lens"] is None else s["lens"].tolist()
    at = torch.arange(S, device=DEV)
    hidden = (at[:, None] < at) | ((at[:, None] - at >= c["window"]) & (at >= c["sinks"]))
    for b, n in enumerate(lens):
        for h in range(nq if n else 0):
            kh = h * nk // nq
            leaf = [t.detach().requires_grad_() for t in (q[b, :n, h], k[b, :n, kh], v[b, :n, kh])]
            x = (leaf[0] @ leaf[1].T / dh ** 0.5).masked_fill(hidden[:n, :n], -math.inf)
            o = torch.softmax(x, -1) @ leaf[2]
            out["o"][b, :n, h], out["lse"][b, h, :n] = o.detach(), torch.logsumexp(x.detach(), -1)
            if c["train"]:
                dq, dk, dv = torch.autograd.grad(o, leaf, do[b, :n, h])
                out["dq"][b, :n, h] = dq
                out["dk"][b, :n, kh] += dk
                out["dv"][b, :n, kh] += dv
    return {n: t if n == "lse" else t.flatten(0, 1) for n, t in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rotary(s) if case["kind"] == "rotary" else _exact_window(s)
