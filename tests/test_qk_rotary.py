"""Norms of queries and keys with rotary positions (dp_op_qk_rotary_fwd / _bwd) against the formulas in 64 bits.

Tolerances, per element, u = 2^-24 (half a step of fp32): a vector's r = 1/sqrt(mean x^2 + eps) comes from a sum of at most 1024
squares, 16 in a row and the rest in a tree of up to six levels, so 22 u, halved by the root, and 2 u for the root; the products
with r and the gain 2 u; sin and cos 4 u (the fraction of a turn is rounded once, then the function); the turn 3 u of each product:
under 24 u of the larger element of the pair.  The backward's second sum adds 24 u of mean |g dn u|: 64 u of the vector's largest
element covers both.  A result in bf16 is rounded once more, by 2^-8 of its value at most."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_05856_amd import binding as B

DEV = "cuda:0"
U = 2.0 ** -24
gpu = pytest.mark.gpu


def frequencies(half, base=10000.0):
    return (base ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()


def turn(n, pos, freq, scale, inter):
    """n: fp64 [T, heads, dh]."""
    half = freq.numel()
    ang = pos.double()[:, None, None] * freq.double()
    c, s = scale * ang.cos(), scale * ang.sin()
    out = n.clone()
    ia = torch.arange(half) * 2 if inter else torch.arange(half)
    ib = ia + 1 if inter else ia + half
    a, b = n[..., ia], n[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    return out


def plain(x, gain, pos, freq, scale, eps, inter):
    n = x
    if gain is not None:
        n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain
    return turn(n, pos, freq, scale, inter)


def close(got, want, extra=0.0, what=""):
    """Elements of a vector: 64 u of its largest (see above), `extra` (absolute), and the rounding to bf16."""
    got, step = got.double().cpu(), 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    most = want.abs().amax(-1, keepdim=True) if want.dim() > 1 else want.abs()
    bad = (got - want).abs() > 64 * U * most * (1 + step) + step * want.abs() + extra
    assert not bad.any(), (what, bad.nonzero()[:3].tolist(), (got - want).abs().max().item())


def make(T, nq, nk, dh, dt, seed, norm=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, sd=1.0, mean=0.0: (torch.randn(*s, generator=g) * sd + mean).to(dt)   # noqa: E731
    return {"qkv": r(T, nq + 2 * nk, dh), "qg": r(dh, sd=0.2, mean=1.0) if norm else None, "kg": r(dh, sd=0.2, mean=1.0) if norm else None,
            "dqo": r(T, nq, dh), "dko": r(T, nk, dh)}


def run(d, nq, nk, dh, rot, inter, seq, pos=None, eps=1e-6, scale=1.0, packed=True, stream=None):
    """Forward and backward on the GPU; inputs as blocks of a packed tensor, or each on its own."""
    to = lambda t: None if t is None else t.to(DEV)   # noqa: E731
    dt, T = d["qkv"].dtype, d["qkv"].shape[0]
    qkv = to(d["qkv"])
    dqkv = torch.full_like(qkv, 7.0)
    q, k, dq, dk = qkv[:, :nq], qkv[:, nq:nq + nk], dqkv[:, :nq], dqkv[:, nq:nq + nk]
    if not packed:
        q, k, dq, dk = (t.contiguous() for t in (q, k, dq, dk))
    freq = frequencies(rot // 2).to(DEV) if rot else None
    qo, ko = (torch.full((T, n, dh), float("nan"), dtype=dt, device=DEV) for n in (nq, nk))
    qg, kg = to(d["qg"]), to(d["kg"])
    dqg, dkg = (None if g is None else torch.full_like(g, float("nan")) for g in (qg, kg))
    ws = torch.full((B.op_qk_rotary_workspace_bytes(T, nq, nk, dh) // 4,), float("nan"), device=DEV)
    form = {"seq": seq, "interleaved": inter, "eps": eps, "scale": scale, "positions": to(pos), "stream": stream}
    B.op_qk_rotary_fwd(q, k, qg, kg, freq, qo, ko, **form)
    B.op_qk_rotary_bwd(to(d["dqo"]), to(d["dko"]), q, k, qg, kg, freq, dq, dk, dqg, dkg, ws, **form)
    torch.cuda.synchronize()
    bits = torch.int16 if dt == torch.bfloat16 else torch.int32   # (a NaN is unchanged too)
    assert torch.equal(qkv.cpu().view(bits), d["qkv"].view(bits))
    if packed and T:   # nothing but the blocks of queries and keys is written
        assert torch.equal(dqkv[:, nq + nk:], torch.full_like(dqkv[:, nq + nk:], 7.0))
    return {"qo": qo, "ko": ko, "dq": dq, "dk": dk, "dqg": dqg, "dkg": dkg}


def check(got, d, nq, nk, dh, rot, inter, seq, pos=None, eps=1e-6, scale=1.0):
    T = d["qkv"].shape[0]
    pos = torch.arange(T) % seq if pos is None else pos
    freq = frequencies(rot // 2)
    for x, gain, name, dy, n0, n in ((d["qkv"][:, :nq], d["qg"], "q", d["dqo"], 0, nq), (d["qkv"][:, nq:nq + nk], d["kg"], "k", d["dko"], nq, nk)):
        x = x.double().requires_grad_()
        g = None if gain is None else gain.double().requires_grad_()
        y = plain(x, g, pos, freq, scale, eps, inter)
        close(got[name + "o"], y.detach(), what=name + "o")
        dx = torch.autograd.grad(y, [x] if g is None else [x, g], dy.double())
        # dx is a difference of g dn r and u mean(..): 64 u of the larger of the two
        most = 0.0
        if g is not None:
            r = 1 / (x.detach().square().mean(-1, keepdim=True) + eps).sqrt()
            dn = turn(dy.double(), pos, -freq, scale, inter).abs() * g.detach().abs()
            u = (x.detach() * r).abs()
            most = 64 * U * r * (dn.amax(-1, keepdim=True) + u.amax(-1, keepdim=True) * (dn * u).mean(-1, keepdim=True))
        close(got["d" + name], dx[0], extra=most, what="d" + name)
        if g is not None:   # a sum over T * n vectors, each term 64 u off; at most T * n additions deep in no more than 64-long runs and trees
            terms = turn(dy.double(), pos, -freq, scale, inter) * (x.detach() * (1 / (x.detach().square().mean(-1, keepdim=True) + eps).sqrt()))
            close(got["d" + name + "g"], dx[1], extra=(64 + 512) * U * terms.abs().sum((0, 1)) + 1e-30, what="d" + name + "g")
    if got["dqg"] is None:
        assert d["qg"] is None


SHAPES = [  # tokens, query heads, key heads, head dimension, elements turned, sequence
    (1, 1, 1, 2, 2, 1), (1, 2, 1, 64, 64, 1), (5, 3, 1, 16, 0, 5), (7, 2, 2, 6, 4, 3), (130, 25, 25, 64, 32, 65), (33, 4, 1, 128, 128, 33),
    (50, 5, 0, 80, 40, 50), (50, 0, 3, 96, 96, 7), (19, 2, 1, 256, 64, 10), (9, 2, 2, 1024, 1024, 9), (11, 3, 3, 34, 18, 11),
    (4099, 2, 1, 48, 16, 4099), (9000, 8, 2, 32, 32, 1000)]


@gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,nq,nk,dh,rot,seq", SHAPES)
def test_forward_and_gradients(T, nq, nk, dh, rot, seq, dt):
    for inter in (False, True):
        for norm in (True, False):
            d = make(T, nq, nk, dh, dt, 7 + T, norm)
            check(run(d, nq, nk, dh, rot, inter, seq, packed=inter), d, nq, nk, dh, rot, inter, seq)


@gpu
def test_one_gain_alone_and_a_scale():
    for only in ("qg", "kg"):
        d = make(300, 4, 2, 64, torch.float32, 3)
        d[only] = None
        check(run(d, 4, 2, 64, 48, False, 100, scale=1.3, eps=0.0), d, 4, 2, 64, 48, False, 100, scale=1.3, eps=0.0)


@gpu
@pytest.mark.parametrize("inter", [False, True])
def test_far_and_negative_positions(inter):
    d = make(64, 2, 1, 64, torch.float32, 5)
    pos = torch.tensor([0, 1, -1, 131071, 1 << 20, (1 << 31) - 1, -(1 << 31), 99999999], dtype=torch.int32).repeat(8)
    check(run(d, 2, 1, 64, 64, inter, 1, pos=pos), d, 2, 1, 64, 64, inter, 1, pos=pos)


@gpu
def test_any_alignment_gives_the_aligned_result():
    """Operands one element off an allocation's start take the element-by-element form."""
    T, n, dh = 37, 3, 64
    x = torch.randn(T * n * dh + 1, device=DEV).bfloat16()
    freq = frequencies(32).to(DEV)
    out = torch.empty(T, n, dh, dtype=torch.bfloat16, device=DEV)
    none = out[:, :0]
    off = x[1:].view(T, n, dh)
    B.op_qk_rotary_fwd(off.clone(), none, None, None, freq, out, none, T)
    want = out.clone()
    for view in (off, off.clone()):
        y = torch.empty(T * n * dh + 1, dtype=torch.bfloat16, device=DEV)[1:].view(T, n, dh)
        B.op_qk_rotary_fwd(view, none, None, None, freq, y, none, T)
        assert torch.equal(y, want)


@gpu
def test_in_place_zero_vectors_and_empty():
    d = make(40, 4, 2, 64, torch.bfloat16, 9)
    d["qkv"][3] = 0   # a vector of zeros: r = 1/sqrt(eps), no NaN
    got = run(d, 4, 2, 64, 64, False, 40)
    check(got, d, 4, 2, 64, 64, False, 40)
    qkv, freq = d["qkv"].to(DEV), frequencies(32).to(DEV)
    q, k = qkv[:, :4], qkv[:, 4:6]
    B.op_qk_rotary_fwd(q, k, d["qg"].to(DEV), d["kg"].to(DEV), freq, q, k, 40)
    assert torch.equal(q, got["qo"]) and torch.equal(k, got["ko"])
    dqo, dko, ws = d["dqo"].to(DEV), d["dko"].to(DEV), torch.empty(B.op_qk_rotary_workspace_bytes(40, 4, 2, 64), dtype=torch.uint8, device=DEV)
    x = d["qkv"].to(DEV)
    gq, gk = torch.empty_like(d["qg"], device=DEV), torch.empty_like(d["kg"], device=DEV)
    B.op_qk_rotary_bwd(dqo, dko, x[:, :4].contiguous(), x[:, 4:6].contiguous(), d["qg"].to(DEV), d["kg"].to(DEV), freq, dqo, dko, gq, gk, ws, 40)
    assert torch.equal(dqo, got["dq"]) and torch.equal(dko, got["dk"]) and torch.equal(gq, got["dqg"]) and torch.equal(gk, got["dkg"])
    e = make(0, 4, 2, 64, torch.bfloat16, 9)
    got = run(e, 4, 2, 64, 64, False, 40)
    assert torch.equal(got["dqg"], torch.zeros_like(got["dqg"])) and torch.equal(got["dkg"], torch.zeros_like(got["dkg"]))


@gpu
def test_a_bad_token_stays_alone():
    """NaN and infinity in one token's projection reach no other token."""
    d = make(70, 4, 2, 64, torch.bfloat16, 10)
    clean = run(d, 4, 2, 64, 32, False, 70)
    d["qkv"][20, 1], d["qkv"][21, 5] = float("nan"), float("inf")
    got = run(d, 4, 2, 64, 32, False, 70)
    rows = [t for t in range(70) if t not in (20, 21)]
    for n in ("qo", "ko", "dq", "dk"):
        assert torch.equal(got[n][rows], clean[n][rows]), n
    # elements beyond the turned ones pass as they are
    e = make(4, 1, 1, 64, torch.float32, 11, norm=False)
    e["qkv"][1, 0, 40] = float("inf")
    assert run(e, 1, 1, 64, 32, False, 4)["qo"][1, 0, 40].item() == math.inf


@gpu
def test_gradients_against_differences():
    d = make(6, 2, 1, 16, torch.float32, 12)
    got = run(d, 2, 1, 16, 8, True, 6)
    q, g, pos, f = d["qkv"][:, :2].double(), d["qg"].double(), torch.arange(6), frequencies(4)
    loss = lambda q, g: (plain(q, g, pos, f, 1.0, 1e-6, True) * d["dqo"].double()).sum()   # noqa: E731
    h = 1e-5
    for t, n, i in ((0, 0, 0), (3, 1, 5), (5, 0, 15)):
        e = torch.zeros_like(q)
        e[t, n, i] = h
        assert abs((loss(q + e, g) - loss(q - e, g)) / (2 * h) - got["dq"][t, n, i].item()) < 1e-4
    e = torch.zeros_like(g)
    e[3] = h
    assert abs((loss(q, g + e) - loss(q, g - e)) / (2 * h) - got["dqg"][3].item()) < 1e-4


def shape(**kw):
    d = dict(rows=8, seq=8, q_heads=2, kv_heads=1, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, scale=1.0, ldq_in=128, ldk_in=64, ldq_out=128, ldk_out=64)
    d.update(kw)
    return B.QkRotary(**d)


FAKE = 4096   # (never followed: every call here is refused before a launch)


def fwd(s, dtype=0, **kw):
    a = dict(q=FAKE, k=FAKE, qg=None, kg=None, freq=FAKE, pos=None, qo=FAKE, ko=FAKE)
    a.update(kw)
    return B.lib().dp_op_qk_rotary_fwd(dtype, None if s is None else C.byref(s), a["q"], a["k"], a["qg"], a["kg"], a["freq"], a["pos"], a["qo"], a["ko"], None)


def bwd(s, dtype=0, **kw):
    a = dict(dqo=FAKE, dko=FAKE, q=FAKE, k=FAKE, qg=FAKE, kg=FAKE, freq=FAKE, pos=None, dq=FAKE, dk=FAKE, dqg=FAKE, dkg=FAKE, ws=FAKE)
    a.update(kw)
    return B.lib().dp_op_qk_rotary_bwd(dtype, C.byref(s), *(a[n] for n in ("dqo", "dko", "q", "k", "qg", "kg", "freq", "pos", "dq", "dk", "dqg", "dkg", "ws")), None)


def test_sizes_past_32_bits():
    far = dict(ldq_in=1 << 40, ldk_in=1 << 40, ldq_out=1 << 40, ldk_out=1 << 40)
    for kw in (dict(rows=2 ** 31 - 1), dict(rows=2 ** 30), dict(q_heads=2 ** 30, kv_heads=2 ** 30), dict(q_heads=0, kv_heads=2 ** 31 - 1)):
        assert fwd(shape(**kw, **far)) == -7 and bwd(shape(**kw, **far)) == -7, kw


def test_refusals():
    inval, unsupported = -1, -7
    assert fwd(None) == inval and fwd(shape(), dtype=2) == inval
    for kw in (dict(rows=-1), dict(seq=0), dict(q_heads=-1), dict(kv_heads=-1), dict(head_dim=0), dict(rot_dim=-2), dict(rot_dim=3), dict(rot_dim=66),
               dict(interleaved=2), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(scale=math.nan), dict(ldq_in=127), dict(ldk_in=0),
               dict(ldq_out=64), dict(ldk_out=63)):
        assert fwd(shape(**kw)) == inval and bwd(shape(**kw)) == inval, kw
    for dim in (63, 1026):
        assert fwd(shape(head_dim=dim, rot_dim=0, ldq_in=4096, ldk_in=4096, ldq_out=4096, ldk_out=4096)) == unsupported
    for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(freq=None)):
        assert fwd(shape(), **kw) == inval, kw
    for kw in (dict(dqo=None), dict(dko=None), dict(dq=None), dict(dk=None), dict(q=None), dict(k=None), dict(dqg=None), dict(dkg=None), dict(ws=None), dict(freq=None)):
        assert bwd(shape(), **kw) == inval, kw
    assert "qk_rotary_bwd" in B.lib().dp_last_error().decode()
    # nothing to do: nothing is touched
    assert fwd(shape(rows=0), q=None, k=None, qo=None, ko=None, freq=None) == 0
    assert fwd(shape(q_heads=0, kv_heads=0), q=None, k=None, qo=None, ko=None, freq=None) == 0
    assert bwd(shape(rows=0), qg=None, kg=None, ws=None) == 0


def test_workspace_size():
    assert B.op_qk_rotary_workspace_bytes(0, 4, 2, 64) == 2 * 64 * 4
    assert B.op_qk_rotary_workspace_bytes(1 << 30, 4, 2, 64) <= 1024 * 2 * 64 * 4
    assert B.op_qk_rotary_workspace_bytes(-1, 4, 2, 64) == 0


def test_binding_refuses_tensors_of_the_host():
    t = torch.zeros(4, 2, 64)
    with pytest.raises(B.DpError) as e:
        B.op_qk_rotary_fwd(t, t, None, None, None, t, t, 4)
    assert e.value.status == "DP_E_INVAL"


@gpu
def test_binding_refusals():
    q, k = torch.zeros(4, 2, 64, device=DEV), torch.zeros(4, 1, 64, device=DEV)
    f = torch.zeros(32, device=DEV)
    ok = dict(q=q, k=k, q_gain=None, k_gain=None, inv_freq=f, q_out=q.clone(), k_out=k.clone(), seq=4)
    B.op_qk_rotary_fwd(**ok)
    wide = torch.zeros(4, 2, 128, device=DEV)
    for kw in (dict(q=q.bfloat16()), dict(k=k.bfloat16()), dict(q=q[0]), dict(q=wide[..., ::2]), dict(q=wide[..., :64]), dict(k=k[:3]),
               dict(k_out=torch.zeros(4, 1, 32, device=DEV)), dict(q_gain=torch.ones(32, device=DEV)), dict(inv_freq=f.double()),
               dict(inv_freq=torch.zeros(33, device=DEV)), dict(positions=torch.zeros(4, device=DEV)),
               dict(positions=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(k=k.cpu()), dict(seq=0)):
        with pytest.raises(B.DpError):
            B.op_qk_rotary_fwd(**{**ok, **kw})
    g = torch.ones(64, device=DEV)
    full = dict(dq_out=q, dk_out=k, q=q, k=k, q_gain=g, k_gain=g, inv_freq=f, dq=q.clone(), dk=k.clone(), dq_gain=g.clone(), dk_gain=g.clone(),
                ws=torch.empty(B.op_qk_rotary_workspace_bytes(4, 2, 1, 64), dtype=torch.uint8, device=DEV), seq=4)
    B.op_qk_rotary_bwd(**full)
    for kw in (dict(ws=None), dict(ws=full["ws"][:-1]), dict(dq_gain=None), dict(dk_gain=g[:32]), dict(q=torch.zeros(4, 4, 64, device=DEV)[:, :2]), dict(q=None)):
        with pytest.raises(B.DpError):
            B.op_qk_rotary_bwd(**{**full, **kw})


@gpu
def test_captured_and_replayed():
    """One workspace, a graph of its own for the backward, replays among eager work: the eager bits every time."""
    d = make(1000, 8, 2, 64, torch.bfloat16, 13)
    want = run(d, 8, 2, 64, 64, False, 500)
    x, freq, qg, kg = d["qkv"].to(DEV), frequencies(32).to(DEV), d["qg"].to(DEV), d["kg"].to(DEV)
    q, k, dqo, dko = x[:, :8], x[:, 8:10], d["dqo"].to(DEV), d["dko"].to(DEV)
    out = {n: torch.empty_like(t) for n, t in want.items()}
    ws = torch.empty(B.op_qk_rotary_workspace_bytes(1000, 8, 2, 64), dtype=torch.uint8, device=DEV)
    dq, dk = torch.empty_like(x)[:, :8], torch.empty_like(x)[:, 8:10]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.op_qk_rotary_fwd(q, k, qg, kg, freq, out["qo"], out["ko"], 500)
        B.op_qk_rotary_bwd(dqo, dko, q, k, qg, kg, freq, dq, dk, out["dqg"], out["dkg"], ws, 500)
    for _ in range(4):
        for t in out.values():
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        out["dq"], out["dk"] = dq, dk
        for n in want:
            assert torch.equal(out[n], want[n]), n
        out["dq"], out["dk"] = torch.empty_like(dq), torch.empty_like(dk)
        run(d, 8, 2, 64, 64, False, 500)
