"""Attention with a sliding window and first keys that stay visible (dp_op_window_attention_fwd / _bwd) against the formulas in
64 bits.

Tolerances, per element, from what each step may round (u = 2^-24 is half a step of fp32; h = 2^-8, half a step of bf16, for bf16
tensors, else u):
  a logit x = scale <q, k>: a sum of dh products, off by (dh + 4) u scale <|q|, |k|>; P = exp(x - lse) by that and the row sum's
    share of it (twice), and 8 u for the exponential;  call it P e
  o = P V: P rounded to h (bf16), e, a sum of n terms n u, the result h:       <P, |v|> (h' + 2 e + n u) + h |o|
  D = <dO, O> takes the rounded o:                                              <|dO|, error of o> + (dh + 4) u <|dO|, |o|>
  dS = P (dP - D):   P ((e + h') |dP - D| + error of D + (dh + 4) u <|dO|, |v|>)
  dQ, dK, dV: sums of those errors times |k|, |q|, |dO|, n u of the sum of magnitudes, the result h
with h' = h in bf16 (P and dS are rounded for the products they go into), 0 in fp32; n the number of terms.  As these add up the
worst of every rounding, the whole tensor is held to 2 h in the 2-norm as well (bf16: two roundings of independent elements)."""
import ctypes as C
import math

import pytest
import torch

from paper_2505_05856_amd import binding as B

DEV = "cuda:0"
U = 2.0 ** -24
gpu = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def seen(n, window, sinks, device):
    i, j = torch.arange(n, device=device)[:, None], torch.arange(n, device=device)
    return (j <= i) & ((i - j < window) | (j < sinks))


def reference(d, Bn, S, window, sinks, lens, scale, dt):
    """Results and tolerances, one head at a time, on the inputs' device."""
    T, nq, dh = d["q"].shape
    nk = d["k"].shape[1]
    dev = d["q"].device
    h = 2.0 ** -8 if dt == BF else U
    hp = h if dt == BF else 0.0
    z = lambda n, *s: torch.zeros(T, n, dh, dtype=torch.float64, device=dev)   # noqa: E731
    out = {n: z(c) for n, c in (("o", nq), ("dq", nq), ("dk", nk), ("dv", nk))}
    tol = {n: torch.zeros_like(t) for n, t in out.items()}
    out["lse"] = torch.full((Bn, nq, S), -math.inf, dtype=torch.float64, device=dev)
    tol["lse"] = torch.zeros_like(out["lse"])
    for b, n in enumerate([S] * Bn if lens is None else lens):
        n = max(0, min(S, n))
        if n == 0:
            continue
        see = seen(n, window, sinks, dev)
        for hq in range(nq):
            hk = hq // (nq // nk)
            rows = slice(b * S, b * S + n)
            q, k, v, g = d["q"][rows, hq].double(), d["k"][rows, hk].double(), d["v"][rows, hk].double(), d["do"][rows, hq].double()
            x = (scale * q @ k.T).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(x, -1)
            p = torch.exp(x - lse[:, None])
            ex = ((dh + 4) * U * scale * (q.abs() @ k.abs().T)).masked_fill(~see, 0)
            e = 2 * ex.amax(-1, keepdim=True) + 16 * U
            nu = n * U
            o = p @ v
            to = (p * (hp + 2 * e + nu)) @ v.abs() + h * o.abs()
            D, tD = (g * o).sum(-1, keepdim=True), (g.abs() * to).sum(-1, keepdim=True) + (dh + 4) * U * (g * o).abs().sum(-1, keepdim=True)
            dp = g @ v.T
            ds = p * (dp - D)
            tds = p * ((e + hp) * (dp - D).abs() + tD + (dh + 4) * U * (g.abs() @ v.abs().T))
            out["o"][rows, hq], tol["o"][rows, hq] = o, to
            out["lse"][b, hq, :n], tol["lse"][b, hq, :n] = lse, e[:, 0] + 8 * U * lse.abs()
            out["dq"][rows, hq], tol["dq"][rows, hq] = scale * ds @ k, scale * (tds + nu * ds.abs()) @ k.abs()
            out["dk"][rows, hk] += scale * ds.T @ q
            tol["dk"][rows, hk] += scale * (tds + nu * nq * ds.abs()).T @ q.abs()
            out["dv"][rows, hk] += p.T @ g
            tol["dv"][rows, hk] += (p * (hp + 2 * e + nu * nq)).T @ g.abs()
    for n in ("dq", "dk", "dv"):
        tol[n] += h * out[n].abs()
    return out, tol


def make(Bn, S, nq, nk, dh, dt, seed, lens=None, sd=1.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda n, sd=1.0: (torch.randn(Bn * S, n, dh, generator=gen) * sd).to(dt).to(DEV)   # noqa: E731
    d = {"q": r(nq, sd), "k": r(nk), "v": r(nk), "do": r(nq)}
    if lens is not None:   # rows past a sample's length hold anything
        for b, n in enumerate(lens):
            for t in d.values():
                t[b * S + max(0, n):(b + 1) * S] = float("nan")
    return d


def run(d, Bn, S, window, sinks, lens=None, scale=None, packed=False, bwd=True, stream=None):
    q, k, v, do = d["q"], d["k"], d["v"], d["do"]
    T, nq, dh = q.shape
    nk = k.shape[1]
    nan = lambda t: torch.full_like(t, float("nan"))   # noqa: E731
    dq, dk, dv = nan(q), nan(k), nan(v)
    if packed:
        x, y = torch.cat((q, k, v), 1), torch.full((T, nq + 2 * nk, dh), 7.0, dtype=q.dtype, device=DEV)
        q, k, v = x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:]
        dq, dk, dv = y[:, :nq], y[:, nq:nq + nk], y[:, nq + nk:]
    o, lse = nan(do), torch.full((Bn, nq, S), float("nan"), device=DEV)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    B.op_window_attention_fwd(q, k, v, S, window, sinks, o, lse, lens=ln, scale=scale, stream=stream)
    out = {"o": o, "lse": lse}
    if bwd:
        ws = torch.full((B.op_window_attention_workspace_bytes(q, k, S, window, sinks) // 4,), float("nan"), device=DEV)
        B.op_window_attention_bwd(q, k, v, o, lse, do, S, window, sinks, dq, dk, dv, ws, lens=ln, scale=scale, stream=stream)
        out.update(dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    return out


def check(got, want, tol, dt):
    for n, t in got.items():
        x, y = t.double(), want[n]
        if n == "lse":
            empty = y == -math.inf
            assert torch.equal(x == -math.inf, empty), n
            x, y, e = x[~empty], y[~empty], tol[n][~empty]
        else:
            e = tol[n]
        assert torch.isfinite(x).all(), n
        bad = (x - y).abs() > e + 1e-30
        assert not bad.any(), (n, bad.nonzero()[:4].tolist(), ((x - y).abs() / (e + 1e-30)).max().item())
        big = y.norm()
        if dt == BF and n != "lse" and big > 1e-6 * math.sqrt(max(y.numel(), 1)):
            assert (x - y).norm() <= 2.0 ** -7 * big, (n, ((x - y).norm() / big).item())


def case(Bn, S, nq, nk, dh, window, sinks, lens=None, dt=BF, scale=None, packed=False, seed=1, sd=1.0):
    d = make(Bn, S, nq, nk, dh, dt, seed, lens, sd)
    want, tol = reference(d, Bn, S, window, sinks, lens, dh ** -0.5 if scale is None else scale, dt)
    check(run(d, Bn, S, window, sinks, lens, scale, packed), want, tol, dt)


# sequence lengths around a row, a key tile, a query tile; windows around them; sinks inside the window, past it, past the sequence
SHAPES = [(1, 1, 1, 0), (1, 2, 1, 0), (2, 3, 2, 1), (1, 63, 7, 3), (2, 64, 64, 0), (1, 65, 64, 1), (1, 127, 65, 4), (2, 128, 1, 0), (1, 129, 128, 64),
          (1, 200, 33, 65), (1, 257, 100, 16), (1, 300, 2, 130), (1, 320, 500, 0), (1, 391, 64, 1), (1, 400, 130, 400), (1, 513, 2 ** 31 - 1, 2 ** 31 - 1)]


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("Bn,S,window,sinks", SHAPES)
def test_lengths_windows_and_sinks(Bn, S, window, sinks, dh, dt):
    case(Bn, S, 2, 1, dh, window, sinks, dt=dt, packed=S % 2 == 0)


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("nq,nk,dh", [(3, 3, 8), (2, 2, 32), (6, 2, 80), (8, 1, 96), (5, 5, 64), (12, 4, 128), (2, 1, 136), (2, 2, 256), (1, 1, 16), (4, 2, 24)])
def test_heads(nq, nk, dh, dt):
    case(2, 150, nq, nk, dh, 50, 3, dt=dt, packed=True)


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("lens", [[0, 0, 0, 0], [1, 0, 260, 128], [64, 65, 63, 300], [127, 129, 200, 2], [-5, 1000, 300, 0]])
def test_padded_samples(lens, dt):
    case(4, 300, 4, 2, 64, 70, 5, lens=lens, dt=dt)
    case(4, 300, 4, 1, 128, 300, 200, lens=lens, dt=dt, packed=True)


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
def test_scale_and_steep_logits(dt):
    case(1, 200, 2, 1, 64, 90, 4, dt=dt, scale=0.5, sd=3.0)
    case(1, 200, 2, 2, 128, 90, 4, dt=dt, scale=1.0, sd=4.0)


@gpu
@pytest.mark.parametrize("dt,S,window,sinks,nq,nk", [(BF, 2500, 300, 10, 4, 1), (BF, 3333, 1000, 140, 2, 2), (BF, 2050, 2050, 0, 3, 3), (F32, 1500, 400, 5, 2, 1)])
def test_long(dt, S, window, sinks, nq, nk):
    """Rows whose queries and keys go through many tiles, first keys that thousands of queries see."""
    case(1, S, nq, nk, 128 if dt == BF else 64, window, sinks, dt=dt)
    case(2, S // 2, nq, nk, 64, window // 3, sinks, lens=[S // 2, S // 3], dt=dt, packed=True)


@gpu
@pytest.mark.parametrize("Bn,S,nq,nk,dh,window,sinks,lens", [(4, 130, 66, 66, 64, 33, 2, None), (3, 300, 64, 8, 128, 70, 5, [300, 129, 0]), (1, 390, 180, 90, 40, 512, 0, None),
                                                             (2, 513, 54, 27, 96, 1, 0, [511, 513]), (9, 90, 58, 29, 128, 31, 40, [90, 1, 33, 64, 65, 89, 2, 32, 31])])
def test_short_windows_of_many_heads(Bn, S, nq, nk, dh, window, sinks, lens):
    case(Bn, S, nq, nk, dh, window, sinks, lens=lens, packed=lens is not None)


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("Bn,S,nq,nk,window,sinks,lens", [(1, 1000, 8, 8, 200, 3, None), (2, 700, 8, 4, 100, 130, [700, 333]), (1, 2000, 1, 1, 300, 1, None),
                                                          (5, 400, 3, 3, 64, 0, None), (8, 300, 2, 1, 300, 0, None)])
def test_walks_of_keys_dealt_and_cut(Bn, S, nq, nk, window, sinks, lens, dt):
    """Numbers of key heads that eight does and does not divide, whole and shortened walks, pieces of both."""
    case(Bn, S, nq, nk, 128 if dt == BF else 64, window, sinks, lens=lens, dt=dt)


@gpu
@pytest.mark.parametrize("Bn,S,nq,nk,dh,window,sinks,lens", [(1, 450, 8, 1, 128, 450, 0, None), (2, 500, 8, 1, 64, 330, 3, [500, 217]), (1, 700, 16, 2, 96, 300, 140, None),
                                                             (3, 390, 12, 1, 40, 129, 2, [390, 64, 1]), (1, 1300, 6, 1, 128, 700, 5, None), (8, 200, 22, 2, 64, 200, 0, None)])
def test_many_query_heads_to_a_key_head(Bn, S, nq, nk, dh, window, sinks, lens):
    """Walks of the keys that are long because many heads share them."""
    case(Bn, S, nq, nk, dh, window, sinks, lens=lens, packed=lens is None)


@gpu
@pytest.mark.parametrize("S,window", [(300, 2), (300, 5), (200, 64), (900, 200), (400, 400)])
def test_gradients_are_rounded_twice(S, window):
    """Where a query sees few keys the rounding of O must not reach dQ and dK through <dO, O>: what is left are the rounding of dS and
    that of the result, independent from element to element, each at most h of its element and h / sqrt 3 in the mean square."""
    d = make(2, S, 4, 2, 128, BF, 17, sd=1.4)
    want, _ = reference(d, 2, S, window, 0, None, 128 ** -0.5, BF)
    got = run(d, 2, S, window, 0)
    for n in ("dq", "dk"):
        err = (got[n].double() - want[n]).norm() / want[n].norm()
        assert err < math.sqrt(2 / 3) * 2.0 ** -8, (n, err.item())


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
def test_gradients_against_differences(dt):
    d = make(1, 40, 2, 1, 64, dt, 5)
    got = run(d, 1, 40, 11, 2)

    def loss(**kw):
        x = {n: (kw.get(n, d[n])).double() for n in ("q", "k", "v")}
        y = torch.zeros((), dtype=torch.float64, device=DEV)
        for h in range(2):
            a = (x["q"][:, h] @ x["k"][:, 0].T / 8).masked_fill(~seen(40, 11, 2, DEV), -math.inf)
            y = y + (torch.softmax(a, -1) @ x["v"][:, 0] * d["do"][:, h].double()).sum()
        return y
    for n, at in (("q", (3, 1, 7)), ("q", (39, 0, 63)), ("k", (0, 0, 5)), ("k", (20, 0, 1)), ("v", (1, 0, 9)), ("v", (39, 0, 0))):
        e = torch.zeros(d[n].shape, dtype=torch.float64, device=DEV)
        e[at] = 1e-5
        fd = (loss(**{n: d[n].double() + e}) - loss(**{n: d[n].double() - e})) / 2e-5
        scale = got["d" + n].double().abs().max().item()
        assert abs(fd.item() - got["d" + n][at].item()) < (2 * 2.0 ** -7 if dt == BF else 1e-5) * scale, (n, at)


@gpu
def test_a_window_of_the_sequence_is_causal_attention():
    """Against the library's causal attention (equal numbers of heads): the same softmax within the roundings both make."""
    Bn, S, n, dh = 2, 300, 4, 64
    d = make(Bn, S, n, n, dh, BF, 9)
    got = run(d, Bn, S, S, 0, packed=True)
    qkv = torch.cat([d[x].reshape(Bn * S, -1) for x in "qkv"], 1).contiguous()
    o, lse = torch.empty(Bn * S, n * dh, dtype=BF, device=DEV), torch.empty(Bn, n, S, device=DEV)
    B.op_attention_fwd(qkv, Bn, S, n, dh, True, o, lse)
    dqkv, ws = torch.empty_like(qkv), torch.empty(B.op_workspace_bytes(Bn * S, n), dtype=torch.uint8, device=DEV)
    B.op_attention_bwd(qkv, o, lse, d["do"].reshape(Bn * S, -1).contiguous(), Bn, S, n, dh, True, dqkv, ws)
    for a, b in ((got["o"].reshape(Bn * S, -1), o), (torch.cat([got[x].reshape(Bn * S, -1) for x in ("dq", "dk", "dv")], 1), dqkv)):
        assert (a.double() - b.double()).norm() <= 2.0 ** -7 * b.double().norm()
    assert (got["lse"] - lse).abs().max() < 1e-4


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
def test_bad_numbers_stay_in_their_sample_and_what_is_hidden_is_not_read(dt):
    Bn, S = 3, 200
    d = make(Bn, S, 4, 2, 64, dt, 11)
    clean = run(d, Bn, S, 60, 2)
    d["k"][S + 100], d["v"][S + 120] = float("nan"), float("inf")
    got = run(d, Bn, S, 60, 2)
    for n in ("o", "dq", "dk", "dv"):
        for b in (0, 2):
            assert torch.equal(got[n][b * S:(b + 1) * S], clean[n][b * S:(b + 1) * S]), n
    assert torch.isnan(got["o"][S + 100]).all()
    # rows past a sample's length, whatever they hold, change nothing
    lens = [150, 200, 0]
    e = make(Bn, S, 4, 2, 64, dt, 11)
    f = make(Bn, S, 4, 2, 64, dt, 11, lens=lens)
    a, b = run(e, Bn, S, 60, 2, lens), run(f, Bn, S, 60, 2, lens)
    assert all(torch.equal(a[n], b[n]) for n in a)


@gpu
def test_outputs_alone_and_repeatable():
    d = make(2, 333, 8, 2, 128, BF, 12)
    a, b = run(d, 2, 333, 100, 4), run(d, 2, 333, 100, 4)
    assert all(torch.equal(a[n], b[n]) for n in a)
    o, lse = torch.full_like(a["o"], float("nan")), torch.full_like(a["lse"], float("nan"))
    B.op_window_attention_fwd(d["q"], d["k"], d["v"], 333, 100, 4, o, None)
    B.op_window_attention_fwd(d["q"], d["k"], d["v"], 333, 100, 4, None, lse)
    torch.cuda.synchronize()
    assert torch.equal(o, a["o"]) and torch.equal(lse, a["lse"])


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
def test_any_alignment(dt):
    """Operands one element off an allocation's start, and row strides that are no whole 16 bytes."""
    Bn, S, nq, nk, dh = 1, 130, 2, 1, 64
    d = make(Bn, S, nq, nk, dh, dt, 13)
    want, tol = reference(d, Bn, S, 40, 2, None, dh ** -0.5, dt)

    def odd(t):
        n, ld = t.shape[1], t.shape[1] * dh + 3
        x = torch.full((S * ld + 1,), float("nan"), dtype=dt, device=DEV)[1:].as_strided((S, n, dh), (ld, dh, 1))
        x.copy_(t)
        return x
    q, k, v, do = (odd(d[n]) for n in ("q", "k", "v", "do"))
    o, lse, dq, dk, dv = odd(d["q"]), torch.empty(Bn, nq, S, device=DEV), odd(d["q"]), odd(d["k"]), odd(d["v"])
    ws = torch.empty(B.op_window_attention_workspace_bytes(q, k, S, 40, 2), dtype=torch.uint8, device=DEV)
    B.op_window_attention_fwd(q, k, v, S, 40, 2, o, lse)
    B.op_window_attention_bwd(q, k, v, o, lse, do, S, 40, 2, dq, dk, dv, ws)
    torch.cuda.synchronize()
    check({"o": o, "dq": dq, "dk": dk, "dv": dv, "lse": lse}, want, tol, dt)


@gpu
@pytest.mark.parametrize("ld", [1 << 20, 5 << 20])
def test_far_rows(ld):
    """Rows so far apart that offsets pass 2^32 bytes between samples, or inside one."""
    Bn, S, nq, nk, dh = 3, 600, 2, 1, 64
    d = make(Bn, S, nq, nk, dh, BF, 14)
    room = torch.empty(Bn * S * ld, dtype=BF, device=DEV)
    far = lambda n, at: room[at:].as_strided((Bn * S, n, dh), (ld, dh, 1))   # noqa: E731
    q, k, v, do = far(2, 0), far(1, 128), far(1, 192), far(2, 256)
    for x, n in ((q, "q"), (k, "k"), (v, "v"), (do, "do")):
        x.copy_(d[n])
    o, dq, dk, dv = far(2, 384), far(2, 512), far(1, 640), far(1, 704)
    lse = torch.empty(Bn, nq, S, device=DEV)
    ws = torch.empty(B.op_window_attention_workspace_bytes(q, k, S, 90, 3), dtype=torch.uint8, device=DEV)
    B.op_window_attention_fwd(q, k, v, S, 90, 3, o, lse)
    B.op_window_attention_bwd(q, k, v, o, lse, do, S, 90, 3, dq, dk, dv, ws)
    torch.cuda.synchronize()
    want, tol = reference(d, Bn, S, 90, 3, None, dh ** -0.5, BF)
    check({"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, want, tol, BF)


@gpu
@pytest.mark.parametrize("dt", [BF, F32])
def test_captured_and_replayed(dt):
    """Two graphs that share a workspace and an output, replayed among eager work on another stream's order: the eager bits."""
    d = make(2, 700, 4, 1, 64, dt, 15)
    forms = [(150, 4), (700, 0)]
    want = [run(d, 2, 700, *f) for f in forms]
    q, k, v, do = d["q"], d["k"], d["v"], d["do"]
    o, lse = torch.empty_like(q), torch.empty(2, 4, 700, device=DEV)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(max(B.op_window_attention_workspace_bytes(q, k, 700, *f) for f in forms), dtype=torch.uint8, device=DEV)
    graphs = []
    for f in forms:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.op_window_attention_fwd(q, k, v, 700, *f, o, lse)
            B.op_window_attention_bwd(q, k, v, o, lse, do, 700, *f, dq, dk, dv, ws)
        graphs.append(g)
    for _ in range(3):
        for g, w in zip(graphs, want):
            for t in (o, lse, dq, dk, dv):
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            for n, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
                assert torch.equal(t, w[n]), n
            run(d, 2, 700, 33, 1)
    s = torch.cuda.Stream()   # a stream of the caller's own
    s.wait_stream(torch.cuda.current_stream())
    other = run(d, 2, 700, *forms[0], stream=s)
    assert all(torch.equal(other[n], want[0][n]) for n in other)


FAKE = 4096   # (never followed: every call here is refused before a launch)


def shape(**kw):
    d = dict(batch=2, seq=16, q_heads=4, kv_heads=2, head_dim=64, window=8, sinks=1, scale=0.125, ldq=256, ldk=128, ldv=128, ldo=256)
    d.update(kw)
    return B.WindowAttention(**d)


def fwd(s, dtype=1, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, lens=None, o=FAKE, lse=FAKE)
    a.update(kw)
    return B.lib().dp_op_window_attention_fwd(dtype, None if s is None else C.byref(s), *(a[n] for n in ("q", "k", "v", "lens", "o", "lse")), None)


def bwd(s, dtype=1, **kw):
    names = ("q", "k", "v", "lens", "o", "lse", "d_o", "dq", "dk", "dv", "ws")
    a = {n: FAKE for n in names}
    a.update(lens=None)
    a.update(kw)
    return B.lib().dp_op_window_attention_bwd(dtype, None if s is None else C.byref(s), *(a[n] for n in names), None)


def test_refusals():
    inval, unsupported = -1, -7
    assert fwd(None) == inval and bwd(None) == inval and fwd(shape(), dtype=2) == inval and bwd(shape(), dtype=-1) == inval
    for kw in (dict(batch=-1), dict(seq=-1), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=3), dict(head_dim=0), dict(window=0), dict(window=-4),
               dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(ldq=255), dict(ldk=127), dict(ldv=0),
               dict(ldo=-256)):
        assert fwd(shape(**kw)) == inval and bwd(shape(**kw)) == inval, kw
        assert B.lib().dp_op_window_attention_workspace_bytes(1, C.byref(shape(**kw))) == 0
    for kw in (dict(head_dim=60), dict(head_dim=264), dict(batch=70000, seq=70000)):
        big = dict(ldq=4096, ldk=4096, ldv=4096, ldo=4096)
        assert fwd(shape(**kw, **big)) == unsupported and bwd(shape(**kw, **big)) == unsupported, kw
    for n in ("q", "k", "v"):
        assert fwd(shape(), **{n: None}) == inval
    for n in ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "ws"):
        assert bwd(shape(), **{n: None}) == inval, n
    assert "window_attention_bwd" in B.lib().dp_last_error().decode()
    # nothing to do: nothing is touched
    nothing = {n: None for n in ("q", "k", "v", "o", "lse")}
    assert fwd(shape(seq=0), **nothing) == 0 and fwd(shape(batch=0), **nothing) == 0 and fwd(shape(), o=None, lse=None) == 0
    assert bwd(shape(batch=0), **nothing, d_o=None, dq=None, dk=None, dv=None, ws=None) == 0


def test_sizes_past_the_launches():
    """What 32-bit rows, or the threads of one launch, do not count is refused before anything is read."""
    wide = dict(ldq=1 << 40, ldk=1 << 40, ldv=1 << 40, ldo=1 << 40)
    for kw in (dict(batch=1, seq=2 ** 31 - 1), dict(batch=1, seq=2 ** 30 + 1), dict(batch=2 ** 20, seq=2 ** 11), dict(batch=2 ** 22, seq=1),
               dict(batch=1, seq=2 ** 29, q_heads=2, kv_heads=1), dict(batch=1, seq=1, q_heads=2 ** 30, kv_heads=1), dict(batch=2 ** 31 - 1, seq=1)):
        assert fwd(shape(**kw, **wide)) == -7 and bwd(shape(**kw, **wide)) == -7, kw
        assert B.lib().dp_op_window_attention_workspace_bytes(1, C.byref(shape(**kw, **wide))) == 0
    assert B.lib().dp_op_window_attention_workspace_bytes(1, C.byref(shape(batch=1, seq=2 ** 26, **wide))) > 0


def test_binding_refuses_tensors_of_the_host():
    t = torch.zeros(4, 2, 64)
    with pytest.raises(B.DpError) as e:
        B.op_window_attention_fwd(t, t, t, 4, 2, 0, t, None)
    assert e.value.status == "DP_E_INVAL"


@gpu
def test_binding_refusals():
    q, k = torch.zeros(8, 4, 64, device=DEV), torch.zeros(8, 2, 64, device=DEV)
    lse = torch.zeros(2, 4, 4, device=DEV)
    ok = dict(q=q, k=k, v=k, seq=4, window=3, sinks=0, o=q.clone(), lse=lse)
    B.op_window_attention_fwd(**ok)
    wide = torch.zeros(8, 4, 128, device=DEV)
    for kw in (dict(q=q.bfloat16()), dict(k=k.bfloat16()), dict(v=k[:7]), dict(q=q.view(8, 256)), dict(q=wide[..., ::2]), dict(q=wide[..., :64]),
               dict(k=torch.zeros(8, 3, 64, device=DEV)), dict(seq=3), dict(seq=0), dict(o=k), dict(lse=lse[:1]), dict(lse=lse.double()),
               dict(lens=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(lens=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(v=k.cpu()),
               dict(window=0), dict(scale=-1.0)):
        with pytest.raises(B.DpError):
            B.op_window_attention_fwd(**{**ok, **kw})
    ws = torch.empty(B.op_window_attention_workspace_bytes(q, k, 4, 3, 0), dtype=torch.uint8, device=DEV)
    full = dict(q=q, k=k, v=k.clone(), o=q.clone(), lse=lse, d_o=q.clone(), seq=4, window=3, sinks=0, dq=q.clone(), dk=k.clone(), dv=k.clone(), ws=ws)
    B.op_window_attention_bwd(**full)
    for kw in (dict(ws=None), dict(ws=ws[:-1]), dict(ws=ws.cpu()), dict(o=None), dict(lse=None), dict(d_o=k), dict(dq=torch.zeros(8, 8, 64, device=DEV)[:, :4]),
               dict(dv=q)):
        with pytest.raises(B.DpError):
            B.op_window_attention_bwd(**{**full, **kw})


@gpu
def test_with_norms_and_rotary_positions_as_a_block():
    """A packed projection through norms, rotary positions and windowed attention and back: the gradient of the projection and of
    the gains against automatic differentiation in 64 bits.  The block rounds q and k to bf16 on the way, and their gradients: a
    logit moves by 2 h of its terms, P by that, and each gradient by one more rounding, random in sign: 2^-5 in the 2-norm holds
    four times the 2^-7 of one such rounding."""
    Bn, S, nq, nk, dh, W, sinks = 2, 160, 4, 2, 64, 48, 2
    T = Bn * S
    gen = torch.Generator().manual_seed(21)
    qkv = torch.randn(T, nq + 2 * nk, dh, generator=gen).bfloat16().to(DEV)
    qg, kg = ((torch.randn(dh, generator=gen) * 0.1 + 1).bfloat16().to(DEV) for _ in range(2))
    do = torch.randn(T, nq, dh, generator=gen).bfloat16().to(DEV)
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float().to(DEV)
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
    qr, kr = torch.empty(T, nq, dh, dtype=BF, device=DEV), torch.empty(T, nk, dh, dtype=BF, device=DEV)
    o, lse = torch.empty_like(qr), torch.empty(Bn, nq, S, device=DEV)
    dqr, dkr, dqkv = torch.empty_like(qr), torch.empty_like(kr), torch.full_like(qkv, float("nan"))
    dqg, dkg = torch.empty_like(qg), torch.empty_like(kg)
    ws = torch.empty(max(B.op_window_attention_workspace_bytes(q, k, S, W, sinks), B.op_qk_rotary_workspace_bytes(T, nq, nk, dh)), dtype=torch.uint8, device=DEV)
    B.op_qk_rotary_fwd(q, k, qg, kg, freq, qr, kr, S)
    B.op_window_attention_fwd(qr, kr, v, S, W, sinks, o, lse)
    B.op_window_attention_bwd(qr, kr, v, o, lse, do, S, W, sinks, dqr, dkr, dqkv[:, nq + nk:], ws)
    B.op_qk_rotary_bwd(dqr, dkr, q, k, qg, kg, freq, dqkv[:, :nq], dqkv[:, nq:nq + nk], dqg, dkg, ws, S)
    torch.cuda.synchronize()
    x, a, b = qkv.double().requires_grad_(), qg.double().requires_grad_(), kg.double().requires_grad_()
    ang = (torch.arange(T, device=DEV) % S).double()[:, None, None] * freq.double()

    def rot(t, g):
        n = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g
        u, w = n[..., :32], n[..., 32:]
        return torch.cat((u * ang.cos() - w * ang.sin(), w * ang.cos() + u * ang.sin()), -1)
    Q, K, V = rot(x[:, :nq], a), rot(x[:, nq:nq + nk], b), x[:, nq + nk:]
    see, outs = seen(S, W, sinks, DEV), []
    for h in range(nq):
        hk = h // (nq // nk)
        parts = []
        for s in range(Bn):
            r = slice(s * S, (s + 1) * S)
            parts.append(torch.softmax((Q[r, h] @ K[r, hk].T / 8).masked_fill(~see, -math.inf), -1) @ V[r, hk])
        outs.append(torch.cat(parts))
    ref = torch.stack(outs, 1)
    grads = torch.autograd.grad(ref, (x, a, b), do.double())
    for got, want in ((o, ref.detach()), (dqkv, grads[0]), (dqg, grads[1]), (dkg, grads[2])):
        assert (got.double() - want).norm() <= 2.0 ** -5 * want.norm()
