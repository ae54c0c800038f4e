"""Attention with a sliding window and sinks against its formulas in fp64: forward, gradients, the single-token step
on its ring cache, and the places where such kernels go wrong.

Tolerances, all derived from the roundings on the way (u = 2^-24; half: half a step of the output's type, 2^-8 of the
value for bf16 and 2^-24 for fp32):
  a score is a sum of d products, off by d u of its mass M = scale sum |q k|; with the factor, the subtraction of the
  maximum and the exponential, numerator and normaliser, P is off by eP = (2 (d + 4) M + 2 n + 8) u of itself;
  P and dS of bf16 rows that see few tokens enter in two parts, 2^-16 of themselves, otherwise rounded, 2^-8;
  y, kept for D = dy . y with 8 more bits, is off by 2^-16 there;
  products of sums add n u of their mass."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_10743_amd as K
    return K


def make(B, T, H, Hk, d, dtype, past=0, lengths=None, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    z = lambda *s: (size * torch.randn(*s, generator=g)).to(TYPES[dtype])
    x = dict(q=z(B, T, H, d), k=z(B, past + T, Hk, d), v=z(B, past + T, Hk, d), dy=z(B, T, H, d), len=None)
    if lengths is not None:
        x["len"] = torch.tensor(lengths, dtype=torch.int32)
    return x


def expected(x, window, sinks, scale=None, parts=True, grads=True):
    """The formulas in fp64 on the CPU: {name: (value, tolerance)}.  parts: the rows see few tokens."""
    q, k, v, dy = (x[n].double() for n in ("q", "k", "v", "dy"))
    bf16 = x["q"].dtype == torch.bfloat16
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    part = 0.0 if not bf16 else 2.0 ** -16 if parts else 2.0 ** -8
    B, T, H, d = q.shape
    Tk, Hk = k.shape[1:3]
    G, past = H // Hk, Tk - T
    scale = 1 / math.sqrt(d) if scale is None else scale
    n = torch.full((B,), Tk) if x["len"] is None else x["len"].long().clamp(0, Tk)
    p = past + torch.arange(T)[:, None]
    j = torch.arange(Tk)[None]
    see = (j <= p) & ((j > p - window) | (j < sinks))
    live = p[None] < n[:, None, None]                                     # [B, T, 1]
    see = (see[None] & live & (j[None] < n[:, None, None]))[:, None]      # [B, 1, T, Tk]
    qv, dyv = (torch.where(live[..., None], t, 0.0).permute(0, 2, 1, 3) for t in (q, dy))
    kk, vv = (torch.where((j[0][None] < n[:, None])[..., None, None], t, 0.0).permute(0, 2, 1, 3).repeat_interleave(G, 1)
              for t in (k, v))
    s = (scale * qv @ kk.transpose(-1, -2)).masked_fill(~see, -math.inf)
    M = (scale * qv.abs() @ kk.abs().transpose(-1, -2)).masked_fill(~see, 0.0).amax(-1, keepdim=True)
    top = s.amax(-1, keepdim=True).clamp_min(-1e300)
    e = torch.exp(s - top)
    tot = e.sum(-1, keepdim=True)
    P = e / torch.where(tot > 0, tot, 1.0)
    eP = (2 * (d + 4) * M + 2 * Tk + 8) * U
    y = P @ vv
    back = lambda t: t.permute(0, 2, 1, 3)
    ty = (P * (eP + part)) @ vv.abs()
    out = {"y": (back(y), back(ty + half * y.abs()))}
    if not grads:
        return out
    A = dyv.abs() @ vv.abs().transpose(-1, -2)
    dP = dyv @ vv.transpose(-1, -2)
    D = (dyv * y).sum(-1, keepdim=True)
    kept = 2.0 ** -24 if not bf16 else 2.0 ** -16 if parts else 2.0 ** -8
    eD = (dyv.abs() * (ty + kept * y.abs())).sum(-1, keepdim=True) + (d + 1) * U * (dyv * y).abs().sum(-1, keepdim=True)
    dS = P * (dP - D)
    tS = dS.abs() * (eP + part + 4 * U) + P * ((d + 1) * U * A + eD)
    share = lambda t: back(t.reshape(B, Hk, G, Tk, d).sum(2))
    dq = scale * dS @ kk
    tq = scale * (tS + Tk * U * dS.abs()) @ kk.abs()
    dk = share(scale * dS.transpose(-1, -2) @ qv)
    tk = share(scale * (tS + G * T * U * dS.abs()).transpose(-1, -2) @ qv.abs())
    dv = share(P.transpose(-1, -2) @ dyv)
    tv = share((P * (eP + part + G * T * U)).transpose(-1, -2) @ dyv.abs())
    out.update(dq=(back(dq), back(tq + half * dq.abs())), dk=(dk, tk + half * dk.abs()), dv=(dv, tv + half * dv.abs()))
    return out


def check(name, got, want):
    ref, tol = want
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, name
    assert torch.isfinite(got).all(), name
    worst = ((got - ref).abs() / (tol + 1e-35)).max().item() if got.numel() else 0.0
    print(f"{name} {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.2f} times the tolerance"


def dev(x):
    return {n: t if t is None else t.to(DEV) for n, t in x.items()}


def run(kla, x, window, sinks, scale=None):
    x = dev(x)
    out = kla.kla_window_attn_forward(x["q"], x["k"], x["v"], window, sinks, x["len"], scale=scale, save=True)
    g = kla.kla_window_attn_backward(x["q"], x["k"], x["v"], window, sinks, x["len"], out["y"], out["saved"], x["dy"],
                                     scale=scale)
    return dict(y=out["y"], **g)


CASES = [  # B, T, past, H, Hk, d, window, sinks, lengths
    (1, 1, 0, 1, 1, 64, 1, 0, None),
    (2, 2, 0, 2, 1, 16, 2, 1, None),
    (2, 33, 0, 2, 2, 32, 1, 0, None),
    (2, 65, 0, 4, 2, 64, 7, 3, None),
    (1, 129, 0, 3, 1, 128, 64, 1, None),
    (2, 130, 0, 2, 1, 16, 200, 5, None),
    (2, 200, 0, 2, 2, 128, 33, 64, None),
    (1, 191, 0, 2, 1, 64, 1, 4, None),
    (3, 100, 0, 6, 2, 32, 20, 2, [100, 0, 37]),
    (3, 77, 60, 2, 1, 64, 50, 3, [137, 1, 61]),
    (2, 5, 150, 4, 4, 128, 40, 10, [155, 152]),
    (1, 3, 190, 8, 1, 32, 500, 0, None),
    (2, 160, 3, 2, 1, 128, 128, 33, [-5, 1000]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:8])) + ("-len" if c[8] else ""))
def test_forward_and_gradients(kla, case, dtype):
    B, T, past, H, Hk, d, window, sinks, lengths = case
    x = make(B, T, H, Hk, d, dtype, past, lengths)
    got, ref = run(kla, x, window, sinks), expected(x, window, sinks)
    for n in ref:
        check(n, got[n], ref[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,T,G", [(256, 3, 900, 2), (700, 0, 700, 1), (100, 64, 1500, 2)])
def test_long_rows(kla, window, sinks, T, G, dtype):
    """Windows that run over many tiles, and first tokens seen by several segments of queries."""
    x = make(1, T, G, 1, 64, dtype, seed=3)
    got, ref = run(kla, x, window, sinks), expected(x, window, sinks, parts=window + sinks < 256)
    for n in ref:
        check(n, got[n], ref[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_queries_of_many_tokens(kla, dtype):
    """The keys are dealt to many workgroups and joined, with rows that see none of a part."""
    x = make(2, 9, 2, 1, 128, dtype, past=1400, lengths=[1409, 1403], seed=4)
    ref = expected(x, 1300, 2, parts=False)
    got = run(kla, x, 1300, 2)
    for n in ref:
        check(n, got[n], ref[n])
    x["len"] = torch.tensor([1409, 0], dtype=torch.int32)
    got = run(kla, x, 1300, 2)
    assert all((t[1] == 0).all() for t in got.values())


def test_scale_and_large_scores(kla):
    """Scores of some hundred: the largest takes nearly all of a row."""
    x = make(2, 70, 2, 2, 64, "f32", size=4.0, seed=6)
    for scale in (0.01, 1.0):
        got, ref = run(kla, x, 30, 2, scale), expected(x, 30, 2, scale)
        for n in ref:
            check(n, got[n], ref[n])


def test_gradients_are_differences(kla):
    """Central differences of the fp64 formulas against the kernel's fp32 gradients, in random directions."""
    x = make(2, 20, 4, 2, 32, "f32", past=6, lengths=[26, 19], seed=9)
    got = run(kla, x, 9, 2)
    gen = torch.Generator().manual_seed(1)
    for n in ("q", "k", "v"):
        d = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        f = lambda h: (expected({**x, n: x[n].double() + h * d}, 9, 2, grads=False)["y"][0] * x["dy"].double()).sum()
        diff = ((f(1e-5) - f(-1e-5)) / 2e-5).item()
        mine = (got["d" + n].double().cpu() * d).sum().item()
        mass = (got["d" + n].double().cpu() * d).abs().sum().item()
        assert abs(diff - mine) <= 1e-5 * mass, n   # h^2 and 1e-16 / h of the mass, and fp32 gradients


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_not_finite_values_stay_where_they_are_seen(kla, d, bad, dtype):
    """A value, a key, a query and an output gradient that are not finite reach the rows that see them and no other."""
    T, W, sinks = 150, 20, 2
    see = torch.tensor([[j <= p and (j > p - W or j < sinks) for j in range(T)] for p in range(T)])
    clean = make(1, T, 2, 1, d, dtype, seed=8)
    ref = expected(clean, W, sinks)   # of the rows without an influence, within the tolerance of any result
    for n, at in (("v", 70), ("k", 70), ("q", 70), ("dy", 70), ("v", 0)):
        x = {m: t if t is None else t.clone() for m, t in clean.items()}
        x[n][0, at, 0, 3] = bad
        got = run(kla, x, W, sinks)
        hit = torch.zeros(T, dtype=torch.bool)   # queries with an influence of it
        hit[at] = True
        if n in ("k", "v"):
            hit = see[:, at]
        keys = (see & hit[:, None]).any(0)       # tokens that those see
        for m, rows in (("y", ~hit if n != "dy" else hit | ~hit), ("dq", ~hit), ("dk", ~keys), ("dv", ~keys)):
            check(f"{n} {m}", got[m][0, rows.to(DEV)], tuple(t[0, rows] for t in ref[m]))
        if n == "v" or math.isnan(bad):
            assert n == "dy" or not torch.isfinite(got["y"][0, hit.to(DEV)].float()).all()


def test_rows_without_a_score(kla):
    """A row whose visible scores are all -inf has y = 0 and no gradient."""
    x = make(1, 40, 1, 1, 64, "f32", seed=2)
    x["q"][0, :, 0] = 0.0
    x["q"][0, 20, 0, 0] = 1.0
    x["k"][0, 16:21, 0, 0] = -math.inf
    x["q"][0, 16:20, 0, 0] = x["q"][0, 21:, 0, 0] = 1.0
    got = kla.kla_window_attn_forward(*(x[n].to(DEV) for n in ("q", "k", "v")), 5)["y"]
    assert (got[0, 20] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_the_ends(kla, dtype):
    """Rows past a sequence's tokens hold anything, are not read, and get zeros."""
    x = make(3, 90, 2, 1, 64, dtype, lengths=[90, 41, 0], seed=5)
    ref = expected(x, 30, 3)
    for n in ("q", "k", "v", "dy"):
        for b, end in ((1, 41), (2, 0)):
            x[n][b, end:] = math.nan
    got = run(kla, x, 30, 3)
    for n in ref:
        check(n, got[n], ref[n])
        assert (got[n][1, 41:] == 0).all() and (got[n][2] == 0).all()


def ring(x, n, window, sinks):
    """The caches of the first n tokens of k, v [T, Hk, d]."""
    out = [torch.zeros(sinks + window, *t.shape[1:], dtype=t.dtype) for t in x]
    for t in range(n):
        slot = t if t < sinks else sinks + (t - sinks) % window
        for o, y in zip(out, x):
            o[slot] = y[t]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,d,H,Hk", [(1, 0, 16, 1, 1), (7, 2, 64, 4, 2), (40, 5, 128, 3, 1), (100, 0, 32, 40, 2),
                                                 (9, 1, 16, 17, 1)])
def test_steps_follow_the_prompt(kla, window, sinks, d, H, Hk, dtype):
    """Caches from prompts of several lengths, then token by token: each step's y is the whole sequence's row."""
    B, T = 3, 60
    x = make(B, T, H, Hk, d, dtype, seed=11)
    ref = expected(x, window, sinks, parts=False, grads=False)["y"]
    X = dev(x)
    start = [0, 13, 50]
    out = kla.kla_window_attn_forward(X["q"], X["k"], X["v"], window, sinks,
                                      torch.tensor(start, dtype=torch.int32, device=DEV), want_cache=True)
    ck, cv = out["cache_k"], out["cache_v"]
    for b in range(B):
        rk, rv = ring((x["k"][b], x["v"][b]), start[b], window, sinks)
        assert torch.equal(ck[b].cpu(), rk) and torch.equal(cv[b].cpu(), rv)
    pos = torch.tensor(start, dtype=torch.int32, device=DEV)
    rows = torch.arange(B, device=DEV)
    for _ in range(10):
        at = pos.long()
        got = kla.kla_window_attn_step(X["q"][rows, at], X["k"][rows, at], X["v"][rows, at], ck, cv, pos, sinks)
        r, c = rows.cpu(), at.cpu()
        check("y", got["y"], (ref[0][r, c], ref[1][r, c]))
        pos += 1
    for b in range(B):
        rk, rv = ring((x["k"][b], x["v"][b]), start[b] + 10, window, sinks)
        assert torch.equal(ck[b].cpu(), rk) and torch.equal(cv[b].cpu(), rv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_reads_and_writes_its_slots_only(kla, dtype):
    """Slots without a token may hold anything, inactive sequences stay as they are; long caches dealt to many
    workgroups, positions far behind the ring's first turn."""
    t, S, H, Hk, d, window, sinks = TYPES[dtype], 4, 4, 2, 64, 1500, 6
    g = torch.Generator().manual_seed(3)
    z = lambda *s: torch.randn(*s, generator=g).to(t)
    q, k, v, ck, cv = z(S, H, d), z(S, Hk, d), z(S, Hk, d), z(S, 1506, Hk, d), z(S, 1506, Hk, d)
    pos = [3, 1000, -1, 2 ** 31 - 1]
    ck[0, 4:], cv[0, 4:], ck[1, 1001:], cv[1, 1001:], ck[2], cv[2] = (math.nan,) * 6
    X = [u.to(DEV) for u in (q, k, v, ck, cv)]
    y = kla.kla_window_attn_step(*X, torch.tensor(pos, dtype=torch.int32, device=DEV), sinks)["y"].cpu()
    for b, p in enumerate(pos):
        if p >= 0:
            slot = p if p < sinks else sinks + (p - sinks) % window
            ck[b, slot], cv[b, slot] = k[b], v[b]
    same = lambda a, b: torch.equal(a.cpu().contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    assert same(X[3], ck) and same(X[4], cv)
    assert (y[2] == 0).all()
    for b, p in enumerate(pos):
        if p < 0:
            continue
        n = min(p + 1, 1506)
        x = dict(q=q[b][None, None], k=ck[b:b + 1, :n], v=cv[b:b + 1, :n], dy=q[b][None, None], len=None)
        ref = expected(x, 1506, 0, parts=False, grads=False)["y"]
        check("y", y[b][None, None], ref)


def test_offsets_past_32_bits(kla):
    """Caches, keys and values of more than 2^31 elements: the last sequence, whose few tokens are known."""
    S, slots, Hk, d, window = 3, (1 << 20) + 8, 8, 128, 1 << 20
    cache = torch.zeros(2, S, slots, Hk, d, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator().manual_seed(5)
    z = lambda *s: torch.randn(*s, generator=g).bfloat16()
    q, k, v, old = z(S, Hk, d), z(S, Hk, d), z(S, Hk, d), z(2, 4, Hk, d)
    cache[0, 2, :4], cache[1, 2, :4] = old[0].to(DEV), old[1].to(DEV)
    y = kla.kla_window_attn_step(q.to(DEV), k.to(DEV), v.to(DEV), cache[0], cache[1],
                                 torch.tensor([-1, -1, 4], dtype=torch.int32, device=DEV), 8)["y"].cpu()
    x = dict(q=q[2][None, None], k=torch.cat((old[0], k[2:])).unsqueeze(0), v=torch.cat((old[1], v[2:])).unsqueeze(0),
             dy=q[2][None, None], len=None)
    check("step", y[2][None, None], expected(x, 100, 0, parts=False, grads=False)["y"])
    assert torch.equal(cache[0, 2, 4].cpu(), k[2]) and torch.equal(cache[1, 2, 4].cpu(), v[2])
    # the same memory as keys and values of a long past: the queries are the last three tokens
    tail = make(1, 3, Hk, Hk, d, "bf16", past=60, seed=7)
    cache[0, 2, -63:], cache[1, 2, -63:] = tail["k"][0].to(DEV), tail["v"][0].to(DEV)
    q3, dy3 = torch.zeros(S, 3, Hk, d, dtype=torch.bfloat16), torch.zeros(S, 3, Hk, d, dtype=torch.bfloat16)
    q3[2], dy3[2] = tail["q"][0], tail["dy"][0]
    n = torch.tensor([0, 0, slots], dtype=torch.int32, device=DEV)
    out = kla.kla_window_attn_forward(q3.to(DEV), cache[0], cache[1], 40, 0, n, save=True)
    g = kla.kla_window_attn_backward(q3.to(DEV), cache[0], cache[1], 40, 0, n, out["y"], out["saved"], dy3.to(DEV))
    ref = expected(tail, 40, 0)
    check("y", out["y"][2:], ref["y"])
    check("dq", g["dq"][2:], ref["dq"])
    check("dk", g["dk"][2:, -63:], ref["dk"])
    check("dv", g["dv"][2:, -63:], ref["dv"])
    assert (g["dk"][2, :-63] == 0).all() and (g["dv"][2, :-63] == 0).all()


def test_autograd_of_a_fused_projection(kla):
    """q, k, v as parts of one tensor, keys shared by heads, and a gradient of y that is broadcast."""
    B, T, H, Hk, d, W = 2, 70, 4, 2, 32, 25
    g = torch.Generator().manual_seed(2)
    f = torch.randn(B, T, H + 2 * Hk, d, generator=g)
    fused = f.to(DEV).requires_grad_(True)
    y = kla.kla_window_attn(*fused.split([H, Hk, Hk], 2), W, 3)
    (df,) = torch.autograd.grad(y, [fused], torch.ones((), device=DEV).expand_as(y))
    q, k, v = f.split([H, Hk, Hk], 2)
    ref = expected(dict(q=q, k=k, v=v, dy=torch.ones_like(q), len=None), W, 3)
    check("y", y, ref["y"])
    for n, part in zip(("dq", "dk", "dv"), df.split([H, Hk, Hk], 2)):
        check(n, part, ref[n])
    fused2 = f.to(DEV).requires_grad_(True)
    y = kla.kla_window_attn(*fused2.split([H, Hk, Hk], 2), W, 3)
    with pytest.raises(NotImplementedError, match="second"):
        torch.autograd.grad(y.sum(), [fused2], create_graph=True)


def test_given_outputs_and_places(kla):
    X = dev(make(2, 40, 2, 1, 64, "f32", seed=1))
    y = torch.empty_like(X["q"])
    v0 = y._version
    out = kla.kla_window_attn_forward(X["q"], X["k"], X["v"], 9, y=y)
    assert out["y"].data_ptr() == y.data_ptr() and y._version > v0 and out["saved"] is None and out["cache_k"] is None
    with pytest.raises(ValueError, match="overlap"):
        kla.kla_window_attn_forward(X["q"], X["k"], X["v"], 9, y=X["q"])
    # inputs off 16 bytes are copied; caches, which are updated in place, are refused there
    off = torch.empty(X["q"].numel() + 1, device=DEV)[1:].view_as(X["q"]).copy_(X["q"])
    assert torch.equal(kla.kla_window_attn_forward(off, X["k"], X["v"], 9)["y"], y)
    q, k = X["q"][:, 0].contiguous(), X["k"][:, 0].contiguous()
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    ck, cv = torch.zeros(2, 5, 1, 64, device=DEV), torch.zeros(2, 5, 1, 64, device=DEV)
    bad = torch.zeros(2 * 5 * 64 + 1, device=DEV)[1:].view(2, 5, 1, 64)
    with pytest.raises(ValueError, match="16 bytes"):
        kla.kla_window_attn_step(q, k, k, bad, cv, pos)
    with pytest.raises(ValueError, match="overlap"):
        kla.kla_window_attn_step(q, k, k, ck, ck, pos)
    with pytest.raises(ValueError, match="more slots"):
        kla.kla_window_attn_step(q, k, k, ck, cv, pos, 5)
    v0 = ck._version
    kla.kla_window_attn_step(q, k, k, ck, cv, pos)
    assert ck._version > v0
    with pytest.raises(ValueError, match="as many tokens"):
        kla.kla_window_attn_forward(X["q"], X["k"][:, :9].contiguous(), X["v"][:, :9].contiguous(), 9)
    with pytest.raises(ValueError, match="saved"):
        kla.kla_window_attn_backward(X["q"], X["k"], X["v"], 9, 0, None, y, torch.empty(8, dtype=torch.uint8, device=DEV), y)
    for bad_args in ((0, 0), (9, 65), (9, -1)):
        with pytest.raises((ValueError, kla.KLAError)):
            kla.kla_window_attn_forward(X["q"], X["k"], X["v"], *bad_args)
    with pytest.raises(kla.KLAError):
        kla.kla_window_attn_forward(X["q"], X["k"], X["v"], 9, scale=-1.0)


def test_no_tokens(kla):
    for T, past in ((0, 0), (0, 5)):
        X = dev(make(2, T, 2, 1, 32, "bf16", past=past))
        out = kla.kla_window_attn_forward(X["q"], X["k"], X["v"], 4, 2, save=True, want_cache=True)
        assert out["y"].shape == (2, 0, 2, 32)
        g = kla.kla_window_attn_backward(X["q"], X["k"], X["v"], 4, 2, None, out["y"], out["saved"], X["dy"])
        assert (g["dk"] == 0).all() and (g["dv"] == 0).all() and g["dk"].shape == X["k"].shape
        for b in range(2):
            rk, rv = ring((X["k"][b].cpu(), X["v"][b].cpu()), past, 4, 2)
            assert torch.equal(out["cache_k"][b].cpu(), rk) and torch.equal(out["cache_v"][b].cpu(), rv)


def test_results_are_the_same_every_time(kla):
    x = make(2, 300, 4, 2, 128, "bf16", seed=13)
    a, b = run(kla, x, 64, 4), run(kla, x, 64, 4)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_captured_training_step_and_decode(kla):
    """Both in graphs, replayed with eager work between; two graphs that share a pool."""
    X = dev(make(2, 150, 4, 2, 64, "bf16", seed=21))
    leaves = [X[n].clone().requires_grad_(True) for n in ("q", "k", "v")]
    g = torch.Generator(device=DEV).manual_seed(1)
    S, slots = 3, 700
    q, k, v = (torch.randn(S, h, 64, generator=g, device=DEV).bfloat16() for h in (4, 2, 2))
    ck, cv = (torch.randn(S, slots, 2, 64, generator=g, device=DEV).bfloat16() for _ in range(2))
    pos = torch.tensor([5, 690, 4000], dtype=torch.int32, device=DEV)

    def train():
        y = kla.kla_window_attn(*leaves, 20, 3)
        return [y.detach(), *torch.autograd.grad(y, leaves, X["dy"])]

    def step():
        return kla.kla_window_attn_step(q, k, v, ck, cv, pos, 4)["y"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            train(), step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        out1 = train()
    with torch.cuda.graph(two, pool=one.pool()):
        out2 = step()
    for i in range(4):
        with torch.no_grad():
            for t in leaves:
                t.copy_(torch.randn(t.shape, generator=g, device=DEV))
            pos += 17
            q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        keep = [ck.clone(), cv.clone()]
        one.replay()
        got = [t.clone() for t in out1]
        two.replay()
        torch.cuda.synchronize()
        y, ck1 = out2.clone(), ck.clone()
        fresh = [t.detach().clone().requires_grad_(True) for t in leaves]
        ye = kla.kla_window_attn(*fresh, 20, 3)
        want = [ye.detach(), *torch.autograd.grad(ye, fresh, X["dy"])]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        ck.copy_(keep[0]), cv.copy_(keep[1])
        assert torch.equal(step(), y) and torch.equal(ck, ck1), i


def test_other_streams(kla):
    """Work on a stream of the caller's own, two at once."""
    xs = [make(2, 200, 4, 2, 64, "f32", seed=s) for s in (1, 2)]
    want = [run(kla, x, 50, 2) for x in xs]
    X = [dev(x) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for s, x in zip(streams, X):
        with torch.cuda.stream(s):
            out = kla.kla_window_attn_forward(x["q"], x["k"], x["v"], 50, 2, save=True)
            got.append(dict(y=out["y"], **kla.kla_window_attn_backward(x["q"], x["k"], x["v"], 50, 2, None, out["y"],
                                                                       out["saved"], x["dy"])))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[n], b[n]) for n in a)
