"""Norms of queries and keys for each head with the position rotation, against the formulas in fp64.

Tolerances (u = 2^-24; half: half a step of the output's type).  r = 1 / sqrt(mean x^2 + eps): the sum of n squares is
off by n u at most, its root by half of that, with the hardware's step n u / 2 + 3 u.  An angle in fp64 turns is off by
2^-53 of itself and becomes fp32 within half a turn, 2^-24 of a turn: cosine and sine are off by 8 u.  So an output is
off by (n / 2 + 14) u of |u_a| + |u_b| and its rounding."""
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


def frequencies(pairs, base=10000.0):
    return base ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1)) if pairs else None


def make(lead, H, Hk, n, pairs, dtype, far=None, weights=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    z = lambda *s: torch.randn(*s, generator=g)
    x = dict(q=z(*lead, H, n), k=3 * z(*lead, Hk, n), dq_out=z(*lead, H, n), dk_out=z(*lead, Hk, n))
    x = {m: t.to(TYPES[dtype]) for m, t in x.items()}
    x.update(wq=1 + 0.3 * z(n) if weights else None, wk=1 + 0.3 * z(n) if weights else None, freq=frequencies(pairs), pos=None)
    if far is not None:
        x["pos"] = torch.randint(-far, far + 1, lead, generator=g, dtype=torch.int32)
    return x


def turned(u, freq, pos, interleaved, back=False):
    if freq is None:
        return u
    P = freq.numel()
    phi = pos.double()[..., None, None] * freq
    c, s = phi.cos(), phi.sin() * (-1 if back else 1)
    at = (lambda t: (t[..., 0:2 * P:2], t[..., 1:2 * P:2])) if interleaved else (lambda t: (t[..., :P], t[..., P:2 * P]))
    out = u.clone()
    (a, b), (oa, ob) = at(u), at(out)
    oa.copy_(a * c - b * s)
    ob.copy_(b * c + a * s)
    return out


def both(u, freq, interleaved):
    """|u_a| + |u_b| at both elements of a pair."""
    if freq is None:
        return u.abs()
    P, out = freq.numel(), u.abs().clone()
    at = (lambda t: (t[..., 0:2 * P:2], t[..., 1:2 * P:2])) if interleaved else (lambda t: (t[..., :P], t[..., P:2 * P]))
    a, b = at(out)
    s = a + b
    a.copy_(s)
    b.copy_(s)
    return out


def expected(x, eps, interleaved):
    out = {}
    lead = x["q"].shape[:-2]
    pos = x["pos"]
    if pos is None:
        pos = torch.arange(lead[-1]).expand(lead)
    half = HALF["bf16" if x["q"].dtype == torch.bfloat16 else "f32"]
    for m in ("q", "k"):
        v, w, g = x[m].double(), x["w" + m], x[f"d{m}_out"].double()
        n = v.shape[-1]
        w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
        c = (n / 2 + 14) * U
        r = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
        hat = v * r
        y = turned(hat * w, x["freq"], pos, interleaved)
        out[m] = (y, c * both(hat * w, x["freq"], interleaved) + half * y.abs())
        du = turned(g, x["freq"], pos, interleaved, back=True)
        tdu = 10 * U * both(g, x["freq"], interleaved)
        mean = (du * w * hat).mean(-1, keepdim=True)
        tmean = ((tdu + (c + (n + 4) * U) * du.abs()) * w.abs() * hat.abs()).mean(-1, keepdim=True)
        dx = r * (du * w - hat * mean)
        tdx = r * (tdu * w.abs() + hat.abs() * tmean + (2 * c + 4 * U) * (du * w).abs() + (2 * c + 4 * U) * (hat * mean).abs())
        out["d" + m] = (dx, tdx + half * dx.abs())
        if x["w" + m] is not None:
            rows = v.numel() // n
            dims = tuple(range(v.dim() - 1))
            out["dw" + m] = ((du * hat).sum(dims), (tdu * hat.abs() + (c + 4 * U) * (du * hat).abs()).sum(dims)
                             + rows * U * (du * hat).abs().sum(dims))
    return out


def check(name, got, want):
    ref, tol = want
    got = got.detach().double().cpu()
    assert got.shape == ref.shape and torch.isfinite(got).all(), name
    worst = ((got - ref).abs() / (tol + 1e-35)).max().item() if got.numel() else 0.0
    print(f"{name} {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.2f} times the tolerance"


def run(kla, x, eps=1e-6, interleaved=False):
    X = {m: t if t is None else t.to(DEV) for m, t in x.items()}
    args = (X["q"], X["k"], X["wq"], X["wk"], X["freq"], X["pos"])
    q, k = kla.kla_qk_norm_rope_forward(*args, eps, interleaved=interleaved)
    g = kla.kla_qk_norm_rope_backward(*args, X["dq_out"], X["dk_out"], eps, interleaved=interleaved)
    return dict(q=q, k=k, **g)


CASES = [  # lead, H, Hk, n, pairs, far, weights
    ((1, 1), 1, 1, 16, 8, None, True),
    ((1, 1), 3, 1, 128, 64, 2 ** 31 - 1, True),
    ((2, 37), 4, 2, 64, 32, None, True),
    ((2, 37), 5, 5, 64, 8, 1000, True),
    ((3, 5), 12, 3, 32, 0, None, True),
    ((3, 5), 2, 7, 128, 24, 10 ** 6, False),
    ((1, 1100), 16, 4, 128, 64, 10 ** 5, True),
    ((1, 700), 1, 1, 16, 8, None, True),
    ((5,), 6, 2, 32, 16, 10 ** 6, True),
    ((2, 300), 40, 8, 64, 32, None, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_forward_and_gradients(kla, case, interleaved, dtype):
    lead, H, Hk, n, pairs, far, weights = case
    x = make(lead, H, Hk, n, pairs, dtype, far, weights)
    got, ref = run(kla, x, 1e-6, interleaved), expected(x, 1e-6, interleaved)
    for m in ref:
        check(m, got[m], ref[m])
    assert (got["dwq"] is None) == (not weights)


def test_gradients_are_differences(kla):
    x = make((2, 6), 3, 1, 32, 8, "f32", 50, seed=4)
    got = run(kla, x, 1e-3, True)
    gen = torch.Generator().manual_seed(1)
    for m in ("q", "k", "wq", "wk"):
        d = torch.randn(x[m].shape, generator=gen, dtype=torch.float64)

        def f(h):
            e = expected({**x, m: x[m].double() + h * d}, 1e-3, True)
            return sum((e[t][0] * x[f"d{t}_out"].double()).sum() for t in ("q", "k"))
        diff = ((f(1e-5) - f(-1e-5)) / 2e-5).item()
        part = got["d" + m].double().cpu() * d
        assert abs(diff - part.sum().item()) <= 1e-5 * part.abs().sum().item(), m


def test_zero_rows_and_eps(kla):
    """A row of zeros is zero, its gradient dout w / sqrt(eps); an infinity or NaN stays in its row."""
    x = make((2, 9), 2, 2, 64, 32, "f32", seed=3)
    x["q"][0, 3, 1] = 0.0
    got, ref = run(kla, x, 1e-4), expected(x, 1e-4, False)
    assert (got["q"][0, 3, 1] == 0).all()
    for m in ref:
        check(m, got[m], ref[m])
    clean = run(kla, x)
    x["q"][1, 2, 0, 5] = math.nan
    x["k"][0, 0, 1, 7] = math.inf
    got = run(kla, x)
    for m, (b, t, h) in (("q", (1, 2, 0)), ("k", (0, 0, 1))):
        for name in (m, "d" + m):
            a, c = got[name].clone(), clean[name].clone()
            assert not torch.isfinite(a[b, t, h]).all()
            a[b, t, h] = c[b, t, h] = 0
            assert torch.equal(a, c), name


def test_autograd_of_a_fused_projection(kla):
    B, T, H, Hk, n = 2, 21, 4, 2, 64
    g = torch.Generator().manual_seed(2)
    f = torch.randn(B, T, H + 2 * Hk, n, generator=g)
    w = (1 + 0.1 * torch.randn(2, n, generator=g)).to(DEV).requires_grad_(True)
    freq, fused = frequencies(32).to(DEV), f.to(DEV).requires_grad_(True)
    q, k, _ = fused.split([H, Hk, Hk], 2)
    oq, ok = kla.kla_qk_norm_rope(q, k, w[0], w[1], freq)
    df, dw = torch.autograd.grad([oq], [fused, w], [torch.ones_like(oq)])   # k's output unused
    x = dict(q=f[:, :, :H], k=f[:, :, H:H + Hk], wq=w[0].detach().cpu(), wk=w[1].detach().cpu(), freq=frequencies(32), pos=None,
             dq_out=torch.ones(B, T, H, n), dk_out=torch.zeros(B, T, Hk, n))
    ref = expected(x, 1e-6, False)
    for m, t in (("q", oq), ("k", ok), ("dq", df[:, :, :H]), ("dwq", dw[0])):
        check(m, t, ref[m])
    assert (df[:, :, H:] == 0).all() and (dw[1] == 0).all()
    with pytest.raises(ValueError, match="constants"):
        kla.kla_qk_norm_rope(q, k, w[0], w[1], freq.clone().requires_grad_(True))
    oq, _ = kla.kla_qk_norm_rope(q, k, w[0], w[1], freq)
    with pytest.raises(NotImplementedError, match="second"):
        torch.autograd.grad(oq.sum(), [fused], create_graph=True)


def test_refusals_and_places(kla):
    x = {m: t if t is None else t.to(DEV) for m, t in make((2, 9), 4, 2, 64, 32, "f32").items()}
    f = lambda **o: kla.kla_qk_norm_rope_forward(*({**x, **o}[m] for m in ("q", "k", "wq", "wk", "freq", "pos")))
    want = f()
    off = torch.empty(x["q"].numel() + 1, device=DEV)[1:].view_as(x["q"]).copy_(x["q"])
    assert torch.equal(f(q=off)[0], want[0])
    for bad in (dict(freq=x["freq"].float()), dict(freq=x["freq"][None]), dict(k=x["k"].bfloat16()), dict(wq=x["wq"][:8].clone()),
                dict(q=x["q"].transpose(1, 2)), dict(pos=torch.zeros(2, 9, dtype=torch.int64, device=DEV)),
                dict(q=x["q"][:, 0].contiguous(), k=x["k"][:, 0].contiguous())):
        with pytest.raises(ValueError):
            f(**bad)
    for bad in (dict(freq=frequencies(12).to(DEV)), dict(freq=frequencies(40).to(DEV)),
                dict(q=x["q"][..., :48].contiguous(), k=x["k"][..., :48].contiguous(), wq=None, wk=None, freq=None)):
        with pytest.raises(kla.KLAError):
            f(**bad)


def test_no_tokens(kla):
    for lead in ((2, 0), (0, 3), (0,)):
        x = make(lead, 2, 1, 32, 16, "bf16", far=5)
        got = run(kla, x)
        assert got["q"].shape == x["q"].shape and (got["dwq"] == 0).all() and (got["dwk"] == 0).all()


def test_offsets_past_32_bits(kla):
    """More than 2^31 elements of q: the last tokens are those of the same rows alone."""
    T, H, n = (1 << 20) + 5, 16, 128
    q = torch.zeros(1, T, H, n, dtype=torch.bfloat16, device=DEV)
    x = make((1, 7), H, 1, n, 64, "bf16", far=10 ** 6, seed=2)
    q[0, -7:] = x["q"][0].to(DEV)
    k = torch.zeros(1, T, 1, n, dtype=torch.bfloat16, device=DEV)
    k[0, -7:] = x["k"][0].to(DEV)
    pos = torch.zeros(1, T, dtype=torch.int32, device=DEV)
    pos[0, -7:] = x["pos"][0].to(DEV)
    dq, dk = torch.zeros_like(q), torch.zeros_like(k)
    dq[0, -7:], dk[0, -7:] = x["dq_out"][0].to(DEV), x["dk_out"][0].to(DEV)
    args = (q, k, x["wq"].to(DEV), x["wk"].to(DEV), x["freq"].to(DEV), pos)
    ref = expected(x, 1e-6, False)
    oq, ok = kla.kla_qk_norm_rope_forward(*args)
    check("q", oq[:, -7:], ref["q"])
    check("k", ok[:, -7:], ref["k"])
    g = kla.kla_qk_norm_rope_backward(*args, dq, dk)
    for m in ("dq", "dk"):
        check(m, g[m][:, -7:], ref[m])
    for m in ("dwq", "dwk"):
        check(m, g[m], ref[m])


def test_captured_and_replayed(kla):
    x = {m: t if t is None else t.to(DEV) for m, t in make((2, 200), 4, 2, 64, 32, "bf16", far=100).items()}
    leaves = [x[m].clone().requires_grad_(True) for m in ("q", "k", "wq", "wk")]

    def step(ls):
        out = kla.kla_qk_norm_rope(*ls, x["freq"], x["pos"])
        return [t.detach() for t in out] + list(torch.autograd.grad(out, ls, [x["dq_out"], x["dk_out"]]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(leaves), step(leaves)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(leaves)
    for i in range(4):
        with torch.no_grad():
            for t in leaves:
                t.copy_(torch.randn(t.shape, device=DEV))
            x["pos"] += 3
        graph.replay()
        torch.cuda.synchronize()
        want = step([t.detach().clone().requires_grad_(True) for t in leaves])
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
