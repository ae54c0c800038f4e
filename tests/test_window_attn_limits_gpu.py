"""Attention with a sliding window at the ends of its ranges: scores whose references have few digits left, rows without
a score, weights of zero beside infinities, and what bf16 keeps of the rows of few tokens.  Tolerances as in
test_window_attn_gpu.py."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_window_attn_gpu import DEV, TYPES, U, check, dev, expected, kla, make, run  # noqa: E402,F401

pytestmark = pytest.mark.gpu

FAR = [  # B, T, past, H, Hk, d, window, sinks: one workgroup a row, and keys dealt to several, joined in either way
    (2, 40, 0, 2, 1, 64, 9, 2),
    (1, 3, 1400, 2, 1, 64, 1500, 0),
    (1, 1024, 0, 4, 2, 128, 1024, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", FAR, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("unit,key", [(12, 1.0), (14, 0.375), (14, -0.375), (14, 1.0), (14, -1.0)])
def test_scores_whose_reference_has_few_digits(kla, case, dtype, unit, key):
    """All scores of a row are alike, key 2^(2 unit) and exact, so P is 1 / n as for scores of `key`, and the gradients
    are those times 2^unit.  Exponents of up to 32 about a reference whose steps are up to 32 are off by 2^-20 ln 2,
    11 u, less than the 2 (d + 4) u of scores that are sums."""
    B, T, past, H, Hk, d, window, sinks = case
    x = make(B, T, H, Hk, d, dtype, past, seed=12)
    x["q"].zero_()[..., 0] = 1.0
    x["k"].zero_()[..., 0] = key
    ref = expected(x, window, sinks, 1.0, parts=min(window + sinks, past + T) < 256)
    far = {**x, "q": x["q"] * 2.0 ** unit, "k": x["k"] * 2.0 ** unit}
    got = run(kla, far, window, sinks, 1.0)
    for n in ref:
        f = 2.0 ** unit if n in ("dq", "dk") else 1.0
        check(n, got[n], tuple(f * t for t in ref[n]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_past_the_range_are_not_zeros(kla, dtype):
    """Past 2^30 in units of scale log2(e) score no fp32 reference may lie near enough to a score for its exponential: a
    row that sees one token is that token's, gradient too, or NaN; in the prompt, in pieces and in the step."""
    T, d = 1000, 64
    x = make(1, T, 1, 1, d, dtype, seed=14)
    g = torch.Generator().manual_seed(15)
    x["q"].zero_()[0, :, 0, 0] = torch.exp2(27 + 13 * torch.rand(T, generator=g)).to(TYPES[dtype])
    x["k"].zero_()[0, :, 0, 0] = torch.tensor([1.0, -1.0]).repeat(T // 2).to(TYPES[dtype])
    near = (x["q"][0, :, 0, 0].double() * math.log2(math.e) < 2.0 ** 30)
    assert near.any() and not near.all()
    zero = {**x, "q": torch.zeros_like(x["q"])}
    ref = expected(zero, 1, 0, 1.0)
    ref["step"] = expected(zero, 1, 0, 1.0, parts=False, grads=False)["y"]
    got = run(kla, x, 1, 0, 1.0)
    X = dev(x)
    one = lambda n: X[n][0].contiguous()
    cache = lambda: torch.zeros(T, 1, 1, d, dtype=TYPES[dtype], device=DEV)
    got["step"] = kla.kla_window_attn_step(one("q"), one("k"), one("v"), cache(), cache(),
                                           torch.zeros(T, dtype=torch.int32, device=DEV), scale=1.0)["y"][None]
    for n in ("y", "dv", "step"):
        value, tol = ref[n]
        r = got[n].double().cpu()
        lost = torch.isnan(r[0, :, 0]).all(-1)
        assert not lost[near].any()
        check(n, r[:, ~lost], (value[:, ~lost], tol[:, ~lost]))


def without_row(x, r):
    """The inputs of which row r of the queries takes no part in a gradient."""
    x = {n: t if t is None else t.clone() for n, t in x.items()}
    x["q"][:, r] = 0.0
    x["dy"][:, r] = 0.0
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d,W,sinks", [(1, 64, 20, 2), (1, 128, 20, 2), (6, 128, 40, 0), (90, 32, 20, 2)])
def test_an_infinite_query_without_a_score_has_no_gradient(kla, B, d, W, sinks, dtype):
    """All scores of rows 70 and 250 are -inf by the query's infinity: zeros for the row, and nothing of it in dk and dv,
    also where an upstream gradient of the row is not finite."""
    T = 300
    x = make(B, T, 2, 1, d, dtype, seed=16)
    x["k"][..., 3] = x["k"][..., 3].abs() + 0.5
    ref = expected(without_row(x, [70, 250]), W, sinks)
    x["q"][:, [70, 250], :, 3] = -math.inf
    for bad in (None, math.inf, math.nan):
        if bad is not None:
            x["dy"][:, [70, 250], :, 1] = bad
        got = run(kla, x, W, sinks)
        rows = torch.ones(T, dtype=torch.bool)
        rows[[70, 250]] = False
        for n in ("y", "dq"):
            assert (got[n][:, [70, 250]] == 0).all(), n
            check(n, got[n][:, rows.to(DEV)], tuple(t[:, rows] for t in ref[n]))
        for n in ("dk", "dv"):
            check(n, got[n], ref[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_infinite_keys_that_leave_a_row_without_a_score(kla, d, dtype):
    """Row 70 sees keys of -inf alone: zeros, and finite dk and dv for all tokens.  In the reference those keys take no
    weight because their scores are -38."""
    T, W, r = 150, 5, 70
    x = make(1, T, 2, 1, d, dtype, seed=17)
    x["q"][..., 0] = 1.0
    bad = slice(r - W + 1, r + 1)
    y = {n: t if t is None else t.clone() for n, t in x.items()}
    y["dy"][:, r] = 0.0
    y["k"][:, bad, :, 0] = -38.0 * math.sqrt(d)
    ref = expected(y, W, 0)
    x["k"][:, bad, :, 0] = -math.inf
    got = run(kla, x, W, 0)
    assert (got["y"][:, r] == 0).all() and (got["dq"][:, r] == 0).all()
    other, clear, finite = (torch.ones(T, dtype=torch.bool) for _ in range(3))
    other[r] = False
    clear[r - W + 1:r + W] = False    # rows that see none of those keys
    finite[bad] = False
    check("y", got["y"][:, other.to(DEV)], tuple(t[:, other] for t in ref["y"]))
    check("dq", got["dq"][:, clear.to(DEV)], tuple(t[:, clear] for t in ref["dq"]))
    for n in ("dk", "dv"):
        check(n, got[n][:, finite.to(DEV)], tuple(t[:, finite] for t in ref[n]))
        assert (got[n][:, bad] == 0).all(), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_a_weight_of_zero_times_a_visible_infinity(kla, d, dtype):
    """0 times an infinite key that a row sees is NaN, whichever sign the zero of dS has; rows that do not see it stay
    finite."""
    T, W, j = 150, 20, 70
    x = make(1, T, 1, 1, d, dtype, seed=18)
    x["q"][..., 0] = 1.0
    x["k"][0, j, 0, 0] = -math.inf
    for sign in (1.0, -1.0):
        x["v"][0, j] = sign * x["v"][0, j].abs()
        x["dy"].copy_(x["dy"].abs())
        dq = run(kla, x, W, 0)["dq"][0, :, 0]
        sees = torch.zeros(T, dtype=torch.bool, device=DEV)
        sees[j + 1:j + W] = True   # row j itself sees other keys too
        sees[j] = True
        assert torch.isnan(dq[sees, 0]).all(), sign
        assert torch.isfinite(dq[~sees]).all() and torch.isfinite(dq[:, 1:]).all()


EARLY = [  # B, T, past, H, Hk, d, window, sinks: the last two with keys dealt to several workgroups, joined in either way
    (2, 300, 0, 2, 1, 64, 300, 2),
    (3, 200, 70, 2, 1, 32, 256, 0),
    (2, 150, 127, 1, 1, 128, 260, 0),
    (2, 300, 100, 2, 2, 16, 270, 4),
    (2, 1024, 0, 1, 1, 64, 1024, 0),
    (2, 1000, 40, 2, 1, 128, 1040, 3),
]


def early_rows(x, window, sinks):
    """expected() where positions under 128 count as rows of few tokens and the others do not: y and dq row by row, dk
    and dv of either rows' dy alone, added up."""
    T, past = x["q"].shape[1], x["k"].shape[1] - x["q"].shape[1]
    early = past + torch.arange(T) < 128
    part = [expected({**x, "dy": x["dy"] * m[None, :, None, None]}, window, sinks, parts=p) for p, m in
            ((True, early), (False, ~early))]
    rows = early[None, :, None, None]
    ref = {n: tuple(torch.where(rows, a, b) for a, b in zip(part[0][n], part[1][n])) for n in ("y", "dq")}
    ref.update({n: tuple(a + b for a, b in zip(part[0][n], part[1][n])) for n in ("dk", "dv")})
    return ref, early


@pytest.mark.parametrize("case", EARLY, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("alike", [False, True], ids=["normal", "alike"])
def test_first_positions_under_a_wide_window(kla, case, alike):
    """Positions under 128 keep P and dS in two parts and y with 8 more bits, whatever the window.  alike: values that are
    one bf16 step apart, so that y lies between two of them and dq is what the kept bits leave of D; without them dq
    would miss its tolerance in most rows."""
    B, T, past, H, Hk, d, window, sinks = case
    x = make(B, T, H, Hk, d, "bf16", past, seed=19)
    if alike:
        g = torch.Generator().manual_seed(20)
        x["v"] = (1 + 2.0 ** -7 * torch.randint(0, 2, x["v"].shape, generator=g)).bfloat16()
        x["dy"] *= torch.nn.functional.one_hot(torch.randint(0, d, x["dy"].shape[:3], generator=g), d)   # one term of D
    ref, early = early_rows(x, window, sinks)
    if alike:   # what D would be off by with y rounded to bf16 alone, in dq
        y = ref["y"][0]
        off = (x["dy"].double() * (y.bfloat16().double() - y)).sum(-1, keepdim=True)
        plain = expected(x, window, sinks, parts=True)["dq"]
        mean = expected({**x, "v": x["k"]}, window, sinks, grads=False)["y"][0]
        miss = (off * mean / math.sqrt(d)).abs() > 2 * plain[1]
        assert miss[:, early].any(-1).double().mean() > 0.7
    got = run(kla, x, window, sinks)
    for n in ref:
        check(n, got[n], ref[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_dealt_keys(kla, dtype):
    """Parts of many rows, joined by a thread for every four columns, with the context that the backward takes."""
    x = make(1, 1024, 4, 2, 128, dtype, lengths=[1000], seed=21)
    ref = expected(x, 1024, 0, parts=False)
    got = run(kla, x, 1024, 0)
    for n in ref:
        check(n, got[n], ref[n])
        if n in ("y", "dq"):
            assert (got[n][:, 1000:] == 0).all()


@pytest.mark.parametrize("size", [3.0, 6.0, 20.0])
def test_peaked_rows(kla, size):
    """Scores of deviation 3 to 20: the largest weight is 0.35 to 0.9, and D is as large as dy . v in rows that see many
    tokens and keep no further bits."""
    x = make(1, 600, 2, 1, 128, "bf16", seed=22)
    x["q"] = (x["q"].float() * size).bfloat16()
    ref = expected(x, 512, 0, parts=False)
    got = run(kla, x, 512, 0)
    for n in ref:
        check(n, got[n], ref[n])


def sharp(B, T, H, Hk, d, past=0, seed=0):
    """bf16 inputs whose scores are exact whole numbers, products of one element each, in peaked rows: the largest of a
    row takes most of it.  One term of dy a row."""
    x = make(B, T, H, Hk, d, "bf16", past, seed=seed)
    g = torch.Generator().manual_seed(seed)
    one = lambda t: torch.nn.functional.one_hot(torch.randint(0, d, t.shape[:3], generator=g), d)
    x["k"] = (2 * x["k"].float()).round().bfloat16()
    x["q"] = (one(x["q"]) * torch.randint(1, 4, (*x["q"].shape[:3], 1), generator=g)).bfloat16()
    x["dy"] *= one(x["dy"])
    return x


def normed(x, window, sinks, grads=True):
    """expected() of one-part weights where y is divided by the sum of the weights as they entered, and keeps 8 more
    bits: y is off by 2^-8 of P |v - y|, D by what y is and 2^-16."""
    q, k, v, dy = (x[n].double() for n in ("q", "k", "v", "dy"))
    B, T, H, d = q.shape
    Tk, Hk = k.shape[1:3]
    p, j = Tk - T + torch.arange(T)[:, None], torch.arange(Tk)[None]
    see = (j <= p) & ((j > p - window) | (j < sinks))
    heads = lambda t: t.permute(0, 2, 1, 3)
    qv, dyv = heads(q), heads(dy)
    kk, vv = (heads(t).repeat_interleave(H // Hk, 1) for t in (k, v))
    s = (qv @ kk.transpose(-1, -2)).masked_fill(~see, -math.inf)
    M = (qv.abs() @ kk.abs().transpose(-1, -2)).masked_fill(~see, 0.0).amax(-1, keepdim=True)
    P = torch.softmax(s, -1)
    eP = (2 * (d + 4) * M + 2 * Tk + 8) * U
    y = P @ vv
    # one column of v after another: sum_j P_j |v_j - y|
    apart = torch.stack([(P * (vv[..., None, :, c] - y[..., c, None]).abs()).sum(-1) for c in range(d)], -1)
    ty = (P * eP) @ vv.abs() + 2.0 ** -8 * apart
    out = {"y": (heads(y), heads(ty + 2.0 ** -8 * y.abs()))}
    if not grads:
        return out
    A = dyv.abs() @ vv.abs().transpose(-1, -2)
    D = (dyv * y).sum(-1, keepdim=True)
    eD = (dyv.abs() * (ty + 2.0 ** -16 * y.abs())).sum(-1, keepdim=True) + (d + 1) * U * (dyv * y).abs().sum(-1, keepdim=True)
    dS = P * (dyv @ vv.transpose(-1, -2) - D)
    tS = dS.abs() * (eP + 2.0 ** -8 + 4 * U) + P * ((d + 1) * U * A + eD)
    dq, tq = dS @ kk, (tS + Tk * U * dS.abs()) @ kk.abs()
    share = lambda t: heads(t.reshape(B, Hk, H // Hk, Tk, d).sum(2))
    n = H // Hk * T * U
    dk, tk = share(dS.transpose(-1, -2) @ qv), share((tS + n * dS.abs()).transpose(-1, -2) @ qv.abs())
    out.update(dq=(heads(dq), heads(tq + 2.0 ** -8 * dq.abs())), dk=(dk, tk + 2.0 ** -8 * dk.abs()))
    return out


@pytest.mark.parametrize("B,T,past,H,Hk,d,window,sinks", [(2, 500, 0, 2, 1, 64, 300, 2), (1, 400, 130, 2, 2, 128, 256, 0),
                                                          (2, 300, 200, 1, 1, 32, 270, 4), (1, 600, 40, 2, 1, 128, 640, 0)])
def test_gradients_of_peaked_rows_that_see_many_tokens(kla, B, T, past, H, Hk, d, window, sinks):
    """A heavy weight's rounding leaves y where its sum takes it too, and D keeps 16 bits of y: else D, as large as
    dy . v, is off by 2^-8 of it, many times the row's dS."""
    x = sharp(B, T, H, Hk, d, past, seed=23)
    ref, got = normed(x, window, sinks), run(kla, x, window, sinks, 1.0)
    for n in ref:
        check(n, got[n], ref[n])


@pytest.mark.parametrize("S,window,H,Hk,d", [(3, 700, 4, 2, 64), (2, 2000, 2, 2, 128), (200, 60, 16, 4, 32)])
def test_step_of_peaked_rows(kla, S, window, H, Hk, d):
    x = sharp(S, 1, H, Hk, d, window - 1, seed=24)
    X = dev(x)
    got = kla.kla_window_attn_step(X["q"][:, 0], X["k"][:, -1].contiguous(), X["v"][:, -1].contiguous(), X["k"].clone(),
                                   X["v"].clone(), torch.full((S,), window - 1, dtype=torch.int32, device=DEV), scale=1.0)
    check("y", got["y"][:, None], normed(x, window, 0, grads=False)["y"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_context_without_a_gradient(kla, dtype):
    """Where nothing takes a gradient the differentiable form holds y and nothing more, with the same y."""
    x = dev(make(2, 1100, 2, 1, 64, dtype, lengths=[1100, 901], seed=25))
    args = (x["q"], x["k"], x["v"], 1100, 3, x["len"])
    leaf = x["q"].clone().requires_grad_(True)
    with_context = kla.kla_window_attn(leaf, *args[1:]).detach()
    raw = kla.kla_window_attn_forward(*args)["y"]
    for given, off in ((args, False), ((leaf,) + args[1:], True)):
        with torch.set_grad_enabled(not off):
            peaks = []
            for call in (lambda: kla.kla_window_attn_forward(*args)["y"], lambda: kla.kla_window_attn(*given)):
                torch.cuda.synchronize()
                torch.cuda.reset_peak_memory_stats()
                asked = lambda n: torch.cuda.memory_stats()["requested_bytes.all." + n]
                before = asked("current")
                y = call()
                peaks.append(asked("peak") - before)
        assert not y.requires_grad and torch.equal(y, with_context) and torch.equal(y, raw)
        assert peaks[1] == peaks[0], peaks
    with torch.autograd.forward_ad.dual_level(), pytest.raises((NotImplementedError, RuntimeError)):
        kla.kla_window_attn(torch.autograd.forward_ad.make_dual(args[0], torch.ones_like(args[0])), *args[1:])
