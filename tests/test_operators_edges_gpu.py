"""Edges of linear attention, layer norm and the token log probabilities: sums that cancel, values at the ends of
fp32's range, infinities, operands off 16 bytes and outputs that lie over inputs, against the formulas in fp64.

A rounding is off by half a step: bf16 2^-8, fp32 2^-24 of the value.  A product of the matrix cores adds to its
sum with at most 2^-23 of the larger of the two."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_linear_attn_gpu import DEV, TYPES, check, expected, kla, make, run  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def zeros(B, T, H, dk, dv, dtype, g):
    """Inputs of linear attention that are all zero."""
    x = dict(q=(dk,), k=(dk,), v=(dv,), dy=(dv,))
    x = {n: torch.zeros(B, T, H, *w, dtype=TYPES[dtype]) for n, w in x.items()}
    x.update(s0=torch.zeros(B, H, dk, dv), ds=torch.zeros(B, H, dk, dv), g=torch.full((H,), g), len=None)
    return x


def pair(shape, gen, dtype):
    """Vectors of two values that are opposite, at places 2 n and 2 n + 1, and zeros."""
    a = torch.zeros(*shape, dtype=TYPES[dtype])
    n = 2 * torch.randint(0, shape[-1] // 2, shape[:-1], generator=gen)[..., None]
    c = (1 + torch.rand(*shape[:-1], 1, generator=gen)).to(a.dtype)
    return a.scatter_(-1, n, c).scatter_(-1, n + 1, -c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [16, 32, 128])
@pytest.mark.parametrize("g", [0.0, -0.01])
def test_large_states_that_cancel(kla, g, width, dtype):
    """y, dq from a start state and dk, dv from a final state's gradient whose neighbouring rows and columns are the
    same but for 2^-13, multiplied by opposite values.

    Each output is a difference of two products with the state.  Its parts enter one after another, at most
    three times two products, each adding with 2^-23 of half the mass: 3 x 2^-23 of the mass, the decay's
    roundings 2^-22 of it; the factors' roundings scale the difference, which is small."""
    gen = torch.Generator().manual_seed(width)
    B, T, H = 3, 40, 2
    for what in ("start", "final"):
        x = zeros(B, T, H, width, width, dtype, g)
        one = torch.randn(B, H, width // 2, width // 2, generator=gen).repeat_interleave(2, -1).repeat_interleave(2, -2)
        near = one * (1 + 2.0 ** -13 * (2 * torch.rand(one.shape, generator=gen) - 1))
        if what == "start":
            x["s0"], names = near, ("y", "dq")
            x["q"], x["dy"] = (pair((B, T, H, width), gen, dtype) for _ in range(2))
        else:
            x["ds"], names = near, ("dk", "dv")
            x["k"], x["v"] = (pair((B, T, H, width), gen, dtype) for _ in range(2))
        got, ref, mass = run(kla, x), expected(x), expected(x, torch.abs)
        for n in names:
            tol = 5 * 2.0 ** -23 * mass[n] + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * ref[n].abs()
            assert ref[n].abs().max() > 2.0 ** -14 * mass[n].max() > 0
            worst = ((got[n].double().cpu() - ref[n]).abs() / tol).nan_to_num(0.0).max().item()
            print(f"{n} {worst:.3f} of the tolerance", flush=True)
            assert worst <= 1.0, f"{n}: {worst:.2f} times the tolerance"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_cancel(kla, dtype):
    """Two tokens whose keys are the same but for 2^-13 in one slot and whose values are opposite.

    The second's y is the difference of its two scores times a value.  A score is a sum of 16 products, off by
    16 x 2^-24 of itself; the three parts of each score add with 2^-23 of it: (16 + 6) x 2^-24 of the mass."""
    gen = torch.Generator().manual_seed(7)
    B, T, H, w = 64, 2, 8, 16
    x = zeros(B, T, H, w, w, dtype, 0.0)
    t = TYPES[dtype]
    x["q"][:, 1] = (0.5 + torch.rand(B, H, w, generator=gen)).to(t)
    x["k"][:] = (0.5 + torch.rand(B, 1, H, w, generator=gen)).to(t)
    x["k"][..., 15] = 0
    x["k"][:, 1, :, 15] = (2.0 ** -10 * torch.rand(B, H, generator=gen)).to(t)
    c = (1 + torch.rand(B, H, w, generator=gen)).to(t)
    x["v"][:, 0], x["v"][:, 1] = c, -c
    got, ref, mass = run(kla, x)["y"], expected(x)["y"], expected(x, torch.abs)["y"]
    tol = 22 * 2.0 ** -24 * mass + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * ref.abs()
    worst = ((got.double().cpu() - ref).abs() / tol).nan_to_num(0.0)[:, 1].max().item()
    print(f"y {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, f"{worst:.2f} times the tolerance"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g", [0.0, -0.01, -0.04, -0.17, -0.6, -6.0])
@pytest.mark.parametrize("B,T,w", [(1, 320, 16), (1, 1100, 16), (2, 100, 128)])
def test_states_near_the_top_of_the_range(kla, B, T, w, g, dtype):
    """States and their gradients up to 1e38, from large values, keys and gradients and from a large start, at decays
    of which a chunk's takes next to nothing and everything.  The factors that read them are small, so that every
    sum over absolute values is within fp32's range."""
    for big, beside in (("v", "k"), ("k", "v"), ("dy", "q")):
        x = make(B, T, 1, w, w, dtype, True, False, 17, g)
        for n in ("q", "k", "v", "dy"):
            x[n] = x[n] * (1.0 if n in (big, beside) else 2.0 ** -10)
        end, start, other = ("ds0", "ds", "s0") if big == "dy" else ("sT", "s0", "ds")
        x[start], x[other] = x[start] * (1e38 / 5), x[other] * 1e-3
        # the tokens' share of the state as large as the start's, where that leaves them in the range
        one = expected({**x, start: 0 * x[start]}, torch.abs)[end].max().item()
        x[big] = x[big] * 2.0 ** math.floor(math.log2(min(1e38 / one, 1e38 / x[big].abs().max().item())))
        mass = expected(x, torch.abs)
        assert all(u.max() < 3.3e38 for u in mass.values()), {n: u.max().item() for n, u in mass.items()}
        assert max(mass[end].max(), x[big].abs().max()) > 2e37
        check(run(kla, x), x, f"g {g} large {big}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g", [0.0, -0.01, -0.6])
def test_states_near_the_bottom_of_the_range(kla, g, dtype):
    """States of 1e-34 and less, which are held to 2^-116 each: 16 of them in an output, with factors under 8."""
    for scale in (1e-30, 1e-34, 1e-37):
        x = make(1, 100, 2, 16, 16, dtype, True, False, 19, g)
        for n in ("q", "k", "v", "dy"):
            x[n] = x[n].clamp(-4, 4) * (1 if n in ("q", "k") else scale)
        x["s0"], x["ds"] = x["s0"] * scale, x["ds"] * scale
        got, ref, mass = run(kla, x), expected(x), expected(x, torch.abs)
        for n in ("y", "sT", "dv", "ds0"):   # dq and dk are products of two such numbers
            tol = 132 * 2.0 ** -24 * mass[n] + 2.0 ** -8 * ref[n].abs() + 16 * 8 * 2.0 ** -116
            assert ((got[n].double().cpu() - ref[n]).abs() <= tol).all(), (n, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinity_stays_in_its_column(kla, dtype):
    """Of a value and of a start state: the columns beside it are as without it, its own is not finite from there on,
    and infinite in fp32."""
    clean = make(1, 100, 2, 32, 64, dtype, True, False, 23)
    want = run(kla, clean)
    for name, at, first in (("v", (0, 41, 1, 5), 41), ("s0", (0, 1, 3, 5), 0)):
        x = {n: None if u is None else u.clone() for n, u in clean.items()}
        x[name][at] = math.inf
        got = run(kla, x)
        rest = [d for d in range(64) if d != 5]
        assert torch.equal(got["y"][0, :, 0], want["y"][0, :, 0]) and torch.equal(got["sT"][0, 0], want["sT"][0, 0])
        # the chunk of an infinite value is added up in another order: rounding of one sum
        assert torch.allclose(got["y"][0, :, 1, rest], want["y"][0, :, 1, rest], rtol=2.0 ** -7 if dtype == "bf16" else 1e-4,
                              atol=1e-4)
        assert torch.equal(got["sT"][0, 1][:, rest], want["sT"][0, 1][:, rest])
        own = got["y"][0, :, 1, 5]
        assert torch.allclose(own[:first], want["y"][0, :first, 1, 5], rtol=2.0 ** -7, atol=1e-4)
        assert not torch.isfinite(own[first:]).any()
        if name == "s0" and dtype == "f32":
            assert torch.equal(own.cpu(), math.inf * x["q"][0, :, 1, 3].sign())


def off16(u):
    """The same values in a tensor that is dense but does not start on 16 bytes, as a row of stacked ones."""
    o = torch.empty(u.numel() + 1, dtype=u.dtype, device=u.device)[1:].view_as(u).copy_(u)
    assert o.is_contiguous() and o.data_ptr() % 16
    return o


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_attention_of_operands_off_16_bytes(kla, dtype):
    x = {n: None if u is None else u.to(DEV) for n, u in make(3, 70, 5, 32, 64, dtype, True, True, 25).items()}
    calls = (lambda d: kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"]),
             lambda d: kla.kla_linear_attn_backward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"], d["dy"], d["ds"]),
             lambda d: kla.kla_linear_attn_step(*(d[n] for n in ("q1", "k1", "v1")), d["g"], x["s0"].clone()))

    def train(d):
        ins = [d[n].detach().requires_grad_(True) for n in ("q", "k", "v", "s0")]
        y, sT = kla.kla_linear_attn(*ins[:3], d["g"], ins[3], d["len"])
        return dict(enumerate([y, sT, *torch.autograd.grad([y, sT], ins, [d["dy"], d["ds"]])]))
    x.update({n + "1": x[n][:, 0].contiguous() for n in ("q", "k", "v")})
    for call in (*calls, train):
        want = call(x)
        for n in x:
            got = call({**x, n: off16(x[n])})
            assert all(torch.equal(want[m], got[m]) for m in want), n
    stacked = torch.stack([2 * x["g"], x["g"]])   # [layers, 5]
    got = train({**x, "g": stacked[1]})
    assert all(torch.equal(a, got[m]) for m, a in train(x).items())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [64, 1001])
def test_layer_norm_of_operands_off_16_bytes(kla, n, dtype):
    g = torch.Generator(device=DEV).manual_seed(n)
    z = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x = dict(x=z(7, n).to(TYPES[dtype]), w=1 + z(n), b=z(n), dy=z(7, n).to(TYPES[dtype]))
    x["mean"], x["rstd"] = kla.kla_layer_norm_forward(x["x"], x["w"], x["b"])[1:]
    calls = (lambda d: kla.kla_layer_norm_forward(d["x"], d["w"], d["b"]),
             lambda d: kla.kla_layer_norm_backward(d["x"], d["w"], d["mean"], d["rstd"], d["dy"]))

    def train(d):
        ins = [d[m].detach().requires_grad_(True) for m in ("x", "w", "b")]
        y = kla.kla_layer_norm(*ins)
        return (y, *torch.autograd.grad(y, ins, d["dy"]))
    for call in (*calls, train):
        want = call(x)
        for m in x:
            assert all(map(torch.equal, want, call({**x, m: off16(x[m])}))), m
    layers = {m: torch.stack([2 * x[m], x[m], 0 * x[m]]) for m in ("w", "b")}   # the second layer's row
    assert all(map(torch.equal, train(x), train({**x, "w": layers["w"][1], "b": layers["b"][1]})))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_logp_of_operands_off_16_bytes(kla, dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    z = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x = dict(x=z(5, 333).to(TYPES[dtype]), t=torch.randint(0, 333, (5,), generator=g, device=DEV), dl=z(5), de=z(5))
    fwd = lambda d: kla.kla_token_logp_forward(d["x"], d["t"], want_entropy=True, top=4, save=True)
    x.update({m: fwd(x)[m] for m in ("stat", "entropy")})

    def train(d):
        u = d["x"].detach().requires_grad_(True)
        out = kla.kla_token_logp(u, d["t"], want_entropy=True)
        return (*out, *torch.autograd.grad(out, u, [d["dl"], d["de"]]))
    for call in (lambda d: tuple(fwd(d).values()), train,
                 lambda d: (kla.kla_token_logp_backward(d["x"], d["t"], d["stat"], d["entropy"], d["dl"], d["de"]),)):
        want = call(x)
        for m in x:
            assert all(map(torch.equal, want, call({**x, m: off16(x[m])}))), m


def test_outputs_apart_from_decays_and_lengths(kla):
    """Other workgroups read them while an output that lies over them would be written."""
    x = make(2, 8, 4, 16, 16, "f32", True, True, 1)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    y = torch.empty_like(d["v"])
    g = y.view(-1)[-4:].copy_(d["g"])
    with pytest.raises(ValueError, match="y must not overlap"):
        kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], g, d["s0"], y=y)
    n = y.view(-1)[:2].view(torch.int32).copy_(d["len"])
    with pytest.raises(ValueError, match="y must not overlap"):
        kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], n, y=y)
    one = [d[n][:, 0].contiguous() for n in ("q", "k", "v")]
    y = torch.empty_like(one[2])
    with pytest.raises(ValueError, match="y must not overlap"):
        kla.kla_linear_attn_step(*one, y.view(-1)[4:8].copy_(d["g"]), d["s0"], y=y)
    with pytest.raises(ValueError, match="state must not overlap"):
        kla.kla_linear_attn_step(*one, d["s0"].view(-1)[8:12].fill_(-1.0), d["s0"])


@pytest.mark.parametrize("n", [7, 100, 1001, 2048, 5000, 16384])
def test_layer_norm_of_constant_rows(kla, n):
    """No spread: the output is the bias, however large the value is against sqrt(eps).

    The mean's sum is off by D <= 48 x 2^-24 |x| and what it leaves, the same in every element, is exact and adds up
    exactly; its mean is off by 2^-22 D, which rstd = eps^-1/2 raises 316 times: 48 x 2^-46 |x| 316."""
    x = torch.tensor([1000.1, -77.77, 3.0e4 + 0.125, 0.3, 0.0], device=DEV)[:, None].repeat(1, n)
    g = torch.Generator(device=DEV).manual_seed(n)
    w, b, dy = (torch.randn(s, generator=g, device=DEV) for s in ((n,), (n,), (5, n)))
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    dx, dw, db = kla.kla_layer_norm_backward(x, w, mean, rstd, dy)
    off = 48 * 2.0 ** -46 * 317 * x.abs()
    assert ((out - b).abs() <= off * w.abs() + 2.0 ** -23 * b.abs()).all()
    assert torch.equal(mean, x[:, 0])
    assert ((rstd * 1e-5 ** 0.5 - 1).abs() <= 2.0 ** -22 + off[:, 0] ** 2).all()
    assert (dw.abs() <= (off * dy.abs()).sum(0)).all()
    d = (dy * w).double()
    want = 1e-5 ** -0.5 * (d - d.mean(-1, keepdim=True))
    # sums of 48 roundings, and the roundings of rstd, of the difference and of the product
    assert ((dx - want).abs() <= 64 * 2.0 ** -24 * 1e-5 ** -0.5 * (d.abs() + d.abs().mean(-1, keepdim=True))).all()


@pytest.mark.parametrize("n", [100, 1001, 4096])
@pytest.mark.parametrize("shift,spread", [(1000.0, 0.02), (-5e4, 3.0), (3.0, 1e-4)])
def test_layer_norm_far_from_zero(kla, n, shift, spread):
    """Rows whose offset is large against their spread.

    x - mu is exact for a mu near x; the sum that gives mu is off by D <= 48 x 2^-24 |shift|, which the second mean
    takes out but for 64 x 2^-24 of the mean of |x - mu|, at most that of |x - mean| and D."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x = shift + spread * torch.randn(20, n, generator=g, device=DEV)
    w, b = (torch.randn(n, generator=g, device=DEV) for _ in range(2))
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    X = x.double()
    m = X.mean(-1, keepdim=True)
    var = (X - m).square().mean(-1, keepdim=True)
    r = 1 / torch.sqrt(var + 1e-5)
    D = 48 * 2.0 ** -24 * X.abs().amax(-1, keepdim=True)
    left = 64 * 2.0 ** -24 * ((X - m).abs() + (X - m).abs().mean(-1, keepdim=True) + D)
    rel = 64 * 2.0 ** -24 * (1 + (D * r).square())   # of the mean square, which has the mean's square taken off
    want = (X - m) * r * w + b
    assert ((out - want).abs() <= (left * r + rel * (X - m).abs() * r) * w.abs() + 2.0 ** -23 * (want.abs() + b.abs())).all()
    assert ((mean - m[:, 0]).abs() <= left[:, 0] + 2.0 ** -24 * m[:, 0].abs()).all()
    assert ((rstd / r[:, 0] - 1).abs() <= rel[:, 0]).all()


def test_gradients_of_unlikely_tokens(kla):
    """fp32 logits under a first one of 0, far enough for their sum to be 1: the gradient of token v is -e^{x_v}.

    2^x is off by 2^-23 and the product that adds what x lost by 2^-24; the product with 1 / s = 1 is exact."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x = -(25 + 60 * torch.rand(6, 1000, generator=g, device=DEV))
    x[:, 0] = 0
    x[1] = torch.where(x[1] < 0, x[1].round(), x[1])
    target = torch.zeros(6, dtype=torch.int64, device=DEV)
    out = kla.kla_token_logp_forward(x, target, save=True)
    assert torch.equal(out["stat"], torch.tensor([0.0, 1.0], device=DEV).expand(6, 2))
    dx = kla.kla_token_logp_backward(x, target, out["stat"], None, torch.ones(6, device=DEV))
    want = -torch.exp(x.double())[:, 1:]
    off = ((dx[:, 1:].double() - want) / want).abs().max().item()
    assert off <= 2.0 ** -22, off
    x[2, 5] = -math.inf
    dx = kla.kla_token_logp_backward(x, target, out["stat"], None, torch.ones(6, device=DEV))
    assert dx[2, 5] == 0 and torch.isfinite(dx).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_segments_of_a_long_sequence(kla, dtype):
    """More than 96 chunks a segment where there were two workgroups a CU: the other number of segments, in both
    directions, with a padded sequence's tokens ending inside one."""
    x = make(1, 49170, 32, 16, 16, dtype, True, True, 31)
    x["len"] = torch.tensor([49170 - 500], dtype=torch.int32)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("at", [1, 95, 96, 550, 1098])
def test_values_that_are_not_finite_in_a_cut_sequence(kla, dtype, bad, at):
    """In the first segment, at a border, in the middle and in the last: earlier outputs (in the backward, later
    gradients), the other sequence and the other head stay as they are."""
    clean = make(2, 1100, 2, 32, 32, dtype, True, True, 33)
    clean["len"] = torch.tensor([1100, 700], dtype=torch.int32)
    want = run(kla, clean)
    for name in ("q", "k", "v", "dy"):
        x = {n: None if u is None else u.clone() for n, u in clean.items()}
        x[name][0, at, 1] = bad
        got = run(kla, x)
        for n in ("y", "dq", "dk", "dv"):
            assert torch.equal(got[n][1], want[n][1]) and torch.equal(got[n][0, :, 0], want[n][0, :, 0]), (name, n)
            late = n in ("dk", "dv")
            a, b = (u[n][0, at + 1:, 1] if late else u[n][0, :at, 1] for u in (got, want))
            assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if dtype == "bf16" else 1e-4, atol=1e-4), (name, n)
        for n in ("sT", "ds0"):
            assert torch.equal(got[n][1], want[n][1]) and torch.equal(got[n][0, 0], want[n][0, 0]), (name, n)
        if name in ("k", "v"):
            assert not torch.isfinite(got["y"][0, at:, 1]).all() and not torch.isfinite(got["sT"][0, 1]).all()
        else:
            assert not torch.isfinite(got["ds0"][0, 1]).all()
            assert torch.equal(got["sT"], want["sT"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dv", [16, 32, 64, 128])
def test_wide_rows_in_many_sequences(kla, dv, dtype):
    """More than two workgroups a CU in the forward too: one wave for the rows of a state 128 wide in bf16."""
    x = make(180, 35, 3, 128, dv, dtype, True, True, dv)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_values_of_large_keys(kla, dtype):
    """Values of 1e-33 and less, held to 2^-116 each, of keys of 1e6: the state and y keep that times the keys."""
    for scale in (1e-26, 1e-33, 1e-36):
        x = make(1, 100, 2, 16, 16, dtype, True, False, 35, -0.02)
        x["k"], x["v"], x["dy"], x["s0"], x["ds"] = x["k"] * 1e6, x["v"] * scale, 0 * x["dy"], 0 * x["s0"], 0 * x["ds"]
        got, ref, mass = run(kla, x), expected(x), expected(x, torch.abs)
        per = expected({**x, "v": torch.ones_like(x["v"])}, torch.abs)   # of values that are one
        for n in ("y", "sT"):
            tol = 132 * 2.0 ** -24 * mass[n] + 2.0 ** -8 * ref[n].abs() + 2.0 ** -116 * per[n] + 2.0 ** -116
            assert ((got[n].double().cpu() - ref[n]).abs() <= tol).all(), (n, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_a_fused_projection(kla, dtype):
    """q, k and v as views of one tensor, or with heads before tokens: the same values and gradients as dense ones."""
    x = {n: None if u is None else u.to(DEV) for n, u in make(2, 60, 3, 32, 64, dtype, True, True, 37).items()}

    def train(make_qkv, leaves):
        leaves = [u.detach().requires_grad_(True) for u in leaves]
        y, sT = kla.kla_linear_attn(*make_qkv(*leaves), x["g"], x["s0"], x["len"])
        return y, sT, torch.autograd.grad([y, sT], leaves, [x["dy"], x["ds"]])
    y, sT, (dq, dk, dv) = train(lambda *u: u, [x["q"], x["k"], x["v"]])
    fused = torch.cat([x[n].flatten(2) for n in ("q", "k", "v")], -1)   # [B, T, H (2 dk + dv)]
    y1, sT1, (df,) = train(lambda f: [u.unflatten(2, (3, -1)) for u in f.split([96, 96, 192], -1)], [fused])
    assert torch.equal(y, y1) and torch.equal(sT, sT1)
    assert torch.equal(df, torch.cat([u.flatten(2) for u in (dq, dk, dv)], -1))
    turned = [x[n].transpose(1, 2).contiguous() for n in ("q", "k", "v")]
    y2, sT2, grads = train(lambda *u: [w.transpose(1, 2) for w in u], turned)
    assert torch.equal(y, y2) and torch.equal(sT, sT2)
    assert all(torch.equal(a.transpose(1, 2), b) for a, b in zip((dq, dk, dv), grads))
