"""Linear attention with a decay for each head against the recurrence in fp64, token by token, and
its adjoint; the recurrence itself against central differences.

Tolerances.  Each output is a sum of products; mass is the same sum over absolute values.  Sums are
fp32: a product of N-term sums, added up over a chunk and carried from chunk to chunk (each carry one
multiplication and one addition, the older ones decayed), is off by at most
(N + 64 + 4 chunks) 2^-24 mass.  bf16 outputs add their rounding, 2^-8 of the value, and come from scores
and states carried to 16 bits: 2 x 2^-16 mass."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_10743_amd as lib
    lib._load()
    return lib


def reference(q, k, v, g, s0, n, dy=None, ds=None):
    """fp64 on the CPU, one token after another; n: tokens of each sequence."""
    B, T, H, dk = q.shape
    gam = torch.exp(g)[:, None, None]
    out = {"y": torch.zeros(B, T, H, v.shape[-1], dtype=torch.float64), "sT": s0.clone(), "ds0": ds.clone() if ds is not None else None}
    for name, like in (("dq", q), ("dk", k), ("dv", v)):
        out[name] = torch.zeros_like(like)
    for b in range(B):
        S = s0[b]
        for t in range(int(n[b])):
            S = gam * S + k[b, t][:, :, None] * v[b, t][:, None, :]
            out["y"][b, t] = (q[b, t][:, :, None] * S).sum(1)
            if dy is not None:
                out["dq"][b, t] = (S * dy[b, t][:, None, :]).sum(2)
        out["sT"][b] = S
        if dy is None:
            continue
        Z = ds[b]
        for t in range(int(n[b]) - 1, -1, -1):
            G = Z + q[b, t][:, :, None] * dy[b, t][:, None, :]
            out["dk"][b, t] = (G * v[b, t][:, None, :]).sum(2)
            out["dv"][b, t] = (G * k[b, t][:, :, None]).sum(1)
            Z = gam * G
        out["ds0"][b] = Z
    return out


def make(B, T, H, dk, dv, dtype, state, ragged, seed, g=None):
    z = lambda *s: torch.randn(*s, generator=gen)
    gen = torch.Generator().manual_seed(seed)
    t = TYPES[dtype]
    x = dict(q=z(B, T, H, dk), k=z(B, T, H, dk) / math.sqrt(dk), v=z(B, T, H, dv), dy=z(B, T, H, dv))
    x = {n: u.to(t) for n, u in x.items()}
    x["g"] = -torch.exp2(-8 * torch.rand(H, generator=gen)) if g is None else torch.full((H,), g)
    x["s0"] = z(B, H, dk, dv) if state else None
    x["ds"] = z(B, H, dk, dv) if state else None
    x["len"] = None
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=gen, dtype=torch.int32)
        n[0], n[-1] = 0, T
        x["len"] = n
    return x


def expected(x, sign=lambda u: u):
    d = {n: None if u is None else sign(u.double()) for n, u in x.items() if n not in ("len", "g")}
    B, T, H, dk = d["q"].shape
    zero = torch.zeros(B, H, dk, d["v"].shape[-1], dtype=torch.float64)
    n = x["len"] if x["len"] is not None else torch.full((B,), T)
    return reference(d["q"], d["k"], d["v"], x["g"].double(), zero if d["s0"] is None else d["s0"], n, d["dy"],
                     zero if d["ds"] is None else d["ds"])


def run(kla, x):
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    out = kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
    out.update(kla.kla_linear_attn_backward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"], d["dy"], d["ds"]))
    torch.cuda.synchronize()
    return out


def check(got, x, what="", names=("y", "sT", "dq", "dk", "dv", "ds0")):
    ref, mass = expected(x), expected(x, torch.abs)
    T = x["q"].shape[1]
    N = max(x["q"].shape[-1], x["v"].shape[-1])
    for n in names:
        out = got[n].double().cpu()
        assert torch.isfinite(out).all(), f"{n} is not finite {what}"
        tol = (N + 64 + 4 * (T // 32 + 1)) * 2.0 ** -24 * mass[n] + 1e-30
        if got[n].dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * ref[n].abs() + 2 * 2.0 ** -16 * mass[n]
        elif n not in ("sT", "ds0"):
            tol = tol + 2.0 ** -24 * ref[n].abs()
        worst = ((out - ref[n]).abs() / tol).max().item() if out.numel() else 0.0
        print(f"{n} {worst:.3f} of the tolerance", flush=True)
        assert worst <= 1.0, f"{n}: {worst:.2f} times the tolerance {what}"


def test_reference_against_differences():
    x = {n: None if u is None else u.double() if u.is_floating_point() else u
         for n, u in make(2, 5, 2, 16, 16, "f32", True, True, 3).items()}
    n = x["len"]
    args = lambda y: (y["q"], y["k"], y["v"], y["g"], y["s0"], n)
    loss = lambda y: sum((reference(*args(y))[m] * x[d]).sum() for m, d in (("y", "dy"), ("sT", "ds")))
    got = reference(*args(x), x["dy"], x["ds"])
    g = torch.Generator().manual_seed(1)
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("s0", "ds0")):
        way = torch.randn(x[name].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        up, down = (loss({**x, name: x[name] + s * h * way}) for s in (1, -1))
        # the loss is bilinear in each argument with the rest held: differences are exact but for rounding
        assert abs((up - down) / (2 * h) - (got[grad] * way).sum()) < 1e-6


WIDTHS = [(16, 16), (16, 128), (32, 32), (32, 64), (64, 16), (64, 128), (128, 16), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
def test_widths(kla, dk, dv, dtype):
    x = make(2, 70, 3, dk, dv, dtype, True, False, dk + dv)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 97])
def test_lengths(kla, T, dtype):
    x = make(2, T, 2, 32, 32, dtype, T % 2 == 0, False, T)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(2, 1), (2, 15), (2, 17), (2, 32), (2, 97), (70, 1), (70, 40)])
def test_wide_rows_in_few_and_many_sequences(kla, B, T, dtype):
    """The rows of a state 128 wide are one wave's or two's, by the number of workgroups."""
    x = make(B, T, 3, 128, 128, dtype, True, True, B + T)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H", [(2, 3), (8, 3), (70, 3)])
@pytest.mark.parametrize("dk,dv", [(a, b) for a in (16, 32, 64, 128) for b in (16, 32, 64, 128) if a != b])
def test_two_widths(kla, dk, dv, B, H, dtype):
    """The backward runs passes of both shapes side by side."""
    x = make(B, 45, H, dk, dv, dtype, True, True, dk + dv + B)
    check(run(kla, x), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("state", [False, True])
def test_ragged_batch(kla, state, dtype):
    x = make(7, 75, 3, 64, 32, dtype, state, True, 11)
    got = run(kla, x)
    check(got, x)
    for n in ("y", "dq", "dk", "dv"):
        for b, m in enumerate(x["len"].tolist()):
            assert not got[n][b, m:].any(), f"{n} past the tokens of a sequence"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,dk,dv,ragged", [(1, 2100, 1, 64, 64, False), (2, 1111, 1, 32, 128, True),
                                                (3, 1300, 2, 16, 16, True), (1, 1025, 3, 128, 64, False),
                                                (1, 1056, 1, 128, 128, False)])
def test_few_long_sequences(kla, B, T, H, dk, dv, ragged, dtype):
    """Enough chunks and few enough sequences that they are cut into segments."""
    x = make(B, T, H, dk, dv, dtype, True, ragged, T)
    if ragged:
        x["len"][-1] = T - 1
    check(run(kla, x), x)


@pytest.mark.parametrize("g", [0.0, -1e-4, -5.0, -200.0, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decays(kla, g, dtype):
    x = make(2, 90, 2, 32, 32, dtype, True, False, 5, g)
    check(run(kla, x), x)
    x = make(1, 700, 1, 16, 16, dtype, True, False, 6, g)
    check(run(kla, x), x)


def test_no_tokens(kla):
    x = make(2, 0, 3, 32, 16, "bf16", True, False, 1)
    got = run(kla, x)
    assert got["y"].shape == (2, 0, 3, 16) and got["dk"].shape == (2, 0, 3, 32)
    assert torch.equal(got["sT"].cpu(), x["s0"]) and torch.equal(got["ds0"].cpu(), x["ds"])
    x["s0"] = x["ds"] = None
    got = run(kla, x)
    assert not got["sT"].any() and not got["ds0"].any()


def test_lengths_are_taken_into_the_sequence(kla):
    x = make(3, 40, 2, 32, 16, "f32", True, True, 2)
    x["len"] = torch.tensor([-7, 33, 41], dtype=torch.int32)
    got = run(kla, x)
    x["len"] = torch.tensor([0, 33, 40], dtype=torch.int32)
    want = run(kla, x)
    check(want, x)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_heads_by_eight_and_a_given_output(kla):
    """Sequences in groups of eight go to the dies in another order; the output may be the caller's."""
    x = make(4, 50, 4, 128, 128, "bf16", True, True, 6)
    check(run(kla, x), x)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    want = kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
    y = torch.full_like(d["v"], math.nan)
    got = kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"], want_state=False, y=y)
    assert got["y"] is not None and torch.equal(y, want["y"]) and got["sT"] is None
    ys = torch.full_like(d["v"][:, 0], math.nan)
    s = d["s0"].clone()
    out = kla.kla_linear_attn_step(*(d[n][:, 0].contiguous() for n in ("q", "k", "v")), d["g"], s, y=ys)
    assert torch.isfinite(ys).all() and torch.equal(out["y"], ys) and out["state"] is s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_small_values(kla, dtype):
    """States near the ends of fp32's range, fast and slow decays.

    dq is the product of dy and the state: about 1e17 * 1e34 = 1e51 at the large scale, past the 3.4e38 of either
    type, so the formula itself has no finite value there and the others are checked."""
    for g in (-0.01, -0.3):
        for scale in (1e17, 1e-17):
            x = make(1, 200, 1, 16, 16, dtype, True, False, 3, g)
            for n in ("k", "v", "dy"):
                x[n] = x[n] * scale
            x["s0"], x["ds"] = x["s0"] * scale ** 2, x["ds"] * scale
            names = ("y", "sT", "dk", "dv", "ds0") if scale > 1 else ("y", "sT", "dq", "dk", "dv", "ds0")
            check(run(kla, x), x, f"g {g} scale {scale}", names)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [1, 45, 98])
@pytest.mark.parametrize("bad,width", [(math.nan, 32), (math.inf, 32), (math.nan, 128), (math.inf, 128)])
def test_values_that_are_not_finite_stay_in_their_future(kla, dtype, bad, width, at):
    """A bad value at one token leaves the outputs of earlier ones as they are, and in the backward the
    gradients of later ones."""
    clean = make(1, 100, 2, width, width, dtype, True, False, 9)
    want = run(kla, clean)
    for name in ("q", "k", "v", "dy"):
        x = {n: None if u is None else u.clone() for n, u in clean.items()}
        x[name][0, at, 1] = bad
        got = run(kla, x)
        head = lambda n: (got[n][:, :, 0], want[n][:, :, 0])
        for n in ("y", "dq", "dk", "dv"):
            assert torch.equal(*head(n)), f"{n} of the other head changed"
            late = n in ("dk", "dv")   # they look ahead, the others back
            a, b = (u[n][0, at + 1:, 1] if late else u[n][0, :at, 1] for u in (got, want))
            # a chunk that holds the value is added up in another order: rounding of one product sum
            assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if dtype == "bf16" else 1e-4, atol=1e-4), (name, n)
        if name in ("k", "v"):
            assert not torch.isfinite(got["y"][0, at:, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,H,dk,dv", [(1, 1, 16, 16), (1, 16, 128, 128), (5, 3, 32, 64), (4, 2, 64, 32), (3, 2, 128, 16),
                                       (2, 3, 16, 128), (9, 16, 128, 128)])
def test_step(kla, S, H, dk, dv, dtype):
    x = make(S, 4, H, dk, dv, dtype, True, False, S + dk)
    ref, mass = expected(x), expected(x, torch.abs)
    s = x["s0"].to(DEV)
    g = x["g"].to(DEV)
    for t in range(4):
        q, k, v = (x[n][:, t].contiguous().to(DEV) for n in ("q", "k", "v"))
        y = kla.kla_linear_attn_step(q, k, v, g, s)["y"]
        r, m = ref["y"][:, t], mass["y"][:, t]
        # dk products, and per token a rounded factor, product and sum
        tol = (dk + 8 * (t + 1)) * 2.0 ** -24 * m + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * r.abs()
        assert ((y.double().cpu() - r).abs() <= tol).all(), t
    assert ((s.double().cpu() - ref["sT"]).abs() <= 32 * 2.0 ** -24 * mass["sT"]).all()


def test_prompt_then_tokens(kla):
    """A prompt's state serves the single tokens that follow, and a prompt may be read in pieces."""
    x = make(3, 96, 2, 64, 64, "f32", False, False, 21)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    whole = kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"])
    cut = lambda a, b: [d[n][:, a:b].contiguous() for n in ("q", "k", "v")]
    one = kla.kla_linear_attn_forward(*cut(0, 41), d["g"])
    two = kla.kla_linear_attn_forward(*cut(41, 90), d["g"], one["sT"])
    ys = [one["y"], two["y"]]
    s = two["sT"]
    for t in range(90, 96):
        ys.append(kla.kla_linear_attn_step(*(u[:, 0].contiguous() for u in cut(t, t + 1)), d["g"], s)["y"][:, None])
    check({**run(kla, x), "y": torch.cat(ys, 1), "sT": s}, x)
    assert torch.allclose(whole["sT"], s, rtol=1e-4, atol=1e-5)


def test_autograd(kla):
    x = make(2, 50, 2, 32, 64, "f32", True, True, 4)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    ins = [d[n].requires_grad_(True) for n in ("q", "k", "v", "s0")]
    y, sT = kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
    grads = torch.autograd.grad([y, sT], ins, [d["dy"], d["ds"]])
    check(dict(zip(("y", "sT", "dq", "dk", "dv", "ds0"), (y.detach(), sT.detach(), *grads))), x)
    # an output that is not used has no gradient, and a start state that is broadcast sums its own
    one = torch.randn(1, 2, 32, 64, device=DEV, requires_grad=True)
    _, sT = kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"], one.expand(2, -1, -1, -1).contiguous(), d["len"])
    (g1,) = torch.autograd.grad(sT, one, d["ds"])
    want = (torch.exp(d["g"].double()[:, None, None] * d["len"].view(-1, 1, 1, 1)) * d["ds"].double()).sum(0, keepdim=True)
    assert torch.allclose(g1.double(), want, rtol=1e-5, atol=1e-6)
    y, _ = kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
    odd = torch.empty(d["dy"].numel() + 1, device=DEV)[1:].view_as(d["dy"]).copy_(d["dy"])   # off 16 bytes
    assert torch.equal(torch.autograd.grad(y, d["q"], odd, retain_graph=True)[0], torch.autograd.grad(y, d["q"], d["dy"])[0])
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"])[0], d["q"], d["dy"], create_graph=True)
    with pytest.raises(ValueError, match="constants"):
        kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"].clone().requires_grad_(True))


def test_repeats_bit_for_bit_and_in_a_graph(kla):
    """Also on another stream, replayed with other work between."""
    x = make(1, 900, 2, 64, 64, "bf16", True, False, 8)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    call = lambda: {**kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"]),
                    **kla.kla_linear_attn_backward(d["q"], d["k"], d["v"], d["g"], d["s0"], None, d["dy"], d["ds"])}
    want = call()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        again = call()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(want[n], again[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(4):
        for u in out.values():
            u.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], out[n]) for n in want), i
        call()
        torch.randn(1 << 20, device=DEV).sum().item()


def test_training_step_in_a_graph(kla):
    """Forward and backward through autograd, captured whole and replayed on new inputs."""
    x = make(2, 600, 2, 32, 64, "bf16", True, True, 12)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    ins = [d[n].requires_grad_(True) for n in ("q", "k", "v", "s0")]

    def step():
        y, sT = kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
        return (y.detach(), sT.detach(), *torch.autograd.grad([y, sT], ins, [d["dy"], d["ds"]]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        with torch.no_grad():
            for u in (*ins, d["dy"]):
                u.add_(0.125 * torch.randn_like(u))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), i


def test_past_32_bits(kla):
    """More than 2^31 elements, in the batch and along one sequence whose states forget all but the last 100 tokens."""
    x = make(16, 2048, 16, 128, 128, "bf16", False, True, 5)
    small = run(kla, x)
    copies = 33
    big = run(kla, {n: None if u is None else u if n == "g" else u.to(DEV).repeat(copies, *[1] * (u.dim() - 1)) for n, u in x.items()})
    assert big["y"].numel() > 2 ** 31
    for n in ("y", "sT", "dq", "dk", "dv"):
        assert (big[n].view(copies, *small[n].shape) == small[n]).all(), n
    del big
    H, T, last = 128, 132000, 320
    gen = torch.Generator(device=DEV).manual_seed(6)
    z = lambda: torch.randn(1, T, H, 128, generator=gen, device=DEV, dtype=torch.bfloat16)
    x = dict(q=z(), k=z(), v=z(), dy=z(), g=torch.full((H,), -1.0), s0=None, ds=None, len=None)
    assert x["q"].numel() > 2 ** 31
    got = run(kla, x)
    heads = [0, H - 1]
    end = {n: x[n][:, -last:, heads].cpu() for n in ("q", "k", "v", "dy")}
    end.update(g=x["g"][heads], s0=None, ds=None, len=None)
    # y and dq of the last tokens, which the tokens before `last` reach by e^-128 at most, under fp32's smallest
    tail = {n: got[n][:, -last:, heads].cpu() for n in ("y", "dq", "dk", "dv")}
    ref, mass = expected(end), expected(end, torch.abs)
    for n, at in (("y", 128), ("dq", 128), ("dk", 0), ("dv", 0)):
        a, r, m = (u[:, at:] for u in (tail[n].double(), ref[n], mass[n]))
        tol = (128 + 64 + 4 * 11) * 2.0 ** -24 * m + 2.0 ** -8 * r.abs() + 2 * 2.0 ** -16 * m + 1e-30
        assert ((a - r).abs() <= tol).all(), n


@pytest.mark.parametrize("T", [40, 700])
def test_a_decay_that_is_no_number(kla, T):
    """Its head has no value; the others keep theirs."""
    x = make(2, T, 2, 32, 32, "f32", True, False, 15)
    want = run(kla, x)
    x["g"] = torch.tensor([math.nan, x["g"][1]])
    got = run(kla, x)
    for n in ("y", "sT", "dq", "dk", "dv", "ds0"):
        head = (lambda u, h: u[:, :, h]) if n in ("y", "dq", "dk", "dv") else lambda u, h: u[:, h]
        assert torch.equal(head(got[n], 1), head(want[n], 1)), n
    assert torch.isnan(got["sT"][:, 0]).all() and torch.isnan(got["y"][:, 1:, 0]).all()
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    out = kla.kla_linear_attn_step(*(d[n][:, 0].contiguous() for n in ("q", "k", "v")), d["g"], d["s0"])
    assert torch.isnan(out["y"][:, 0]).all() and torch.isfinite(out["y"][:, 1]).all()


def test_outputs_apart_from_inputs(kla):
    """An output that overlaps an input is refused, and a state that a backward saved is known to have changed."""
    x = make(2, 8, 2, 16, 16, "f32", True, False, 1)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    one = [d[n][:, 0].contiguous() for n in ("q", "k", "v")]
    for n in ("q", "k", "v"):
        with pytest.raises(ValueError, match="y must not overlap"):
            kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"], d["s0"], y=d[n])
    for u in one:
        with pytest.raises(ValueError, match="y must not overlap"):
            kla.kla_linear_attn_step(*one, d["g"], d["s0"], y=u)
    with pytest.raises(ValueError, match="state must not overlap"):
        kla.kla_linear_attn_step(d["s0"].view(-1)[:64].view(2, 2, 16), *one[1:], d["g"], d["s0"])
    y, sT = kla.kla_linear_attn(d["q"].requires_grad_(True), d["k"], d["v"], d["g"], d["s0"])
    kla.kla_linear_attn_step(*one, d["g"], d["s0"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        kla.kla_linear_attn_step(*one, d["g"], torch.zeros_like(d["s0"]))


def test_threads(kla):
    """Two threads, each on a stream of its own, give what one gives."""
    import threading
    xs = [make(2, 600, 2, 64, 64, "bf16", True, True, 30 + i) for i in range(2)]
    want = [run(kla, x) for x in xs]
    got = [[], []]

    def work(i):
        d = {n: None if u is None else u.to(DEV) for n, u in xs[i].items()}
        ins = [d[n].requires_grad_(True) for n in ("q", "k", "v", "s0")]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(10):
                y, sT = kla.kla_linear_attn(d["q"], d["k"], d["v"], d["g"], d["s0"], d["len"])
                grads = torch.autograd.grad([y, sT], ins, [d["dy"], d["ds"]])
                got[i].append(dict(zip(("y", "sT", "dq", "dk", "dv", "ds0"), (y, sT, *grads))))
            stream.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(got[i]) == 10
        for out in got[i]:
            assert all(torch.equal(out[n], want[i][n]) for n in out)


def test_refusals(kla):
    x = make(2, 8, 2, 32, 16, "f32", True, False, 1)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    fwd = lambda **c: kla.kla_linear_attn_forward(*({**d, **c}[n] for n in ("q", "k", "v", "g", "s0", "len")))
    for bad, match in ((dict(q=d["q"][0]), r"q must be \[B, T, H, dk\]"), (dict(k=d["k"][:, :4].contiguous()), "k has shape"),
                       (dict(v=d["v"].bfloat16()), "v must share"), (dict(v=d["v"].transpose(1, 2).contiguous().transpose(1, 2)), "v must be contiguous"),
                       (dict(g=d["g"].double()), "g must be a contiguous float32"), (dict(g=d["g"][:1]), "g must be a contiguous float32"),
                       (dict(s0=d["s0"][:1]), "s0 must be a contiguous float32"),
                       (dict(len=torch.zeros(2, dtype=torch.int64, device=DEV)), "lengths must be a contiguous int32"),
                       (dict(len=torch.zeros(2, dtype=torch.int32)), "lengths must be a contiguous int32"),
                       (dict(q=d["q"].cpu()), "must live on a GPU")):
        with pytest.raises(ValueError, match=match):
            fwd(**bad)
    with pytest.raises(TypeError, match="unsupported dtype"):
        fwd(q=d["q"].half())
    with pytest.raises(kla.KLAError) as e:
        fwd(q=d["q"][..., :24].contiguous(), k=d["k"][..., :24].contiguous(), s0=None)
    assert e.value.status == 2
    with pytest.raises(ValueError, match="dy has shape"):
        kla.kla_linear_attn_backward(d["q"], d["k"], d["v"], d["g"], None, None, d["dy"][:1])
    q, k, v = (d[n][:, 0].contiguous() for n in ("q", "k", "v"))
    with pytest.raises(ValueError, match="state must be a contiguous float32"):
        kla.kla_linear_attn_step(q, k, v, d["g"], d["s0"][:1])
    with pytest.raises(ValueError, match="k has shape"):
        kla.kla_linear_attn_step(q, k[:1], v, d["g"], d["s0"])


def test_domain_check(kla, monkeypatch):
    monkeypatch.setenv("KLA_CHECK", "1")
    x = make(1, 8, 2, 16, 16, "f32", False, False, 1)
    d = {n: None if u is None else u.to(DEV) for n, u in x.items()}
    kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], d["g"])
    for bad in (0.5, math.nan):
        g = d["g"].clone()
        g[1] = bad
        with pytest.raises(kla.KLAError) as e:
            kla.kla_linear_attn_forward(d["q"], d["k"], d["v"], g)
        assert e.value.status == 6
