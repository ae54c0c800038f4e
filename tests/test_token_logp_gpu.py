"""Log probabilities of tokens, entropies, top alternatives and the logits' gradient against their
formulas in fp64, and those against differences.

Tolerances.  A sum over V tokens is added up in at most V / 256 + 64 steps by a thread and across
threads, so sums are off by that many 2^-24 of themselves (es); e^d is off by 2^-23 (1 + 2 |d|) of
itself, the argument's rounding."""
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


def formula(x, target, dlogp, dent):
    """fp64: x [R, V], the rest [R]; target -1 for none."""
    empty = torch.isneginf(x).all(-1, keepdim=True)
    lp = torch.log_softmax(torch.where(empty, 0.0, x), -1)
    p = torch.where(empty, 0.0, lp.exp())
    have = target >= 0
    logp = torch.where(have, lp.gather(-1, target.clamp_min(0)[:, None])[:, 0], 0.0)
    logp = torch.where(have & empty[:, 0], -math.inf, logp)
    plp = torch.where(p > 0, p * lp, 0.0)
    entropy = -plp.sum(-1)
    d = torch.where(have, dlogp, 0.0)[:, None]
    dx = -d * p
    dx.scatter_add_(-1, target.clamp_min(0)[:, None], d)
    dx = dx - dent[:, None] * (plp + p * entropy[:, None])
    return logp, entropy, torch.where(empty, 0.0, dx), lp, p


def test_formula_against_differences():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4, 11, generator=g, dtype=torch.float64)
    x[1, 3] = -math.inf
    target = torch.tensor([0, 10, -1, 4])
    dlogp, dent = torch.randn(4, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    way = torch.randn(4, 11, generator=g, dtype=torch.float64)
    loss = lambda x: sum((a * b).sum() for a, b in zip(formula(x, target, dlogp, dent)[:2], (dlogp, dent)))
    h = 1e-6
    assert abs((loss(x + h * way) - loss(x - h * way)) / (2 * h) - (formula(x, target, dlogp, dent)[2] * way).sum()) < 1e-6


def best_of(x, K):
    """The largest, the lower index first among equals."""
    return torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :K]


def check(kla, x, target, top=0, entropy=True, seed=0):
    lead, V = x.shape[:-1], x.shape[-1]
    g = torch.Generator(device=DEV).manual_seed(seed)
    dlogp, dent = (torch.randn(lead, generator=g, device=DEV) for _ in range(2))
    out = kla.kla_token_logp_forward(x, target, want_entropy=entropy, top=top, save=True)
    dx = kla.kla_token_logp_backward(x, target, out["stat"], out["entropy"], dlogp, dent if entropy else None)
    torch.cuda.synchronize()
    X = x.double().view(-1, V)
    tg = target.expand(lead).reshape(-1)
    if not entropy:
        dent = torch.zeros_like(dent)
    DL, DE = dlogp.double().view(-1), dent.double().view(-1)
    logp, ent, rdx, lp, p = formula(X, tg, DL, DE)
    es = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -20
    alive = torch.isfinite(logp)
    assert torch.equal(out["logp"].view(-1)[~alive], logp[~alive].float())
    tol = es + 2.0 ** -22 * (logp.abs() + math.log(V) + 1)
    assert ((out["logp"].double().view(-1) - logp).abs() <= tol)[alive].all()
    if entropy:
        # u / s and log s: each as near as the sums, relative to themselves
        assert ((out["entropy"].double().view(-1) - ent).abs() <= 4 * es * (1 + math.log(V))).all()
    lpf = torch.where(p > 0, lp, 0.0)
    ep = es + 2.0 ** -22 * (1 + lpf.abs() + math.log(V))
    size = p * (DL.abs()[:, None] + DE.abs()[:, None] * (lpf.abs() + ent[:, None] + 4 * (1 + math.log(V))))
    tol = 2 * ep * size + (2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -23) * rdx.abs() + 1e-30
    tol = tol + 2.0 ** -22 * torch.zeros_like(tol).scatter_(1, tg.clamp_min(0)[:, None], DL.abs()[:, None])
    # probabilities under fp32's smallest normal number are taken as none
    tol = tol + 2.0 ** -120
    assert torch.isfinite(dx).all()
    worst = ((dx.double().view(-1, V) - rdx).abs() / tol).max().item()
    print(f"dlogits {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0
    if top:
        idx = best_of(X, top)
        assert torch.equal(out["top_index"].view(-1, top), idx)
        want = lp.gather(-1, idx)
        want = torch.where(torch.isneginf(X).all(-1, keepdim=True), -math.inf, want)
        got = out["top_logp"].double().view(-1, top)
        fin = torch.isfinite(want)
        assert torch.equal(got[~fin], want[~fin])
        assert ((got - want).abs() <= es + 2.0 ** -22 * (want.abs() + math.log(V) + 1))[fin].all()
    return out, dx


def make(lead, V, dtype, seed, scale=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (scale * torch.randn(*lead, V, generator=g, device=DEV)).to(TYPES[dtype])
    target = torch.randint(-1, V, lead[-1:], generator=g, device=DEV)
    return x, target


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 5, 8, 31, 63, 64, 255, 257, 1000, 1001, 2053, 8192, 8201, 32003])
def test_vocabularies(kla, V, dtype):
    check(kla, *make((5,), V, dtype, V), top=min(V, 9))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,top", [(1, 50257, 32), (2, 128000, 16), (1, 300001, 7), (40, 9000, 1), (1100, 5003, 8),
                                        (1030, 131, 5)])
def test_few_and_many_rows(kla, rows, V, top, dtype):
    """Rows cut over several workgroups, and rows that are not."""
    check(kla, *make((rows,), V, dtype, rows + V), top=top)


@pytest.mark.parametrize("top", [0, 1, 2, 31, 32])
def test_top(kla, top):
    check(kla, *make((20,), 700, "bf16", top), top=top, entropy=top % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_draws_share_their_targets(kla, dtype):
    x, target = make((4, 37), 999, dtype, 3)
    check(kla, x, target)
    x, _ = make((3, 2, 37), 120, dtype, 4)
    check(kla, x, target.clamp_max(119), top=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,rows", [(400, 8), (40000, 3)])
def test_masked_tokens(kla, V, rows, dtype):
    """-inf and the type's lowest value in masked places, rows with fewer tokens left than alternatives,
    one and none."""
    x, target = make((rows + 4,), V, dtype, V)
    off = torch.rand(rows + 4, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) < 0.5
    x.masked_fill_(off, -math.inf)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, V // 2] = 1.5
    target[1] = V // 2
    x[2] = -math.inf
    x[2, 3:8] = torch.arange(5, device=DEV).to(x.dtype)
    lowest = torch.finfo(x.dtype).min
    x[3] = lowest
    x[4, ::2] = lowest
    target[0], target[3] = 5, 2
    target[2] = 0   # itself masked: -inf
    out, dx = check(kla, x, target, top=12)
    assert out["logp"][0] == -math.inf and out["entropy"][0] == 0 and not dx[0].any()
    assert out["top_index"][0].tolist() == list(range(12))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties(kla, dtype):
    """Equal logits: the lower index first, also where all are equal, and zeros of both signs."""
    x, target = make((6,), 5000, dtype, 2)
    x[0] = 0.25
    x[1] = x[1].round()
    x[2] = 0.0
    x[2, 1::2] = -0.0
    x[3, 4000:] = 20.0
    x[4] = -1.0
    x[4, 77], x[4, 4999] = 2.0, 2.0
    check(kla, x, target, top=32)
    check(kla, x.repeat(1, 8)[:2].contiguous(), target[:2], top=20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rising_rows(kla, dtype):
    """Rows in order, whose first elements say nothing about the largest."""
    x, target = make((3,), 40000, dtype, 5)
    x = x.sort(-1).values.contiguous()
    x[1] = x[1].flip(0)
    check(kla, x, target, top=8)
    check(kla, x.repeat(300, 1), target.repeat(300), top=32)


def test_large_logits(kla):
    for scale, at in ((1.0, 3e4), (100.0, 0.0), (1.0, -1e6)):
        x, target = make((7,), 1500, "f32", 9, scale)
        check(kla, x + at, target, top=4)


def test_values_that_are_not_finite(kla):
    x, target = make((5,), 3000, "f32", 10)
    clean = x.clone()
    want = kla.kla_token_logp_forward(clean, target, want_entropy=True, top=3)
    x[1, 17] = math.nan
    x[3, 5] = math.inf
    target[1] = target[3] = 2
    got = kla.kla_token_logp_forward(x, target, want_entropy=True, top=3, save=True)
    for n in ("logp", "entropy", "top_logp", "top_index"):
        assert torch.equal(got[n][[0, 2, 4]], want[n][[0, 2, 4]]), n
    assert torch.isnan(got["logp"][1]) and 17 not in got["top_index"][1].tolist()
    assert got["top_index"][3, 0] == 5 and torch.isnan(got["entropy"][3])
    one = torch.ones(5, device=DEV)
    dx = kla.kla_token_logp_backward(x, target, got["stat"], got["entropy"], one)
    assert torch.isfinite(dx[[0, 2, 4]]).all() and torch.isnan(dx[1]).any()
    few = torch.full((1, 6), math.nan, device=DEV)
    few[0, 4] = 1.0
    out = kla.kla_token_logp_forward(few, torch.tensor([-1], device=DEV), top=3)
    assert out["top_index"].tolist() == [[4, -1, -1]] and torch.isnan(out["top_logp"]).all()


def test_targets_outside(kla):
    x, target = make((4,), 300, "f32", 11)
    target[:] = torch.tensor([-100, 300, 299, 0], device=DEV)
    out = kla.kla_token_logp_forward(x, target, save=True)
    assert out["logp"][0] == 0 and torch.isnan(out["logp"][1]) and torch.isfinite(out["logp"][2:]).all()
    dx = kla.kla_token_logp_backward(x, target, out["stat"], None, torch.ones(4, device=DEV))
    assert not dx[0].any() and torch.isnan(dx[1]).any() and torch.isfinite(dx[2:]).all()


def test_no_rows(kla):
    x, target = make((3, 0), 50, "bf16", 1)
    out = kla.kla_token_logp_forward(x, target, want_entropy=True, top=2, save=True)
    assert out["logp"].shape == (3, 0) and out["top_index"].shape == (3, 0, 2)
    assert kla.kla_token_logp_backward(x, target, out["stat"], out["entropy"], out["logp"]).shape == (3, 0, 50)


def test_autograd(kla):
    x, target = make((3, 8), 65, "f32", 12)
    x.requires_grad_(True)
    g = torch.Generator(device=DEV).manual_seed(1)
    dlogp, dent = (torch.randn(3, 8, generator=g, device=DEV) for _ in range(2))
    logp, ent = kla.kla_token_logp(x, target, want_entropy=True)
    (dx,) = torch.autograd.grad([logp, ent], x, [dlogp, dent], retain_graph=True)
    X = x.detach().double().view(-1, 65)
    tg = target.expand(3, 8).reshape(-1)
    f = lambda a, b: formula(X, tg, a.double().view(-1), b.double().view(-1))[2].view(3, 8, 65)
    assert torch.allclose(dx.double(), f(dlogp, dent), atol=1e-5)
    (de,) = torch.autograd.grad(ent, x, dent)   # one of the two alone
    assert torch.allclose(de.double(), f(0 * dlogp, dent), atol=1e-5)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(ent, x, dent, create_graph=True)
    # slices that start off 16 bytes, of the logits, the targets and the gradients
    (do,) = torch.autograd.grad(kla.kla_token_logp(x[1, 1:], target[1:]), x, torch.cat([dlogp[1], dlogp[0]])[1:8])
    assert torch.allclose(do[1, 1:].double(), f(dlogp, 0 * dent)[1, 1:], atol=1e-5) and not do[0].any()
    (dl,) = torch.autograd.grad(kla.kla_token_logp(x, target), x, dlogp)
    assert torch.allclose(dl.double(), f(dlogp, 0 * dent), atol=1e-5)


def test_repeats_bit_for_bit_and_in_a_graph(kla):
    for lead, V in (((2,), 40000), ((1200,), 700)):
        x, target = make(lead, V, "bf16", 13)
        dlogp = torch.randn(lead, device=DEV)

        def call():
            out = kla.kla_token_logp_forward(x, target, want_entropy=True, top=8, save=True)
            return (*out.values(), kla.kla_token_logp_backward(x, target, out["stat"], out["entropy"], dlogp, dlogp))
        want = call()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            again = call()
        torch.cuda.current_stream().wait_stream(stream)
        assert all(map(torch.equal, want, again))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        for i in range(4):
            for u in out:
                u.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(map(torch.equal, want, out)), i
            call()
            torch.randn(1 << 20, device=DEV).sum().item()


def test_past_32_bits(kla):
    """More than 2^31 logits: rows are independent, so copies of a block give copies of its results."""
    rows, V, copies = 1000, 131072, 17
    x, target = make((rows,), V, "bf16", 9)

    def call(x, target, rep):
        out = kla.kla_token_logp_forward(x, target, want_entropy=True, top=5, save=True)
        d = torch.linspace(-1, 1, rows, device=DEV).repeat(rep)
        return (*out.values(), kla.kla_token_logp_backward(x, target, out["stat"], out["entropy"], d, -d))
    small = call(x, target, 1)
    X = x.repeat(copies, 1)
    assert X.numel() > 2 ** 31
    big = call(X, target.repeat(copies), copies)
    torch.cuda.synchronize()
    for a, b in zip(big, small):
        assert (a.view(copies, *b.shape) == b).all()


def test_refusals(kla):
    x, target = make((2, 4), 50, "f32", 14)
    with pytest.raises(ValueError, match="target has shape"):
        kla.kla_token_logp_forward(x, target[:3])
    with pytest.raises(ValueError, match="target must be a contiguous int64"):
        kla.kla_token_logp_forward(x, target.int())
    with pytest.raises(ValueError, match="target must be a contiguous int64"):
        kla.kla_token_logp_forward(x, target.cpu())
    with pytest.raises(ValueError, match="logits must be contiguous"):
        kla.kla_token_logp_forward(x.transpose(0, 1), torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError, match="must live on a GPU"):
        kla.kla_token_logp_forward(x.cpu(), target)
    with pytest.raises(TypeError, match="unsupported dtype"):
        kla.kla_token_logp_forward(x.double(), target)
    with pytest.raises(ValueError, match="top must not be negative"):
        kla.kla_token_logp_forward(x, target, top=-1)
    for top in (33, 51):
        with pytest.raises(kla.KLAError) as e:
            kla.kla_token_logp_forward(x, target, top=top)
        assert e.value.status == 2
    out = kla.kla_token_logp_forward(x, target, save=True)
    with pytest.raises(kla.KLAError) as e:   # the entropy's gradient needs the entropy
        kla.kla_token_logp_backward(x, target, out["stat"], None, None, out["logp"])
    assert e.value.status == 1
    with pytest.raises(ValueError, match="stat must be a contiguous float32"):
        kla.kla_token_logp_backward(x, target, out["logp"], None, out["logp"])
