"""Layer norm, forward and backward, against its formula in fp64, and that against differences.

Tolerances.  A row's sums run over at most 32 elements in a lane and 10 steps across lanes, so a mean
is off by at most 48 x 2^-24 of the mean of absolute values, and xh by 64 x 2^-24 (|x| + mean|x|) rstd
(ex below) with the rounding of rstd and of the products.  bf16 outputs add 2^-8 of the value."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_10743_amd as lib
    lib._load()
    return lib


def formula(x, w, b, eps, dy):
    mean = x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    y = xh * w + (0.0 if b is None else b)
    d = dy * w
    dx = rstd * (d - d.mean(-1, keepdim=True) - xh * (d * xh).mean(-1, keepdim=True))
    return y, dx, (dy * xh).sum(0), dy.sum(0), mean[:, 0], rstd[:, 0]


def test_formula_against_differences():
    g = torch.Generator().manual_seed(2)
    z = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x, w, b, dy = z(3, 9), z(9), z(9), z(3, 9)
    _, dx, dw, db, _, _ = formula(x, w, b, 1e-5, dy)
    loss = lambda x, w, b: (formula(x, w, b, 1e-5, dy)[0] * dy).sum()
    h = 1e-6
    for i, (grad, shape) in enumerate(((dx, (3, 9)), (dw, (9,)), (db, (9,)))):
        way = z(*shape)
        up, down = (loss(*[u + s * h * way if j == i else u for j, u in enumerate((x, w, b))]) for s in (1, -1))
        assert abs((up - down) / (2 * h) - (grad * way).sum()) < 1e-6


def check(kla, x, w, b, dy, eps=1e-5):
    t = x.dtype
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b, eps)
    dx, dw, db = kla.kla_layer_norm_backward(x, w, mean, rstd, dy, want_bias=b is not None)
    torch.cuda.synchronize()
    n = x.shape[-1]
    X, W, D = x.double().view(-1, n), w.double(), dy.double().view(-1, n)
    Bd = None if b is None else b.double()
    ry, rdx, rdw, rdb, rm, rr = formula(X, W, Bd, eps, D)
    r = rr[:, None]
    ex = E * (X.abs() + X.abs().mean(-1, keepdim=True)) * r
    xh = (X - rm[:, None]) * r
    d = (D * W).abs()
    last = 2.0 ** -8 if t == torch.bfloat16 else 2.0 ** -24
    mean_ = lambda u: u.mean(-1, keepdim=True)
    # rstd: half the relative error of the mean square, which is that of 2 |x - mean| ex / rstd
    er = E + mean_(xh.abs() * ex)
    tol = {"out": (last + E) * ry.abs() + (ex + er * xh.abs()) * W.abs() + (0 if b is None else 2.0 ** -23 * Bd.abs()),
           "dx": last * rdx.abs() + r * ((E + 2 * er) * (d + mean_(d) + xh.abs() * mean_(d * xh.abs()))
                                          + ex * mean_(d * xh.abs()) + xh.abs() * mean_(d * ex)),
           "dw": ((ex + (E + er) * xh.abs()) * D.abs()).sum(0), "db": E * D.abs().sum(0),
           "mean": E * X.abs().mean(-1), "rstd": er[:, 0] * rr}
    for name, got, ref in (("out", out, ry), ("dx", dx, rdx), ("dw", dw, rdw), ("db", db, rdb), ("mean", mean, rm),
                           ("rstd", rstd, rr)):
        if got is None:
            continue
        got = got.double().reshape(ref.shape)
        assert torch.isfinite(got).all(), name
        worst = ((got - ref).abs() / (tol[name] + 1e-30)).max().item() if got.numel() else 0.0
        print(f"{name} {worst:.3f} of the tolerance", flush=True)
        assert worst <= 1.0, f"{name}: {worst:.2f} times the tolerance"


def make(rows, n, dtype, bias, seed, shift=0.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = lambda *s: torch.randn(*s, generator=g, device=DEV)
    t = TYPES[dtype]
    return (shift + z(rows, n)).to(t), 1 + 0.2 * z(n), z(n) if bias else None, z(rows, n).to(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 16, 100, 127, 128, 129, 512, 513, 1000, 1001, 1024, 1026, 2047, 2048, 2056,
                               4096, 4100, 4101, 8192, 8200, 8191, 16384, 16383])
def test_widths(kla, n, dtype):
    check(kla, *make(5, n, dtype, n % 3 != 0, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", [(1, 64), (17, 64), (33, 96), (3000, 40), (2500, 960), (4500, 256), (600, 4096),
                                    (300, 5000), (9000, 33)])
def test_rows(kla, rows, n, dtype):
    """More rows than the workgroups take at once, and numbers of rows that leave groups without one."""
    check(kla, *make(rows, n, dtype, True, rows))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_from_zero_and_constant_rows(kla, dtype):
    check(kla, *make(6, 640, dtype, True, 1, shift=300.0))
    x, w, b, dy = make(4, 320, dtype, True, 2)
    x[1] = 3.0
    x[2] = 0.0
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    assert torch.allclose(out[1:3].float(), b.expand(2, -1), atol=2.0 ** -8 * b.abs().max().item())
    assert torch.allclose(rstd[1:3], torch.full((2,), 1e-5 ** -0.5, device=DEV), rtol=1e-5)
    check(kla, x, w, b, dy)


def test_eps(kla):
    x, w, b, dy = make(4, 50, "f32", True, 3)
    check(kla, 1e-3 * x, w, b, dy, eps=1e-2)
    check(kla, x, w, b, dy, eps=0.0)


def test_a_row_that_is_not_finite_is_alone(kla):
    for n in (100, 1001, 4096):
        x, w, b, dy = make(40, n, "f32", True, 4)
        want = kla.kla_layer_norm_forward(x, w, b)[0]
        x[7, 3] = math.nan
        x[9, 0] = math.inf
        got, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
        dx = kla.kla_layer_norm_backward(x, w, mean, rstd, dy)[0]
        keep = [i for i in range(40) if i not in (7, 9)]
        assert torch.equal(got[keep], want[keep]) and torch.isfinite(dx[keep]).all()
        assert torch.isnan(got[7]).all() and torch.isnan(got[9]).any()


def test_no_rows(kla):
    x, w, b, dy = make(0, 32, "bf16", True, 5)
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    dx, dw, db = kla.kla_layer_norm_backward(x, w, mean, rstd, dy)
    assert out.shape == dx.shape == (0, 32) and not dw.any() and not db.any()


def test_autograd(kla):
    x, w, b, dy = make(24, 96, "f32", True, 6)
    x3 = x.view(2, 12, 96).transpose(0, 1).requires_grad_(True)   # any shape, any strides
    w.requires_grad_(True)
    b.requires_grad_(True)
    y = kla.kla_layer_norm(x3, w, b, 1e-5)
    assert y.shape == (12, 2, 96)
    d3 = dy.view(12, 2, 96)
    dx, dw, db = torch.autograd.grad(y, (x3, w, b), d3)
    ref = formula(x3.detach().double().reshape(24, 96), w.detach().double(), b.detach().double(), 1e-5, dy.double())
    for got, want in zip((y.detach(), dx, dw, db), ref):
        assert torch.allclose(got.double().reshape(want.shape), want, rtol=1e-5, atol=1e-5)
    odd = torch.empty(24 * 96 + 1, device=DEV)[1:].view(12, 2, 96).copy_(d3)   # off 16 bytes
    assert torch.equal(torch.autograd.grad(kla.kla_layer_norm(x3, w, b), w, odd)[0], dw)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(kla.kla_layer_norm(x3, w, b), w, d3, create_graph=True)
    (dw2,) = torch.autograd.grad(kla.kla_layer_norm(x3, w), w, d3)
    assert torch.equal(dw2, dw)


def test_repeats_bit_for_bit_and_in_a_graph(kla):
    x, w, b, dy = make(3000, 768, "bf16", True, 7)

    def call():
        out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
        return (out, *kla.kla_layer_norm_backward(x, w, mean, rstd, dy))
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
    """More than 2^31 elements: rows are independent, so copies of a block give copies of its results."""
    n, rows, copies = 16384, 1000, 135
    x, w, b, dy = make(rows, n, "bf16", True, 9)
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    dx, dw, db = kla.kla_layer_norm_backward(x, w, mean, rstd, dy)
    X, DY = x.repeat(copies, 1), dy.repeat(copies, 1)
    assert X.numel() > 2 ** 31
    OUT, MEAN, RSTD = kla.kla_layer_norm_forward(X, w, b)
    DX, DW, DB = kla.kla_layer_norm_backward(X, w, MEAN, RSTD, DY)
    torch.cuda.synchronize()
    for big, small in ((OUT, out), (MEAN, mean), (RSTD, rstd), (DX, dx)):
        assert (big.view(copies, *small.shape) == small).all()
    # both sums are off by at most 2^-24 of the terms' size for each of the additions in a row
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for big, small, size in ((DW, dw, (dy.double() * xh).abs().sum(0)), (DB, db, dy.double().abs().sum(0))):
        off = (copies * rows / 256 + 64) * 2.0 ** -24 * copies * size
        assert ((big.double() - copies * small.double()).abs() <= 2 * off).all()


def test_refusals(kla):
    x, w, b, dy = make(4, 32, "f32", True, 8)
    with pytest.raises(ValueError, match="x must be contiguous"):
        kla.kla_layer_norm_forward(x.t(), w, b)
    with pytest.raises(ValueError, match="must live on a GPU"):
        kla.kla_layer_norm_forward(x.cpu(), w, b)
    with pytest.raises(ValueError, match="w must be a contiguous float32"):
        kla.kla_layer_norm_forward(x, w[:16], b)
    with pytest.raises(ValueError, match="bias must be a contiguous float32"):
        kla.kla_layer_norm_forward(x, w, b.bfloat16())
    with pytest.raises(TypeError, match="unsupported dtype"):
        kla.kla_layer_norm_forward(x.half(), w, b)
    out, mean, rstd = kla.kla_layer_norm_forward(x, w, b)
    with pytest.raises(ValueError, match="dout has shape"):
        kla.kla_layer_norm_backward(x, w, mean, rstd, dy[:2])
    with pytest.raises(ValueError, match="mean must be a contiguous float32"):
        kla.kla_layer_norm_backward(x, w, mean[:2], rstd, dy)
    for n, eps in ((16385, 1e-5), (0, 1e-5), (8, -1.0), (8, math.nan)):
        with pytest.raises(kla.KLAError) as e:
            kla.kla_layer_norm_forward(torch.zeros(2, n, device=DEV), torch.zeros(n, device=DEV), None, eps)
        assert e.value.status == 2
