"""A layer of a hybrid stack as a model uses it: layer norm, a fused projection, the norms of queries and keys with the
rotation, windowed attention, the output projection, then linear attention as the next layer's mixer, the head and the
tokens' log probabilities, with every gradient, against the same in fp64; then the serving form of the same layer."""
import math
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_10743_amd as K
    return K


def norm(x, w, b):
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    return (x - mean) / torch.sqrt(var + 1e-5) * w + b


def rope(q, k, wq, wk, freq, pos):
    out = []
    for x, w in ((q, wq), (k, wk)):
        u = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        phi = pos.double()[..., None, None] * freq
        P = freq.numel()
        a, b = u[..., :P], u[..., P:2 * P]
        out.append(torch.cat((a * phi.cos() - b * phi.sin(), b * phi.cos() + a * phi.sin(), u[..., 2 * P:]), -1))
    return out


def attn(q, k, v, window, sinks, lengths):
    T, G = q.shape[1], q.shape[2] // k.shape[2]
    k, v = (t.repeat_interleave(G, 2) for t in (k, v))
    i = torch.arange(T, device=q.device)
    see = (i <= i[:, None]) & ((i > i[:, None] - window) | (i < sinks))
    s = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(q.shape[-1])
    y = torch.einsum("bhij,bjhd->bihd", torch.softmax(s.masked_fill(~see, -math.inf), -1), v)
    return torch.where((i < lengths[:, None])[..., None, None], y, 0.0)


def mixer(q, k, v, g, s0, lengths):
    S, ys = torch.zeros(q.shape[0], q.shape[2], q.shape[3], v.shape[3], dtype=q.dtype, device=q.device), []
    for t in range(q.shape[1]):
        live = (t < lengths).view(-1, 1, 1, 1)
        S = torch.where(live, torch.exp(g)[:, None, None] * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        ys.append(torch.where(live[..., 0], (q[:, t, :, :, None] * S).sum(-2), 0.0))
    return torch.stack(ys, 1), S


def logp(u, t):
    lp = torch.log_softmax(u, -1)
    return torch.where(t >= 0, lp.gather(-1, t.clamp_min(0)[..., None])[..., 0], 0.0)


SIZES = dict(B=3, T=83, C=72, H=4, Hk=2, d=32, W=20, sinks=3, V=301)


def layer(p, x, pos, lengths, f, z=SIZES):
    """Up to the attention layer's output, and the rotated keys and the values."""
    h = f["norm"](x, p["w1"], p["b1"])
    qkv = (h @ p["wqkv"]).unflatten(-1, (z["H"] + 2 * z["Hk"], z["d"]))
    q, k, v = qkv.split([z["H"], z["Hk"], z["Hk"]], -2)
    q, k = f["rope"](q, k, p["wq"], p["wk"], p["freq"], pos)
    y = f["attn"](q, k, v, z["W"], z["sinks"], lengths)
    return x + y.flatten(-2) @ p["wo"], q, k, v


def model(p, x, pos, target, lengths, f):
    x, *_ = layer(p, x, pos, lengths, f)
    a, b, c = (t.unflatten(-1, (2, 16)) for t in (f["norm"](x, p["w2"], p["b2"]) @ p["wabc"]).chunk(3, -1))
    y, _ = f["mixer"](a, b, c, p["g"], None, lengths)
    return f["logp"]((x + y.flatten(-2) @ p["wy"]) @ p["head"], target)


def make(seed=5):
    z = SIZES
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s, c=1.0: (c * torch.randn(*s, generator=gen)).to(DEV)
    C, H, Hk, d = z["C"], z["H"], z["Hk"], z["d"]
    p = dict(w1=1 + r(C, c=0.1), b1=r(C, c=0.1), wqkv=r(C, (H + 2 * Hk) * d, c=C ** -0.5), wq=1 + r(d, c=0.2), wk=1 + r(d, c=0.2),
             wo=r(H * d, C, c=0.1), w2=1 + r(C, c=0.1), b2=r(C, c=0.1), wabc=r(C, 96, c=0.3 * C ** -0.5), wy=r(32, C, c=0.1),
             head=r(C, z["V"], c=0.3), g=torch.tensor([-0.05, -0.6], device=DEV),
             freq=(10000.0 ** (-torch.arange(8, dtype=torch.float64) / 8)).to(DEV))
    x = r(z["B"], z["T"], C)
    pos = (torch.arange(z["T"], dtype=torch.int32) + torch.tensor([[0], [1000], [7]], dtype=torch.int32)).to(DEV)
    lengths = torch.tensor([z["T"], 0, 61], dtype=torch.int32, device=DEV)
    target = torch.randint(0, z["V"], (z["B"], z["T"]), generator=gen).to(DEV)
    target = torch.where(torch.arange(z["T"], device=DEV) < lengths[:, None], target, -1)
    return p, x, pos, lengths, target


def test_training_step(kla):
    p, x, pos, lengths, target = make()
    ours = dict(norm=kla.kla_layer_norm, rope=kla.kla_qk_norm_rope, attn=kla.kla_window_attn, mixer=kla.kla_linear_attn,
                logp=kla.kla_token_logp)
    plain = dict(norm=norm, rope=rope, attn=attn, mixer=mixer, logp=logp)
    fixed = ("g", "freq")
    names = [n for n in p if n not in fixed]
    res = []
    for f, cast in ((ours, lambda t: t), (plain, torch.Tensor.double)):
        q = {n: (cast(u).detach().requires_grad_(True) if n not in fixed else u) for n, u in p.items()}
        xin = cast(x).detach().requires_grad_(True)
        out = model(q, xin, pos, target, lengths, f)
        res.append([out.detach(), *torch.autograd.grad(out.sum(), [xin] + [q[n] for n in names])])
    for n, a, b in zip(["logp", "x"] + names, *res):
        assert torch.isfinite(a).all(), n
        rel = ((a.double() - b).norm() / b.norm()).item()
        # fp32 products and sums of some hundred terms, one operator after another: each about 2^-24 sqrt(100)
        print(f"{n} {rel:.2e}", flush=True)
        assert rel < 2e-5, f"{n}: {rel:.2e}"


def test_serving(kla):
    """A prompt with its cache, then single tokens: the layer's outputs are those of the whole sequence."""
    p, x, pos, _, _ = make(9)
    z = SIZES
    whole = torch.full((z["B"],), z["T"], dtype=torch.int32, device=DEV)
    d = {n: u.double() if u.is_floating_point() else u for n, u in p.items()}
    want, *_ = layer(d, x.double(), pos, whole, dict(norm=norm, rope=rope, attn=attn))
    start = torch.tensor([40, 7, 0], dtype=torch.int32, device=DEV)
    cache = {}

    def prompt(q, k, v, W, sinks, lengths):
        out = kla.kla_window_attn_forward(q.contiguous(), k.contiguous(), v.contiguous(), W, sinks, lengths, want_cache=True)
        cache.update(out)
        return out["y"]
    got, *_ = layer(p, x, pos, start, dict(norm=kla.kla_layer_norm, rope=kla.kla_qk_norm_rope, attn=prompt))
    for b, n in enumerate(start.tolist()):
        assert torch.allclose(got[b, :n].double(), want[b, :n], atol=2e-5)
    seen, rows = start.clone(), torch.arange(z["B"], device=DEV)
    step = lambda q, k, v, W, sinks, lengths: kla.kla_window_attn_step(q, k, v.contiguous(), cache["cache_k"], cache["cache_v"],
                                                                        lengths, sinks)["y"]
    for _ in range(43):
        at = seen.long().clamp_max(z["T"] - 1)
        live = seen < z["T"]
        y, *_ = layer(p, x[rows, at], pos[rows, at], torch.where(live, seen, -1),
                      dict(norm=kla.kla_layer_norm, rope=lambda *a: kla.kla_qk_norm_rope_forward(*(t.contiguous() for t in a)),
                           attn=step))
        assert torch.allclose(y[live].double(), want[rows, at][live], atol=2e-5)
        seen += 1


def test_captured_backward_beside_an_eager_graph(kla):
    """Refused while a graph of the same leaves lives that the default stream made; right once it is gone."""
    z = lambda *s: torch.randn(*s, device=DEV)
    q, k, v, w = (z(*s).requires_grad_(True) for s in ((2, 40, 4, 32), (2, 40, 2, 32), (2, 40, 2, 32), (32,)))
    for call, ins in ((lambda: kla.kla_window_attn(q, k, v, 9, 2), (q, k, v)), (lambda: kla.kla_qk_norm_rope(q, k, w, w)[0], (q, w))):
        alive = call()
        up = torch.randn_like(alive)
        want = torch.autograd.grad(alive, ins, up, retain_graph=True)
        torch.cuda.synchronize()
        with pytest.raises(RuntimeError, match="drop its outputs first"):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                torch.autograd.grad(call(), ins, up)
        torch.cuda.synchronize()
        del alive
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = torch.autograd.grad(call(), ins, up)
        for _ in range(3):
            for u in got:
                u.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(map(torch.equal, got, want))
            call()


def test_threads(kla):
    """Two threads, each on a stream of its own, give what one gives."""
    sets = []
    for i in range(2):
        gen = torch.Generator(device=DEV).manual_seed(i)
        r = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()
        sets.append([r(2, 300, 4, 64), r(2, 300, 2, 64), r(2, 300, 2, 64), r(2, 300, 4, 64)])

    def run(q, k, v, dy):
        ins = [t.detach().requires_grad_(True) for t in (q, k, v)]
        y = kla.kla_window_attn(*kla.kla_qk_norm_rope(*ins[:2]), ins[2], 50, 2)
        return [y.detach(), *torch.autograd.grad(y, ins, dy)]
    want = [run(*s) for s in sets]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                got[i].append(run(*sets[i]))
            stream.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(got[i]) == 10 and all(torch.equal(a, b) for out in got[i] for a, b in zip(out, want[i]))
