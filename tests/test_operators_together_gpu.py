"""The operators as a model uses them: layer norm, linear attention from a carried state, layer norm,
draws of the readout, the head, the draws' token log probabilities and the loss over them, with every
gradient, against the same in fp64 from their definitions; then the serving form of the same model."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def mixer(q, k, v, g, s0, lengths):
    """The recurrence, token by token, differentiable."""
    S, ys = s0, []
    gam = torch.exp(g)[:, None, None]
    for t in range(q.shape[1]):
        live = (t < lengths).view(-1, 1, 1, 1)
        S = torch.where(live, gam * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        ys.append(torch.where(live[..., 0], (q[:, t, :, :, None] * S).sum(-2), 0.0))
    return torch.stack(ys, 1), S


def norm(x, w, b):
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    return (x - mean) / torch.sqrt(var + 1e-5) * w + b


def model(p, x, target, lengths, eps, fwd):
    """fwd: the operators by name; returns the loss per token and the final state."""
    B, T, C = x.shape
    H, dk, dv = p["s0"].shape[1:]
    h = fwd["norm"](x, p["w1"], p["b1"])
    q, k, v = ((h @ p[n]).view(B, T, H, -1) for n in ("wq", "wk", "wv"))
    y, sT = fwd["mixer"](q.contiguous(), k.contiguous(), v.contiguous(), p["g"], p["s0"], lengths)
    out = fwd["norm"](x + y.reshape(B, T, H * dv) @ p["wo"], p["w2"], p["b2"])
    draws = out + p["sigma"] * eps                                   # [S, B, T, C]
    logp, ent = fwd["logp"]((draws @ p["head"]).contiguous(), target)
    S = eps.shape[0]
    nll = fwd["nll"](logp.reshape(S, B * T).contiguous())
    return nll.view(B, T) - 0.1 * ent.mean(0), sT


def test_training_step_and_serving():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_10743_amd as kla
    gen = torch.Generator().manual_seed(5)
    z = lambda *s, c=1.0: (c * torch.randn(*s, generator=gen)).to(DEV)
    B, T, H, dk, dv, C, V, S = 3, 45, 2, 16, 32, 72, 501, 4
    p = dict(w1=1 + z(C, c=0.1), b1=z(C, c=0.1), w2=1 + z(C, c=0.1), b2=z(C, c=0.1), wq=z(C, H * dk, c=C ** -0.5),
             wk=z(C, H * dk, c=0.3 * C ** -0.5), wv=z(C, H * dv, c=C ** -0.5), wo=z(H * dv, C, c=0.1), head=z(C, V, c=0.3),
             s0=z(B, H, dk, dv), sigma=torch.tensor(0.3, device=DEV))
    p["g"] = torch.tensor([-0.05, -0.6], device=DEV)
    x, eps = z(B, T, C), z(S, B, T, C)
    lengths = torch.tensor([45, 0, 31], dtype=torch.int32, device=DEV)
    target = torch.randint(0, V, (B, T), generator=gen).to(DEV)
    target = torch.where(torch.arange(T, device=DEV) < lengths[:, None], target, -1)
    names = [n for n in p if n != "g"]
    ours = dict(norm=kla.kla_layer_norm, mixer=kla.kla_linear_attn,
                logp=lambda u, t: kla.kla_token_logp(u, t, want_entropy=True), nll=kla.KLAMCNLL.apply)

    def logp64(u, t):
        lp = torch.log_softmax(u, -1)
        got = torch.where(t >= 0, lp.gather(-1, t.clamp_min(0).expand(u.shape[:-1])[..., None])[..., 0], 0.0)
        return got, -(lp.exp() * lp).sum(-1)
    plain = dict(norm=norm, mixer=mixer, logp=logp64, nll=lambda u: math.log(S) - torch.logsumexp(u, 0))
    dsT = z(B, H, dk, dv)
    res = []
    for fwd, cast in ((ours, torch.Tensor.float), (plain, torch.Tensor.double)):
        q = {n: cast(u).detach().requires_grad_(n != "g") for n, u in p.items()}
        xin = cast(x).requires_grad_(True)
        loss, sT = model(q, xin, target, lengths, cast(eps), fwd)
        total = (loss * (target >= 0)).sum() + (sT * cast(dsT)).sum()
        res.append([loss.detach(), sT.detach(), *torch.autograd.grad(total, [xin] + [q[n] for n in names])])
    for n, a, b in zip(["loss", "sT", "x"] + names, *res):
        assert torch.isfinite(a).all(), n
        rel = ((a.double() - b).norm() / b.norm()).item()
        # fp32 products and sums of some hundred terms, one operator after another
        assert rel < 2e-5, f"{n}: {rel:.2e}"
    # serving: the prompt's state, then one token at a time; the last token's alternatives
    q = {n: u.detach() for n, u in p.items()}
    h = kla.kla_layer_norm_forward(x, q["w1"], q["b1"])[0]
    qkv = [(h @ q[n]).view(B, T, H, -1).contiguous() for n in ("wq", "wk", "wv")]
    cut = lambda a, b: [u[:, a:b].contiguous() for u in qkv]
    full = kla.kla_linear_attn_forward(*qkv, q["g"], q["s0"])
    state = kla.kla_linear_attn_forward(*cut(0, 40), q["g"], q["s0"])["sT"]
    for t in range(40, T):
        y = kla.kla_linear_attn_step(*(u[:, t].contiguous() for u in qkv), q["g"], state)["y"]
        assert torch.allclose(y, full["y"][:, t], rtol=1e-4, atol=1e-4)
    assert torch.allclose(state, full["sT"], rtol=1e-4, atol=1e-4)
    out = kla.kla_layer_norm_forward(x[:, -1] + y.reshape(B, -1) @ q["wo"], q["w2"], q["b2"])[0]
    logits = out @ q["head"]
    got = kla.kla_token_logp_forward(logits, target[:, -1].contiguous(), top=5)
    want = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(got["top_index"], want)
    assert torch.allclose(got["top_logp"], torch.log_softmax(logits.double(), -1).gather(1, want).float(), atol=1e-5)


def test_captured_backward_beside_an_eager_graph():
    """Refused while a graph of the same leaves lives that the default stream made; right once it is gone."""
    import paper_2602_10743_amd as kla
    z = lambda *s: torch.randn(*s, device=DEV)
    g = torch.tensor([-0.1, -0.01], device=DEV)
    q, k, v, x, w, b, logits = (z(*s).requires_grad_(True) for s in ((2, 40, 2, 32), (2, 40, 2, 32), (2, 40, 2, 32), (50, 64),
                                                                    (64,), (64,), (50, 100)))
    target = torch.randint(0, 100, (50,), device=DEV)
    for call, ins in ((lambda: kla.kla_linear_attn(q, k, v, g)[0], (q, k, v)), (lambda: kla.kla_layer_norm(x, w, b), (x, w, b)),
                      (lambda: kla.kla_token_logp(logits, target), (logits,))):
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
