"""The operators around the filter layer that a language model of such layers needs, as measured cases.

``listed()`` names them, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes what a
program holds before the call, ``run`` is one pass through an operator -- in plain torch where
``own`` is false, through the package's entry points where it is true --, ``work`` the bytes and
operations a pass cannot do without, and ``exact`` the same outputs in 64 bits from the
definitions, one token after another.

Kinds of case:
  attn_train    linear attention with a decay for each head in a training step: kla_linear_attn
                and the gradients of every input
  attn_prefill  a prompt through it for serving: kla_linear_attn_forward, y and the final state
  attn_decode   one token for S sequences, the state updated in place: kla_linear_attn_step
  norm_train    layer norm in a training step: kla_layer_norm and the gradients of x, w, bias
  norm_infer    its forward alone: kla_layer_norm_forward
  logp_train    log probabilities of target tokens under S draws of the logits, and entropies, in
                a training step: kla_token_logp and the gradient of the logits
  logp_score    the same forward with the top alternatives: kla_token_logp_forward
"""
import math

import torch

own = False   # the package's entry points instead of plain torch

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _kla():
    import paper_2602_10743_amd
    return paper_2602_10743_amd


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the mixer of a 1.3B-parameter language model, one training step: the benchmark's shape
        dict(name="attn_train_lm", kind="attn_train", B=8, T=2048, H=16, dk=128, dv=128, dtype="bf16", state=False,
             ragged=False),
        # a padded batch of a smaller model, resumed from a carried state that is trained through
        dict(name="attn_train_ragged", kind="attn_train", B=3, T=777, H=5, dk=64, dv=128, dtype="bf16", state=True,
             ragged=True),
        # an fp32 state-tracking model, one training step
        dict(name="attn_train_f32", kind="attn_train", B=64, T=512, H=4, dk=32, dv=32, dtype="f32", state=False,
             ragged=False),
        # one 64k-token context read before generation
        dict(name="attn_prefill_64k", kind="attn_prefill", B=1, T=65536, H=16, dk=128, dv=128, dtype="bf16",
             state=False, ragged=False),
        # a full serving batch, one token each
        dict(name="attn_decode_512", kind="attn_decode", S=512, H=16, dk=128, dv=128, dtype="bf16"),
        # one interactive sequence, one token: latency only
        dict(name="attn_decode_1", kind="attn_decode", S=1, H=16, dk=128, dv=128, dtype="bf16"),
        # the norm in front of a layer of the language model, one training step
        dict(name="norm_train_lm", kind="norm_train", rows=16384, n=2048, dtype="bf16", bias=True),
        # an odd width in fp32, no bias
        dict(name="norm_train_odd_f32", kind="norm_train", rows=2331, n=1001, dtype="f32", bias=False),
        # the norm of a few interactive sequences' tokens
        dict(name="norm_infer_3", kind="norm_infer", rows=3, n=2048, dtype="bf16", bias=True),
        # the Monte Carlo readout's log probabilities: four draws of a batch's logits, trained
        dict(name="logp_train_mc", kind="logp_train", S=4, rows=2048, V=50257, dtype="bf16", entropy=True),
        # tokens scored with their eight best alternatives, part of the vocabulary masked out, fp32 logits
        dict(name="logp_score_f32", kind="logp_score", S=1, rows=1000, V=32000, dtype="f32", top=8, masked=True),
        # the next token's alternatives for two interactive sequences
        dict(name="logp_score_2", kind="logp_score", S=1, rows=2, V=128000, dtype="bf16", top=16, masked=False),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn_train", "attn_train", "attn_train", "attn_prefill", "attn_prefill", "attn_decode",
                       "norm_train", "norm_infer", "logp_train", "logp_score"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("attn_train", "attn_prefill"):
        w = (16, 32, 64, 64, 128, 128)
        B = _logint(rng, 1, 64)
        T = _logint(rng, 1, 2048 if kind == "attn_train" else 65536)
        H = rng.randint(1, 16)
        most = (1 << 18) if kind == "attn_train" else (1 << 20)
        if dtype == "f32":
            most >>= 2
        while B > 1 and B * T * H > most:
            B -= 1
        while T > 1 and B * T * H > most:
            T -= T // 8 + 1
        return dict(kind=kind, B=B, T=max(T, 1), H=H, dk=rng.choice(w), dv=rng.choice(w), dtype=dtype,
                    state=rng.random() < 0.5, ragged=rng.random() < 0.4)
    if kind == "attn_decode":
        return dict(kind=kind, S=_logint(rng, 1, 512), H=rng.randint(1, 16), dk=rng.choice([32, 64, 128]),
                    dv=rng.choice([16, 64, 128]), dtype=dtype)
    if kind in ("norm_train", "norm_infer"):
        n = _logint(rng, 8, 8192)
        if rng.random() < 0.6:
            n = (n + 7) // 8 * 8
        rows = _logint(rng, 1, min(16384, (1 << 25) // n))
        return dict(kind=kind, rows=rows, n=n, dtype=dtype, bias=rng.random() < 0.7)
    V = _logint(rng, 200, 128000)
    S = rng.randint(1, 6) if kind == "logp_train" else 1
    rows = _logint(rng, 1, max(1, min(4096, (1 << (27 if kind == "logp_train" else 25)) // (V * S))))
    c = dict(kind=kind, S=S, rows=rows, V=V, dtype=dtype)
    if kind == "logp_train":
        return dict(c, entropy=rng.random() < 0.5)
    return dict(c, top=rng.randint(0, 32), masked=rng.random() < 0.4)


def _tokens(case):
    return (case["S"] if case["kind"] == "attn_decode" else case["B"] * case["T"]) * case["H"]


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    kind, t = case["kind"], _TYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    z = lambda *s: torch.randn(*s, generator=g, device="cuda")
    if kind.startswith("attn"):
        H, dk, dv = case["H"], case["dk"], case["dv"]
        lead = (case["S"], H) if kind == "attn_decode" else (case["B"], case["T"], H)
        x = dict(q=z(*lead, dk).to(t), k=torch.nn.functional.normalize(z(*lead, dk), dim=-1).to(t),
                 v=z(*lead, dv).to(t), kind=kind)
        # decays 1 - 2^-e, e from 3 to 10 over the heads: memories of eight to a thousand tokens
        x["g"] = torch.log1p(-torch.exp2(-(3.0 + 7.0 * torch.rand(H, generator=g, device="cuda"))))
        if kind == "attn_decode":
            x["s"] = z(*lead, dk, dv)
            return x
        B, T = case["B"], case["T"]
        x["s0"] = z(B, H, dk, dv) if case["state"] else None
        x["len"] = None
        if case["ragged"]:
            x["len"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        if kind == "attn_train":
            x["dy"] = z(*lead, dv).to(t)
            x["ds"] = 0.1 * z(B, H, dk, dv) if case["state"] else None
            for n in ("q", "k", "v", "s0"):
                if x[n] is not None:
                    x[n].requires_grad_(True)
        return x
    if kind.startswith("norm"):
        rows, n = case["rows"], case["n"]
        x = dict(x=(0.5 + 2.0 * z(rows, n)).to(t), w=1.0 + 0.1 * z(n), b=0.1 * z(n) if case["bias"] else None, kind=kind)
        if kind == "norm_train":
            x["dy"] = z(rows, n).to(t)
            for m in ("x", "w", "b"):
                if x[m] is not None:
                    x[m].requires_grad_(True)
        return x
    S, rows, V = case["S"], case["rows"], case["V"]
    logits = torch.randn(S, rows, V, generator=g, device="cuda", dtype=t).mul_(2.0)
    target = torch.randint(0, V, (rows,), generator=g, device="cuda")
    # the model has learnt something: its targets stand out
    logits.scatter_add_(2, target.expand(S, rows)[..., None], (4.0 + z(S, rows, 1)).to(t))
    # a twentieth of the tokens are padding
    target = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.05, -1, target)
    x = dict(logits=logits, target=target, kind=kind)
    if kind == "logp_train":
        x["logits"].requires_grad_(True)
        x["dlogp"] = z(S, rows)
        x["dent"] = 0.01 * z(S, rows) if case["entropy"] else None
        return x
    if case["masked"]:   # a quarter of the vocabulary is not allowed
        off = torch.rand(V, generator=g, device="cuda") < 0.25
        x["logits"].masked_fill_(off, -math.inf)
    x["top"] = min(case["top"], V)
    return x


# ------------------------------------------------------------------ one pass
def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


# ---- through the package
def _own_attn_train(s):
    ins = [s[n] for n in ("q", "k", "v", "s0") if s[n] is not None]
    y, sT = _kla().kla_linear_attn(s["q"], s["k"], s["v"], s["g"], s["s0"], s["len"])
    outs, ups = ([y], [s["dy"]]) if s["ds"] is None else ([y, sT], [s["dy"], s["ds"]])
    return {"y": y.detach(), "sT": sT.detach(), "grads": list(torch.autograd.grad(outs, ins, ups))}


def _own_attn_prefill(s):
    out = _kla().kla_linear_attn_forward(s["q"], s["k"], s["v"], s["g"], s["s0"], s["len"])
    return {"y": out["y"], "sT": out["sT"]}


def _own_attn_decode(s):
    out = _kla().kla_linear_attn_step(s["q"], s["k"], s["v"], s["g"], s["s"])
    return {"y": out["y"], "s": out["state"]}


def _own_norm_train(s):
    y = _kla().kla_layer_norm(s["x"], s["w"], s["b"], 1e-5)
    return {"y": y.detach(), "grads": list(torch.autograd.grad(y, [s[n] for n in ("x", "w", "b") if s[n] is not None],
                                                               s["dy"]))}


def _own_norm_infer(s):
    return {"y": _kla().kla_layer_norm_forward(s["x"], s["w"], s["b"], 1e-5)[0]}


def _own_logp_train(s):
    want = s["dent"] is not None
    out = _kla().kla_token_logp(s["logits"], s["target"], want_entropy=want)
    outs, ups = (list(out), [s["dlogp"], s["dent"]]) if want else ([out], [s["dlogp"]])
    (dx,) = torch.autograd.grad(outs, [s["logits"]], ups)
    return {"logp": outs[0].detach(), "entropy": outs[1].detach() if want else [], "dlogits": dx}


def _own_logp_score(s):
    out = _kla().kla_token_logp_forward(s["logits"], s["target"], want_entropy=True, top=s["top"])
    return {"logp": out["logp"], "entropy": out["entropy"], "top_logp": out["top_logp"] if s["top"] else [],
            "top_index": out["top_index"] if s["top"] else []}


_OWN = {"attn_train": _own_attn_train, "attn_prefill": _own_attn_prefill, "attn_decode": _own_attn_decode,
        "norm_train": _own_norm_train, "norm_infer": _own_norm_infer, "logp_train": _own_logp_train,
        "logp_score": _own_logp_score}


# ---- in plain torch, 32 bits
def _decayed_sums(q, k, v, g, length=64):
    """out_t = sum_{s <= t} exp(g (t - s)) (q_t . k_s) v_s over [B, T, H, *] fp32 tensors: inside chunks
    of `length` tokens by a masked product, between them by the states at the chunks' ends."""
    B, T, H, N = q.shape
    D, c = v.shape[-1], min(length, T)
    n = (T + c - 1) // c
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * c - T)).view(B, n, c, H, -1).permute(0, 3, 1, 2, 4)
               .contiguous() for x in (q, k, v))
    i = torch.arange(c, device=q.device, dtype=torch.float32)
    lag = i[:, None] - i
    g = g.view(H, 1, 1)
    y = (q @ k.transpose(-1, -2) * torch.where(lag >= 0, torch.exp(g * lag.clamp_min(0)), 0.0)[:, None]) @ v
    if n > 1:
        ends = (k * torch.exp(g * (c - 1 - i))[..., None]).transpose(-1, -2) @ v
        m = torch.arange(n, device=q.device, dtype=torch.float32)
        gap = m[:, None] - 1 - m
        starts = torch.where(gap >= 0, torch.exp(g * c * gap.clamp_min(0)), 0.0) @ ends.view(B, H, n, N * D)
        y = y + torch.exp(g * (i + 1))[..., None] * (q @ starts.view(B, H, n, N, D))
    return y.permute(0, 2, 3, 1, 4).reshape(B, n * c, H, D)[:, :T]


def _plain_attn(s, train):
    q, k, v = (s[n].detach().float() for n in ("q", "k", "v"))
    B, T, H, dk = q.shape
    dv, g, t = v.shape[-1], s["g"], s["q"].dtype
    s0 = None if s["s0"] is None else s["s0"].detach()
    at = torch.arange(T, device=q.device, dtype=torch.float32).view(1, T, 1)
    left = T - 1 - at
    whole = torch.exp(g * T).expand(B, H)
    if s["len"] is not None:
        left = s["len"].view(B, 1, 1) - 1 - at
        live = (left >= 0)[..., None]
        q, k, v = (torch.where(live, x, 0.0) for x in (q, k, v))
        left = left.clamp_min(0)
        whole = torch.exp(g * s["len"].view(B, 1))
    since, until = torch.exp(g * (at + 1))[..., None], torch.exp(g * left)[..., None]   # to the start, to the end
    heads = lambda x: x.expand(B, T, H, x.shape[-1]).permute(0, 2, 1, 3).contiguous()      # [B, H, T, *]
    back = lambda x: x.permute(0, 2, 1, 3)
    y = _decayed_sums(q, k, v, g)
    sT = heads(k * until).transpose(-1, -2) @ heads(v)
    if s0 is not None:
        y = y + back(heads(q * since) @ s0)
        sT = sT + whole[..., None, None] * s0
    out = {"y": y.to(t), "sT": sT}
    if not train:
        return out
    dy = s["dy"].float()
    if s["len"] is not None:
        dy = torch.where(live, dy, 0.0)
    flip = lambda *x: (u.flip(1) for u in x)
    dq = _decayed_sums(dy, v, k, g)
    dk_ = _decayed_sums(*flip(v, dy, q), g).flip(1)
    dv_ = _decayed_sums(*flip(k, q, dy), g).flip(1)
    grads = [dq, dk_, dv_]
    if s0 is not None:
        grads[0] = dq + back(heads(dy * since) @ s0.transpose(-1, -2))
        grads[1] = dk_ + back(heads(v * until) @ s["ds"].transpose(-1, -2))
        grads[2] = dv_ + back(heads(k * until) @ s["ds"])
    grads = [u.to(t) for u in grads]
    if s0 is not None:
        grads.append(heads(q * since).transpose(-1, -2) @ heads(dy) + whole[..., None, None] * s["ds"])
    return dict(out, grads=grads)


def _plain_attn_decode(s):
    s["s"].mul_(torch.exp(s["g"])[:, None, None]).add_(s["k"].float()[..., None] * s["v"].float()[..., None, :])
    return {"y": (s["q"].float()[..., None, :] @ s["s"])[..., 0, :].to(s["q"].dtype), "s": s["s"]}


def _plain_norm(s, train):
    x, w = s["x"].detach().float(), s["w"].detach()
    mid = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt(mid.square().mean(-1, keepdim=True) + 1e-5)
    hat = mid * rstd
    y = hat * w if s["b"] is None else hat * w + s["b"].detach()
    out = {"y": y.to(s["x"].dtype)}
    if not train:
        return out
    dy = s["dy"].float()
    d = dy * w
    dx = rstd * (d - d.mean(-1, keepdim=True) - hat * (d * hat).mean(-1, keepdim=True))
    grads = [dx.to(s["x"].dtype), (dy * hat).sum(0)] + ([] if s["b"] is None else [dy.sum(0)])
    return dict(out, grads=grads)


def _plain_logp(s):
    """Log softmax of the logits in fp32, the targets' entries (0 where there is no target), entropies."""
    x = s["logits"].detach().float()
    lp = x - x.amax(-1, keepdim=True)
    p = lp.exp()
    total = p.sum(-1, keepdim=True)
    lp = lp - total.log()
    p = p / total
    target = s["target"].expand(x.shape[:-1])
    logp = lp.gather(-1, target.clamp_min(0)[..., None])[..., 0]
    logp = torch.where(target >= 0, logp, 0.0)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(-1)
    return lp, p, target, logp, entropy


def _plain_logp_train(s):
    lp, p, target, logp, entropy = _plain_logp(s)
    d = torch.where(target >= 0, s["dlogp"], 0.0)[..., None]
    dx = -d * p
    dx.scatter_add_(-1, target.clamp_min(0)[..., None], d)
    if s["dent"] is not None:
        dx -= torch.where(p > 0, s["dent"][..., None] * p * (lp + entropy[..., None]), 0.0)
    return {"logp": logp, "entropy": [] if s["dent"] is None else entropy, "dlogits": dx.to(s["logits"].dtype)}


def _plain_logp_score(s):
    lp, p, target, logp, entropy = _plain_logp(s)
    if not s["top"]:
        return {"logp": logp, "entropy": entropy, "top_logp": [], "top_index": []}
    # a key that orders by value, the lower index first among equals
    bits = (s["logits"].float() + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits)
    V = lp.shape[-1]
    best = (order * (1 << 20) + (V - 1 - torch.arange(V, device=lp.device))).topk(s["top"], dim=-1).values
    index = V - 1 - (best & ((1 << 20) - 1))
    return {"logp": logp, "entropy": entropy, "top_logp": lp.gather(-1, index), "top_index": index}


_PLAIN = {"attn_train": lambda s: _plain_attn(s, True), "attn_prefill": lambda s: _plain_attn(s, False),
          "attn_decode": _plain_attn_decode, "norm_train": lambda s: _plain_norm(s, True),
          "norm_infer": lambda s: _plain_norm(s, False), "logp_train": _plain_logp_train,
          "logp_score": _plain_logp_score}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind.startswith("attn"):
        n, dk, dv = _tokens(case), case["dk"], case["dv"]
        if kind == "attn_decode":
            return {"bytes": n * (8 * dk * dv + (2 * dk + 2 * dv) * e), "flops": n * 5 * dk * dv}
        states = 4 * case["B"] * case["H"] * dk * dv
        if kind == "attn_prefill":
            return {"bytes": n * (2 * dk + 2 * dv) * e + states * (2 if case["state"] else 1), "flops": n * 5 * dk * dv}
        # forward; backward: q, k, v, dy once, dq, dk, dv, and the states and their gradients
        return {"bytes": n * ((2 * dk + 2 * dv) + (2 * dk + 2 * dv) + (2 * dk + dv)) * e + states * (6 if case["state"] else 1),
                "flops": n * 17 * dk * dv}
    if kind.startswith("norm"):
        m = case["rows"] * case["n"]
        if kind == "norm_infer":
            return {"bytes": 2 * m * e + 8 * case["n"], "flops": 8 * m}
        return {"bytes": 5 * m * e + 16 * case["n"], "flops": 20 * m}
    m, rows = case["S"] * case["rows"] * case["V"], case["S"] * case["rows"]
    if kind == "logp_train":
        return {"bytes": 3 * m * e + 16 * rows, "flops": 10 * m}
    return {"bytes": m * e + rows * (16 + 12 * min(case["top"], case["V"])), "flops": 5 * m}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    x = {n: u.detach().double() if u.is_floating_point() else u for n, u in s.items() if isinstance(u, torch.Tensor)}
    kind = case["kind"]
    if kind == "attn_decode":
        state = torch.exp(x["g"])[:, None, None] * x["s"] + x["k"][..., :, None] * x["v"][..., None, :]
        return {"y": (x["q"][..., :, None] * state).sum(-2), "s": state}
    if kind.startswith("attn"):
        return _exact_attn(x, case)
    if kind.startswith("norm"):
        return _exact_norm(x, case)
    return _exact_logp(x, case, s.get("top", 0))


def _exact_attn(x, case):
    """The recurrence S_t = exp(g) S_{t-1} + k_t v_t^T, y_t = S_t^T q_t and its adjoint, token by token."""
    train, T = case["kind"] == "attn_train", case["T"]
    q, k, v = (x[n].permute(1, 0, 2, 3).contiguous() for n in ("q", "k", "v"))   # [T, B, H, *]
    dy = x["dy"].permute(1, 0, 2, 3).contiguous() if train else None
    gamma = torch.exp(x["g"])[:, None, None]
    S = x["s0"].clone() if case["state"] else q.new_zeros(*q.shape[1:], v.shape[-1])
    n = x["len"] if case["ragged"] else None
    live = None if n is None else (torch.arange(T, device=q.device)[:, None] < n).view(T, -1, 1, 1, 1)
    y, dq, dk, dv = (None if u is None else torch.zeros_like(u) for u in (v, q if train else None, k, v))
    for t in range(T):
        new = torch.addcmul(gamma * S, k[t][..., None], v[t][..., None, :])
        S = new if live is None else torch.where(live[t], new, S)
        y[t] = torch.matmul(q[t][..., None, :], S)[..., 0, :]
        if train:
            dq[t] = torch.matmul(S, dy[t][..., None])[..., 0]
    out = {"y": y, "sT": S}
    if live is not None:
        out["y"] = torch.where(live[..., 0], y, 0.0)
    out["y"] = out["y"].permute(1, 0, 2, 3).contiguous()
    if not train:
        return out
    Z = x["ds"].clone() if case["state"] else torch.zeros_like(S)   # the adjoint of the state after token t
    for t in range(T - 1, -1, -1):
        G = torch.addcmul(Z, q[t][..., None], dy[t][..., None, :])
        dk[t] = torch.matmul(G, v[t][..., None])[..., 0]
        dv[t] = torch.matmul(k[t][..., None, :], G)[..., 0, :]
        Z = gamma * G if live is None else torch.where(live[t], gamma * G, Z)
    grads = [dq, dk, dv] if live is None else [torch.where(live[..., 0], u, 0.0) for u in (dq, dk, dv)]
    grads = [u.permute(1, 0, 2, 3).contiguous() for u in grads]
    return dict(out, grads=grads + ([Z] if case["state"] else []))


def _exact_norm(x, case):
    with torch.enable_grad():
        names = [n for n in ("x", "w", "b") if n in x]
        leaves = [x[n].requires_grad_(True) for n in names]
        var, mean = torch.var_mean(x["x"], dim=-1, correction=0, keepdim=True)
        y = (x["x"] - mean) / torch.sqrt(var + 1e-5) * x["w"]
        if "b" in x:
            y = y + x["b"]
        if case["kind"] == "norm_infer":
            return {"y": y.detach()}
        return {"grads": list(torch.autograd.grad(y, leaves, x["dy"])), "y": y.detach()}


def _exact_logp(x, case, top):
    logits, target = x["logits"], x["target"].expand(case["S"], case["rows"])
    lse = torch.logsumexp(logits, -1, keepdim=True)
    lp = logits - lse
    p = torch.exp(lp)
    logp = torch.where(target < 0, 0.0, torch.take_along_dim(lp, target.clamp_min(0)[..., None], -1)[..., 0])
    entropy = torch.special.entr(p).sum(-1)
    if case["kind"] == "logp_score":
        out = {"logp": logp, "entropy": entropy, "top_logp": [], "top_index": []}
        if top:
            best = torch.sort(logits, dim=-1, descending=True, stable=True).indices[..., :top]
            out.update(top_logp=torch.take_along_dim(lp, best, -1), top_index=best)
        return out
    d = torch.where(target < 0, 0.0, x["dlogp"])
    dx = -d[..., None] * p
    dx.scatter_add_(-1, target.clamp_min(0)[..., None], d[..., None])
    if case["entropy"]:
        dx -= x["dent"][..., None] * (-torch.special.entr(p) + p * entropy[..., None])
    return {"logp": logp, "entropy": entropy if case["entropy"] else [], "dlogits": dx}
