"""The attention layer that a hybrid stack has between filter layers, as measured cases.

``listed()`` names them, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes what a
program holds before the call, ``run`` is one pass through an operator -- in plain torch where
``own`` is false, through the package's entry points where it is true --, ``work`` the bytes and
operations a pass cannot do without, and ``exact`` the same outputs in 64 bits from the
definitions, one head after another.

Kinds of case:
  rope_train    norms of queries and keys for each head and the position rotation in a training
                step: kla_qk_norm_rope and the gradients of q, k and both weights
  rope_infer    the same forward alone, at given positions: kla_qk_norm_rope_forward
  attn_train    attention with a sliding window and first tokens that stay visible, in a training
                step: kla_window_attn and the gradients of q, k, v
  attn_prefill  a prompt, or the next piece of one, through it for serving:
                kla_window_attn_forward, y and (where the whole prompt is read) the cache
  attn_decode   one token for S sequences, the cache updated in place: kla_window_attn_step
"""
import math

import torch

own = False   # the package's entry points instead of plain torch

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6


def _kla():
    import paper_2602_10743_amd
    return paper_2602_10743_amd


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # queries and keys of a 1.3B-parameter language model's attention layer, one training step
        dict(name="rope_train_lm", kind="rope_train", B=8, T=2048, H=16, Hk=16, d=128, rot=128, interleaved=False,
             base=10000.0, far=0, dtype="bf16"),
        # a smaller fp32 model with shared keys that rotates half of each head, pieces of longer documents
        dict(name="rope_train_f32", kind="rope_train", B=5, T=333, H=12, Hk=3, d=64, rot=32, interleaved=True,
             base=10000.0, far=500000, dtype="f32"),
        # a 64k-token prompt
        dict(name="rope_infer_64k", kind="rope_infer", B=1, T=65536, H=16, Hk=4, d=128, rot=128, interleaved=False,
             base=1000000.0, far=0, dtype="bf16"),
        # the next token of three interactive sequences: latency only
        dict(name="rope_infer_3", kind="rope_infer", B=3, T=1, H=16, Hk=4, d=128, rot=128, interleaved=False,
             base=1000000.0, far=1000000, dtype="bf16"),
        # the attention layer of the language model, one training step
        dict(name="attn_train_lm", kind="attn_train", B=8, T=2048, H=16, Hk=16, d=128, window=512, sinks=4,
             ragged=False, dtype="bf16"),
        # a padded batch of a smaller model with shared keys
        dict(name="attn_train_ragged", kind="attn_train", B=3, T=777, H=6, Hk=2, d=64, window=100, sinks=3,
             ragged=True, dtype="bf16"),
        # an fp32 state-tracking model, one training step
        dict(name="attn_train_f32", kind="attn_train", B=64, T=512, H=4, Hk=4, d=32, window=128, sinks=0,
             ragged=False, dtype="f32"),
        # one 64k-token context read before generation, shared keys
        dict(name="attn_prefill_64k", kind="attn_prefill", B=1, T=65536, past=0, H=16, Hk=4, d=128, window=2048,
             sinks=4, ragged=False, dtype="bf16"),
        # the next 500 tokens of two prompts whose first 1500 are read, all of them visible, fp32
        dict(name="attn_prefill_more_f32", kind="attn_prefill", B=2, T=500, past=1500, H=8, Hk=8, d=64, window=2000,
             sinks=0, ragged=False, dtype="f32"),
        # a full serving batch, one token each
        dict(name="attn_decode_512", kind="attn_decode", S=512, H=16, Hk=4, d=128, window=1024, sinks=4, seen=4096,
             dtype="bf16"),
        # one interactive sequence, one token: latency only
        dict(name="attn_decode_1", kind="attn_decode", S=1, H=16, Hk=4, d=128, window=4096, sinks=4, seen=20000,
             dtype="bf16"),
        # a few short fp32 sequences
        dict(name="attn_decode_7_f32", kind="attn_decode", S=7, H=6, Hk=3, d=64, window=250, sinks=1, seen=200,
             dtype="f32"),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope_train", "rope_infer", "attn_train", "attn_train", "attn_train", "attn_prefill",
                       "attn_prefill", "attn_decode", "attn_decode"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([16, 32, 64, 64, 128, 128])
    Hk = rng.randint(1, 8)
    H = Hk * rng.choice([1, 1, 2, 3, 4, 8])
    c = dict(kind=kind, H=H, Hk=Hk, d=d, dtype=dtype)
    if kind.startswith("rope"):
        T = _logint(rng, 1, 8192)
        B = _logint(rng, 1, max(1, min(64, (1 << 25) // ((H + Hk) * d * T))))
        while T > 1 and B * T * (H + Hk) * d > 1 << 26:
            T -= T // 8 + 1
        return dict(c, B=B, T=T, rot=rng.choice([d, d, d, d // 32 * 16, 16, 0]), interleaved=rng.random() < 0.3,
                    base=rng.choice([10000.0, 500000.0, 1000000.0]),
                    far=rng.choice([0, _logint(rng, 1, 1000000)]) if kind == "rope_train" else _logint(rng, 1, 1000000))
    # from two tokens on: one that sees itself alone has gradients of zero, which leave nothing to compare
    c.update(window=_logint(rng, 2, 4096), sinks=rng.choice([0, 0, rng.randint(1, 8), rng.randint(1, 64)]))
    slots = c["window"] + c["sinks"]
    if kind == "attn_decode":
        most = (1 << 29) if dtype == "bf16" else (1 << 28)   # elements of both caches
        S = _logint(rng, 1, max(1, min(512, most // (2 * slots * Hk * d))))
        return dict(c, S=S, seen=rng.choice([4 * slots, _logint(rng, 1, 4 * slots)]))
    T = _logint(rng, 2, 2048 if kind == "attn_train" else 16384)
    past = rng.choice([0, _logint(rng, 1, 4096)]) if kind == "attn_prefill" else 0
    B = _logint(rng, 1, 16)
    most = 1 << (30 if dtype == "bf16" else 28)   # scores of the plain form, a quarter of them kept
    size = lambda B, T: B * H * T * (min(c["window"], T + past) + 64)
    while B > 1 and (size(B, T) * 2 > most or B * T * H * d > 1 << 25):
        B -= 1
    while T > 2 and (size(B, T) * 2 > most or B * T * H * d > 1 << 26):
        T -= T // 8 + 1
    return dict(c, B=B, T=T, **({"past": past} if kind == "attn_prefill" else {}), ragged=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    kind, t = case["kind"], _TYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    z = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.int32)
    H, Hk, d = case["H"], case["Hk"], case["d"]
    if kind.startswith("rope"):
        B, T, rot = case["B"], case["T"], case["rot"]
        # projections whose heads differ in size by a factor of a few
        size = lambda h: torch.exp(0.5 * z(h, 1))
        x = dict(kind=kind, q=(z(B, T, H, d) * size(H)).to(t), k=(z(B, T, Hk, d) * size(Hk)).to(t),
                 wq=1.0 + 0.2 * z(d), wk=1.0 + 0.2 * z(d), interleaved=case["interleaved"], pos=None, freq=None)
        if rot:
            x["freq"] = case["base"] ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
            if case["far"]:   # each sequence is a piece that starts somewhere in a long document
                x["pos"] = ints(0, case["far"] + 1, B, 1) + torch.arange(T, device="cuda", dtype=torch.int32)
        if kind == "rope_train":
            x["dq"], x["dk"] = z(B, T, H, d).to(t), z(B, T, Hk, d).to(t)
            for n in ("q", "k", "wq", "wk"):
                x[n].requires_grad_(True)
        return x
    x = dict(kind=kind, window=case["window"], sinks=case["sinks"])
    if kind == "attn_decode":
        S, slots = case["S"], case["window"] + case["sinks"]
        x.update(q=z(S, H, d).to(t), k=z(S, Hk, d).to(t), v=z(S, Hk, d).to(t))
        x.update(ck=z(S, slots, Hk, d).to(t), cv=z(S, slots, Hk, d).to(t))
        x["pos"] = ints(case["seen"] // 2, case["seen"] + 1, S)
        return x
    B, T = case["B"], case["T"]
    past = case.get("past", 0)
    x.update(q=z(B, T, H, d).to(t), k=z(B, past + T, Hk, d).to(t), v=z(B, past + T, Hk, d).to(t), len=None)
    if case["ragged"]:
        x["len"] = ints(0, past + T + 1, B)
        x["len"][x["len"] == 1] = 0   # as in draw()
    x["cache"] = kind == "attn_prefill" and past == 0
    if kind == "attn_train":
        x["dy"] = z(B, T, H, d).to(t)
        for n in ("q", "k", "v"):
            x[n].requires_grad_(True)
    return x


# ------------------------------------------------------------------ one pass
def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


# ---- through the package
def _own_rope_train(s):
    q, k = _kla().kla_qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["pos"], _EPS,
                                   interleaved=s["interleaved"])
    grads = torch.autograd.grad([q, k], [s["q"], s["k"], s["wq"], s["wk"]], [s["dq"], s["dk"]])
    return {"q": q.detach(), "k": k.detach(), "grads": list(grads)}


def _own_rope_infer(s):
    q, k = _kla().kla_qk_norm_rope_forward(s["q"], s["k"], s["wq"], s["wk"], s["freq"], s["pos"], _EPS,
                                           interleaved=s["interleaved"])
    return {"q": q, "k": k}


def _own_attn_train(s):
    y = _kla().kla_window_attn(s["q"], s["k"], s["v"], s["window"], s["sinks"], s["len"])
    return {"y": y.detach(), "grads": list(torch.autograd.grad(y, [s["q"], s["k"], s["v"]], s["dy"]))}


def _own_attn_prefill(s):
    out = _kla().kla_window_attn_forward(s["q"], s["k"], s["v"], s["window"], s["sinks"], s["len"],
                                         want_cache=s["cache"])
    return {n: [] if out[n] is None else out[n] for n in ("y", "cache_k", "cache_v")}


def _own_attn_decode(s):
    out = _kla().kla_window_attn_step(s["q"], s["k"], s["v"], s["ck"], s["cv"], s["pos"], s["sinks"])
    return {n: out[n] for n in ("y", "cache_k", "cache_v")}


_OWN = {"rope_train": _own_rope_train, "rope_infer": _own_rope_infer, "attn_train": _own_attn_train,
        "attn_prefill": _own_attn_prefill, "attn_decode": _own_attn_decode}


# ---- in plain torch, 32 bits
def _angles(s, x):
    """cos and sin of position * frequency, [B, T, 1, rot / 2]: the angles in 64 bits, for far positions."""
    B, T = x.shape[:2]
    pos = torch.arange(T, device=x.device).expand(B, T) if s["pos"] is None else s["pos"]
    phi = pos[..., None, None].double() * s["freq"]
    return phi.cos().float(), phi.sin().float()


def _pairs(x, rot, interleaved):
    """The first and second elements of the rotated pairs, and the elements that stay."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b, rest = _pairs(x, rot, interleaved)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _plain_rope(s, train):
    out, dx, dw = [], [], []
    cs = None if s["freq"] is None else _angles(s, s["q"])
    for n in ("q", "k"):
        x, w = s[n].detach().float(), s["w" + n].detach()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
        hat = x * r
        u = hat * w
        out.append((u if cs is None else _rotated(u, *cs, s["interleaved"])).to(s[n].dtype))
        if train:
            du = s["d" + n].float()
            if cs is not None:
                du = _rotated(du, cs[0], -cs[1], s["interleaved"])
            g = du * w
            dx.append((r * (g - hat * (g * hat).mean(-1, keepdim=True))).to(s[n].dtype))
            dw.append((du * hat).sum((0, 1, 2)))
    return dict({"q": out[0], "k": out[1]}, **({"grads": dx + dw} if train else {}))


def _bands(s):
    """Queries in blocks of c positions, each with the c + L keys that its window can reach and the first tokens apart.

    Returns q [B, Hk, n, G c, d] and the keys and values of the blocks [B, Hk, n, L + c, d], all fp32, the first tokens
    [B, Hk, 1, sinks, d], and what is visible, [B, 1, n, c, L + c] and [B, 1, n, c, sinks]."""
    q, k, v = (s[n].detach().float() for n in ("q", "k", "v"))
    B, T, H, d = q.shape
    Tk, Hk, W = k.shape[1], k.shape[2], s["window"]
    past = Tk - T
    c = max(64, W)
    c, L = (T, min(W - 1, past)) if T <= c else (c, c)
    n = (T + c - 1) // c
    pos = past + torch.arange(n * c, device=q.device).view(n, c, 1)
    at = past - L + torch.arange(n, device=q.device).view(n, 1, 1) * c + torch.arange(L + c, device=q.device)
    first = torch.arange(min(s["sinks"], Tk), device=q.device)
    end = torch.full((B, 1, 1, 1), Tk, device=q.device) if s["len"] is None else s["len"].view(B, 1, 1, 1)
    see = ((at <= pos) & (at > pos - W) & (at >= 0))[None] & (at < end) & (pos < end)
    see_first = (first <= pos - W)[None] & (first < end) & (pos < end)
    # a padded batch's rows past the ends hold anything
    live = (torch.arange(Tk, device=q.device)[:, None] < end.view(B, 1, 1))[..., None]
    k, v, q = torch.where(live, k, 0.0), torch.where(live, v, 0.0), torch.where(live[:, past:], q, 0.0)
    pad = torch.nn.functional.pad
    blocks = lambda x: pad(x[:, max(0, past - L):], (0, 0, 0, 0, max(0, L - past), n * c - T)).unfold(1, L + c, c) \
        .permute(0, 2, 1, 4, 3).contiguous()
    heads = lambda x: x[:, :first.numel()].permute(0, 2, 1, 3)[:, :, None].contiguous()
    return (_grouped(q, Hk, n, c), blocks(k), blocks(v), heads(k), heads(v), see[:, None], see_first[:, None])


def _grouped(x, Hk, n, c):
    """[B, T, H, d] -> [B, Hk, n, G c, d]"""
    B, T, H, d = x.shape
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * c - T)).view(B, n, c, Hk, H // Hk, d)
    return x.permute(0, 3, 1, 4, 2, 5).reshape(B, Hk, n, H // Hk * c, d)


def _flat(x, G, T):
    """[B, Hk, n, G c, d] -> [B, T, H, d]"""
    B, Hk, n, _, d = x.shape
    x = x.view(B, Hk, n, G, -1, d).permute(0, 2, 4, 1, 3, 5)
    return x.reshape(B, -1, Hk * G, d)[:, :T].contiguous()


def _plain_attn(s, train):
    t = s["q"].dtype
    B, T, H, d = s["q"].shape
    Tk, Hk = s["k"].shape[1:3]
    G, scale = H // Hk, 1.0 / math.sqrt(d)
    q, k, v, k0, v0, see, see0 = _bands(s)
    n, c = see.shape[2:4]
    L = see.shape[4] - c

    def scores(keys, visible):
        x = (q @ keys.transpose(-1, -2)).mul_(scale).view(B, Hk, n, G, c, -1)
        return x.masked_fill_(~visible[:, :, :, None], -math.inf).view(B, Hk, n, G * c, -1)
    p, p0 = scores(k, see), scores(k0, see0)
    top = p.amax(-1, keepdim=True)
    if p0.shape[-1]:
        top = torch.maximum(top, p0.amax(-1, keepdim=True))
    top = top.clamp_min(-3e38)   # rows that see nothing
    p, p0 = p.sub_(top).exp_(), (p0 - top).exp()
    total = p.sum(-1, keepdim=True) + p0.sum(-1, keepdim=True)
    total = torch.where(total > 0, total, 1.0)
    p, p0 = p.div_(total), p0 / total
    y = p @ v + p0 @ v0
    out = {"y": _flat(y, G, T).to(t)}
    if not train:
        return out
    dy = s["dy"].float()
    if s["len"] is not None:
        dy = torch.where((torch.arange(T, device=dy.device) < s["len"][:, None])[..., None, None], dy, 0.0)
    dy = _grouped(dy, Hk, n, c)
    D = (dy * y).sum(-1, keepdim=True)
    ds, ds0 = p * (dy @ v.transpose(-1, -2) - D) * scale, p0 * (dy @ v0.transpose(-1, -2) - D) * scale
    dq = _flat(ds @ k + ds0 @ k0, G, T)

    def keys(x, x0, of):
        """Sums over the queries: each block's own keys, the keys before them from the next block, the first tokens."""
        g = x.transpose(-1, -2) @ of
        own_part, before = g[:, :, :, L:], g[:, :, :, :L]
        if n > 1:
            own_part = own_part + torch.nn.functional.pad(before[:, :, 1:], (0, 0, 0, 0, 0, 1))
        got = own_part.reshape(B, Hk, n * c, d)[:, :, :T]   # no past in training
        first = (x0.transpose(-1, -2) @ of).sum(2)
        got[:, :, :first.shape[2]] += first
        return got.permute(0, 2, 1, 3).contiguous()
    return dict(out, grads=[dq.to(t), keys(ds, ds0, q).to(t), keys(p, p0, dy).to(t)])


def _plain_prefill(s):
    out = _plain_attn(s, False)
    if not s["cache"]:
        return dict(out, cache_k=[], cache_v=[])
    B, T, W, sinks = *s["k"].shape[:2], s["window"], s["sinks"]
    end = torch.full((B, 1), T, device=s["k"].device) if s["len"] is None else s["len"].view(B, 1)
    slot = torch.arange(sinks + W, device=s["k"].device)
    # the last token before the end that has this slot
    last = end - 1 - (end - 1 - slot) % W
    token = torch.where(slot < sinks, slot, last)
    held = torch.where(slot < sinks, slot < end, token >= sinks)[..., None, None]
    rows = torch.arange(B, device=slot.device)[:, None]
    of = lambda x: torch.where(held, x[rows, token.clamp(0, max(T - 1, 0))], torch.zeros((), dtype=x.dtype, device=x.device))
    return dict(out, cache_k=of(s["k"]), cache_v=of(s["v"]))


def _plain_decode(s):
    S, H, d = s["q"].shape
    slots, Hk = s["ck"].shape[1:3]
    sinks, pos = s["sinks"], s["pos"].long()
    slot = torch.where(pos < sinks, pos, sinks + (pos - sinks) % s["window"])
    rows = torch.arange(S, device=pos.device)
    s["ck"][rows, slot], s["cv"][rows, slot] = s["k"], s["v"]
    q = s["q"].float().view(S, Hk, H // Hk, d)
    x = (q @ s["ck"].float().permute(0, 2, 3, 1).contiguous()) / math.sqrt(d)
    x = torch.where((torch.arange(slots, device=pos.device) <= pos[:, None])[:, None, None], x, -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    y = (p / p.sum(-1, keepdim=True)) @ s["cv"].float().permute(0, 2, 1, 3).contiguous()
    return {"y": y.view(S, H, d).to(s["q"].dtype), "cache_k": s["ck"], "cache_v": s["cv"]}


_PLAIN = {"rope_train": lambda s: _plain_rope(s, True), "rope_infer": lambda s: _plain_rope(s, False),
          "attn_train": lambda s: _plain_attn(s, True), "attn_prefill": _plain_prefill, "attn_decode": _plain_decode}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    H, Hk, d = case["H"], case["Hk"], case["d"]
    if kind.startswith("rope"):
        m = case["B"] * case["T"] * (H + Hk) * d
        # forward x and out; backward x, the outputs' gradients and the inputs'
        return {"bytes": (5 if kind == "rope_train" else 2) * m * e + 32 * d, "flops": (27 if kind == "rope_train" else 8) * m}
    W, sinks = case["window"], case["sinks"]
    if kind == "attn_decode":
        held = case["S"] * min(W + sinks, max(1, 3 * case["seen"] // 4))
        # the visible tokens' keys and values, the new token's written, q and y
        return {"bytes": 2 * (held + case["S"]) * Hk * d * e + 2 * case["S"] * H * d * e, "flops": 4 * held * H * d}
    T, past = case["T"], case.get("past", 0)
    Tk, part = T + past, 0.5 if case["ragged"] else 1.0
    # sum over the positions p of min(p + 1, W) and of the first tokens behind the window
    upto = lambda n: n * (n + 1) // 2 if n <= W else W * (W + 1) // 2 + (n - W) * W
    behind = lambda n: sum(min(sinks, max(0, p - W + 1)) for p in range(min(n, W + sinks))) + max(0, n - W - sinks) * sinks
    pairs = part * case["B"] * H * (upto(Tk) - upto(past) + behind(Tk) - behind(past))
    qy, kv = part * case["B"] * T * H * d * e, part * case["B"] * Tk * Hk * d * e
    if kind == "attn_prefill":
        cache = 2 * case["B"] * min(Tk, W + sinks) * Hk * d * e if past == 0 else 0
        return {"bytes": 2 * qy + 2 * kv + cache, "flops": 4 * d * pairs}
    # forward q, k, v, y; backward q, k, v, y, dy and the three gradients
    return {"bytes": 6 * qy + 6 * kv, "flops": 14 * d * pairs}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("rope"):
        return _exact_rope(s, case)
    if case["kind"] == "attn_decode":
        return _exact_decode(s)
    return _exact_attn(s, case)


def _exact_rope(s, case):
    """The rotation as a product of complex numbers, the gradients by differentiation."""
    train = case["kind"] == "rope_train"
    outs, leaves, ups = [], [], []
    with torch.enable_grad():
        for n in ("q", "k"):
            x, w = (s[m].detach().double().requires_grad_(True) for m in (n, "w" + n))
            u = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + _EPS) * w
            if case["rot"]:
                rot, T = case["rot"], case["T"]
                pos = torch.arange(T, device=x.device)[None] if s["pos"] is None else s["pos"]
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos[:, :, None, None] * s["freq"])
                pair = u[..., :rot].unflatten(-1, (rot // 2, 2) if case["interleaved"] else (2, rot // 2))
                pair = pair if case["interleaved"] else pair.transpose(-1, -2)
                c = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
                c = (c if case["interleaved"] else c.transpose(-1, -2)).flatten(-2)
                u = torch.cat((c, u[..., rot:]), -1)
            outs.append(u)
            leaves.append((x, w))
            if train:
                ups.append(s["d" + n].double())
        out = {"q": outs[0].detach(), "k": outs[1].detach()}
        if train:
            (x0, w0), (x1, w1) = leaves
            out["grads"] = list(torch.autograd.grad(outs, [x0, x1, w0, w1], ups))
    return out


def _exact_attn(s, case):
    train = case["kind"] == "attn_train"
    x = {n: s[n].detach().double() for n in ("q", "k", "v", "dy") if n in s}
    B, T, H, d = x["q"].shape
    Tk, Hk, W = x["k"].shape[1], x["k"].shape[2], case["window"]
    y = torch.zeros_like(x["q"])
    dq, dk, dv = torch.zeros_like(x["q"]), torch.zeros_like(x["k"]), torch.zeros_like(x["v"])
    ends = [Tk] * B if s["len"] is None else s["len"].tolist()
    step = max(1, (1 << 27) // max(Tk, 1))
    for b in range(B):
        n = ends[b]
        for h in range(H):
            k, v = x["k"][b, :n, h * Hk // H], x["v"][b, :n, h * Hk // H]
            for lo in range(0, max(0, n - (Tk - T)), step):
                hi = min(lo + step, n - (Tk - T))
                q = x["q"][b, lo:hi, h]
                behind = (Tk - T + torch.arange(lo, hi, device=q.device))[:, None] - torch.arange(n, device=q.device)
                hidden = (behind < 0) | ((behind >= W) & (torch.arange(n, device=q.device) >= case["sinks"]))
                p = torch.softmax(torch.where(hidden, -math.inf, q @ k.T / d ** 0.5), -1)
                y[b, lo:hi, h] = p @ v
                if train:
                    g = x["dy"][b, lo:hi, h]
                    dp = g @ v.T
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / d ** 0.5
                    dq[b, lo:hi, h] = ds @ k
                    dk[b, :n, h * Hk // H] += ds.T @ q
                    dv[b, :n, h * Hk // H] += p.T @ g
    if train:
        return {"y": y, "grads": [dq, dk, dv]}
    out = {"y": y, "cache_k": [], "cache_v": []}
    if s["cache"]:
        for n in ("k", "v"):
            c = torch.zeros(B, W + case["sinks"], Hk, d, dtype=torch.float64, device=y.device)
            for b in range(B):
                keep = torch.tensor([t for t in range(ends[b]) if t < case["sinks"] or t >= ends[b] - W], dtype=torch.long,
                                    device=y.device)
                c[b, torch.where(keep < case["sinks"], keep, case["sinks"] + (keep - case["sinks"]) % W)] = x[n][b, keep]
            out["cache_" + n] = c
    return out


def _exact_decode(s):
    x = {n: s[n].double() for n in ("q", "k", "v", "ck", "cv")}
    S, H, d = x["q"].shape
    Hk, sinks = x["k"].shape[1], s["sinks"]
    y = torch.zeros_like(x["q"])
    for b, p in enumerate(s["pos"].tolist()):
        slot = p if p < sinks else sinks + (p - sinks) % s["window"]
        x["ck"][b, slot], x["cv"][b, slot] = x["k"][b], x["v"][b]
        held = min(p + 1, x["ck"].shape[1])
        k, v = (x[n][b, :held].repeat_interleave(H // Hk, 1) for n in ("ck", "cv"))
        w = torch.softmax((k * x["q"][b]).sum(-1) / d ** 0.5, 0)
        y[b] = (w[..., None] * v).sum(0)
    return {"y": y, "cache_k": x["ck"], "cache_v": x["cv"]}
