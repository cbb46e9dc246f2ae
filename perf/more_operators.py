"""Cases of the operators around a recurrent model, in their plain form and as the library's.

``listed()`` names the fixed cases, ``draw(rng)`` gives another one of the same
ranges, ``prepare`` makes a case's inputs on the GPU, ``run`` takes one pass and
``exact`` gives the same outputs in 64 bits, written apart from the plain form.
With ``own`` false ``run`` works in elementary torch operations; with ``own``
true it calls the library.

Kinds of pass:

* ``lookup`` - rows of an item table by id, scaled; the padding id gives zeros.
* ``embed``  - the lookup and its gradient by item, as a table of its own or added to the
  gradient that the prediction layer has left in it.
* ``qk``     - queries and keys of each head normalised and rotated by their positions.
* ``qktrain`` - the same and its gradients, those of the norms' weights among them.
* ``policy`` - a clipped policy loss with a KL term over logits of all items, and its gradient.
* ``muon``   - one optimiser step whose update is orthogonalised by Newton-Schulz products.
"""
from __future__ import annotations

import math

import torch

own = False

PAD = 0                            # the padding id
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
LR, MOMENTUM, DECAY, MUON_EPS, STEPS = 0.02, 0.95, 0.1, 1e-7, 5
COEFFS = (3.4445, -4.7750, 2.0315)  # of the Newton-Schulz step


def listed():
    return [
        # The last items of a few users, looked up before a decode step: one launch's latency.
        {"name": "lookup_few_bf16", "kind": "lookup", "io": "bf16", "B": 16, "L": 1,
         "V": 1000000, "D": 128},
        # MovieLens-1M's training batch: left-padded histories of up to 200 items.
        {"name": "embed_train_batch", "kind": "embed", "io": "f32", "B": 2048, "L": 200,
         "V": 3416, "D": 64, "into": False},
        # Long histories over a catalogue of a million items; the table is the prediction
        # layer's too, whose gradient is there already.
        {"name": "embed_train_catalogue_bf16", "kind": "embed", "io": "bf16", "B": 256, "L": 2048,
         "V": 1000000, "D": 128, "into": True},
        # Decode for a few users far into their histories.
        {"name": "qk_step_few_bf16", "kind": "qk", "io": "bf16", "B": 8, "L": 1, "H": 2, "HK": 2,
         "D": 128, "rot": 128, "norm": "rms", "weights": True, "start": 1000000},
        # A training batch for the delta rule, 2 heads of 64, with weights.
        {"name": "qk_train_batch_bf16", "kind": "qktrain", "io": "bf16", "B": 1024, "L": 200,
         "H": 2, "HK": 2, "D": 64, "rot": 64, "norm": "rms", "weights": True, "start": 0},
        # Long histories in fp32, lengths of one, half of each head rotated.
        {"name": "qk_train_long", "kind": "qktrain", "io": "f32", "B": 64, "L": 2048, "H": 4,
         "HK": 2, "D": 128, "rot": 64, "norm": "l2", "weights": False, "start": 0},
        # Four answers over a catalogue of 50,000 items: few long rows.
        {"name": "policy_few", "kind": "policy", "io": "f32", "N": 4, "V": 50000},
        # A batch of answers over MovieLens-1M's items.
        {"name": "policy_batch", "kind": "policy", "io": "f32", "N": 2048, "V": 3416},
        # Many answers over a large catalogue, logits in bf16.
        {"name": "policy_large_bf16", "kind": "policy", "io": "bf16", "N": 4096, "V": 131072},
        # The two-layer model's own matrices at MovieLens-1M's width.
        {"name": "muon_model_f32", "kind": "muon", "io": "f32", "D": 64, "layers": 2},
        # The same layers at the largest width, in bf16.
        {"name": "muon_wide_bf16", "kind": "muon", "io": "bf16", "D": 256, "layers": 2},
        # Matrices of a large model, one of odd sizes.
        {"name": "muon_large_f32", "kind": "muon", "io": "f32",
         "shapes": "2x2048x2048 1x8192x2048 1x999x1501"},
    ]


def _spread(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["lookup", "embed", "embed", "qk", "qktrain", "qktrain", "policy", "policy",
                       "muon", "muon"])
    io = rng.choice(["f32", "bf16"])
    if kind in ("lookup", "embed"):
        D = rng.choice([48, 64, 64, 100, 128, 128, 256, 33])
        V = int(_spread(rng, 20, 6.0e7 / D))
        n = _spread(rng, 1, 6.0e7 / D if kind == "embed" else 2.0e6 / D)
        L = 1 if kind == "lookup" else max(1, int(_spread(rng, 1, min(2048, n))))
        case = {"kind": kind, "io": io, "B": max(1, int(n / L)), "L": L, "V": V, "D": D}
        return case if kind == "lookup" else {**case, "into": bool(rng.random() < 0.5)}
    if kind in ("qk", "qktrain"):
        D = rng.choice([64, 64, 128, 128, 32, 72, 17, 256, 100])
        H = rng.choice([1, 2, 2, 4, 8])
        HK = max(1, H // rng.choice([1, 1, 2]))
        n = _spread(rng, 1, (1.0e8 if kind == "qktrain" else 4.0e6) / ((H + HK) * D))
        L = 1 if kind == "qk" and rng.random() < 0.6 else max(1, int(_spread(rng, 1, min(4096, n))))
        return {"kind": kind, "io": io, "B": max(1, int(n / L)), "L": L, "H": H, "HK": HK, "D": D,
                "rot": rng.choice([0, D // 2 * 2, D // 2 * 2, D // 4 * 2]),
                "norm": rng.choice(["rms", "l2"]), "weights": bool(rng.random() < 0.6),
                "start": rng.choice([0, 0, int(_spread(rng, 1, 2.0e6))])}
    if kind == "policy":
        N = int(round(_spread(rng, 1, 8192)))
        return {"kind": kind, "io": io, "N": N, "V": int(_spread(rng, 2, min(400000, 2.0e8 / N)))}
    if rng.random() < 0.5:
        return {"kind": "muon", "io": io, "D": rng.choice([33, 48, 64, 100, 128, 200, 256]),
                "layers": rng.choice([1, 2, 3])}
    shapes = ["%dx%dx%d" % (rng.choice([1, 1, 2, 3]), int(_spread(rng, 1, 2000)),
                            int(_spread(rng, 1, 2000))) for _ in range(rng.choice([1, 2, 3]))]
    return {"kind": "muon", "io": io, "shapes": " ".join(shapes)}


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["io"] == "f32" else torch.bfloat16


def _shapes(case):
    """[(count, rows, cols)] of the matrices of a step."""
    if "shapes" in case:
        return [tuple(int(x) for x in s.split("x")) for s in case["shapes"].split()]
    D, n = case["D"], case["layers"]
    E = 2 * D  # projections to and from the recurrent layer, its gates, the feed-forward's two
    return [(2 * n, E, D), (2 * n, E, E), (n, D, E), (n, 4 * D, D), (n, D, 4 * D)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt, s = case["kind"], _dtype(case), {"case": case}

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo

    if kind in ("lookup", "embed"):
        B, L, V, D = case["B"], case["L"], case["V"], case["D"]
        # Popularity falls as one over the rank; ranks lie anywhere in the table.
        cdf = torch.cumsum(1.0 / torch.arange(1, V, device="cuda", dtype=torch.float64), 0)
        rank = torch.searchsorted(cdf, uniform(0, 1, B, L).double() * cdf[-1]).clamp(max=V - 2)
        ids = torch.randperm(V - 1, generator=g, device="cuda")[rank] + 1
        if L > 1:  # left-padded rows
            least = max(1, int(0.655 * L))
            lengths = torch.randint(least, L + 1, (B, 1), generator=g, device="cuda")
            ids = ids.masked_fill(torch.arange(L, device="cuda")[None] < L - lengths, PAD)
        s["ids"] = ids.int()
        s["table"] = normal(V, D, scale=0.1).to(dt)
        s["scale"] = math.sqrt(D)
        if kind == "embed":
            s["dout"] = normal(B, L, D, scale=1e-2).to(dt)
            s["into"] = normal(V, D, scale=1e-2).to(dt) if case["into"] else None
        return s
    if kind in ("qk", "qktrain"):
        B, L, H, HK, D = case["B"], case["L"], case["H"], case["HK"], case["D"]
        s["q"], s["k"] = normal(B, L, H, D).to(dt), normal(B, L, HK, D, scale=2.0).to(dt)
        s["wq"], s["wk"] = (uniform(0.5, 1.5, D), uniform(0.5, 1.5, D)) if case["weights"] \
            else (None, None)
        # Each row starts somewhere: users' histories differ in what was read before.
        first = torch.randint(0, case["start"] + 1, (B, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(L, device="cuda")[None]).int()
        s["base"], s["eps"] = 10000.0, 1e-6
        if kind == "qktrain":
            s["dq"], s["dk"] = normal(B, L, H, D).to(dt), normal(B, L, HK, D).to(dt)
        return s
    if kind == "policy":
        N, V = case["N"], case["V"]
        logits = normal(N, V, scale=3.0)
        # Items that a user has had already are masked; one row in 64 has no item left.
        seen = uniform(0, 1, N, V) < 0.05 * uniform(0, 1, N, 1)
        seen |= (torch.arange(N, device="cuda") % 64 == 63)[:, None]
        logits = logits.masked_fill_(seen, -math.inf)
        s["temperature"] = 0.8
        # The items were chosen by an older policy: this one's odds, somewhat off.
        noise = uniform(1e-7, 1, N, V).log_().neg_().log_().neg_()
        s["ids"] = torch.argmax(noise.add_(logits, alpha=1 / 0.8), 1).int()
        s["logits"] = logits.to(dt)
        del noise, seen
        logp = torch.log_softmax(logits.div_(0.8), 1).gather(1, s["ids"].long()[:, None])[:, 0]
        empty = torch.arange(N, device="cuda") % 64 == 63
        empty |= ~torch.isfinite(logp)
        s["ids"] = s["ids"].masked_fill(empty, -1)
        logp = logp.masked_fill(empty, 0.0)
        s["old_logp"] = logp + normal(N, scale=0.2)
        s["ref_logp"] = logp + normal(N, scale=0.3)
        s["advantage"] = normal(N)
        s["weight"] = torch.full((N,), 1.0 / max(1, N - N // 64), device="cuda")
        return s
    # Matrices of a shape lie behind one another in one buffer.
    groups = _shapes(case)
    s["p"] = [normal(n, r, c, scale=c ** -0.5).to(dt) for n, r, c in groups]
    # Gradients of little rank and noise, momenta of the same kind.
    low = lambda n, r, c: normal(n, r, 4) @ normal(n, 4, c) + normal(n, r, c)  # noqa: E731
    s["g"] = [(low(*x) * 1e-3).to(dt) for x in groups]
    s["m"] = [low(*x) * 1e-3 for x in groups]
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind in ("lookup", "embed"):
        return _embed_plain(s, kind)
    if kind in ("qk", "qktrain"):
        return _qk_plain(s, kind == "qktrain")
    return _policy_plain(s) if kind == "policy" else _muon_plain(s)


def _run_own(s, kind):
    from paper_2406_12580_amd import recblr as rb
    if kind in ("lookup", "embed"):
        out = rb.embed(s["table"], s["ids"], scale=s["scale"], pad_id=PAD)
        if kind == "lookup":
            return {"out": out}
        return {"out": out, "dtable": rb.embed_backward(
            s["ids"], s["dout"], s["case"]["V"], scale=s["scale"], pad_id=PAD, into=s["into"])}
    if kind in ("qk", "qktrain"):
        how = dict(wq=s["wq"], wk=s["wk"], positions=s["positions"], rotate=s["case"]["rot"],
                   base=s["base"], norm=s["case"]["norm"], eps=s["eps"])
        qn, kn = rb.qk_norm(s["q"], s["k"], **how)
        if kind == "qk":
            return {"q": qn, "k": kn}
        d = rb.qk_norm_backward(s["q"], s["k"], s["dq"], s["dk"], **how)
        return {"q": qn, "k": kn, **d}
    if kind == "policy":
        loss, logp, dlogits = rb.policy_loss(
            s["logits"], s["ids"], s["old_logp"], s["advantage"], ref_logp=s["ref_logp"],
            weight=s["weight"], temperature=s["temperature"], clip_low=CLIP_LOW,
            clip_high=CLIP_HIGH, kl=KL)
        return {"loss": loss, "logp": logp, "dlogits": dlogits}
    if "opt" not in s:  # a program makes its optimiser once, around the momenta that it holds
        one = lambda ts: [t for x in ts for t in x.unbind(0)]  # noqa: E731
        s["opt"] = rb.Muon(one(s["p"]), lr=LR, momentum=MOMENTUM, nesterov=True,
                           weight_decay=DECAY, steps=STEPS, eps=MUON_EPS, state=one(s["m"]))
        s["grads"] = one(s["g"])
    s["opt"].step(s["grads"])
    return {"p": s["p"], "m": s["m"]}


# ------------------------------------------------------------------ plain forms

def _embed_plain(s, kind):
    ids = s["ids"].long()
    pad = (ids == PAD)[..., None]
    out = (s["table"][ids].float() * s["scale"]).masked_fill_(pad, 0.0).to(s["table"].dtype)
    if kind == "lookup":
        return {"out": out}
    V, D = s["table"].shape
    rows = s["dout"].float().masked_fill(pad, 0.0).reshape(-1, D)
    d = torch.zeros(V, D, device="cuda").index_add_(0, ids.reshape(-1), rows).mul_(s["scale"])
    if s["into"] is None:
        return {"out": out, "dtable": d.to(s["dout"].dtype)}
    return {"out": out, "dtable": s["into"].copy_(d.add_(s["into"]))}


def _qk_plain(s, train):
    case = s["case"]
    R, D = case["rot"], case["D"]
    # Angles in 64 bits: those of far positions are thousands of turns.
    rate = s["base"] ** (-2.0 * torch.arange(R // 2, device="cuda", dtype=torch.float64)
                         / max(R, 1))
    angle = (s["positions"].double()[..., None] * rate)[:, :, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    share = 1.0 / D if case["norm"] == "rms" else 1.0

    def turn(x, sin):
        a, b, rest = x[..., :R // 2], x[..., R // 2:R], x[..., R:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)

    def forward(x, w):
        r = torch.rsqrt((x.float().square().sum(-1, keepdim=True)) * share + s["eps"])
        u = x.float() * r
        return r, u, turn(u if w is None else u * w, sin).to(x.dtype)

    def backward(x, w, r, u, dy):
        g = turn(dy.float(), -sin)
        a = g if w is None else g * w
        dx = (r * (a - u * ((u * a).sum(-1, keepdim=True) * share))).to(x.dtype)
        dw = None if w is None else (g * u).sum((0, 1, 2), dtype=torch.float64).float()
        return dx, dw

    rq, uq, q = forward(s["q"], s["wq"])
    rk, uk, k = forward(s["k"], s["wk"])
    if not train:
        return {"q": q, "k": k}
    dq, dwq = backward(s["q"], s["wq"], rq, uq, s["dq"])
    dk, dwk = backward(s["k"], s["wk"], rk, uk, s["dk"])
    return {"q": q, "k": k, "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def _policy_plain(s):
    T, ids = s["temperature"], s["ids"].long()
    live, at = ids >= 0, ids.clamp(min=0)[:, None]
    x = s["logits"].float()
    x = (x - x.amax(1, keepdim=True)) / T
    e = torch.exp(x)
    total = e.sum(1)
    lp = x.gather(1, at)[:, 0] - torch.log(total)
    ratio, A, d = torch.exp(lp - s["old_logp"]), s["advantage"], s["ref_logp"] - lp
    free, held = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    rows = s["weight"] * (-torch.minimum(free, held) + KL * (torch.exp(d) - d - 1))
    c = s["weight"] * (KL * (1 - torch.exp(d)) - torch.where(free <= held, free, 0.0)) / T
    c = torch.where(live, c, 0.0)
    grad = e.mul_(torch.where(live, -c / total, 0.0)[:, None]).scatter_add_(1, at, c[:, None])
    grad = torch.where(live[:, None], grad, 0.0)
    loss = torch.where(live, rows, 0.0).sum(0, keepdim=True)
    return {"loss": loss, "logp": torch.where(live, lp, 0.0),
            "dlogits": grad.to(s["logits"].dtype)}


def _muon_plain(s):
    a, b, c = COEFFS
    for p, g, m in zip(s["p"], s["g"], s["m"]):  # a shape's matrices at a time
        g = g.float()
        m.mul_(MOMENTUM).add_(g, alpha=1 - MOMENTUM)
        x = m * MOMENTUM + g * (1 - MOMENTUM)
        tall = x.shape[1] > x.shape[2]
        x = x.transpose(1, 2).contiguous() if tall else x
        norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
        x = x / (norm + MUON_EPS).float()
        for _ in range(STEPS):
            A = torch.bmm(x, x.transpose(1, 2).contiguous())
            x = a * x + torch.bmm(b * A + c * torch.bmm(A, A), x)
        x = x.transpose(1, 2) if tall else x
        scale = math.sqrt(max(1.0, p.shape[1] / p.shape[2]))
        p.copy_(p.float() * (1 - LR * DECAY) - LR * scale * x)
    return {"p": s["p"], "m": s["m"]}


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once, each output written once; symmetric products by half of them."""
    kind, e = case["kind"], 4 if case["io"] == "f32" else 2
    if kind in ("lookup", "embed"):
        N, V, D = case["B"] * case["L"], case["V"], case["D"]
        hit = min(N, V)  # rows of the table that are met
        fwd = 4.0 * N + (hit + N) * D * e
        if kind == "lookup":
            return {"bytes": fwd, "flops": 1.0 * N * D}
        grad = 2.0 * hit if case["into"] else 1.0 * V
        return {"bytes": fwd + N * D * e + grad * D * e, "flops": 2.0 * N * D + hit * D}
    if kind in ("qk", "qktrain"):
        rows = case["B"] * case["L"] * (case["H"] + case["HK"])
        n = 1.0 * rows * case["D"]
        if kind == "qk":
            return {"bytes": 2 * n * e + 4.0 * case["B"] * case["L"], "flops": 8 * n}
        return {"bytes": 5 * n * e + 4.0 * case["B"] * case["L"], "flops": 25 * n}
    if kind == "policy":
        n = 1.0 * case["N"] * case["V"]
        return {"bytes": 2 * n * e + 24.0 * case["N"], "flops": 8 * n}
    size, flops = 0.0, 0.0
    for n, r, c in _shapes(case):
        m, k = min(r, c), max(r, c)
        size += n * r * c
        flops += n * STEPS * (3.0 * m * m * k + 1.0 * m * m * m)
    return {"bytes": size * (3 * e + 8), "flops": flops + 10 * size}


# ------------------------------------------------------------------ 64-bit reference

def _embed64(s, kind):
    V, D = s["table"].shape
    ids = s["ids"].reshape(-1).long()
    table = s["table"].double()
    table[PAD] = 0.0
    out = {"out": (table * s["scale"]).index_select(0, ids).reshape(*s["ids"].shape, D)}
    if kind == "lookup":
        return out
    del table
    # Sorted by item, an item's rows are a difference of running sums.
    order = torch.argsort(ids, stable=True)
    run_sum = torch.cumsum(s["dout"].reshape(-1, D).double()[order], 0)
    run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
    item = torch.arange(V, device="cuda")
    first = torch.searchsorted(ids[order].contiguous(), item)
    last = torch.searchsorted(ids[order].contiguous(), item, right=True)
    d = s["scale"] * (run_sum[last] - run_sum[first])
    d[PAD] = 0.0
    out["dtable"] = d if s["into"] is None else d + s["into"].double()
    return out


def _qk64(s, train):
    case = s["case"]
    R, D = case["rot"], case["D"]
    # Pairs as complex numbers, turned by e^(i angle).
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    rate = torch.exp(-2.0 * i / max(R, 1) * math.log(s["base"]))
    t = s["positions"].double()[:, :, None, None] * rate
    spin = torch.complex(torch.cos(t), torch.sin(t))
    share = 1.0 / D if case["norm"] == "rms" else 1.0
    out = {}
    for n in ("q", "k"):
        x, w = s[n].double(), s["w" + n]
        w = torch.ones(D, dtype=torch.float64, device="cuda") if w is None else w.double()
        length = torch.sqrt(share * (x * x).sum(-1, keepdim=True) + s["eps"])
        y = w * x / length
        z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * spin
        out[n] = torch.cat([z.real, z.imag, y[..., R:]], -1)
        if not train:
            continue
        dy = s["d" + n].double()
        z = torch.complex(dy[..., :R // 2], dy[..., R // 2:R]) * spin.conj()
        dy = torch.cat([z.real, z.imag, dy[..., R:]], -1)
        out["d" + n] = w * dy / length \
            - share * x * (w * dy * x).sum(-1, keepdim=True) / length ** 3
        if s["w" + n] is not None:
            out["dw" + n] = (dy * x / length).reshape(-1, D).sum(0)
    return out


def _policy64(s):
    """By the definition, a few rows at a time."""
    N, V = s["logits"].shape
    T = s["temperature"]
    loss = torch.zeros(1, dtype=torch.float64, device="cuda")
    logp = torch.zeros(N, dtype=torch.float64, device="cuda")
    grad = torch.zeros(N, V, dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 26 // V)
    for a in range(0, N, step):
        rows = a + torch.nonzero(s["ids"][a:a + step] >= 0)[:, 0]
        if not len(rows):
            continue
        pick = s["ids"][rows].long()[:, None]
        p = torch.softmax(s["logits"][rows].double() / T, 1)
        lp = torch.log_softmax(s["logits"][rows].double() / T, 1).gather(1, pick)[:, 0]
        logp[rows] = lp
        old, ref, A, w = (s[n][rows].double() for n in ("old_logp", "ref_logp", "advantage",
                                                        "weight"))
        r = torch.exp(lp - old)
        inside = torch.where(A >= 0, r <= 1 + CLIP_HIGH, r >= 1 - CLIP_LOW)
        gain = torch.where(inside, r, torch.where(A >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW)) * A
        loss += (w * (KL * (torch.expm1(ref - lp) - (ref - lp)) - gain)).sum()
        c = w * (-KL * torch.expm1(ref - lp) - torch.where(inside, r * A, 0.0))
        p.neg_().scatter_add_(1, pick, torch.ones_like(pick, dtype=torch.float64))
        grad[rows] = p * (c / T)[:, None]
    return {"loss": loss, "logp": logp, "dlogits": grad}


def _muon64(s):
    a, b, c = COEFFS
    out = {"p": [], "m": []}
    for p, g, m in zip(s["p"], s["g"], s["m"]):
        new_p, new_m = torch.empty_like(p, dtype=torch.float64), torch.empty_like(m.double())
        for i in range(len(p)):
            gi = g[i].double()
            mi = MOMENTUM * m[i].double() + (1 - MOMENTUM) * gi
            x = MOMENTUM * mi + (1 - MOMENTUM) * gi
            x = x / (torch.linalg.matrix_norm(x) + MUON_EPS)
            for _ in range(STEPS):  # from the shorter side: x (aI + b G + c G^2), or its mirror
                if x.shape[0] > x.shape[1]:
                    G = x.T @ x
                    x = a * x + x @ (b * G + c * (G @ G))
                else:
                    G = x @ x.T
                    x = a * x + (b * G + c * (G @ G)) @ x
            r, k = p.shape[1:]
            new_p[i] = (1 - LR * DECAY) * p[i].double() - LR * max(1.0, r / k) ** 0.5 * x
            new_m[i] = mi
        out["p"].append(new_p)
        out["m"].append(new_m)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("lookup", "embed"):
        return _embed64(s, kind)
    if kind in ("qk", "qktrain"):
        return _qk64(s, kind == "qktrain")
    return _policy64(s) if kind == "policy" else _muon64(s)
