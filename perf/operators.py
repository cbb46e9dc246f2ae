"""Cases of the sequence, optimiser and answer operators, in their plain form and as the library's.

``listed()`` names the fixed cases, ``draw(rng)`` gives another one of the same
ranges, ``prepare`` makes a case's inputs on the GPU, ``run`` takes one pass and
``exact`` gives the same outputs in 64 bits, written apart from the plain form.
With ``own`` false ``run`` works in elementary torch operations; with ``own``
true it calls the library.

Kinds of pass:

* ``train``   - gated delta rule, forward and backward of a batch of histories:
  S_t = a_t (I - b_t k_t k_t^T) S_{t-1} + b_t k_t v_t^T, o_t = scale S_t^T q_t,
  a_t = e^{g_t}; value head j reads query and key head j / (HV / H).
* ``prefill`` - the forward alone, from a given state.
* ``step``    - one token of the same recurrence for a batch of users.
* ``adamw``   - one AdamW step over a list of tensors, moments in 32 or 8 bits.
* ``sample``  - one item a row from logits: temperature, top-k, top-p, min-p.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
QBLOCK = 256  # elements that share a scale of the 8-bit moments


def listed():
    return [
        # A handful of short histories in fp32: the smallest training call, all latency.
        {"name": "delta_train_small", "kind": "train", "io": "f32", "B": 4, "L": 50, "H": 2,
         "HV": 2, "Dk": 32, "Dv": 32, "h0": False},
        # A training batch of histories of up to 200 items, width 2 x 64, left-padded.
        {"name": "delta_train_batch_bf16", "kind": "train", "io": "bf16", "B": 1024, "L": 200,
         "H": 2, "HV": 2, "Dk": 64, "Dv": 64, "h0": False},
        # Long histories in fp32, two value heads to each query and key head.
        {"name": "delta_train_long", "kind": "train", "io": "f32", "B": 64, "L": 2048, "H": 2,
         "HV": 4, "Dk": 64, "Dv": 64, "h0": False},
        # One very long history in bf16: few heads, much sequence, a state carried in.
        {"name": "delta_train_verylong_bf16", "kind": "train", "io": "bf16", "B": 1, "L": 16384,
         "H": 2, "HV": 4, "Dk": 128, "Dv": 128, "h0": True},
        # Serving: odd sizes everywhere, histories read in from a kept state.
        {"name": "delta_prefill_ragged_bf16", "kind": "prefill", "io": "bf16", "B": 37, "L": 777,
         "H": 1, "HV": 3, "Dk": 72, "Dv": 100, "h0": True},
        # Decode for a few users at once: one launch's latency.
        {"name": "delta_step_few_bf16", "kind": "step", "io": "bf16", "B": 8, "H": 2, "HV": 4,
         "Dk": 128, "Dv": 128},
        # Decode for thousands of users: every state read and written once.
        {"name": "delta_step_many_bf16", "kind": "step", "io": "bf16", "B": 8192, "H": 2, "HV": 4,
         "Dk": 64, "Dv": 64},
        # The two-layer model's own tensors (MovieLens-1M sizes): many, most of them small.
        {"name": "adamw_model_f32", "kind": "adamw", "io": "f32", "bits": 32, "V": 3416, "D": 64,
         "layers": 2},
        # A table of a million items beside the same layers, bf16, moments in 8 bits.
        {"name": "adamw_table_bf16_8bit", "kind": "adamw", "io": "bf16", "bits": 8, "V": 1000000,
         "D": 128, "layers": 2},
        # An answer for a few users over a catalogue of 50,000 items.
        {"name": "sample_few", "kind": "sample", "io": "f32", "B": 4, "V": 50000},
        # A whole evaluation batch over MovieLens-1M's items.
        {"name": "sample_batch", "kind": "sample", "io": "f32", "B": 2048, "V": 3416},
        # A large catalogue, logits in bf16 (many equal ones).
        {"name": "sample_large_bf16", "kind": "sample", "io": "bf16", "B": 64, "V": 131072},
    ]


def _spread(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["train", "train", "train", "prefill", "step", "adamw", "sample", "sample"])
    io = rng.choice(["f32", "bf16"])
    if kind == "adamw":
        return {"kind": kind, "io": io, "bits": rng.choice([8, 32]),
                "V": int(_spread(rng, 50, 600000)), "D": rng.choice([48, 64, 100, 128]),
                "layers": rng.choice([1, 2, 3])}
    if kind == "sample":
        B = int(round(_spread(rng, 1, 2048)))
        return {"kind": kind, "io": io, "B": B,
                "V": int(_spread(rng, 100, min(200000, 8.0e6 / B)))}
    # Head widths: the configurations' own and odd ones; value heads share keys or not.
    Dk, Dv = rng.choice([(64, 64), (64, 64), (128, 128), (32, 32), (64, 128), (72, 100), (17, 40)])
    H = rng.choice([1, 2, 2, 4])
    HV = H * rng.choice([1, 1, 2, 3])
    if kind == "step":
        return {"kind": kind, "io": io, "B": max(1, int(_spread(rng, 1, 1.2e8 / (HV * Dk * Dv)))),
                "H": H, "HV": HV, "Dk": Dk, "Dv": Dv}
    rows = _spread(rng, 4 * HV, 4.0e5 * 4096 / max(4096, Dk * Dv)) / HV
    L = max(1, int(_spread(rng, min(8, rows), min(8192, rows))))
    return {"kind": kind, "io": io, "B": max(1, int(rows / L)), "L": L, "H": H, "HV": HV,
            "Dk": Dk, "Dv": Dv, "h0": bool(rng.random() < 0.5)}


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["io"] == "f32" else torch.bfloat16


def _tensors(case):
    """[(size, decayed)] of the model's parameter tensors: matrices and the item table decay,
    biases, norms and per-channel vectors do not."""
    D, V = case["D"], case["V"]
    E = 2 * D
    one = [(E * D, 1), (E, 0), (E * D, 1), (E, 0), (E * 4, 1), (E, 0), (E * E, 1), (E, 0),
           (E * E, 1), (E, 0), (E, 0), (D * E, 1), (D, 0), (D, 0), (D, 0), (4 * D * D, 1),
           (4 * D, 0), (4 * D * D, 1), (D, 0), (D, 0), (D, 0)]
    return [(V * D, 1), (D, 0), (D, 0)] + one * case["layers"]


def _code_values(scale, code, power, lo, top):
    """What codes stand for: the block's scale times ((code + lo) / top) ** power, signed."""
    x = (code.double() + lo) / top
    return scale.double() * torch.sign(x) * x.abs() ** power


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt, s = case["kind"], _dtype(case), {"case": case}

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo

    if kind == "adamw":
        sizes = _tensors(case)
        s["sizes"] = [n for n, _ in sizes]
        s["decay"] = [DECAY * d for _, d in sizes]
        # One flat buffer, each tensor at a multiple of 64 elements, as the model step has it.
        starts, off = [], 0
        for n, _ in sizes:
            starts.append(off)
            off += -(-n // 64) * 64
        s["params"] = normal(off, scale=0.1).to(dt)
        s["grads"] = (normal(off, scale=1e-3) * torch.exp(normal(off))).to(dt)
        s["t"] = 10  # updates done so far
        views = lambda t: [t[o:o + n] for o, n in zip(starts, s["sizes"])]  # noqa: E731
        s["p"], s["g"] = views(s["params"]), views(s["grads"])
        s["starts"] = starts
        if case["bits"] == 32:
            s["m1"], s["m2"] = normal(off, scale=1e-3), uniform(1e-8, 1e-5, off)
            s["m"], s["v"] = views(s["m1"]), views(s["m2"])
        else:
            # Codes lie as their elements do; each tensor's scales start anew.
            s["c1"] = torch.randint(-127, 128, (off,), generator=g, device="cuda").to(torch.int8)
            s["c2"] = torch.randint(0, 256, (off,), generator=g, device="cuda").to(torch.uint8)
            blocks = [-(-n // QBLOCK) for n in s["sizes"]]
            s["s1"], s["s2"] = uniform(1e-4, 1e-2, sum(blocks)), uniform(1e-8, 1e-5, sum(blocks))
            cut = lambda t: list(torch.split(t, blocks))  # noqa: E731
            s["m"], s["v"] = views(s["c1"]), views(s["c2"])
            s["ms"], s["vs"] = cut(s["s1"]), cut(s["s2"])
        # Which tensor, and which block of the scales, an element of the flat buffer is of.
        size = torch.tensor(s["sizes"], device="cuda")
        start = torch.tensor(starts, device="cuda")
        at = torch.arange(off, device="cuda")
        which = torch.searchsorted(start, at, right=True) - 1
        inside = at - start[which]
        s["live"] = inside < size[which]
        s["wd"] = torch.tensor(s["decay"], device="cuda", dtype=torch.float32)[which]
        if case["bits"] == 8:
            nb = (size + QBLOCK - 1) // QBLOCK
            first = torch.cumsum(nb, 0) - nb
            s["block"] = torch.where(s["live"], first[which] + inside // QBLOCK, 0)
        return s
    if kind == "sample":
        B, V = case["B"], case["V"]
        s["logits"] = normal(B, V, scale=3.0)
        # Items that a user has had already are masked; one row in 64 has no item left.
        seen = uniform(0, 1, B, V) < 0.05 * uniform(0, 1, B, 1)
        seen |= (torch.arange(B, device="cuda") % 64 == 63)[:, None]
        s["logits"] = s["logits"].masked_fill(seen, -math.inf).to(dt).contiguous()
        s["u"] = uniform(0, 1, B)
        s["temperature"] = torch.where(uniform(0, 1, B) < 0.05, 0.0, uniform(0.5, 1.5, B))
        k = torch.exp(uniform(0, math.log(max(2, V // 2)), B)).int()
        s["top_k"] = torch.where(uniform(0, 1, B) < 0.4, torch.zeros_like(k), k)
        s["top_p"] = torch.where(uniform(0, 1, B) < 0.3, 1.0, uniform(0.3, 1.0, B))
        s["min_p"] = torch.where(uniform(0, 1, B) < 0.7, 0.0, uniform(0.0, 0.1, B))
        return s
    B, L, H, HV, Dk, Dv = case["B"], case.get("L", 1), case["H"], case["HV"], case["Dk"], case["Dv"]
    # Queries and keys leave a SiLU and are brought to length one; decays and strengths as
    # their gates give them (half-lives of ten to some thousand items).
    unit = lambda x: x / x.norm(dim=-1, keepdim=True).clamp_min(1e-6)  # noqa: E731
    silu = lambda x: x * torch.sigmoid(x)  # noqa: E731
    s["q"] = unit(silu(normal(B, L, H, Dk))).to(dt)
    s["k"] = unit(silu(normal(B, L, H, Dk))).to(dt)
    s["v"] = silu(normal(B, L, HV, Dv)).to(dt)
    rate = torch.exp(uniform(math.log(2e-4), math.log(0.1), HV))
    s["g"] = (-rate * uniform(0.2, 2.0, B, L, HV)).to(dt)
    s["beta"] = torch.sigmoid(normal(B, L, HV)).to(dt)
    if kind == "train" and B >= 8:  # left-padded rows: a padded step leaves the state alone
        least = max(1, int(0.655 * L))
        lengths = torch.randint(least, L + 1, (B, 1, 1), generator=g, device="cuda")
        pad = torch.arange(L, device="cuda")[None, :, None] < L - lengths
        s["g"], s["beta"] = s["g"].masked_fill(pad, 0), s["beta"].masked_fill(pad, 0)
    if kind == "step":
        for n in ("q", "k", "v", "g", "beta"):
            s[n] = s[n][:, 0].contiguous()
        s["h_prev"] = normal(B, HV, Dk, Dv, scale=0.3)
        return s
    s["h0"] = normal(B, HV, Dk, Dv, scale=0.3) if case["h0"] else None
    if kind == "train":
        s["do"] = normal(B, L, HV, Dv).to(dt)
        s["dhT"] = normal(B, HV, Dk, Dv, scale=0.3) if case["h0"] else None
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "train":
        return _train_plain(s)
    if kind == "prefill":
        with torch.no_grad():
            o, hT = _delta_plain(s["q"], s["k"], s["v"], s["g"], s["beta"], s["h0"])
        return {"o": o.to(s["v"].dtype), "hT": hT}
    if kind == "step":
        return _step_plain(s)
    if kind == "adamw":
        return _adamw_plain(s)
    return _sample_plain(s)


def _run_own(s, kind):
    from paper_2406_12580_amd import recblr as rb
    if kind in ("train", "prefill"):
        a = (s["q"], s["k"], s["v"], s["g"], s["beta"])
        if kind == "prefill":
            o, hT, _ = rb.delta_forward(*a, h0=s["h0"])
            return {"o": o, "hT": hT}
        o, hT, states = rb.delta_forward(*a, h0=s["h0"], keep_states=True)
        d = rb.delta_backward(*a, states, s["do"], dhT=s["dhT"], need_dh0=s["h0"] is not None)
        return {"o": o, "hT": hT, **{n: t for n, t in d.items() if t is not None}}
    if kind == "step":
        o, h = rb.delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["h_prev"])
        return {"o": o, "h": h}
    if kind == "sample":
        ids, prob = rb.sample(s["logits"], s["u"], temperature=s["temperature"],
                              top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"ids": ids, "prob": prob}
    bits = s["case"]["bits"]
    if "opt" not in s:  # a program makes its optimiser once, around the moments that it holds
        s["opt"] = rb.AdamW(s["p"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                            weight_decay=s["decay"], state_bits=bits,
                            state=(s["m"], s["v"]) if bits == 32
                            else (s["m"], s["v"], s["ms"], s["vs"]), step=s["t"])
    s["opt"].step(s["g"])
    if bits == 32:
        return {"params": s["params"], "m1": s["m1"], "m2": s["m2"]}
    m1, m2 = torch.zeros_like(s["wd"]), torch.zeros_like(s["wd"])
    views = lambda t: [t[o:o + n] for o, n in zip(s["starts"], s["sizes"])]  # noqa: E731
    s["opt"].moments(out=(views(m1), views(m2)))
    return {"params": s["params"], "m1": m1, "m2": m2}


# ------------------------------------------------------------------ plain forms

CHUNK = 64


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower triangular blocks: inverses of twice the size at a time."""
    n = A.shape[-1]
    if n == 1:
        return torch.ones_like(A)
    m = n // 2
    a, d = _unit_lower_inverse(A[..., :m, :m]), _unit_lower_inverse(A[..., m:, m:])
    b = -d @ (A[..., m:, :m] @ a)
    top = torch.cat([a, torch.zeros_like(b.transpose(-1, -2))], -1)
    return torch.cat([top, torch.cat([b, d], -1)], -2)


def _delta_plain(q, k, v, g, beta, h0):
    """Outputs and the last state in 32 bits, 64 steps at a time: within a block the updates
    u solve (I + tril(b (k k^T) decay)) u = b (v - e^c k S), c the running sum of g."""
    B, L, H, Dk = q.shape
    HV, Dv = v.shape[2], v.shape[3]
    n = -(-L // CHUNK)

    def blocks(t):  # [B, L, heads, d] -> [B * HV, n, CHUNK, d], padded behind the last step
        t = t.float().transpose(1, 2)
        t = t.repeat_interleave(HV // t.shape[1], 1)
        t = torch.nn.functional.pad(t, (0, 0, 0, n * CHUNK - L))
        return t.reshape(B * HV, n, CHUNK, t.shape[-1])

    q, k, v, g, b = blocks(q), blocks(k), blocks(v), blocks(g[..., None]), blocks(beta[..., None])
    c = torch.cumsum(g.double(), 2)
    tri = torch.ones(CHUNK, CHUNK, device=q.device, dtype=torch.bool).tril()
    G = torch.exp((c - c.transpose(2, 3)).masked_fill(~tri, -math.inf)).float()
    e, left, whole = c.exp().float(), (c[:, :, -1:] - c).exp().float(), c[:, :, -1:].exp().float()
    kT = k.transpose(2, 3).contiguous()
    T = _unit_lower_inverse((b * (k @ kT) * G).tril(-1))
    P = (q @ kT) * G
    S = torch.zeros(B * HV, Dk, Dv, device=q.device) if h0 is None else h0.reshape(B * HV, Dk, Dv)
    out, scale = [], Dk ** -0.5
    for j in range(n):
        u = T[:, j] @ (b[:, j] * (v[:, j] - e[:, j] * (k[:, j] @ S)))
        out.append(scale * (e[:, j] * (q[:, j] @ S) + P[:, j] @ u))
        S = whole[:, j] * S + kT[:, j] @ (left[:, j] * u)
    o = torch.stack(out, 1).reshape(B, HV, n * CHUNK, Dv)[:, :, :L].transpose(1, 2).contiguous()
    return o, S.reshape(B, HV, Dk, Dv)


def _train_plain(s):
    names = ["q", "k", "v", "g", "beta"] + (["h0"] if s["h0"] is not None else [])
    leaf = {n: s[n].float().requires_grad_() for n in names}
    with torch.enable_grad():
        o, hT = _delta_plain(*(leaf[n] for n in names[:5]), leaf.get("h0"))
        loss = (o * s["do"].float()).sum()
        if s["dhT"] is not None:
            loss = loss + (hT * s["dhT"]).sum()
        grads = torch.autograd.grad(loss, [leaf[n] for n in names])
    out = {"d" + n: t.to(s[n].dtype) for n, t in zip(names, grads)}
    return {"o": o.detach().to(s["v"].dtype), "hT": hT.detach(), **out}


def _step_plain(s):
    r = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[n].float().repeat_interleave(r, 1).unsqueeze(-1) for n in ("q", "k"))
    S = s["h_prev"] * torch.exp(s["g"].float())[..., None, None]
    u = s["beta"].float()[..., None] * (s["v"].float() - (S * k).sum(-2))
    S = S + k * u.unsqueeze(-2)
    o = (S * q).sum(-2) * k.shape[-2] ** -0.5
    return {"o": o.to(s["v"].dtype), "h": S}


def _adamw_plain(s):
    bits8 = s["case"]["bits"] == 8
    # 8-bit moments in 64 bits: a value next to the border of two codes has to fall on one side.
    ft = torch.float64 if bits8 else torch.float32
    s["t"] += 1
    g, p = s["grads"].to(ft), s["params"].float()
    if bits8:
        m = _code_values(s["s1"][s["block"]], s["c1"], 2, 0, 127)
        v = _code_values(s["s2"][s["block"]], s["c2"], 4, 1, 256)
    else:
        m, v = s["m1"], s["m2"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    upd = (m / (1 - BETA1 ** s["t"])) / (torch.sqrt(v / (1 - BETA2 ** s["t"])) + EPS)
    new = p * (1 - LR * s["wd"]) - LR * upd.float()
    live = s["live"]
    s["params"].copy_(torch.where(live, new.to(s["params"].dtype), s["params"]))
    if not bits8:
        s["m1"].copy_(torch.where(live, m, s["m1"]))
        s["m2"].copy_(torch.where(live, v, s["m2"]))
        return {"params": s["params"], "m1": s["m1"], "m2": s["m2"]}
    outs = []
    for val, sc, code, power, lo, top in ((m, "s1", "c1", 2, 0, 127), (v, "s2", "c2", 4, 1, 256)):
        big = torch.zeros_like(s[sc], dtype=ft)
        big.scatter_reduce_(0, s["block"], torch.where(live, val.abs(), 0.0), "amax")
        s[sc].copy_(big.float())
        per = s[sc].double()[s["block"]]
        x = torch.where(per > 0, val.abs() / per, 0.0) ** (1.0 / power) * top
        c = torch.sign(val) * torch.round(x).clamp(0, top) if lo == 0 else \
            (torch.round(x) - 1).clamp(0, 255)
        s[code].copy_(torch.where(live, c.to(s[code].dtype), s[code]))
        outs.append(torch.where(live, _code_values(per, s[code], power, lo, top), 0.0).float())
    return {"params": s["params"], "m1": outs[0], "m2": outs[1]}


def _sample_plain(s):
    """Weights and their sums in 64 bits: a sum next to a border decides which item is taken."""
    x = s["logits"].double()
    B, V = x.shape
    top = x.amax(1, keepdim=True)
    empty = ~torch.isfinite(top[:, 0])
    t = s["temperature"].double()[:, None]
    w = torch.where(t > 0, torch.exp((x - top) / t), (x == top).double())
    w = torch.where(empty[:, None], torch.zeros_like(w), w)
    _, order = torch.sort(x, dim=1, descending=True, stable=True)
    ws = torch.gather(w, 1, order)
    rank = torch.arange(V, device=x.device)[None]
    k = torch.where((s["top_k"] > 0) & (t[:, 0] > 0), s["top_k"].long(), V)
    k = torch.where(t[:, 0] > 0, k, 1)[:, None]
    ws = torch.where(rank < k, ws, torch.zeros_like(ws))
    cum = torch.cumsum(ws, 1)
    p = s["top_p"].double()[:, None]
    keep = (rank < k) & ((cum - ws < p * cum[:, -1:]) | (p >= 1) | (rank == 0))
    keep &= (ws >= s["min_p"].double()[:, None] * ws[:, :1])
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, torch.zeros_like(ws)))
    cum = torch.cumsum(kept, 1)
    ids = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1)
    last = V - 1 - torch.argmax((kept.flip(1) > 0).int(), 1)
    ids = torch.minimum(ids, last)
    prob = torch.gather(kept, 1, ids[:, None])[:, 0] / cum[:, -1]
    return {"ids": torch.where(empty, -1, ids).int(),
            "prob": torch.where(empty, torch.zeros_like(prob), prob).float()}


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once, each output written once, and the recurrence's products as the
    definition has them, for a whole chunk of steps at a time where there is one."""
    kind, e = case["kind"], 4 if case["io"] == "f32" else 2
    if kind == "adamw":
        n = sum(m for m, _ in _tensors(case))
        # Parameter, gradient and both moments in, parameter and moments out; the values that
        # 8-bit moments stand for once more, as they are returned.
        per = 3 * e + (16 if case["bits"] == 32 else 4 + 4 * 8 / QBLOCK + 10)
        return {"bytes": n * per, "flops": 20.0 * n}
    if kind == "sample":
        n = case["B"] * case["V"]
        return {"bytes": n * e + 28.0 * case["B"], "flops": 10.0 * n}
    B, L, H, HV, Dk, Dv = case["B"], case.get("L", 1), case["H"], case["HV"], case["Dk"], case["Dv"]
    qk, vo, gate, st = B * L * H * Dk * e, B * L * HV * Dv * e, B * L * HV * e, B * HV * Dk * Dv * 4.0
    if kind == "step":
        return {"bytes": 2 * qk + 2 * vo + 2 * gate + 2 * st, "flops": 7.0 * B * HV * Dk * Dv}
    given = 1 if case["h0"] else 0
    fwd = 2 * qk + 2 * vo + 2 * gate + st * (1 + given)
    flops = 7.0 * B * L * HV * Dk * Dv
    if kind == "prefill":
        return {"bytes": fwd, "flops": flops}
    bwd = 4 * qk + 3 * vo + 4 * gate + 2 * st * given
    return {"bytes": fwd + bwd, "flops": 3 * flops}


# ------------------------------------------------------------------ 64-bit reference

def _time_first64(t, r=1):
    """[B, L, heads, ...] -> [L, B * value heads, ...] in 64 bits."""
    t = t.double()
    if t.dim() == 3:
        t = t[..., None]
    t = t.repeat_interleave(r, 2).movedim(1, 0)
    return t.reshape(t.shape[0], -1, t.shape[-1]).contiguous()


def _delta64(s, train):
    """The recurrence one step after the other, and its adjoint step by step backwards."""
    B, L, H, Dk = s["q"].shape
    HV, Dv = s["v"].shape[2:]
    r, scale = HV // H, Dk ** -0.5
    q, k = _time_first64(s["q"], r), _time_first64(s["k"], r)
    v, b = _time_first64(s["v"]), _time_first64(s["beta"])
    a = torch.exp(_time_first64(s["g"]))[..., None]
    N = B * HV
    S = torch.zeros(N, Dk, Dv, dtype=torch.float64, device=q.device)
    if s["h0"] is not None:
        S += s["h0"].double().reshape(N, Dk, Dv)
    o, err = torch.empty_like(v), torch.empty_like(v)
    kept = torch.empty(L + 1, N, Dk, Dv, dtype=torch.float64, device=q.device) if train else None
    if train:
        kept[0] = S
    for t in range(L):
        S = a[t] * S
        err[t] = v[t] - (S * k[t].unsqueeze(-1)).sum(1)
        S = S + k[t].unsqueeze(-1) * (b[t] * err[t]).unsqueeze(1)
        o[t] = scale * (S * q[t].unsqueeze(-1)).sum(1)
        if train:
            kept[t + 1] = S

    def back(t, heads):  # [L, B * heads, d] -> [B, L, heads, d]
        return t.reshape(L, B, heads, -1).movedim(0, 1)

    out = {"o": back(o, HV), "hT": S.reshape(B, HV, Dk, Dv)}
    if not train:
        return out
    do = _time_first64(s["do"])
    dS = torch.zeros_like(S) if s["dhT"] is None else s["dhT"].double().reshape(N, Dk, Dv).clone()
    dq, dk, dv, dg, db = (torch.empty_like(x) for x in (q, k, v, a[..., 0], b))
    for t in range(L - 1, -1, -1):
        dS = dS + scale * q[t].unsqueeze(-1) * do[t].unsqueeze(1)
        dq[t] = scale * (kept[t + 1] * do[t].unsqueeze(1)).sum(-1)
        du = (dS * k[t].unsqueeze(-1)).sum(1)
        db[t] = (du * err[t]).sum(-1, keepdim=True)
        de = b[t] * du
        dv[t] = de
        before = a[t] * kept[t]
        dk[t] = (dS * (b[t] * err[t]).unsqueeze(1)).sum(-1) - (before * de.unsqueeze(1)).sum(-1)
        dS = dS - k[t].unsqueeze(-1) * de.unsqueeze(1)
        dg[t] = (dS * before).sum((1, 2)).unsqueeze(-1)
        dS = a[t] * dS
    shared = lambda x: back(x, HV).reshape(B, L, H, r, Dk).sum(3)  # noqa: E731
    out.update(dq=shared(dq), dk=shared(dk), dv=back(dv, HV), dg=back(dg, HV)[..., 0],
               dbeta=back(db, HV)[..., 0])
    if s["h0"] is not None:
        out["dh0"] = dS.reshape(B, HV, Dk, Dv)
    return out


def _adamw64(s):
    t = s["t"] + 1
    outs = {n: torch.zeros(s["params"].shape, dtype=torch.float64, device="cuda")
            for n in ("params", "m1", "m2")}
    outs["params"] += s["params"].double()
    if s["case"]["bits"] == 32:
        outs["m1"] += s["m1"]
        outs["m2"] += s["m2"]
    for i, (o, n) in enumerate(zip(s["starts"], s["sizes"])):
        p, g = s["p"][i].double(), s["g"][i].double()
        if s["case"]["bits"] == 32:
            m, v = s["m"][i].double(), s["v"][i].double()
        else:
            wide = lambda x: x.double().repeat_interleave(QBLOCK)[:n]  # noqa: E731,B023
            c1 = s["m"][i].double() / 127
            m = wide(s["ms"][i]) * c1 * c1.abs()
            v = wide(s["vs"][i]) * ((s["v"][i].double() + 1) / 256) ** 4
        m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
        step = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        outs["params"][o:o + n] = p - LR * (step + s["decay"][i] * p)
        if s["case"]["bits"] == 8:
            fill = -n % QBLOCK

            def scale(x):  # each block's largest, as it is kept: in 32 bits
                x = torch.nn.functional.pad(x.abs(), (0, fill)).reshape(-1, QBLOCK)  # noqa: B023
                return x.amax(1).float().double().repeat_interleave(QBLOCK)[:n]  # noqa: B023

            sm, sv = scale(m), scale(v)
            cm = torch.round(127 * torch.sqrt(m.abs() / sm)).clamp(max=127) / 127
            cv = (torch.round(256 * torch.sqrt(torch.sqrt(v / sv))).clamp(1, 256)) / 256
            m, v = torch.sign(m) * sm * cm ** 2, sv * cv ** 4
        outs["m1"][o:o + n], outs["m2"][o:o + n] = m, v
    return outs


def _sample64(s):
    """Row by row: items in falling order, each border found on the sorted weights."""
    x = s["logits"].double().cpu().numpy()
    B, V = x.shape
    u, temp, tp, mp = (s[n].double().cpu().numpy() for n in ("u", "temperature", "top_p", "min_p"))
    tk = s["top_k"].cpu().numpy()
    ids, prob = np.full(B, -1, np.int32), np.zeros(B)
    for r in range(B):
        best = x[r].max()
        if not np.isfinite(best):
            continue
        if temp[r] <= 0:
            ids[r], prob[r] = int(np.argmax(x[r])), 1.0
            continue
        w = np.exp((x[r] - best) / temp[r])
        order = np.argsort(-x[r], kind="stable")
        if tk[r] > 0:
            order = order[:tk[r]]
        run_sum = np.cumsum(w[order])
        if tp[r] < 1:
            order = order[:1 + int(np.searchsorted(run_sum, tp[r] * run_sum[-1]))]
        order = order[w[order] >= mp[r]]
        order = np.sort(order)
        run_sum = np.cumsum(w[order])
        at = order[min(int(np.searchsorted(run_sum, u[r] * run_sum[-1], side="right")),
                       len(order) - 1)]
        ids[r], prob[r] = at, w[at] / run_sum[-1]
    return {"ids": torch.from_numpy(ids), "prob": torch.from_numpy(prob)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "adamw":
        return _adamw64(s)
    if kind == "sample":
        return _sample64(s)
    if kind != "step":
        return _delta64(s, kind == "train")
    r = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[n].double().repeat_interleave(r, 1) for n in ("q", "k"))
    S = torch.exp(s["g"].double())[..., None, None] * s["h_prev"].double()
    err = s["v"].double() - torch.einsum("bhkv,bhk->bhv", S, k)
    S = S + torch.einsum("bhk,bhv->bhkv", k, s["beta"].double()[..., None] * err)
    return {"o": torch.einsum("bhkv,bhk->bhv", S, q) * q.shape[-1] ** -0.5, "h": S}
