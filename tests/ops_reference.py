"""64-bit references of the operators of recblr_ops.h, in plain numpy, from their definitions.

Shared by the CPU tests (which check the references against differences and closed cases) and
the GPU tests (which check the library against the references).
"""
import math

import numpy as np


# ------------------------------------------------------------------ gated delta rule

def delta(q, k, v, g, beta, h0=None, do=None, dhT=None, scale=None):
    """The recurrence one step after the other and, given do, its adjoint.

    q, k [B,L,H,Dk], v [B,L,HV,Dv], g, beta [B,L,HV], states [B,HV,Dk,Dv]."""
    q, k, v, g, beta = (np.asarray(t, dtype=np.float64) for t in (q, k, v, g, beta))
    B, L, H, Dk = q.shape
    HV, Dv = v.shape[2:]
    r = HV // H
    scale = Dk ** -0.5 if scale is None else scale
    qe, ke = np.repeat(q, r, axis=2), np.repeat(k, r, axis=2)
    a = np.exp(g)
    S = np.zeros((B, HV, Dk, Dv)) if h0 is None else np.array(h0, dtype=np.float64)
    kept, err, o = [S], np.zeros_like(v), np.zeros_like(v)
    for t in range(L):
        D = a[:, t, :, None, None] * S
        err[:, t] = v[:, t] - np.einsum("bhkv,bhk->bhv", D, ke[:, t])
        S = D + np.einsum("bhk,bhv->bhkv", ke[:, t], beta[:, t, :, None] * err[:, t])
        o[:, t] = scale * np.einsum("bhkv,bhk->bhv", S, qe[:, t])
        kept.append(S)
    out = {"o": o, "hT": S, "kept": kept}
    if do is None:
        return out
    do = np.asarray(do, dtype=np.float64)
    dS = np.zeros_like(S) if dhT is None else np.array(dhT, dtype=np.float64)
    dq, dk = np.zeros_like(qe), np.zeros_like(ke)
    dv, dg, db = np.zeros_like(v), np.zeros_like(g), np.zeros_like(beta)
    for t in range(L - 1, -1, -1):
        dq[:, t] = scale * np.einsum("bhkv,bhv->bhk", kept[t + 1], do[:, t])
        dS = dS + scale * np.einsum("bhk,bhv->bhkv", qe[:, t], do[:, t])
        du = np.einsum("bhkv,bhk->bhv", dS, ke[:, t])
        db[:, t] = (du * err[:, t]).sum(-1)
        dv[:, t] = beta[:, t, :, None] * du
        D = a[:, t, :, None, None] * kept[t]
        dk[:, t] = (np.einsum("bhkv,bhv->bhk", dS, beta[:, t, :, None] * err[:, t])
                    - np.einsum("bhkv,bhv->bhk", D, dv[:, t]))
        dD = dS - np.einsum("bhk,bhv->bhkv", ke[:, t], dv[:, t])
        dg[:, t] = (dD * D).sum((-2, -1))
        dS = a[:, t, :, None, None] * dD
    share = lambda x: x.reshape(B, L, H, r, Dk).sum(3)  # noqa: E731
    out.update(dq=share(dq), dk=share(dk), dv=dv, dg=dg, dbeta=db, dh0=dS)
    return out


# ------------------------------------------------------------------ AdamW

BLOCK = 256


def moment_values(m, v, s1, s2):
    """What 8-bit codes and scales stand for."""
    wide = lambda s, n: np.repeat(np.asarray(s, np.float64), BLOCK)[:n]  # noqa: E731
    x = np.asarray(m, np.float64) / 127
    y = (np.asarray(v, np.float64) + 1) / 256
    return wide(s1, len(x)) * x * np.abs(x), wide(s2, len(y)) * y ** 4


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, wd):
    """One step on values: (p, m, v) in 64 bits."""
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p * (1 - lr * wd) - lr * step, m, v


# ------------------------------------------------------------------ sampling

def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(ids, prob) row by row: items sorted, borders on exact sums (math.fsum)."""
    x = np.asarray(logits, dtype=np.float64)
    B, V = x.shape
    at = lambda t, r, d: d if t is None else float(np.asarray(t, np.float64)[r])  # noqa: E731
    ids, prob = np.full(B, -1, np.int32), np.zeros(B)
    for r in range(B):
        temp = at(temperature, r, 1.0)
        if V == 0 or math.isnan(temp) or np.isnan(x[r]).any() or not np.isfinite(x[r].max()):
            continue
        best = x[r].max()
        if temp <= 0:
            ids[r], prob[r] = int(np.argmax(x[r])), 1.0
            continue
        w = np.where(x[r] == -np.inf, 0.0, np.exp((x[r] - best) / temp))
        # weights are multiples of 2^-F, as recblr_ops.h has it
        one = 2.0 ** min(51, 62 - math.ceil(math.log2(V)))
        whole, w = w, np.rint(w * one) / one
        order = np.argsort(-x[r], kind="stable")
        k, p = int(at(top_k, r, 0)), at(top_p, r, 1.0)
        if k > 0:
            order = order[:k]
        if p < 1:
            want, n = p * math.fsum(w[order]), 1
            while n < len(order) and math.fsum(w[order[:n]]) < want:
                n += 1
            order = order[:n]
        order = np.sort(order[w[order] >= min(at(min_p, r, 0.0), 1.0)])
        order = order[w[order] > 0]
        total = math.fsum(w[order])
        target = at(u, r, 0.0) * total
        pick = order[-1]
        sums = np.cumsum(w[order])
        over = np.nonzero(sums > target)[0]
        if len(over):
            pick = order[over[0]]
        ids[r], prob[r] = pick, whole[pick] / total
    return ids, prob
