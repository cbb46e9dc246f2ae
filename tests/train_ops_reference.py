"""64-bit references of the item lookup, the norms of queries and keys, the policy loss and Muon,
in plain numpy, from their definitions (recblr_ops.h).

Shared by the CPU tests (which check the references against differences and closed cases) and
the GPU tests (which check the library against the references).
"""
import numpy as np


# ------------------------------------------------------------------ item lookup

def embed(table, ids, scale=1.0, pad_id=-1):
    table = np.asarray(table, np.float64)
    V, D = table.shape
    out = np.full((*ids.shape, D), np.nan)
    for at in np.ndindex(*ids.shape):
        i = int(ids[at])
        if i == pad_id:
            out[at] = 0.0
        elif 0 <= i < V:
            out[at] = scale * table[i]
    return out


def embed_backward(ids, dout, V, scale=1.0, pad_id=-1, into=None):
    """(gradient, the sum of the sizes of what it is a sum of)."""
    dout = np.asarray(dout, np.float64)
    D = dout.shape[-1]
    ids = np.asarray(ids).reshape(-1)
    rows = dout.reshape(-1, D)
    keep = (ids != pad_id) & (ids >= 0) & (ids < V)
    d, size = np.zeros((V, D)), np.zeros((V, D))
    np.add.at(d, ids[keep], scale * rows[keep])
    np.add.at(size, ids[keep], np.abs(scale * rows[keep]))
    if into is not None:
        d, size = d + into, size + np.abs(into)
    return d, size


# ------------------------------------------------------------------ norms of queries and keys

def _angles(positions, D, rotate, base):
    rate = np.asarray(base, np.float64) ** (-2.0 * np.arange(rotate // 2) / max(rotate, 1))
    return np.asarray(positions, np.float64)[..., None, None] * rate


def turn(x, positions, rotate, base, back=False):
    """x [..., heads, D] with its first `rotate` elements turned."""
    if rotate == 0:
        return x.copy()
    h = rotate // 2
    t = _angles(positions, x.shape[-1], rotate, base) * (-1.0 if back else 1.0)
    out = x.copy()
    out[..., :h] = x[..., :h] * np.cos(t) - x[..., h:rotate] * np.sin(t)
    out[..., h:rotate] = x[..., h:rotate] * np.cos(t) + x[..., :h] * np.sin(t)
    return out


def amplitude(x, rotate):
    """Of each element, the size of the pair that it is turned with (its own where it is not)."""
    out = np.abs(x)
    h = rotate // 2
    if h:
        both = np.hypot(x[..., :h], x[..., h:rotate])
        out[..., :h], out[..., h:rotate] = both, both
    return out


def qk_norm(x, w, positions, rotate, base=10000.0, norm="rms", eps=1e-6, dy=None):
    """Of queries or keys x [..., heads, D]: dict with y and, given dy, dx and dw, and what their
    errors are measured by (r, u, the amplitudes of w g, and dw's terms' sizes)."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    w = np.ones(D) if w is None else np.asarray(w, np.float64)
    s = 1.0 / D if norm == "rms" else 1.0
    r = 1.0 / np.sqrt(s * (x * x).sum(-1, keepdims=True) + eps)
    u = x * r
    out = {"y": turn(w * u, positions, rotate, base), "r": r, "u": u, "s": s}
    if dy is None:
        return out
    dy = np.asarray(dy, np.float64)
    g = turn(dy, positions, rotate, base, back=True)
    a = w * g
    out["dx"] = r * (a - s * u * (u * a).sum(-1, keepdims=True))
    lead = tuple(range(x.ndim - 1))
    out["dw"] = (g * u).sum(lead)
    amp = amplitude(g, rotate)
    out["a_size"] = np.abs(w) * amp
    out["dw_size"] = (amp * np.abs(u)).sum(lead)
    return out


# ------------------------------------------------------------------ policy loss

def policy(logits, ids, old_logp, advantage, ref_logp=None, weight=None, temperature=1.0,
           clip_low=0.2, clip_high=0.2, kl=0.0):
    """dict of loss, logp, dlogits, row losses and the rows' derivatives c by logp."""
    x = np.asarray(logits, np.float64)
    N, V = x.shape
    loss, logp, grad = np.zeros(N), np.zeros(N), np.zeros((N, V))
    cs, xa = np.zeros(N), np.zeros(N)
    lo, hi = 1.0 - float(np.float32(clip_low)), 1.0 + float(np.float32(clip_high))
    T = float(np.float32(temperature))
    for n in range(N):
        i = int(ids[n])
        if i < 0:
            continue
        if i >= V:
            loss[n] = logp[n] = np.nan
            grad[n] = np.nan
            continue
        with np.errstate(all="ignore"):
            z = (x[n] - x[n].max()) / T
            e = np.exp(z)
            p = e / e.sum()
            lp = z[i] - np.log(e.sum())
            A, w = float(advantage[n]), 1.0 if weight is None else float(weight[n])
            r = np.exp(lp - float(old_logp[n]))
            inside = not r > hi if A >= 0 else not r < lo
            gain = r * A if inside else (hi if A >= 0 else lo) * A
            c = -gain if inside else 0.0
            row = -gain
            if kl > 0:
                d = float(ref_logp[n]) - lp
                row += kl * (np.expm1(d) - d)
                c -= kl * np.expm1(d)
        loss[n], logp[n], cs[n], xa[n] = w * row, lp, w * c, z[i]
        grad[n] = -w * c / T * p
        grad[n, i] += w * c / T
    return {"loss": loss.sum(), "rows": loss, "logp": logp, "dlogits": grad, "c": cs, "xa": xa}


# ------------------------------------------------------------------ Muon

NS = (3.4445, -4.7750, 2.0315)


def newton_schulz(x, steps):
    """(the result, the norms of the iterates, the first of them x's)."""
    a, b, c = NS
    x = np.asarray(x, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    norms = [np.linalg.norm(x)]
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
        norms.append(np.linalg.norm(x))
    return (x.T if tall else x), norms


def muon(p, g, m, lr, momentum, nesterov, wd, scale, steps=5, eps=1e-7):
    """(p, m, the orthogonalised update, its iterates' norms) of one matrix."""
    p, g, m = (np.asarray(t, np.float64) for t in (p, g, m))
    m = momentum * m + (1 - momentum) * g
    u = momentum * m + (1 - momentum) * g if nesterov else m
    x, norms = newton_schulz(u / (np.linalg.norm(u) + eps), steps)
    return p * (1 - lr * wd) - lr * scale * x, m, x, norms
