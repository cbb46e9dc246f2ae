"""The item lookup, the norms of queries and keys, the policy loss and Muon without a GPU: their
refusals, and the references of their GPU tests.

Pointers are fake addresses: every call is refused by host-side validation (or has nothing to
do), so no HIP call is made.
"""
import math
import os
import re

import numpy as np
import pytest

import train_ops_reference as ref
from paper_2406_12580_amd import build as hipbuild
from test_wave_order import _assembly, _lds_runs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000000


def addr(k):
    return A + k * (64 << 20)


@pytest.fixture(scope="module")
def rb():
    from paper_2406_12580_amd import recblr
    return recblr


def test_header_constants(rb):
    text = open(os.path.join(ROOT, "include", "recblr_ops.h")).read()
    val = lambda n: int(re.search(n + r" = (\d+)", text).group(1))  # noqa: E731
    assert val("RECBLR_NORM_L2") == rb.NORM_L2 and val("RECBLR_NORM_RMS") == rb.NORM_RMS


# ------------------------------------------------------------------ item lookup

def lookup(rb, **kw):
    a = dict(table=addr(0), ids=addr(1), out=addr(2), N=10, V=7, D=4, scale=1.0, pad=-1, io=0)
    a.update(kw)
    return rb.recblr_embed_forward(*a.values(), None)


def gradient(rb, **kw):
    a = dict(ids=addr(1), dout=addr(0), dtable=addr(2), N=10, V=7, D=4, scale=1.0, pad=-1, add=0,
             io=0, ws=None, nws=0)
    a.update(kw)
    return rb.recblr_embed_backward(*a.values(), None)


@pytest.mark.parametrize("call", [lookup, gradient])
def test_embed_refuses(rb, call):
    bad = rb.ERR_INVALID_ARGUMENT
    assert call(rb, N=-1) == bad and call(rb, V=-1) == bad and call(rb, D=0) == bad
    assert call(rb, io=2) == rb.ERR_UNSUPPORTED
    assert call(rb, D=4097) == rb.ERR_UNSUPPORTED
    assert call(rb, V=(1 << 31) - 1) == rb.ERR_UNSUPPORTED
    assert call(rb, N=(1 << 28) + 1) == rb.ERR_UNSUPPORTED
    assert call(rb, N=1 << 27, D=128) == rb.ERR_UNSUPPORTED          # 2^34 elements
    assert call(rb, V=(1 << 31) - 2, D=1024) == rb.ERR_UNSUPPORTED
    third = "table" if call is lookup else "dout"
    last = "out" if call is lookup else "dtable"
    for name in ("ids", third, last):
        assert call(rb, **{name: None}) == bad, name
        assert call(rb, **{name: addr(9) + 2}) == bad, name
    assert call(rb, **{last: addr(0) + 8}) == bad                    # over the other tensor
    assert call(rb, **{last: addr(1)}) == bad                        # over the ids


def test_embed_nothing_to_do(rb):
    assert lookup(rb, N=0, table=None, ids=None, out=None) == rb.OK
    assert gradient(rb, V=0, dtable=None) == rb.OK
    assert gradient(rb, N=0, add=1, ids=None, dout=None) == rb.OK


def test_embed_workspace(rb):
    size = rb.recblr_embed_workspace_size
    assert size(4096, 5000, 64, 0) == 0 and size(4097, 5000, 64, 0) > 0
    for bad in ((-1, 10, 4, 0), (5000, 10, 0, 0), (5000, 10, 4, 3), (1 << 29, 10, 4, 0)):
        assert size(*bad) == 0
    n = size(5000, 100, 4, 0)
    assert gradient(rb, N=5000, V=100) == rb.ERR_WORKSPACE
    assert gradient(rb, N=5000, V=100, ws=addr(5), nws=n - 1) == rb.ERR_WORKSPACE
    assert gradient(rb, N=5000, V=100, ws=addr(5) + 128, nws=n) == rb.ERR_WORKSPACE
    assert gradient(rb, N=5000, V=100, ws=addr(2), nws=n) == rb.ERR_INVALID_ARGUMENT


# ------------------------------------------------------------------ norms of queries and keys

QK = dict(q=addr(0), k=addr(1), q_pitch=16, k_pitch=8, wq=None, wk=None, positions=addr(2))
QK_SIZES = dict(N=5, H=2, HK=1, D=8, rotate=8, base=10000.0, norm=0, eps=1e-6, io=0)


def norm(rb, **kw):
    a = dict(**QK, q_out=addr(3), k_out=addr(4), **QK_SIZES)
    a.update(kw)
    return rb.recblr_qk_norm_forward(*a.values(), None)


def norm_back(rb, **kw):
    a = dict(**QK, dq_out=addr(3), dk_out=addr(4), dq=addr(5), dk=addr(6), dwq=None, dwk=None,
             **QK_SIZES, ws=None, nws=0)
    a.update(kw)
    return rb.recblr_qk_norm_backward(*a.values(), None)


@pytest.mark.parametrize("call", [norm, norm_back])
def test_qk_norm_refuses(rb, call):
    bad = rb.ERR_INVALID_ARGUMENT
    assert call(rb, N=-1) == bad and call(rb, H=0) == bad and call(rb, HK=0) == bad
    assert call(rb, D=0, rotate=0) == bad
    assert call(rb, io=2) == rb.ERR_UNSUPPORTED
    assert call(rb, D=257, q_pitch=1000, k_pitch=1000) == rb.ERR_UNSUPPORTED
    assert call(rb, H=4097, q_pitch=1 << 20) == rb.ERR_UNSUPPORTED
    assert call(rb, N=(1 << 31) - 256) == rb.ERR_UNSUPPORTED
    assert call(rb, q_pitch=1 << 31) == rb.ERR_UNSUPPORTED
    assert call(rb, q_pitch=15) == bad and call(rb, k_pitch=7) == bad
    assert call(rb, rotate=10) == bad and call(rb, rotate=3) == bad and call(rb, rotate=-2) == bad
    assert call(rb, norm=2) == bad
    for x in (0.0, -1.0, math.nan):
        assert call(rb, eps=x) == bad and call(rb, base=x) == bad
    for name in ("q", "k", "positions"):
        assert call(rb, **{name: None}) == bad, name
    for name in ("q", "k", "positions", "wq", "wk"):
        assert call(rb, **{name: addr(20) + 2}) == bad, name
    assert call(rb, N=0, q=None, k=None) == rb.OK


def test_qk_norm_refuses_outputs(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    for name in ("q_out", "k_out"):
        assert norm(rb, **{name: None}) == bad and norm(rb, **{name: addr(9) + 2}) == bad
    for name in ("dq_out", "dk_out", "dq", "dk"):
        assert norm_back(rb, **{name: None}) == bad, name
        assert norm_back(rb, **{name: addr(9) + 2}) == bad, name
    assert norm(rb, q_out=addr(0)) == bad and norm(rb, k_out=addr(3) + 4) == bad
    assert norm(rb, q_out=addr(0) + 16 * 4 * 5 - 4) == bad           # the last element of q
    assert norm(rb, q_out=addr(0) + 16 * 4 * 5 - 4, q_pitch=32) == bad  # between two tokens
    assert norm_back(rb, dq=addr(3)) == bad and norm_back(rb, dk=addr(5)) == bad
    # weights and their gradients come together, and these need workspace
    assert norm_back(rb, dwq=addr(7)) == bad and norm_back(rb, wk=addr(7)) == bad
    assert norm_back(rb, wq=addr(7), dwq=addr(8)) == rb.ERR_WORKSPACE
    n = rb.recblr_qk_norm_workspace_size(5, 2, 1, 8, 0)
    assert n > 0
    assert norm_back(rb, wq=addr(7), dwq=addr(7), ws=addr(9), nws=n) == bad
    assert norm_back(rb, wq=addr(7), dwq=addr(8), ws=addr(5), nws=n) == bad
    assert norm_back(rb, wq=addr(7), dwq=addr(8), ws=addr(9), nws=n - 1) == rb.ERR_WORKSPACE
    assert rb.recblr_qk_norm_workspace_size(5, 2, 1, 300, 0) == 0


# ------------------------------------------------------------------ policy loss

def policy(rb, **kw):
    a = dict(logits=addr(0), ids=addr(1), old=addr(2), adv=addr(3), ref=addr(4), weight=None,
             loss=addr(5), logp=addr(6), dlogits=addr(7), N=2, V=10, temperature=1.0, lo=0.2,
             hi=0.2, kl=0.1, io=0, ws=addr(8), nws=1 << 20)
    a.update(kw)
    return rb.recblr_policy_loss(*a.values(), None)


def test_policy_refuses(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    assert policy(rb, N=-1) == bad and policy(rb, V=-1) == bad and policy(rb, V=0) == bad
    assert policy(rb, io=2) == rb.ERR_UNSUPPORTED
    assert policy(rb, V=(1 << 24) + 1) == rb.ERR_UNSUPPORTED
    assert policy(rb, N=1 << 22) == rb.ERR_UNSUPPORTED
    assert policy(rb, N=1 << 20, V=1 << 16) == rb.ERR_UNSUPPORTED
    for x in (0.0, -1.0, math.nan, math.inf, 1e-31):
        assert policy(rb, temperature=x) == bad, x
    for name in ("lo", "hi", "kl"):
        for x in (-0.1, math.nan, math.inf):
            assert policy(rb, **{name: x}) == bad, (name, x)
    for name in ("logits", "ids", "old", "adv", "ref", "loss"):
        assert policy(rb, **{name: None}) == bad, name
    for name in ("logits", "ids", "old", "adv", "ref", "weight", "loss", "logp", "dlogits"):
        assert policy(rb, **{name: addr(20) + 2}) == bad, name
    assert policy(rb, dlogits=addr(0) + 4) == bad                    # partly over the logits
    assert policy(rb, logp=addr(2)) == bad and policy(rb, loss=addr(0)) == bad
    assert policy(rb, loss=addr(6) + 4) == bad and policy(rb, dlogits=addr(1)) == bad
    need = rb.recblr_policy_loss_workspace_size(2, 10, 0)
    assert need > 0
    assert policy(rb, ws=None) == policy(rb, nws=need - 1) == rb.ERR_WORKSPACE
    assert policy(rb, ws=addr(8) + 64) == rb.ERR_WORKSPACE
    assert policy(rb, ws=addr(7)) == bad
    for bad_size in ((-1, 10, 0), (2, 0, 0), (2, 10, 5)):
        assert rb.recblr_policy_loss_workspace_size(*bad_size) == 0


# ------------------------------------------------------------------ Muon

def matrices(rb, r, c, count=2, **kw):
    t = (rb.MuonTensor * count)()
    for i in range(count):
        t[i].param, t[i].grad, t[i].m = addr(3 * i), addr(3 * i + 1), addr(3 * i + 2)
        t[i].rows, t[i].cols, t[i].scale = r, c, 1.0
    for name, value in kw.items():
        setattr(t[count - 1], name, value)
    return t


def update(rb, t, count=None, io=0, momentum=0.9, steps=5, eps=1e-7, ws=addr(900), nws=1 << 40):
    return rb.recblr_muon_update(t, len(t) if count is None else count, io, 0.1, momentum, 1,
                                 steps, eps, ws, nws, None)


def test_muon_refuses(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    ok = matrices(rb, 8, 8)
    assert update(rb, ok, io=3) == rb.ERR_UNSUPPORTED
    assert update(rb, ok, count=-1) == bad and update(rb, None, count=1) == bad
    for x in (-0.1, 1.0, math.nan):
        assert update(rb, ok, momentum=x) == bad
    for x in (0.0, -1.0, math.nan):
        assert update(rb, ok, eps=x) == bad
    assert update(rb, ok, steps=0) == bad and update(rb, ok, steps=65) == rb.ERR_UNSUPPORTED
    assert update(rb, matrices(rb, 8, 8, rows=-1)) == bad
    assert update(rb, matrices(rb, 8, 8, cols=(1 << 16) + 1)) == rb.ERR_UNSUPPORTED
    assert update(rb, matrices(rb, 1 << 16, 1 << 16)) == rb.ERR_UNSUPPORTED
    for name in ("param", "grad", "m"):
        assert update(rb, matrices(rb, 8, 8, **{name: None})) == bad, name
        assert update(rb, matrices(rb, 8, 8, **{name: addr(40) + 2})) == bad, name
    assert update(rb, matrices(rb, 8, 8, param=addr(0))) == bad       # the same matrix twice
    assert update(rb, matrices(rb, 8, 8, param=addr(0) + 252)) == bad  # its last element
    assert update(rb, matrices(rb, 8, 8, m=addr(1))) == bad           # momentum over a gradient
    assert update(rb, matrices(rb, 8, 8, count=200, param=addr(3 * 77))) == bad
    assert update(rb, None, count=0) == rb.OK


def test_muon_workspace(rb):
    size = rb.recblr_muon_workspace_size
    assert size(matrices(rb, 128, 128), 2, 0) == 0 == size(matrices(rb, 64, 256), 2, 1)
    assert size(matrices(rb, 0, 5000), 2, 0) == 0
    big = matrices(rb, 300, 500)
    need = size(big, 2, 0)
    assert need > 0 and size(big, 1, 0) < need
    assert size(big, 2, 7) == 0 and size(big, -1, 0) == 0
    assert update(rb, big, ws=None) == rb.ERR_WORKSPACE
    assert update(rb, big, nws=need - 1) == rb.ERR_WORKSPACE
    assert update(rb, big, ws=addr(900) + 8) == rb.ERR_WORKSPACE
    assert update(rb, big, ws=addr(3), nws=need) == rb.ERR_INVALID_ARGUMENT


# ------------------------------------------------------------------ the binding

def test_binding_refuses(rb):
    import torch
    z = torch.zeros
    i = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="on the GPU"):
        rb.embed(z(4, 8), i(3))
    with pytest.raises(ValueError, match="on the GPU"):
        rb.embed_backward(i(3), z(3, 8), 4)
    with pytest.raises(ValueError, match="on the GPU"):
        rb.qk_norm(z(1, 2, 1, 4), z(1, 2, 1, 4))
    with pytest.raises(ValueError, match="on the GPU"):
        rb.qk_norm_backward(z(1, 2, 1, 4), z(1, 2, 1, 4), z(1, 2, 1, 4), z(1, 2, 1, 4))
    with pytest.raises(ValueError, match="on the GPU"):
        rb.policy_loss(z(2, 5), i(2), z(2), z(2))
    with pytest.raises(ValueError, match="on the GPU"):
        rb.Muon([z(4, 4)])
    with pytest.raises(ValueError):
        rb.Muon([])


# ------------------------------------------------------------------ the references

def central(f, x, at, h):
    x = x.copy().reshape(-1)
    x[at] += h
    up = f(x)
    x[at] -= 2 * h
    return (up - f(x)) / (2 * h)


def test_embed_reference():
    table = np.arange(12.0).reshape(4, 3)
    ids = np.array([[1, 0, 9], [3, 1, -5]])
    out = ref.embed(table, ids, 2.0, pad_id=0)
    assert np.array_equal(out[0, 0], [6, 8, 10]) and np.array_equal(out[0, 1], [0, 0, 0])
    assert np.isnan(out[0, 2]).all() and np.isnan(out[1, 2]).all()
    r = np.random.default_rng(0)
    w = r.normal(size=(2, 3, 3))
    ok = np.array([[1, 0, 2], [3, 1, 1]])
    f = lambda t: (ref.embed(t.reshape(4, 3), ok, 2.0, pad_id=0) * w).sum()  # noqa: E731
    d, size = ref.embed_backward(ok, w, 4, 2.0, pad_id=0)
    for at in range(12):  # linear: differences are exact but for rounding
        assert abs(central(f, table, at, 0.5) - d.reshape(-1)[at]) < 1e-12
    assert (size >= np.abs(d) - 1e-15).all() and not d[0].any()


@pytest.mark.parametrize("norm", ["rms", "l2"])
@pytest.mark.parametrize("rotate", [0, 4, 6])
def test_qk_norm_reference_gradients_by_differences(norm, rotate):
    """Central differences: error O(h^2) ~ 1e-9, cancellation 1e-16 / h ~ 1e-11."""
    r = np.random.default_rng(1)
    x, dy, w = r.normal(size=(2, 3, 2, 6)), r.normal(size=(2, 3, 2, 6)), r.normal(size=6)
    pos = r.integers(0, 50, (2, 3))
    f = lambda x_, w_: (ref.qk_norm(x_.reshape(x.shape), w_, pos, rotate, norm=norm)["y"]  # noqa: E731
                        * dy).sum()
    out = ref.qk_norm(x, w, pos, rotate, norm=norm, dy=dy)
    for at in range(0, x.size, 5):
        got = central(lambda t: f(t, w), x, at, 1e-5)
        assert abs(got - out["dx"].reshape(-1)[at]) < 1e-7
    for at in range(6):
        assert abs(central(lambda t: f(x, t), w, at, 1e-5) - out["dw"][at]) < 1e-7


def test_qk_norm_reference_closed_cases():
    """Lengths of one; a quarter turn; the products of turned vectors hang on the distance of
    their positions alone."""
    r = np.random.default_rng(2)
    x = r.normal(size=(1, 5, 1, 8))
    y = ref.qk_norm(x, None, np.arange(5)[None], 8, norm="l2", eps=1e-30)["y"]
    assert np.allclose((y * y).sum(-1), 1.0)
    one = np.zeros((1, 1, 1, 2))
    one[..., 0] = 1.0
    y = ref.turn(one, np.array([[1]]), 2, 1.0)
    assert np.allclose(y.reshape(-1), [math.cos(1.0), math.sin(1.0)])
    a, b = r.normal(size=(1, 1, 1, 8)), r.normal(size=(1, 1, 1, 8))
    dot = lambda p, q: (ref.turn(a, np.array([[p]]), 8, 100.0)  # noqa: E731
                        * ref.turn(b, np.array([[q]]), 8, 100.0)).sum()
    assert abs(dot(3, 10) - dot(1003, 1010)) < 1e-9


def policy_case(N=6, V=7, seed=3):
    r = np.random.default_rng(seed)
    c = dict(logits=r.normal(size=(N, V)) * 2, ids=r.integers(0, V, N),
             old_logp=-1.9 + 0.5 * r.normal(size=N), advantage=r.normal(size=N),
             ref_logp=-1.9 + 0.5 * r.normal(size=N), weight=r.random(N) + 0.1)
    c["ids"][1] = -1
    return c


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_reference_gradients_by_differences(kl):
    """As above, times the gradient's size (the third derivative of e^d is d's own slope again, and
    a row's d is up to six here); no ratio of these rows lies within h of a border."""
    c = policy_case()
    how = dict(temperature=0.7, clip_low=0.1, clip_high=0.3, kl=kl)
    out = ref.policy(**c, **how)
    assert out["logp"][1] == 0 and not out["dlogits"][1].any()
    f = lambda x: ref.policy(**{**c, "logits": x.reshape(c["logits"].shape)}, **how)["loss"]  # noqa: E731
    for at in range(c["logits"].size):
        got = central(f, c["logits"], at, 1e-5)
        assert abs(got - out["dlogits"].reshape(-1)[at]) < 1e-7 * (1 + np.abs(out["dlogits"]).max())


def test_policy_reference_closed_cases():
    """Two items of equal odds; a ratio of one leaves the plain gradient of -A logp; clipped rows
    have none; at the reference's own odds the KL term and its gradient are zero."""
    x, half = np.zeros((1, 2)), np.log(0.5)
    out = ref.policy(x, [0], [half], [2.0])
    assert np.isclose(out["loss"], -2.0) and np.allclose(out["dlogits"], [[-1.0, 1.0]])
    out = ref.policy(x, [0], [half - 1.0], [2.0])
    assert np.isclose(out["loss"], -2.4) and not out["dlogits"].any()
    out = ref.policy(x, [0], [half + 1.0], [-2.0])
    assert np.isclose(out["loss"], 1.6) and not out["dlogits"].any()
    out = ref.policy(x, [0], [half], [0.0], ref_logp=[half], kl=1.0)
    assert out["loss"] == 0.0 and not out["dlogits"].any()
    out = ref.policy(x, [0], [half], [0.0], ref_logp=[half + 1.0], kl=1.0)
    assert np.isclose(out["loss"], math.e - 2.0)


def test_muon_reference():
    """The products act on the singular values alone: U p(S) V^T; a matrix and its transposed
    alike; one step by hand."""
    r = np.random.default_rng(4)
    x = r.normal(size=(4, 7))
    x /= np.linalg.norm(x)
    u, s, vt = np.linalg.svd(x, full_matrices=False)
    a, b, c = ref.NS
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    y, norms = ref.newton_schulz(x, 5)
    assert np.allclose(y, u * s @ vt) and np.isclose(norms[0], 1.0) and len(norms) == 6
    assert np.allclose(ref.newton_schulz(x.T, 5)[0], y.T)
    p, m, x, _ = ref.muon([[2.0]], [[3.0]], [[1.0]], 0.1, 0.5, False, 0.2, 1.0, steps=1, eps=0.0)
    assert np.isclose(m[0, 0], 2.0) and np.isclose(x[0, 0], a + b + c)
    assert np.isclose(p[0, 0], 2.0 * 0.98 - 0.1 * (a + b + c))


def test_singular_values_stay_where_the_planes_hold_them():
    """The polynomial keeps [0, 1.21] in itself, and b s^2 + c s^4 there stays within 3: what the
    kernels scale by 2^12 for fp16 rests on it."""
    a, b, c = ref.NS
    s = np.linspace(0.0, 1.21, 200001)
    f = a * s + b * s ** 3 + c * s ** 5
    assert f.min() >= 0.0 and f.max() <= 1.21
    assert np.abs(b * s ** 2 + c * s ** 4).max() < 3.0


# ------------------------------------------------------------------ hand-overs within a wave

def test_embed_hand_overs(tmp_path):
    """In the compiled kernels: the positions that a wave has found are read behind a fence; a
    digit's next place is read, fenced, written by the last lane that has it, and fenced before
    the next positions' lanes read it."""
    source = os.path.join(hipbuild.CSRC, "embed.hip")
    lines = _assembly(tmp_path, source)
    for kernel in ("few_kernelIfLi1", "few_kernelINS_4bf16ELi4"):
        ops = _lds_runs(lines, kernel)
        print(kernel, ops)
        assert ops.count("F") == 1 and "WFWR" in ops, ops  # found, fence, the heavy ones, found
    for kernel in ("place_kernelILi6", "place_kernelILi9", "place_kernelILi12"):
        ops = _lds_runs(lines, kernel)
        print(kernel, ops)
        steps = ops[ops.rindex("B") + 1:].strip("F") + "F"
        assert len(steps) >= 16 and steps == "RFWF" * (len(steps) // 4), ops
