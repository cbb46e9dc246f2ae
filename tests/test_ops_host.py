"""recblr_ops.h without a GPU: its symbols, its refusals, and the references of its GPU tests.

Pointers are fake addresses: every call is refused by host-side validation (or has nothing to
do), so no HIP call is made.
"""
import ctypes
import math
import os
import re

import numpy as np
import pytest

import ops_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "recblr_ops.h")
A = 0x10000000


def addr(k):
    return A + k * (64 << 20)


@pytest.fixture(scope="module")
def rb():
    from paper_2406_12580_amd import recblr
    return recblr


def test_header_and_library_agree(rb):
    text = open(HEADER).read()
    syms = set(re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?(recblr_\w+)\(", text, re.M))
    assert syms == set(rb.OPS_EXPORTS) == set(rb._OPS_SIGS)
    lib = ctypes.CDLL(rb.LIB_PATH)
    assert all(hasattr(lib, s) for s in syms)


def test_header_constants(rb):
    text = open(HEADER).read()
    val = lambda n: int(re.search(n + r" = (\d+)", text).group(1))  # noqa: E731
    assert val("RECBLR_ADAMW_BLOCK") == rb.ADAMW_BLOCK == ref.BLOCK
    assert val("RECBLR_DELTA_CHUNK") == rb.DELTA_CHUNK
    assert val("RECBLR_OP_DELTA_FORWARD") == rb.OP_DELTA_FORWARD
    assert val("RECBLR_OP_DELTA_BACKWARD") == rb.OP_DELTA_BACKWARD


# ------------------------------------------------------------------ gated delta rule

SIZES = dict(B=2, L=3, H=2, HV=4, Dk=8, Dv=8, scale=1.0, io=0, ws=None, nws=0)


def fwd(rb, **kw):
    a = dict(q=addr(0), k=addr(1), v=addr(2), g=addr(3), beta=addr(4), h0=None, o=addr(5),
             hT=addr(6), states=None, **SIZES)
    a.update(kw)
    return rb.recblr_delta_forward(*[a[n] for n in (
        "q", "k", "v", "g", "beta", "h0", "o", "hT", "states", "B", "L", "H", "HV", "Dk", "Dv",
        "scale", "io", "ws", "nws")], None)


def bwd(rb, **kw):
    a = dict(q=addr(0), k=addr(1), v=addr(2), g=addr(3), beta=addr(4), states=addr(5),
             d_o=addr(6), dhT=None, dq=addr(7), dk=addr(8), dv=addr(9), dg=addr(10),
             dbeta=addr(11), dh0=None, **{**SIZES, "ws": addr(12), "nws": 1 << 24})
    a.update(kw)
    return rb.recblr_delta_backward(*[a[n] for n in (
        "q", "k", "v", "g", "beta", "states", "d_o", "dhT", "dq", "dk", "dv", "dg", "dbeta",
        "dh0", "B", "L", "H", "HV", "Dk", "Dv", "scale", "io", "ws", "nws")], None)


def step(rb, **kw):
    a = dict(q=addr(0), k=addr(1), v=addr(2), g=addr(3), beta=addr(4), h_prev=addr(5), o=addr(6),
             h_next=addr(7), **SIZES)
    a.update(kw)
    return rb.recblr_delta_step(*[a[n] for n in (
        "q", "k", "v", "g", "beta", "h_prev", "o", "h_next", "B", "H", "HV", "Dk", "Dv", "scale",
        "io")], None)


@pytest.mark.parametrize("call", [fwd, bwd, step])
def test_delta_refuses_sizes(rb, call):
    assert call(rb, B=-1) == rb.ERR_INVALID_ARGUMENT
    assert call(rb, H=0) == rb.ERR_INVALID_ARGUMENT
    assert call(rb, HV=3) == rb.ERR_INVALID_ARGUMENT                 # not a multiple of H
    assert call(rb, Dk=0) == rb.ERR_INVALID_ARGUMENT
    assert call(rb, Dk=129) == rb.ERR_UNSUPPORTED
    assert call(rb, Dv=129) == rb.ERR_UNSUPPORTED
    assert call(rb, io=2) == rb.ERR_UNSUPPORTED
    assert call(rb, H=4098, HV=4098) == rb.ERR_UNSUPPORTED
    assert call(rb, B=1 << 24) == rb.ERR_UNSUPPORTED
    assert call(rb, B=0) == rb.OK                                    # nothing to do


def test_delta_refuses_lengths(rb):
    for call in (fwd, bwd):
        assert call(rb, L=-1) == rb.ERR_INVALID_ARGUMENT
        assert call(rb, L=1 << 31) == rb.ERR_UNSUPPORTED
        # more chunks of all heads than workgroups
        assert call(rb, B=1 << 20, L=1 << 20) == rb.ERR_UNSUPPORTED
        assert call(rb, B=1 << 12, H=1, HV=1, L=64 << 12) == rb.ERR_UNSUPPORTED
        # more strips of all heads
        assert call(rb, B=1 << 21, H=2, HV=2, L=1, Dv=128) == rb.ERR_UNSUPPORTED


def test_delta_refuses_pointers(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    for name in ("q", "k", "v", "g", "beta", "o"):
        assert fwd(rb, **{name: None}) == bad, name
        assert fwd(rb, **{name: addr(20) + 2}) == bad, name
        assert step(rb, **{name: None}) == bad, name
    for name in ("h0", "hT", "states"):
        assert fwd(rb, **{name: addr(20) + 2}) == bad, name
    for name in ("h_prev", "h_next"):
        assert step(rb, **{name: None}) == bad and step(rb, **{name: addr(20) + 2}) == bad
    for name in ("q", "k", "v", "g", "beta", "states", "d_o", "dq", "dk", "dv", "dg", "dbeta"):
        assert bwd(rb, **{name: None}) == bad, name
        assert bwd(rb, **{name: addr(20) + 2}) == bad, name


def test_delta_refuses_overlap(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    assert fwd(rb, o=addr(2)) == bad
    assert fwd(rb, hT=addr(5) + 4) == bad
    assert fwd(rb, h0=addr(6)) == bad                                # hT over h0
    assert fwd(rb, states=addr(6)) == bad
    assert bwd(rb, dq=addr(8)) == bad                                # dq over dk
    assert bwd(rb, dv=addr(6)) == bad                                # dv over do
    assert bwd(rb, dh0=addr(5)) == bad                               # dh0 over states
    assert bwd(rb, ws=addr(0)) == bad                                # workspace over q
    assert step(rb, h_next=addr(5) + 4) == bad                       # partly over h_prev
    assert step(rb, o=addr(5)) == bad


def test_delta_workspace(rb):
    size = rb.recblr_delta_workspace_size
    assert size(rb.OP_DELTA_BACKWARD, 2, 3, 2, 4, 8, 8, 0) > 0
    assert bwd(rb, ws=None) == rb.ERR_WORKSPACE
    assert bwd(rb, nws=16) == rb.ERR_WORKSPACE
    assert bwd(rb, ws=addr(12) + 64) == rb.ERR_WORKSPACE
    # many short sequences walk in one kernel; one long one takes workspace
    assert size(rb.OP_DELTA_FORWARD, 1024, 200, 2, 2, 64, 64, 1) == 0
    assert size(rb.OP_DELTA_FORWARD, 1, 16384, 2, 4, 128, 128, 1) > 0
    assert fwd(rb, B=1, L=16384, Dk=128, Dv=128, q=1 << 40, k=2 << 40, v=3 << 40, g=4 << 40,
               beta=5 << 40, o=6 << 40, hT=7 << 40) == rb.ERR_WORKSPACE
    for bad in ((-1, 3, 2, 4, 8, 8, 0), (2, 3, 2, 3, 8, 8, 0), (2, 3, 2, 4, 200, 8, 0),
                (2, 3, 2, 4, 8, 8, 7)):
        assert size(rb.OP_DELTA_BACKWARD, *bad) == 0
    assert size(5, 2, 3, 2, 4, 8, 8, 0) == 0


def test_delta_workspace_of_many_heads(rb):
    """Heads that fill the chip are walked in one kernel each way: no workspace forward, the
    gradients of the states and of the updates alone backward.  (The other way's walk has a
    workgroup to 16 columns: 2^32 threads at the last of these sizes.)"""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    for B, L, Dk, Dv in ((8192, 200, 64, 64), (2048, 200, 64, 128), (50000, 8, 64, 64),
                         (4096, 1000, 16, 16), (1 << 22, 64, 64, 64)):
        for io in (rb.F32, rb.BF16):
            sizes = (B, L, 1, 1, Dk, Dv, io)
            assert rb.recblr_delta_workspace_size(rb.OP_DELTA_FORWARD, *sizes) == 0, sizes
            assert rb.recblr_delta_workspace_size(rb.OP_DELTA_BACKWARD, *sizes) == up(
                4 * B * -(-L // 64) * Dk * Dv) + up(4 * B * L * Dv), sizes


# ------------------------------------------------------------------ AdamW

def tensors(rb, size, count=2, bits=32, **kw):
    t = (rb.AdamWTensor * count)()
    for i in range(count):
        t[i].param, t[i].grad = addr(6 * i), addr(6 * i + 1)
        t[i].m1, t[i].m2 = addr(6 * i + 2), addr(6 * i + 3)
        t[i].scale1, t[i].scale2 = (addr(6 * i + 4), addr(6 * i + 5)) if bits == 8 else (None, None)
        t[i].n = size
    for name, value in kw.items():
        setattr(t[count - 1], name, value)
    return t


def update(rb, t, count=None, bits=32, io=0, step=1, lr=1e-3, b1=0.9, b2=0.999):
    return rb.recblr_adamw_update(t, len(t) if count is None else count, bits, io, step, lr, b1,
                                  b2, 1e-8, None)


def test_adamw_refuses(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    ok = tensors(rb, 8)
    assert update(rb, ok, bits=16) == rb.ERR_UNSUPPORTED
    assert update(rb, ok, io=3) == rb.ERR_UNSUPPORTED
    assert update(rb, ok, step=0) == bad
    assert update(rb, ok, count=-1) == bad
    assert update(rb, None, count=1) == bad
    assert update(rb, ok, b1=1.0) == bad and update(rb, ok, b2=-0.1) == bad
    assert update(rb, ok, b1=math.nan) == bad
    assert update(rb, tensors(rb, 8, n=-1)) == bad
    assert update(rb, tensors(rb, 8, n=(1 << 40) + 1)) == rb.ERR_UNSUPPORTED
    assert update(rb, tensors(rb, 8, n=1 << 36)) == rb.ERR_UNSUPPORTED
    for name in ("param", "grad", "m1", "m2"):
        assert update(rb, tensors(rb, 8, **{name: None})) == bad, name
        assert update(rb, tensors(rb, 8, **{name: addr(40) + 2})) == bad, name
    for name in ("scale1", "scale2"):
        assert update(rb, tensors(rb, 8, bits=8, **{name: None}), bits=8) == bad, name
        assert update(rb, tensors(rb, 8, bits=8, **{name: addr(40) + 2}), bits=8) == bad, name


def test_adamw_refuses_overlap(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    assert update(rb, tensors(rb, 8, param=addr(0))) == bad           # the same tensor twice
    assert update(rb, tensors(rb, 8, param=addr(0) + 28)) == bad      # the last element of it
    assert update(rb, tensors(rb, 8, m1=addr(1))) == bad              # moments over a gradient
    assert update(rb, tensors(rb, 8, m2=addr(8))) == bad              # m2 over m1
    assert update(rb, tensors(rb, 300, bits=8, scale2=addr(4) + 4), bits=8) == bad
    many = tensors(rb, 8, count=200, param=addr(6 * 77))
    assert update(rb, many) == bad


def test_adamw_nothing_to_do(rb):
    assert update(rb, None, count=0) == rb.OK
    assert update(rb, tensors(rb, 0, param=None, grad=None)) == rb.OK
    assert rb.recblr_adamw_moments(None, 0, None, None, None) == rb.OK
    assert rb.recblr_adamw_moments(tensors(rb, 8, bits=8), 2, None, None, None) == rb.OK


def test_adamw_moments_refuses(rb):
    outs = (ctypes.c_void_p * 2)(addr(50), addr(51))
    call = lambda t, a=outs, b=None, n=2: rb.recblr_adamw_moments(t, n, a, b, None)  # noqa: E731
    bad = rb.ERR_INVALID_ARGUMENT
    assert call(tensors(rb, 8, bits=8), n=-1) == bad
    assert call(None) == bad
    assert call(tensors(rb, 8, bits=8, m1=None)) == bad
    assert call(tensors(rb, 8, bits=8, scale1=None)) == bad
    assert call(tensors(rb, 8, bits=8), (ctypes.c_void_p * 2)(addr(50), None)) == bad
    assert call(tensors(rb, 8, bits=8), (ctypes.c_void_p * 2)(addr(50), addr(51) + 2)) == bad
    assert call(tensors(rb, 8, bits=8), (ctypes.c_void_p * 2)(addr(50), addr(8))) == bad


def test_adamw_moments_refuses_overlap(rb):
    """Outputs over other tensors' outputs, codes and scales, not only over their own."""
    def call(n, a, b):
        lists = [x and (ctypes.c_void_p * n)(*x) for x in (a, b)]
        return rb.recblr_adamw_moments(tensors(rb, 300, count=n, bits=8), n, *lists, None)
    bad = rb.ERR_INVALID_ARGUMENT
    out = [addr(600 + i) for i in range(200)]
    assert call(2, [out[0], out[0]], None) == bad                 # one output for two tensors
    assert call(2, [out[0], out[0] + 1196], None) == bad          # the last element of it
    assert call(2, out[:2], [out[2], out[1]]) == bad              # m2's over another's m1
    assert call(2, None, [addr(8), out[1]]) == bad                # over the other's codes
    assert call(2, None, [out[0], addr(4) + 4]) == bad            # over the other's scales
    assert call(200, out[:199] + [out[77]], None) == bad


# ------------------------------------------------------------------ sampling

def draw(rb, **kw):
    a = dict(logits=addr(0), u=addr(1), temperature=None, top_k=None, top_p=None, min_p=None,
             ids=addr(2), prob=addr(3), B=2, V=10, io=0, ws=None, nws=0)
    a.update(kw)
    return rb.recblr_sample(*a.values(), None)


def test_sample_refuses(rb):
    bad = rb.ERR_INVALID_ARGUMENT
    assert draw(rb, B=-1) == bad and draw(rb, V=-1) == bad
    assert draw(rb, io=2) == rb.ERR_UNSUPPORTED
    assert draw(rb, V=(1 << 24) + 1) == rb.ERR_UNSUPPORTED
    assert draw(rb, B=1 << 31) == rb.ERR_UNSUPPORTED
    assert draw(rb, B=1 << 24, V=1) == rb.ERR_UNSUPPORTED
    assert draw(rb, B=1 << 30, V=1 << 20) == rb.ERR_UNSUPPORTED
    for name in ("logits", "u", "ids"):
        assert draw(rb, **{name: None}) == bad, name
    for name in ("logits", "u", "ids", "prob", "temperature", "top_k", "top_p", "min_p"):
        assert draw(rb, **{name: addr(9) + 2}) == bad, name
    assert draw(rb, ids=addr(0)) == bad and draw(rb, prob=addr(2)) == bad
    assert draw(rb, prob=addr(1)) == bad
    need = rb.recblr_sample_workspace_size(2, 10000, 0)
    assert need > 0 and rb.recblr_sample_workspace_size(2, 4096, 0) == 0
    assert draw(rb, V=10000) == rb.ERR_WORKSPACE
    assert draw(rb, V=10000, ws=addr(5), nws=need - 1) == rb.ERR_WORKSPACE
    assert draw(rb, V=10000, ws=addr(5) + 128, nws=need) == rb.ERR_WORKSPACE
    assert draw(rb, V=10000, ws=addr(0), nws=need) == bad             # over the logits
    assert draw(rb, B=0, logits=None, u=None, ids=None) == rb.OK
    assert rb.recblr_sample_workspace_size(-1, 10000, 0) == 0


# ------------------------------------------------------------------ the binding

def test_binding_refuses_cpu_tensors(rb):
    import torch
    z = torch.zeros
    with pytest.raises(ValueError):
        rb.delta_forward(z(1, 2, 1, 4), z(1, 2, 1, 4), z(1, 2, 1, 4), z(1, 2, 1), z(1, 2, 1))
    with pytest.raises(ValueError):
        rb.delta_step(z(1, 1, 4), z(1, 1, 4), z(1, 1, 4), z(1, 1), z(1, 1), z(1, 1, 4, 4))
    with pytest.raises(ValueError):
        rb.sample(z(1, 5), z(1))
    with pytest.raises(ValueError):
        rb.AdamW([z(4)])
    with pytest.raises(ValueError):
        rb.AdamW([])


def test_binding_takes_the_first_argument_by_name(rb):
    """As far as the tensors' device, which is refused for CPU tensors."""
    import torch
    z = torch.zeros
    with pytest.raises(ValueError, match="on the GPU"):
        rb.sample(logits=z(1, 5), u=z(1))
    with pytest.raises(ValueError, match="on the GPU"):
        rb.delta_forward(q=z(1, 2, 1, 4), k=z(1, 2, 1, 4), v=z(1, 2, 1, 4), g=z(1, 2, 1),
                         beta=z(1, 2, 1))
    with pytest.raises(TypeError):
        rb.sample()


# ------------------------------------------------------------------ the references

def _case(B, L, H, HV, Dk, Dv, seed=0):
    r = np.random.default_rng(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    return dict(q=unit(r.normal(size=(B, L, H, Dk))), k=unit(r.normal(size=(B, L, H, Dk))),
                v=r.normal(size=(B, L, HV, Dv)), g=-0.5 * r.random((B, L, HV)),
                beta=r.random((B, L, HV)), h0=0.5 * r.normal(size=(B, HV, Dk, Dv)))


def test_delta_reference_gradients_by_differences():
    """Central differences of a random linear functional of o and hT: error O(h^2) ~ 1e-10 and
    cancellation 1e-16 / h ~ 1e-11, so 1e-7 of the gradient's size leaves room."""
    c = _case(2, 5, 2, 4, 3, 4)
    r = np.random.default_rng(1)
    do, dhT = r.normal(size=c["v"].shape), r.normal(size=c["h0"].shape)

    def loss(**kw):
        out = ref.delta(**{**c, **kw})
        return (out["o"] * do).sum() + (out["hT"] * dhT).sum()

    grads = ref.delta(**c, do=do, dhT=dhT)
    for name in ("q", "k", "v", "g", "beta", "h0"):
        d = grads["d" + name]
        assert d.shape == c[name].shape
        for at in r.integers(0, d.size, 12):
            x = c[name].copy().reshape(-1)
            h = 1e-5
            x[at] += h
            up = loss(**{name: x.reshape(c[name].shape)})
            x[at] -= 2 * h
            down = loss(**{name: x.reshape(c[name].shape)})
            got = (up - down) / (2 * h)
            assert abs(got - d.reshape(-1)[at]) <= 1e-7 * (1 + np.abs(d).max()), (name, at)


def test_delta_reference_closed_cases():
    """beta = 1 and unit keys overwrite what the key read; g = 0, beta = 0 changes nothing."""
    k = np.zeros((1, 2, 1, 3))
    k[0, :, 0, 1] = 1.0
    v = np.array([[1.0, 2.0], [5.0, 7.0]]).reshape(1, 2, 1, 2)
    zero, one = np.zeros((1, 2, 1)), np.ones((1, 2, 1))
    out = ref.delta(k, k, v, zero, one, scale=1.0)
    assert np.allclose(out["o"], v) and np.allclose(out["hT"][0, 0, 1], [5.0, 7.0])
    h0 = np.arange(6.0).reshape(1, 1, 3, 2)
    assert np.array_equal(ref.delta(k, k, v, zero, zero, h0=h0)["hT"], h0)


def test_adamw_reference_values():
    """Codes' ends and middles, by hand; a first step's size is the rate."""
    m, v = ref.moment_values([127, -127, 0, 64], [255, 127, 0, 63], [0.5], [2.0])
    assert np.allclose(m, [0.5, -0.5, 0.0, 0.5 * (64 / 127) ** 2])
    assert np.allclose(v, [2.0, 2.0 / 16, 2.0 / 256 ** 4, 2.0 / 256])
    p, m, v = ref.adamw([1.0, 1.0], [0.25, -4.0], 0.0, 0.0, 1, 0.1, 0.9, 0.99, 0.0, 0.5)
    assert np.allclose(p, [0.95 - 0.1, 0.95 + 0.1]) and np.allclose(m, [0.025, -0.4])
    assert np.allclose(v, [0.01 * 0.0625, 0.16])


def test_sample_reference_shares():
    """Over a fine grid of u every item's share is its weight's."""
    x = np.log(np.array([[4.0, 1.0, 3.0, 2.0]]))
    n = 1000
    u = (np.arange(n) + 0.5) / n
    ids, prob = ref.sample(np.repeat(x, n, 0), u)
    assert [int((ids == i).sum()) for i in range(4)] == [400, 100, 300, 200]
    assert np.allclose(prob, np.array([0.4, 0.1, 0.3, 0.2])[ids])
    ids, _ = ref.sample(np.repeat(x, n, 0), u, top_k=np.full(n, 2))
    assert set(ids) == {0, 2}
    ids, _ = ref.sample(np.repeat(x, n, 0), u, top_p=np.full(n, 0.85))
    assert set(ids) == {0, 2, 3}
    ids, _ = ref.sample(np.repeat(x, n, 0), u, min_p=np.full(n, 0.6))
    assert set(ids) == {0, 2}
