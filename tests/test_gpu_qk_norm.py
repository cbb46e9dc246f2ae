"""The norms of queries and keys on the GPU where sizes and values go far: more tokens than a launch
has workgroups for or than one of a sum takes in a turn, more elements than 31 bits count, heads and
angles far from one.  Ordinary sizes are in test_gpu_train_ops.py.
"""
import numpy as np
import pytest

import train_ops_reference as ref
from test_gpu_train_ops import LAST, U, ints, put, qk_case, rb, within  # noqa: F401

pytestmark = pytest.mark.gpu


def repeated(t, times):
    return t.repeat(times, *([1] * (t.dim() - 1)))


def is_repeated(t, small):
    """Whether t is small, over and over."""
    return bool((t.view(-1, *small.shape) == small).all())


@pytest.mark.parametrize("io,times,H,D,R", [
    ("bf16", 66601, 1, 3, 2),      # 2^26 tokens and more, four to a workgroup of 256
    ("f32", 66601, 1, 2, 2),
    ("bf16", 8401, 2, 128, 128),   # 2^31 elements and more, of vectors
    ("bf16", 8401, 2, 129, 64)])   # and one by one
def test_tokens_beyond_a_launch(rb, io, times, H, D, R):  # noqa: F811
    """1009 tokens over and over have the results of 1009 tokens, bit by bit: a head's arithmetic
    does not hang on where it lies."""
    import torch
    r = np.random.default_rng(0)
    q, k, dq, dk = (put(r.normal(size=(1009, h, D)), io)[0] for h in (H, 1, H, 1))
    pos = ints(r.integers(0, 10000, 1009))
    how = dict(rotate=R, norm="l2")
    want = (*rb.qk_norm(q, k, positions=pos, **how),
            *list(rb.qk_norm_backward(q, k, dq, dk, positions=pos, **how).values())[:2])
    print(io, times, H, D, R, flush=True)
    q, k, dq, dk, pos = (repeated(t, times) for t in (q, k, dq, dk, pos))
    for t, w in zip(rb.qk_norm(q, k, positions=pos, **how), want):
        assert is_repeated(t, w)
    torch.cuda.synchronize()
    got = rb.qk_norm_backward(q, k, dq, dk, positions=pos, **how)
    assert is_repeated(got["dq"], want[2]) and is_repeated(got["dk"], want[3])


def check_far(rb, c, eps):  # noqa: F811
    io, R, D = c["io"], c["rotate"], c["q"].shape[-1]
    how = dict(wq=c["wq"], wk=c["wk"], positions=ints(c["pos"]) if R else None, rotate=R,
               norm=c["norm"], eps=eps)
    qn, kn = rb.qk_norm(c["q"], c["k"], **how)
    got = rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **how)
    least = 2.0 ** (-149 if io == "f32" else -133)
    for name, y in (("q", qn), ("k", kn)):
        o = ref.qk_norm(c[name + "_"], c["w" + name + "_"], c["pos"], R, 10000.0, c["norm"],
                        float(np.float32(eps)), dy=c["d" + name + "_"])
        amp = ref.amplitude(o["y"], R)
        within(name, y, o["y"], (D / 2 + 18) * U * amp + LAST[io] * np.abs(o["y"]) + 4 * least)
        dot = (np.abs(o["u"]) * o["a_size"]).sum(-1, keepdims=True)
        bound = U * o["r"] * ((D / 2 + 24) * o["a_size"]
                              + o["s"] * np.abs(o["u"]) * dot * (2 * D + 48))
        within("d" + name, got["d" + name], o["dx"], bound + LAST[io] * np.abs(o["dx"]) + least)
        if c["w" + name] is not None:
            rows = o["dx"].size // D
            within("dw" + name, got["dw" + name], o["dw"], (rows + D / 2 + 20) * U * o["dw_size"])


# Heads whose squares are beyond fp32's range at one end or the other, beside ordinary ones.
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("norm,weights", [("rms", True), ("l2", False)])
@pytest.mark.parametrize("D,R", [(16, 16), (64, 32), (128, 128), (256, 0), (17, 16), (255, 254)])
@pytest.mark.parametrize("sizes,eps", [((1.0, 1e19, 1e20, 1e25, 1e30, 2e37), 1e-6),
                                       ((1.0, 1e-6, 1e-19, 1e-22, 1e-30, 1e20), 1e-30),
                                       ((1.0, 0.0, 1e-19, 1e-22, 1e-36, 1e30), 1e-45)])
def test_heads_far_from_one(rb, io, norm, weights, D, R, sizes, eps):  # noqa: F811
    """Elements are within 4.5 of these sizes times 2.  Results have the bounds of ordinary heads,
    with a floor of a denormal's rounding in place of 1e-38, times what follows it: of y by the
    weight (below 2) and the rotation, of dx none."""
    print(io, norm, D, R, sizes, flush=True)
    c = qk_case(io, (3, 11), 2, 4, D, R, norm=norm, weights=weights, far=100, seed=D)
    r = np.random.default_rng(1)
    for name in ("q", "k"):
        by = r.permutation(np.resize(sizes, c[name].shape[0] * 11 * c[name].shape[2]))
        x = c[name + "_"] * by.reshape(3, 11, -1, 1)
        c[name], c[name + "_"] = put(x, io)
        assert np.isfinite(c[name + "_"]).all()
    check_far(rb, c, eps)


@pytest.mark.parametrize("D,R", [(64, 64), (256, 128), (33, 32)])
@pytest.mark.parametrize("far", [3, 5000, 1 << 24])
def test_sines_keep_their_digits(rb, D, R, far):  # noqa: F811
    """Heads of a single one at an element of a pair have length one exactly, and are turned to the
    sine and cosine as they are formed.  An angle's rounding to fp32 is U of it, up to pi, times the
    other one of the two; sine and cosine are right to 2 ulps, 4 U of themselves; turns in 64 bits
    are off by three roundings of all of them."""
    r = np.random.default_rng(far)
    n = 40 * R
    pos = r.integers(-far, far + 1, n)
    i = np.arange(n) % R                              # each element of a pair
    x = np.zeros((n, 1, D))
    x[np.arange(n), 0, i] = 1.0
    q, _ = put(x)
    y, _ = rb.qk_norm(q, q, positions=ints(pos), rotate=R, norm="l2", eps=1e-30)
    y = y[:, 0].double().cpu().numpy()
    pair = i % (R // 2)
    turns = pos.astype(np.longdouble) * np.longdouble(10000.0) ** (-2.0 * pair.astype(
        np.longdouble) / R) / (2 * np.longdouble(np.pi) + np.longdouble(2.4492935982947064e-16))
    a = ((turns - np.rint(turns)) * (2 * np.longdouble(np.pi))).astype(np.float64)
    sn, cs = np.sin(a), np.cos(a)
    far_off = 2 * np.pi * 3 * 2.0 ** -52 * np.abs(turns).astype(np.float64)
    first = i < R // 2
    for name, at, want, other in (("cos", i, cs, sn),
                                  ("sin", np.where(first, i + R // 2, i - R // 2),
                                   np.where(first, sn, -sn), cs)):
        off = np.abs(y[np.arange(n), at] - want)
        bound = U * np.abs(a * other) + 4 * U * np.abs(want) + far_off + 1e-16
        print(f"ERR {name}: {np.max(off / bound):.3f} of its bound, rms {np.sqrt(np.mean(off ** 2)) / U:.3f} U")
        assert (off <= bound).all()


# Each number of lanes to a token (0: a wave, an element at a time), by types and widths.
LANES = [("f32", 8, 2), ("f32", 16, 4), ("f32", 32, 8), ("f32", 64, 16), ("f32", 128, 32),
         ("f32", 256, 64), ("bf16", 16, 2), ("bf16", 32, 4), ("bf16", 64, 8), ("bf16", 128, 16),
         ("bf16", 256, 32), ("f32", 17, 0), ("bf16", 100, 0)]


def tokens_of_turns(lanes):
    """(tokens that workgroups of sums take two turns for, and some of them a third with a part of
    it, tokens to a workgroup): 1024 workgroups are the most."""
    each = 256 // (lanes or 64)
    return 1024 * each * 2 + 3 * each + 1, each


@pytest.mark.parametrize("io,D,lanes", LANES)
def test_turns_of_whole_numbers(rb, io, D, lanes):  # noqa: F811
    """Heads of a single 1 or -1 have length one exactly, and turned by no angle stay as they are; with
    gradients of small whole numbers all of the results are whole, and so are sums in any order:
    y = x, dx = dy but for 0 at the one, dw the sums of x dy.  No token is lost or taken twice."""
    import torch
    n, _ = tokens_of_turns(lanes)
    r = np.random.default_rng(D)
    R = D // 2 * 2
    how = dict(positions=ints(np.zeros(n)), rotate=R, norm="l2", eps=1e-30,
               wq=torch.ones(D, device="cuda"), wk=torch.ones(D, device="cuda"))
    x, dy = {}, {}
    for name, heads in (("q", 2), ("k", 1)):
        a = np.zeros((n * heads, D))
        a[np.arange(n * heads), r.integers(0, D, n * heads)] = r.choice([-1.0, 1.0], n * heads)
        x[name] = put(a.reshape(n, heads, D), io)
        dy[name] = put(r.integers(1, 4, (n, heads, D)) * r.choice([-1.0, 1.0], (n, heads, D)), io)
    got = rb.qk_norm_backward(x["q"][0], x["k"][0], dy["q"][0], dy["k"][0], **how)
    for name, y in zip("qk", rb.qk_norm(x["q"][0], x["k"][0], **how)):
        (a, a_), (g, g_) = x[name], dy[name]
        assert torch.equal(y, a)
        assert torch.equal(got["d" + name], g.masked_fill(a != 0, 0.0))
        want = (a_ * g_).sum((0, 1))
        assert np.array_equal(got["dw" + name].double().cpu().numpy(), want)
        # one token's part alone: the last one's, whose workgroup has others' turns before it
        g.zero_()
        g[-1] = 2.0
    alone = rb.qk_norm_backward(x["q"][0], x["k"][0], dy["q"][0], dy["k"][0], **how)
    for name in "qk":
        assert np.array_equal(alone["dw" + name].double().cpu().numpy(),
                              2.0 * x[name][1][-1].sum(0))


@pytest.mark.parametrize("io,D,lanes", LANES)
def test_turns(rb, io, D, lanes):  # noqa: F811
    """A thread adds its own tokens' heads one after another, three turns of them at most, a workgroup
    its 256 / lanes groups (four waves), and the rest is summed in 64 bits: no more additions than
    these lie over a term of dw, whose own error is that of u and of a turned pair, (D / 2 + 18) U."""
    n, each = tokens_of_turns(lanes)
    c = qk_case(io, (n,), 2, 1, D, D // 4 * 2, far=3000, seed=D)
    how = dict(wq=c["wq"], wk=c["wk"], positions=ints(c["pos"]), rotate=c["rotate"])
    got = rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **how)
    for name, heads in (("q", 2), ("k", 1)):
        o = ref.qk_norm(c[name + "_"], c["w" + name + "_"], c["pos"], c["rotate"],
                        eps=float(np.float32(1e-6)), dy=c["d" + name + "_"])
        chain = 3 * heads + each + 1
        within("dw" + name, got["dw" + name], o["dw"], (chain + D / 2 + 18) * U * o["dw_size"])
