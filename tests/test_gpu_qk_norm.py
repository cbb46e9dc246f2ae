"""The norms of queries and keys on the GPU where sizes and values go far: more tokens than a launch
has workgroups for, more elements than 31 bits count.  Ordinary sizes are in test_gpu_train_ops.py.
"""
import numpy as np
import pytest

from test_gpu_train_ops import ints, put, rb  # noqa: F401

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
