"""Muon's workspace and the policy loss's arguments on the GPU, at the ends of what they accept.
Ordinary sizes are in test_gpu_train_ops.py."""
import math

import numpy as np
import pytest

from test_gpu_train_ops import U, dtype_of, ints, rb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_muon_list_in_one_workspace(rb, io):  # noqa: F811
    """Matrices sixteen at a time in the same workspace: what the list gets is what each sixteen
    get by themselves, bit by bit, over and over, and nothing around the workspace is touched."""
    import ctypes
    import torch
    shapes = [(130 + 37 * i % 300, 190 + 53 * i % 400) for i in range(40)]
    shapes[5:5] = [(20, 30), (128, 128)]              # smaller ones between need no workspace
    torch.manual_seed(0)
    draw = lambda dt: [torch.randn(s, device="cuda").to(dt) for s in shapes]  # noqa: E731
    p, g, m = draw(dtype_of(io)), draw(dtype_of(io)), draw(torch.float32)
    want_p, want_m = [t.clone() for t in p], [t.clone() for t in m]
    for a, b in ((0, 18), (18, 34), (34, 42)):        # of 16, 16 and 8 large ones
        rb.Muon(want_p[a:b], state=want_m[a:b], lr=0.1).step(g[a:b])
    opt = rb.Muon(p, state=m, lr=0.1)
    start = [t.clone() for t in p + m]
    n, edge = opt._ws_bytes, 4096
    room = torch.full((n + 2 * edge,), 77, dtype=torch.uint8, device="cuda")
    ws = room[edge:edge + n]
    for t, x in zip(g, opt._table):
        x.grad = t.data_ptr()
    for _ in range(3):
        for t, s in zip(p + m, start):
            t.copy_(s)
        st = rb.recblr_muon_update(opt._table, len(p), rb.io_code(p[0].dtype), 0.1, 0.95, 1, 5,
                                   ctypes.c_double(1e-7), ws.data_ptr(), n,
                                   torch.cuda.current_stream().cuda_stream)
        assert st == rb.OK
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p + m, want_p + want_m))
        assert bool((room[:edge] == 77).all()) and bool((room[edge + n:] == 77).all())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 100), (6, 3001), (130, 5000), (6, 30000), (6, 140000)])
@pytest.mark.parametrize("T", [0.8, 1.1, 0.7])
def test_policy_takes_the_temperature_as_it_is(rb, io, size, T):  # noqa: F811
    """Two items a row, 100 apart, the rarer one chosen: logp is -100 / T but for e^-100, and the
    ratio to an old logp near it shows the temperature's last digits, whose rounding to fp32 would move
    it by 100 / T times up to U.  What it is off by itself: the one power of the sum and the sum, 2
    ulps (4 U), and the loss's rounding, U of a loss of about one."""
    import torch
    N, V = size
    r = np.random.default_rng(V)
    x = torch.full(size, -math.inf, dtype=dtype_of(io), device="cuda")
    top, ids = r.integers(0, V, N), r.integers(0, V, N)
    ids = np.where(ids == top, (top + 1) % V, ids)
    at = np.resize([0.0, 37.0, -28.0], N)
    x[torch.arange(N), torch.from_numpy(top)] = torch.from_numpy(at).cuda().to(x.dtype)
    x[torch.arange(N), torch.from_numpy(ids)] = torch.from_numpy(at - 100).cuda().to(x.dtype)
    old = np.float32(-100.0 / T)
    z = torch.zeros(N, device="cuda")
    one_row = math.exp(-100.0 / T - float(old))
    assert abs(math.exp(-100.0 / float(np.float32(T)) - float(old)) / one_row - 1) > 15 * U
    for row in range(6):
        one = z.clone()
        one[row] = 1.0
        loss, logp, _ = rb.policy_loss(x, ints(ids), z + float(old), z + 1, weight=one,
                                       temperature=T)
        assert abs(float(loss) + one_row) <= 5 * U * one_row, row
        assert np.allclose(logp.double().cpu().numpy(), -100.0 / T, rtol=U, atol=4 * U)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 100), (6, 3001), (130, 5000), (6, 30000), (6, 140000)])
def test_policy_masks_at_any_temperature(rb, io, size):  # noqa: F811
    """Masked items count as nothing also where log2(e) / T lies above a float by less than the least
    one, at temperatures that make all other items alike: log odds of -log of their number, off by
    the sum's roundings (128 + 70 + 16 in a chain) and its own."""
    import torch
    N, V = size
    x = torch.randn(size, device="cuda").to(dtype_of(io))
    x[:, ::3] = -math.inf
    n = V - (V + 2) // 3
    z = torch.zeros(N, device="cuda")
    for T in (2.5118862065898873e+29, 2.5118857130558871e+29, 1e30, 1e29):
        k = 1.4426950408889634 / T
        print(size, T, k - float(np.float32(k)), flush=True)
        loss, logp, grad = rb.policy_loss(x, ints(np.full(N, 1)), z - math.log(n), z + 1,
                                          temperature=T)
        bar = (128 + 70 + 16 + 8 + math.log(n)) * U
        assert np.allclose(logp.double().cpu().numpy(), -math.log(n), rtol=0, atol=bar)
        assert abs(float(loss) + N) <= 2 * N * bar and not grad[:, ::3].any()


def test_policy_without_a_gradient_leaves_out_alone(rb):  # noqa: F811
    """No gradient is asked for: none is returned, and the logits given as its place stay."""
    import torch
    x = torch.randn(5, 40, device="cuda")
    before, z = x.clone(), torch.zeros(5, device="cuda")
    args = (x, ints(np.arange(5)), z - 3, z + 1)
    loss, logp, grad = rb.policy_loss(*args, need_grad=False, out=x)
    assert grad is None and torch.equal(x, before)
    want = rb.policy_loss(*args, out=x)
    assert want[2] is x and torch.equal(want[0], loss) and torch.equal(want[1], logp)


@pytest.mark.parametrize("pad_id", [(1 << 32) + 2, -(1 << 31) - 1, 1 << 31])
def test_embed_padding_beyond_its_type(rb, pad_id):  # noqa: F811
    """An id that int32 does not have is refused, not taken for the one that its low bits are."""
    import torch
    t, ids = torch.randn(6, 8, device="cuda"), ints([1, 2, 3])
    with pytest.raises(ValueError, match="pad_id"):
        rb.embed(t, ids, pad_id=pad_id)
    with pytest.raises(ValueError, match="pad_id"):
        rb.embed_backward(ids, t[:3], 6, pad_id=pad_id)
    assert torch.equal(rb.embed(t, ids, pad_id=-(1 << 31)), t[1:4])
