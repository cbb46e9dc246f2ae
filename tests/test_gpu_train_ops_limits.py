"""Muon's workspace and the policy loss's arguments on the GPU, at the ends of what they accept.
Ordinary sizes are in test_gpu_train_ops.py."""
import pytest

from test_gpu_train_ops import dtype_of, rb  # noqa: F401

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
