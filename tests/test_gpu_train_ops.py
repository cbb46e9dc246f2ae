"""The item lookup, the norms of queries and keys, the policy loss and Muon on the GPU, against
the 64-bit references of train_ops_reference.py.

Bounds, element by element, from the arithmetic (U = 2^-24, the largest relative error of a
rounding to fp32; 2^-8 to bf16):

* Lookup: one product in fp32, then one rounding to the type: equal to that.
* Its gradient: an item's n rows are added in chains of at most 64 within a piece, 16 pieces in a
  group, groups of 1024 in eight chains that are added up (up to 4096 positions: by halves of 8 or
  16, at most 32 of these in a chain, 16 chains): no more than d = min(n, 64 + n / 512 + 24)
  additions lie over a term, and the factor, and what was there: (d + 3) U of the sum of the terms' sizes.
* Norms: the sum of D squares has at most D roundings, the root halves them, division, square
  root, products: r and u are off by (D / 2 + 6) U.  A sine's angle is rounded to fp32 (pi U of
  turns up to a half) and sincospif is right to 2 ulps: 8 U of the pair's size, with the products
  and the sum 12 U.  dx has the product u . a of D terms more.
* Policy loss: e^x is off by 3 U |x| (scale, difference, argument) and 2 ulps; sums have at most
  128 + 16 additions in a chain; log, difference: see policy_bounds.
* Muon: a step's products have operands of 2^-22 and the neglected product of two low parts,
  2^-22: 2^-20 of the operands' norms together, and sums of K in fp32, sqrt(K) U at random
  rounding, 4 times that as a bound; B = b A + c A^2 and X = a X + B X weigh this by |a| + |b| s^2
  + |c| s^4 < 20 at s = 1.2.  An error in X is passed on by a step with a factor of at most 3.9
  (the polynomial's slope and divided differences on [0, 1.2]).  Norms are Frobenius norms.
"""
import math

import numpy as np
import pytest

import ops_reference as ops_ref
import train_ops_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LAST = {"f32": 0.0, "bf16": 2.0 ** -8}  # the rounding to the output's type


@pytest.fixture(scope="module")
def rb():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_12580_amd import recblr
    return recblr


def dtype_of(io):
    import torch
    return torch.float32 if io == "f32" else torch.bfloat16


def put(a, io="f32", offset=0):
    """A numpy array on the GPU in the I/O type, and what it stands for in 64 bits; `offset`:
    elements by which its start is off a multiple of 16 bytes."""
    import torch
    a = np.ascontiguousarray(a)
    t = torch.from_numpy(a).to(dtype_of(io)).cuda()
    if offset:
        room = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
        room[offset:] = t.reshape(-1)
        t = room[offset:].view(a.shape)
    return t, t.double().cpu().numpy()


def ints(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def within(name, got, want, bound):
    """|got - want| <= bound, element by element; NaN and infinities at the same places."""
    got = host(got)
    assert got.shape == np.shape(want), name
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), name
    assert np.array_equal(np.isnan(want), np.isnan(got)), name
    if not fine.any():
        return
    off = np.abs(got - want)[fine]
    bound = np.broadcast_to(bound, np.shape(want))[fine]
    worst = float(np.max(off / np.maximum(bound, 1e-300)))
    print(f"ERR {name}: {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.3f} of its bound"


def poisoned(shape, dtype):
    """A tensor in the middle of a buffer of 7s, and a check that these are untouched."""
    import torch
    n, edge = int(np.prod(shape)), 1024
    room = torch.full((n + 2 * edge,), 7.0, dtype=dtype, device="cuda")

    def untouched():
        return bool((room[:edge] == 7).all()) and bool((room[edge + n:] == 7).all())
    return room[edge:edge + n].view(shape), untouched


# ------------------------------------------------------------------ item lookup

def embed_case(io, N, V, D, seed=0, offset=0, zipf=True):
    r = np.random.default_rng(seed)
    if zipf and V > 1:
        p = 1.0 / np.arange(1, V + 1)
        ids = r.permutation(V)[r.choice(V, N, p=p / p.sum())]
    else:
        ids = r.integers(0, max(V, 1), N)
    table, table_ = put(r.normal(size=(V, D)), io, offset)
    dout, dout_ = put(r.normal(size=(N, D)), io, offset)
    into, into_ = put(r.normal(size=(V, D)), io, offset)
    return dict(ids=ids, table=table, table_=table_, dout=dout, dout_=dout_, into=into,
                into_=into_, io=io)


def check_embed(rb, c, scale=1.5, pad_id=-1, add=False):
    import torch
    io, V = c["io"], c["table"].shape[0]
    out = rb.embed(c["table"], ints(c["ids"]), scale=scale, pad_id=pad_id)
    ids = torch.from_numpy(np.asarray(c["ids"])).cuda().long()
    ok = (ids >= 0) & (ids < V) & (ids != pad_id)
    want = torch.full((*ids.shape, c["table"].shape[1]), math.nan, dtype=c["table"].dtype,
                      device="cuda")
    want[ok] = (c["table"][ids[ok]].float() * scale).to(want.dtype)
    want[ids == pad_id] = 0
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    into = None
    if add:  # a copy that starts where the case's does
        into = torch.empty(c["into"].numel() + 8, dtype=c["into"].dtype, device="cuda")
        skew = c["into"].data_ptr() % 16 // into.element_size()
        into = into[skew:skew + c["into"].numel()].view(c["into"].shape).copy_(c["into"])
    d = rb.embed_backward(ints(c["ids"]), c["dout"], V, scale=scale, pad_id=pad_id, into=into)
    assert not add or d is into
    want, size = ref.embed_backward(c["ids"], c["dout_"], V, float(np.float32(scale)), pad_id,
                                    c["into_"] if add else None)
    keep = np.asarray(c["ids"])
    keep = keep[(keep >= 0) & (keep < V) & (keep != pad_id)]
    n = np.bincount(keep, minlength=V)[:, None] if V else np.zeros((0, 1))
    chain = np.minimum(n, 64 + n / 512 + 24)
    within("dtable", d, want, (chain + 3) * U * size + LAST[io] * np.abs(want))
    if add:  # rows that no id names are as they were
        assert np.array_equal(host(d)[n[:, 0] == 0], c["into_"][n[:, 0] == 0])


# Around the few positions' limit (4096), a wave's and a workgroup's part of them (64, 1024), a
# block (2048), pieces (64); tables of one digit (12 bits), two and three; widths of every way to
# read a row.
EMBED = [(1, 1, 1), (1, 5, 64), (7, 3, 33), (64, 1, 128), (1000, 50, 48), (1024, 4, 256),
         (1025, 4, 64), (1025, 3000, 100), (2048, 4095, 130), (2049, 4096, 64), (5000, 1, 5),
         (6001, 2, 64), (64, 1, 33), (65, 1, 33), (129, 2, 64), (4095, 70, 16),
         (4096, 4000, 8), (4096, 1, 130), (4097, 300, 8), (4100, 1, 64), (9001, 2, 130),
         (10240, 4096, 64), (70, 9, 4096), (4200, 9, 2049), (9000, 70000, 7), (4500, 300, 600), (70000, 5000, 20)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("size", EMBED)
def test_embed(rb, io, add, size):
    print(io, add, size, flush=True)
    check_embed(rb, embed_case(io, *size), add=add)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N", [40, 3000, 200000])
def test_embed_of_one_item(rb, io, N):
    """Every position names the same item: one run over all pieces."""
    c = embed_case(io, N, 9, 64, seed=1)
    c["ids"] = np.full(N, 6)
    check_embed(rb, c)
    check_embed(rb, c, pad_id=6)                     # and it is padding


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N", [200, 4000, 20000])
def test_embed_runs_at_piece_borders(rb, io, N):
    """Runs that end with a piece, one before or behind it, and that fill whole pieces."""
    lengths, ids = [64, 63, 1, 65, 128, 127, 2, 64, 1, 192, 3, 61, 320], []
    for i, n in enumerate(lengths * 20):
        ids += [i] * n
    c = embed_case(io, N, 300, 64, seed=2)
    c["ids"] = np.asarray(ids)[:N]
    check_embed(rb, c)
    check_embed(rb, c, add=True)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_embed_runs_at_group_borders(rb, io):
    """The same with groups of 1024 positions, that are added up by themselves."""
    lengths, ids = [1024, 1023, 1, 1025, 2048, 2047, 2, 1024, 1, 3 * 1024, 3, 1021, 5120], []
    for i, n in enumerate(lengths * 2):
        ids += [i] * n
    c = embed_case(io, len(ids), 100, 64, seed=2)
    c["ids"] = np.asarray(ids)
    check_embed(rb, c)
    c["ids"] = np.random.default_rng(3).permutation(c["ids"])
    check_embed(rb, c, add=True)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1100000, 60000, 5), (1500000, 3, 3), (3000, 17000000, 1),
                                  (1200000, 17000000, 2)])
def test_embed_many(rb, io, size):
    """More positions than the blocks take in one turn; tables of three digits."""
    c = embed_case(io, *size, seed=4, zipf=size[1] < 100000)
    check_embed(rb, c, scale=0.5)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N", [30, 2500, 12000])
def test_embed_ids_of_no_row(rb, io, N):
    """Ids behind the table, negative ones, the type's ends and padding (inside or outside)."""
    for pad in (-1, 0, 1 << 30):
        c = embed_case(io, N, 20, 64, seed=3)
        r = np.random.default_rng(4)
        odd = np.array([-1, 20, 21, 1 << 30, -(1 << 31), (1 << 31) - 1, 0])
        c["ids"] = np.where(r.random(N) < 0.5, c["ids"], odd[r.integers(0, 7, N)])
        check_embed(rb, c, pad_id=pad)
        check_embed(rb, c, pad_id=pad, add=True)
    c["ids"] = np.full(N, -1)                        # none is left
    check_embed(rb, c)
    check_embed(rb, c, add=True)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 4])
@pytest.mark.parametrize("D", [64, 128, 256, 96])
def test_embed_unaligned(rb, io, offset, D):
    check_embed(rb, embed_case(io, 1500, 200, D, seed=5, offset=offset))
    check_embed(rb, embed_case(io, 4500, 200, D, seed=5, offset=offset))
    check_embed(rb, embed_case(io, 15, 200, D, seed=5, offset=offset), add=True)


@pytest.mark.parametrize("N", [100, 3000, 12000])
def test_embed_writes_its_table_only(rb, N):
    """A gradient in the middle of a buffer, at addresses that are no multiples of 16 bytes."""
    import ctypes
    import torch
    for io, shape in (("f32", (37, 33)), ("bf16", (37, 33)), ("bf16", (1, 1))):
        ids, dout = ints(np.arange(N) % shape[0]), torch.ones(N, shape[1], dtype=dtype_of(io),
                                                               device="cuda")
        room = torch.full((shape[0] * shape[1] + 43,), 7.0, dtype=dtype_of(io), device="cuda")
        d = room[21:21 + shape[0] * shape[1]]
        n = rb.recblr_embed_workspace_size(N, *shape, rb.io_code(d.dtype))
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        for V in (shape[0], shape[0] - 1):  # and with one row less, the last of it is left
            d.fill_(7.0)
            st = rb.recblr_embed_backward(ids.data_ptr(), dout.data_ptr(), d.data_ptr(), N, V,
                                          shape[1], ctypes.c_float(1.0), -1, 0,
                                          rb.io_code(d.dtype), ws.data_ptr(), n, None)
            assert st == rb.OK
            torch.cuda.synchronize()
            assert (room[:21] == 7).all() and (room[21 + V * shape[1]:] == 7).all()
            want = np.bincount(np.arange(N) % shape[0], minlength=shape[0])[:V]
            want = host(torch.from_numpy(want).to(d.dtype))  # counts, as the type has them
            assert np.array_equal(host(d[:V * shape[1]]).reshape(V, shape[1]),
                                  np.repeat(want[:, None], shape[1], 1))


def test_embed_shapes(rb):
    """Ids of any shape, none at all, and an empty table."""
    import torch
    t = torch.randn(6, 8, device="cuda")
    out = rb.embed(t, ints([[[1, 2]], [[0, 5]]]))
    assert out.shape == (2, 1, 2, 8) and torch.equal(out[1, 0, 1], t[5])
    assert torch.equal(rb.embed(t, ints([3])[0]), t[3])
    assert rb.embed(t, ints(np.zeros((0, 3)))).shape == (0, 3, 8)
    d = rb.embed_backward(ints(np.zeros((0, 3))), torch.empty(0, 3, 8, device="cuda"), 6)
    assert d.shape == (6, 8) and not d.any()
    assert torch.isnan(rb.embed(t[:0], ints([0]))).all()
    assert rb.embed_backward(ints([0]), torch.ones(1, 8, device="cuda"), 0).shape == (0, 8)
    same = rb.embed_backward(ints(np.zeros(0)), torch.empty(0, 8, device="cuda"), 6, into=t)
    assert same is t
    with pytest.raises(ValueError):
        rb.embed(t.t(), ints([0]))
    with pytest.raises(ValueError):
        rb.embed(t, ints([0]).long())
    with pytest.raises(ValueError):
        rb.embed_backward(ints([0]), torch.ones(1, 8, device="cuda"), 6, into=t.bfloat16())
    with pytest.raises(ValueError):
        rb.embed_backward(ints([0]), torch.ones(2, 8, device="cuda"), 6)


def test_embed_gradient_by_differences(rb):
    """The lookup is linear: a step of one in one element of the table changes w . out by the
    gradient of w, to the roundings of sums of 400 terms."""
    c = embed_case("f32", 400, 12, 16, seed=6)
    d = host(rb.embed_backward(ints(c["ids"]), c["dout"], 12, scale=0.5))
    base = (host(rb.embed(c["table"], ints(c["ids"]), scale=0.5)) * c["dout_"]).sum()
    for v, e in ((0, 0), (3, 7), (11, 15), (5, 5)):
        t = c["table"].clone()
        t[v, e] += 1.0
        moved = (host(rb.embed(t, ints(c["ids"]), scale=0.5)) * c["dout_"]).sum()
        assert abs(moved - base - d[v, e]) <= 400 * 8 * U * np.abs(c["dout_"]).sum() / 100


# ------------------------------------------------------------------ norms of queries and keys

def qk_case(io, lead, H, HK, D, rotate, norm="rms", weights=True, seed=0, far=0, offset=0):
    r = np.random.default_rng(seed)
    c = dict(io=io, rotate=rotate, norm=norm)
    for name, heads in (("q", H), ("k", HK)):
        c[name], c[name + "_"] = put(2.0 * r.normal(size=(*lead, heads, D)), io, offset)
        c["d" + name], c["d" + name + "_"] = put(r.normal(size=(*lead, heads, D)), io, offset)
        c["w" + name], c["w" + name + "_"] = put(0.5 + r.random(D)) if weights else (None, None)
    c["pos"] = r.integers(-far, far + 1, lead)
    return c


def check_qk(rb, c, eps=1e-6, base=10000.0):
    io, R, D = c["io"], c["rotate"], c["q"].shape[-1]
    how = dict(wq=c["wq"], wk=c["wk"], positions=ints(c["pos"]) if R else None, rotate=R,
               base=base, norm=c["norm"], eps=eps)
    qn, kn = rb.qk_norm(c["q"], c["k"], **how)
    got = rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **how)
    eps = float(np.float32(eps))
    for name, y in (("q", qn), ("k", kn)):
        o = ref.qk_norm(c[name + "_"], c["w" + name + "_"], c["pos"], R, base, c["norm"], eps,
                        dy=c["d" + name + "_"])
        amp = ref.amplitude(o["y"], R)
        within(name, y, o["y"], (D / 2 + 6 + 12) * U * amp + LAST[io] * np.abs(o["y"]) + 1e-38)
        dot = (np.abs(o["u"]) * o["a_size"]).sum(-1, keepdims=True)
        bound = U * o["r"] * ((D / 2 + 24) * o["a_size"]
                              + o["s"] * np.abs(o["u"]) * dot * (2 * D + 48))
        within("d" + name, got["d" + name], o["dx"], bound + LAST[io] * np.abs(o["dx"]) + 1e-38)
        if c["w" + name] is None:
            assert got["dw" + name] is None
        else:
            rows = o["dx"].size // D
            within("dw" + name, got["dw" + name], o["dw"], (rows + D / 2 + 20) * U * o["dw_size"])


QK = [((1, 1), 1, 1, 1, 0), ((2, 3), 2, 1, 2, 2), ((3, 5), 2, 2, 32, 32), ((2, 70), 4, 2, 64, 64),
      ((1, 33), 1, 3, 64, 32), ((2, 9), 2, 2, 64, 0), ((2, 9), 2, 1, 128, 64),
      ((7, 30), 2, 2, 128, 128), ((3, 3), 1, 2, 256, 256), ((2, 5), 1, 1, 16, 16),
      ((2, 5), 1, 2, 48, 16), ((2, 5), 3, 1, 96, 96), ((2, 5), 2, 2, 100, 100),
      ((3, 7), 2, 1, 17, 16), ((3, 7), 1, 1, 72, 36), ((2, 4), 2, 2, 255, 254),
      ((1, 6), 1, 1, 8, 8), ((1, 5), 2, 2, 33, 2), ((900, 3), 2, 2, 64, 64)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("norm,weights", [("rms", True), ("l2", False)])
@pytest.mark.parametrize("size", QK)
def test_qk_norm(rb, io, norm, weights, size):
    print(io, norm, weights, size, flush=True)
    check_qk(rb, qk_case(io, *size, norm=norm, weights=weights, far=3000))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D,R", [(64, 64), (100, 100)])
def test_qk_norm_many_tokens(rb, io, D, R):
    """More tokens than workgroups take at once."""
    check_qk(rb, qk_case(io, (9, 1501), 1, 2, D, R, far=3000, seed=1))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D,R", [(64, 64), (17, 16)])
def test_qk_norm_far_positions(rb, io, D, R):
    """Angles of thousands of turns keep their fractions (both sides form them in 64 bits, which
    leaves 2^24 / 2^53 turns of difference)."""
    check_qk(rb, qk_case(io, (4, 25), 2, 2, D, R, far=1 << 24, seed=2))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 4])
def test_qk_norm_unaligned(rb, io, offset):
    check_qk(rb, qk_case(io, (3, 10), 2, 2, 64, 64, far=100, seed=3, offset=offset))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D,HV", [(64, 4), (64, 3), (17, 2)])
def test_qk_norm_of_a_projection(rb, io, D, HV):
    """q and k as they lie in one projection's output, tokens a row of it apart."""
    import torch
    c = qk_case(io, (3, 20), 2, 1, D, D // 2 * 2, far=500, seed=4)
    row = torch.randn(3, 20, 3 + HV, D, device="cuda").to(dtype_of(io))
    row[:, :, :2], row[:, :, 2:3] = c["q"], c["k"]
    c["q"], c["k"] = row[:, :, :2], row[:, :, 2:3]
    assert not c["q"].is_contiguous()
    check_qk(rb, c)
    c["q"] = c["q"].transpose(0, 1)                  # tokens at two distances
    with pytest.raises(ValueError):
        rb.qk_norm(c["q"], c["q"])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 17])
def test_qk_norm_zero_and_tiny_heads(rb, io, D):
    """A head of zeros stays zeros, with a gradient of 1 / sqrt(eps); heads far below eps."""
    c = qk_case(io, (2, 3), 2, 2, D, D // 2 * 2, far=10, seed=5)
    for name in ("q", "k"):
        c[name][0, 0], c[name + "_"][0, 0] = 0, 0
        c[name], c[name + "_"] = put(c[name + "_"] * np.array([1.0, 1e-8])[:, None, None, None], io)
    check_qk(rb, c)


def test_qk_norm_positions(rb):
    """Without positions a row's tokens stand at 0, 1, ...; one token a row is a step of it."""
    import torch
    q = torch.randn(3, 11, 2, 64, device="cuda")
    a, b = rb.qk_norm(q, q)
    pos = ints(np.tile(np.arange(11), (3, 1)))
    assert torch.equal(a, rb.qk_norm(q, q, positions=pos)[0]) and torch.equal(a, b)
    for t in (0, 5, 10):
        one = q[:, t].contiguous()
        s, _ = rb.qk_norm(one, one, positions=ints(np.full(3, t)))
        assert torch.equal(s, a[:, t])
    flat, _ = rb.qk_norm(q.view(33, 2, 64), q.view(33, 2, 64), positions=pos.view(33))
    assert torch.equal(flat, a.view(33, 2, 64))
    with pytest.raises(ValueError):
        rb.qk_norm(q.view(33, 2, 64), q.view(33, 2, 64))
    with pytest.raises(ValueError):
        rb.qk_norm(q, q, positions=pos[:2])
    with pytest.raises(ValueError):
        rb.qk_norm(q, q, norm="max")
    none = rb.qk_norm(q[:0], q[:0])
    assert none[0].shape == (0, 11, 2, 64)
    w = torch.ones(64, device="cuda")
    d = rb.qk_norm_backward(q[:0], q[:0], q[:0], q[:0], wq=w, wk=None)
    assert not d["dwq"].any() and d["dwk"] is None


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 33])
def test_qk_norm_one_weight(rb, io, D):
    """Weights for queries or for keys alone: the other one's are ones, and have no gradient."""
    import torch
    c = qk_case(io, (3, 40), 2, 1, D, D // 2 * 2, far=50)
    pos, one = ints(c["pos"]), torch.ones(D, device="cuda")
    full = dict(wq=c["wq"], wk=c["wk"], positions=pos)
    for wq, wk in ((c["wq"], None), (None, c["wk"])):
        some = dict(full, wq=wq, wk=wk)
        ones = dict(full, wq=one if wq is None else wq, wk=one if wk is None else wk)
        for a, b in zip(rb.qk_norm(c["q"], c["k"], **some), rb.qk_norm(c["q"], c["k"], **ones)):
            assert torch.equal(a, b)
        a = rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **some)
        b = rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **ones)
        for name, w in (("dq", 1), ("dk", 1), ("dwq", wq), ("dwk", wk)):
            assert a[name] is None if w is None else torch.equal(a[name], b[name]), name


def test_qk_norm_nan_stays_in_its_head(rb):
    import torch
    c = qk_case("f32", (2, 9), 2, 2, 64, 64, seed=6)
    good = rb.qk_norm(c["q"], c["k"])
    c["q"][1, 4, 0, 3] = math.nan
    bad = rb.qk_norm(c["q"], c["k"])
    assert torch.isnan(bad[0][1, 4, 0]).all() and torch.equal(good[1], bad[1])
    bad[0][1, 4, 0] = good[0][1, 4, 0]
    assert torch.equal(good[0], bad[0])


# ------------------------------------------------------------------ policy loss

def policy_case(io, N, V, seed=0, offset=0, masked=0.05, spread=3.0):
    r = np.random.default_rng(seed)
    x = spread * r.normal(size=(N, V))
    x = np.where(r.random((N, V)) < masked, -np.inf, x)
    ids = r.integers(0, V, N)
    x[np.arange(N), ids] = spread * r.normal(size=N)
    c = dict(io=io)
    c["logits"], c["logits_"] = put(x, io, offset)
    c["ids"] = ids
    with np.errstate(all="ignore"):
        z = c["logits_"] / 0.8
        lp = z[np.arange(N), ids] - np.log(np.exp(z - z.max(1, keepdims=True)).sum(1)) - z.max(1)
    for name, v in (("old_logp", lp + 0.2 * r.normal(size=N)),
                    ("ref_logp", lp + 0.3 * r.normal(size=N)), ("advantage", r.normal(size=N)),
                    ("weight", r.random(N))):
        c[name], c[name + "_"] = put(v)
    return c


def policy_bounds(c, want, kl, T):
    """What the parts of a row may be off by, in fp32.  z: (l - max) / T; S = sum e^z."""
    x = c["logits_"]
    N, V = x.shape
    with np.errstate(all="ignore"):
        z = (x - x.max(1, keepdims=True)) / T
        e = np.exp(z)
        S = e.sum(1, keepdims=True)
        p = e / S
        zz = np.where(p > 0, np.abs(z), 0.0)
        e_S = (p * (3 * zz + 4)).sum(1) + 150         # relative, in U
        lp = want["logp"]
        e_lp = 3 * np.abs(want["xa"]) + e_S + 2 * np.abs(np.log(S[:, 0])) + np.abs(lp)
        r = np.exp(lp - c["old_logp_"])
        e_r = e_lp + 2 * np.abs(lp - c["old_logp_"]) + 4
        w, A = np.abs(c["weight_"]), np.abs(c["advantage_"])
        row = w * r * A * (e_r + 4)
        if kl > 0:
            d = c["ref_logp_"] - lp
            e_d = e_lp + 2 * np.abs(d) + 4
            row = row + w * kl * (np.exp(d) + 1) * (e_d + 4)
        e_c = row / T + 4 * np.abs(want["c"]) / T
    live = (c["ids"] >= 0) & (c["ids"] < V)
    one = np.zeros_like(p)
    one[np.arange(N)[live], c["ids"][live]] = 1.0
    e_grad = e_c[:, None] * (p + one) + np.abs(want["c"])[:, None] / T * (
        p * (3 * zz + e_S[:, None] + 8) + 2 * one)
    fix = lambda b: np.where(np.isfinite(b), U * b, 0.0)  # noqa: E731
    return fix(e_lp), fix(row + 4 * np.abs(want["rows"])), fix(e_grad)


def check_policy(rb, c, kl=0.05, T=0.8, lo=0.2, hi=0.28, **more):
    args = (c["logits"], ints(c["ids"]), c["old_logp"], c["advantage"])
    how = dict(ref_logp=c["ref_logp"] if kl else None, weight=c["weight"], temperature=T,
               clip_low=lo, clip_high=hi, kl=kl)
    loss, logp, grad = rb.policy_loss(*args, **how, **more)
    want = ref.policy(c["logits_"], c["ids"], c["old_logp_"], c["advantage_"], c["ref_logp_"],
                      c["weight_"], T, lo, hi, kl)
    e_lp, e_row, e_grad = policy_bounds(c, want, kl, T)
    within("logp", logp, want["logp"], e_lp)
    within("loss", loss, np.array([want["loss"]]), e_row.sum() + U * abs(want["loss"]))
    if grad is not None:
        # e^x below 2^-126, the least normal float, counts as 0, and so does such a product
        least = 2.0 ** -126 * (1 + np.abs(want["c"])[:, None] / T)
        within("dlogits", grad, want["dlogits"],
               e_grad + LAST[c["io"]] * np.abs(want["dlogits"]) + least)
    return loss, logp, grad


# Rows of one wave, of 256 and 1024 threads at each number of vectors and beside it; odd widths
# (rows start anywhere); few long rows in pieces.
POLICY = [(1, 1), (5, 2), (9, 7), (3, 64), (6, 255), (6, 257), (4, 511), (4, 1023), (5, 1025),
          (3, 2049), (130, 2050), (200, 4096), (150, 4099), (140, 8193), (130, 16385),
          (129, 32770), (1, 9000), (2, 50000), (3, 20011), (7, 131072), (4, 100003)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", POLICY)
def test_policy(rb, io, size):
    print(io, size, flush=True)
    check_policy(rb, policy_case(io, *size))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [66000, 140000])
def test_policy_rows_longer_than_registers(rb, io, V):
    check_policy(rb, policy_case(io, 130, V, seed=1))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(7, 100), (5, 1000), (140, 3001), (3, 30000), (3, 140000)])
@pytest.mark.parametrize("kl", [0.0, 0.5])
def test_policy_left_out_rows(rb, io, size, kl):
    """Negative ids leave their rows out, whatever these hold; ids behind the last item are NaN."""
    import torch
    c = policy_case(io, *size, seed=2)
    c["ids"][1], c["ids"][2] = -1, -(1 << 31)
    for row, v in ((1, -math.inf), (2, math.nan)):
        c["logits"][row], c["logits_"][row] = v, v
        for n in ("old_logp", "ref_logp", "advantage", "weight"):
            c[n][row], c[n + "_"][row] = math.nan, math.nan
    loss, logp, grad = check_policy(rb, c, kl=kl)
    assert not grad[1:3].any() and not logp[1:3].any()
    c["ids"][0] = size[1]
    loss, logp, grad = rb.policy_loss(c["logits"], ints(c["ids"]), c["old_logp"], c["advantage"])
    assert torch.isnan(loss).all() and torch.isnan(logp[0]) and torch.isnan(grad[0]).all()
    assert torch.isfinite(logp[3:]).all() and torch.isfinite(grad[3:]).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 100), (6, 3001), (130, 3001), (6, 30000), (6, 140000)])
def test_policy_masks(rb, io, size):
    """Masks by -inf and by the type's lowest value, all but the chosen item, all items alike at
    the lowest value, a masked chosen item; temperatures that make differences overflow."""
    import torch
    low = float(torch.finfo(dtype_of(io)).min)
    c = policy_case(io, *size, seed=3)
    ids = c["ids"]
    for row, v in ((0, -math.inf), (1, low), (2, low)):
        keep = c["logits"][row, ids[row]].clone()
        c["logits"][row] = v
        if row < 2:
            c["logits"][row, ids[row]] = keep
    c["logits_"] = host(c["logits"])
    for T in (0.8, 0.1, 30.0):  # odds of policies near the one at that temperature
        lp = ref.policy(c["logits_"], ids, c["old_logp_"], c["advantage_"], temperature=T)["logp"]
        for k, n in enumerate(("old_logp", "ref_logp")):
            c[n], c[n + "_"] = put(lp + 0.2 * np.random.default_rng(k).normal(size=size[0]))
        check_policy(rb, c, T=T)
    c["logits"][3, ids[3]] = -math.inf
    loss, logp, grad = rb.policy_loss(c["logits"], ints(ids), c["old_logp"], c["advantage"])
    assert logp[3] == -math.inf and not grad[3].any() and torch.isfinite(loss).all()
    loss, _, grad = rb.policy_loss(c["logits"], ints(ids), c["old_logp"], c["advantage"],
                                   ref_logp=c["ref_logp"], kl=0.1)
    assert loss == math.inf and torch.isfinite(grad[4:]).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 100), (6, 3001), (130, 5000), (6, 30000), (6, 140000)])
@pytest.mark.parametrize("v", [math.nan, math.inf, -math.inf])
def test_policy_rows_without_odds(rb, io, size, v):
    """A NaN, a +inf or nothing but -inf in a row that counts: NaN there and in the loss alone."""
    import torch
    c = policy_case(io, *size, seed=4)
    args = lambda: (c["logits"], ints(c["ids"]), c["old_logp"], c["advantage"])  # noqa: E731
    _, logp0, grad0 = rb.policy_loss(*args())
    if v == -math.inf:
        c["logits"][4] = v
    else:
        c["logits"][4, (c["ids"][4] + 1) % size[1]] = v
    loss, logp, grad = rb.policy_loss(*args())
    assert torch.isnan(loss).all() and torch.isnan(logp[4]) and torch.isnan(grad[4]).all()
    other = torch.arange(size[0], device="cuda") != 4
    assert torch.equal(logp[other], logp0[other]) and torch.equal(grad[other], grad0[other])


def test_policy_borders(rb):
    """Each side of the clip by the sign of the advantage; an advantage of 0 with a ratio that
    overflows has no surrogate; without a KL term ref_logp is not needed."""
    import torch
    x = torch.zeros(6, 2, device="cuda")
    half = math.log(0.5)
    old = torch.tensor([half - 1, half + 1, half - 1, half + 1, half - 200, half],
                       dtype=torch.float32, device="cuda")
    A = torch.tensor([1.0, 1.0, -1.0, -1.0, 0.0, 2.0], device="cuda")
    ids = ints([0, 0, 1, 1, 0, 0])
    each = [rb.policy_loss(x[i:i + 1], ids[i:i + 1], old[i:i + 1], A[i:i + 1]) for i in range(6)]
    e = math.e
    for i, (loss, c) in enumerate([(-1.2, 0.0), (-1 / e, -1 / e), (e, e), (0.8, 0.0), (0.0, 0.0),
                                   (-2.0, -2.0)]):
        assert abs(float(each[i][0]) - loss) < 1e-5, i
        g = each[i][2][0].tolist()
        want = [c / 2, -c / 2] if i not in (2, 3) else [-c / 2, c / 2]
        assert abs(g[0] - want[0]) < 1e-5 and abs(g[1] - want[1]) < 1e-5, i
    with pytest.raises(ValueError):
        rb.policy_loss(x, ids, old, A, kl=0.1)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 300), (140, 3003), (3, 30001), (130, 70000), (3, 140001)])
def test_policy_in_place(rb, io, size):
    """The gradient over the logits, at any alignment; another alignment than theirs; none."""
    import torch
    for offset in (0, 1, 3):
        c = policy_case(io, *size, seed=5, offset=offset)
        check_policy(rb, c)
        args = lambda: (c["logits"], ints(c["ids"]), c["old_logp"], c["advantage"])  # noqa: E731
        how = dict(ref_logp=c["ref_logp"], weight=c["weight"], temperature=0.8, clip_high=0.28,
                   kl=0.05)
        other, untouched = poisoned(size, c["logits"].dtype)
        check_policy(rb, c, out=other)
        assert untouched()
        alike = put(c["logits_"], io, offset)[0]       # lies to 16 bytes as the logits do
        loss, logp, grad = check_policy(rb, c, out=alike)
        assert grad is alike
        none = rb.policy_loss(*args(), **how, need_grad=False)
        assert none[2] is None and torch.equal(none[0], loss) and torch.equal(none[1], logp)
        inplace = rb.policy_loss(*args(), **how, out=c["logits"])
        assert inplace[2] is c["logits"] and torch.equal(inplace[2], grad)
        assert torch.equal(inplace[0], loss)


ROWS = [(6, 100), (6, 3001), (130, 5000), (6, 30000), (6, 140000)]  # each way to take a row


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_policy_rows_of_one_value(rb, io, size, T):
    """Odds are one in V, whatever the value.  All powers are alike and near one: a power is off
    by its argument, U / 2 of at most 1/32, and by 2 ulps, and a chain of n equal terms by n U at
    most, with n <= 128 a thread, 70 pieces and 16 levels between threads; ratios by that and the
    roundings of logp's other side, U |log V|, and of three products."""
    import torch
    N, V = size
    c = policy_case(io, N, V, masked=0.0)
    values = np.array([1.0, -37.5, 999.0, 1234.5, -20000.0, 123456.0])
    c["logits"][:] = torch.from_numpy(values[np.arange(N) % 6]).to(c["logits"].dtype).cuda()[:, None]
    c["logits"][:, 0] = -math.inf
    ids = 1 + c["ids"] % (V - 1)
    old = torch.full((N,), -math.log(V - 1), device="cuda")
    bar = (128 + 70 + 16 + 8 + abs(math.log(V))) * U
    for row in range(6):
        one = torch.zeros(N, device="cuda")
        one[row] = 1.0
        loss, logp, grad = rb.policy_loss(c["logits"], ints(ids), old, one, weight=one,
                                          temperature=T)
        print(row, abs(float(loss) + math.exp(-math.log(V - 1) - float(old[0]))) / bar)
        assert abs(float(loss) + math.exp(-math.log(V - 1) - float(old[0]))) <= bar
        assert np.allclose(host(logp), -math.log(V - 1), rtol=0, atol=bar + 2 * U * 12)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2048, 1000), (2048, 4000), (512, 131072)])
def test_policy_sums_lean_to_no_side(rb, io, size):
    """The mean error of logp over the rows.  Roundings of logp itself, of numbers of 16 or less, are
    within U 8 and random: their mean is within 5 sigma = 5 U 8 / sqrt(3 N) < U / 1.9 for N = 2048,
    U 1.03 for 512.  What a sum loses on one side would not go with the number of rows: small powers
    added one by one to a sum of 131,072 lose 3 U.  Half a U is left for the powers' own."""
    import torch
    N, V = size
    torch.manual_seed(0)
    x = (3 * torch.randn(N, V, device="cuda")).to(dtype_of(io))
    ids = torch.argmax(x.float() / 0.8 - torch.log(-torch.log(torch.rand(N, V, device="cuda"))), 1)
    z = torch.zeros(N, device="cuda")
    _, logp, _ = rb.policy_loss(x, ids.int(), z, z, temperature=0.8)
    want = torch.cat([torch.log_softmax(c.double() / 0.8, 1).gather(1, i[:, None])[:, 0]
                      for c, i in zip(x.split(128), ids.split(128))])
    assert float(want.abs().max()) < 16
    mean = float((logp.double() - want).mean())
    print(f"mean error {mean / U:.3f} U", flush=True)
    assert abs(mean) <= (5 * 8 / math.sqrt(3 * N) + 0.5) * U


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("size", ROWS)
def test_policy_far_logits(rb, io, size):
    """Logits of a few million, where 2^(l K) against M K would lose their differences, and rows
    that lie so low beside a running sum's first reference; a temperature near the limits."""
    import torch
    N, V = size
    for at, T in ((3e6, 1.0), (-3e6, 1.0), (-6e5, 0.8), (-4.5e5, 1.0), (3e5, 1.0), (1e30, 1e30), (-2.0, 1e-6)):
        c = policy_case(io, N, V, seed=9)
        step = max(abs(at) * 2.0 ** -20, abs(T)) if io == "f32" else max(abs(at) / 128, T)
        x = at + step * torch.round(torch.from_numpy(
            np.where(np.isinf(c["logits_"]), 0.0, c["logits_"])).cuda())
        x[c["logits"] == -math.inf] = -math.inf
        c["logits"].copy_(x)
        c["logits_"] = host(c["logits"])
        lp = ref.policy(c["logits_"], c["ids"], c["old_logp_"], c["advantage_"],
                        temperature=float(np.float32(T)))["logp"]
        for k, n in enumerate(("old_logp", "ref_logp")):
            c[n], c[n + "_"] = put(lp + 0.2 * np.random.default_rng(k).normal(size=N))
        check_policy(rb, c, T=float(np.float32(T)))


@pytest.mark.parametrize("N", [16384, 16385, 40000])
def test_policy_many_rows(rb, N):
    """The loss's sum in one launch and in two."""
    check_policy(rb, policy_case("f32", N, 3, seed=6, masked=0.0))


def test_policy_nothing(rb):
    import torch
    z = torch.zeros(0, device="cuda")
    loss, logp, grad = rb.policy_loss(torch.zeros(0, 5, device="cuda"), ints(np.zeros(0)), z, z)
    assert loss.tolist() == [0.0] and grad.shape == (0, 5)
    with pytest.raises(ValueError):
        rb.policy_loss(torch.zeros(5, 4, device="cuda").t(), ints(np.zeros(4)), z, z)


def test_policy_gradient_by_differences(rb):
    """Along random directions: 64-bit differences of the fp32 loss are no use, so the loss's own
    reference is stepped; what is compared is the library's gradient."""
    c = policy_case("f32", 6, 40, seed=7, masked=0.0)
    _, _, grad = check_policy(rb, c, T=1.0)
    r = np.random.default_rng(8)

    def loss(x):
        return ref.policy(x, c["ids"], c["old_logp_"], c["advantage_"], c["ref_logp_"],
                          c["weight_"], 1.0, 0.2, 0.28, 0.05)["loss"]
    for _ in range(5):
        v = r.normal(size=(6, 40))
        slope = (loss(c["logits_"] + 1e-5 * v) - loss(c["logits_"] - 1e-5 * v)) / 2e-5
        size = np.abs(host(grad) * v).sum()
        assert abs(slope - (host(grad) * v).sum()) <= 1e-7 + 400 * U * size


# ------------------------------------------------------------------ Muon

def muon_case(io, shapes, seed=0, kind="random", momenta=True):
    r = np.random.default_rng(seed)
    c = dict(io=io, shapes=shapes)
    for name in ("p", "g", "m"):
        c[name], c[name + "_"] = [], []
    for rows, cols in shapes:
        g = r.normal(size=(rows, cols))
        if kind == "low":  # four large directions over noise
            g = r.normal(size=(rows, 4)) @ r.normal(size=(4, cols)) + 0.3 * g
        m = r.normal(size=(rows, cols)) if momenta else np.zeros((rows, cols))
        for name, a, t in (("p", r.normal(size=(rows, cols)), io), ("g", g, io), ("m", m, "f32")):
            x, x_ = put(a, t)
            c[name].append(x)
            c[name + "_"].append(x_)
    return c


def muon_bound(norms, K, steps):
    """Of the orthogonalised update's error, Frobenius norm: see above."""
    each = 20 * (2.0 ** -20 + 4 * math.sqrt(K) * U)
    return sum(each * norms[k] * 3.9 ** (steps - k) for k in range(steps)) + 4 * U * norms[0]


def check_muon(rb, c, lr=0.5, momentum=0.9, nesterov=True, wd=0.1, steps=5, scale=None, **more):
    io = c["io"]
    opt = rb.Muon(c["p"], lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=wd,
                  steps=steps, scale=scale, state=c["m"])
    opt.step(c["g"], **more)
    for i, (rows, cols) in enumerate(c["shapes"]):
        s = max(1.0, rows / cols) ** 0.5 if scale is None else scale
        p, m, x, norms = ref.muon(c["p_"][i], c["g_"][i], c["m_"][i], lr, momentum, nesterov, wd,
                                  s, steps)
        size = momentum * np.abs(c["m_"][i]) + (1 - momentum) * np.abs(c["g_"][i])
        within(f"m {rows}x{cols}", c["m"][i], m, 4 * U * size)
        off = np.linalg.norm(host(c["p"][i]) - p)
        # m and u are off by 4 U of their terms' sizes, x by that over the norm, times the slopes
        e_u = 8 * U * np.linalg.norm(size) / max(1e-30, np.linalg.norm(
            momentum * m + (1 - momentum) * c["g_"][i] if nesterov else m)) * 3.9 ** steps
        bound = lr * s * (muon_bound(norms, max(rows, cols), steps) + e_u) + (
            4 * U + LAST[io]) * (np.linalg.norm(c["p_"][i]) + np.linalg.norm(p)) + 1e-30
        print(f"ERR p {rows}x{cols}: {off / bound:.4f} of its bound; of x "
              f"{off / (lr * s) / np.linalg.norm(x):.2e}", flush=True)
        assert off <= bound, (rows, cols)


# One element, vectors, sides around a tile of 32 and of 128, one workgroup's largest and what is
# just beyond it, tall and wide.
MUON = [(1, 1), (1, 7), (7, 1), (2, 3), (31, 33), (32, 32), (33, 31), (64, 64), (48, 96), (96, 48),
        (64, 256), (256, 64), (128, 128), (127, 129), (129, 127), (128, 136), (1, 512), (1, 513),
        (512, 32), (32, 520), (96, 160), (150, 90), (128, 256), (200, 200), (300, 130), (130, 700), (1, 3000)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", MUON)
def test_muon(rb, io, shape):
    print(io, shape, flush=True)
    check_muon(rb, muon_case(io, [shape]))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(520, 1030)], [(1030, 520)], [(1500, 1500)], [(136, 1240)] * 16,
                                    [(462, 532)] * 16, [(750, 790)] * 16, [(1160, 1320)] * 16,
                                    [(1320, 1160)] * 4, [(2500, 2500)], [(4000, 4100)],
                                    [(2001, 1999), (100, 2999), (777, 1301), (90, 80)]])
def test_muon_large(rb, io, shapes):
    """Each tile of each of the products, alone and for many matrices, against 64-bit products on
    the GPU.  Four large directions make every product weigh in the first steps already, whose
    bounds are small beside a part of a matrix that is wrong."""
    import torch
    torch.manual_seed(0)
    draw = lambda *s: torch.randn(s, device="cuda")  # noqa: E731
    for low, steps in ((True, 1), (True, 2), (False, 5)):
        p = [draw(*s).to(dtype_of(io)) * 0.01 for s in shapes]
        g = [(draw(s[0], 4) @ draw(4, s[1]) + 0.1 * draw(*s) if low else draw(*s)).to(dtype_of(io))
             for s in shapes]
        m = [0.1 * draw(*s) for s in shapes]
        before = [(a.double(), b.double()) for a, b in zip(p, m)]
        rb.Muon(p, lr=1.0, momentum=0.9, weight_decay=0.1, scale=0.3, state=m, steps=steps).step(g)
        for i, (rows, cols) in enumerate(shapes):
            p0, m0 = before[i]
            m1 = 0.9 * m0 + 0.1 * g[i].double()
            u = 0.9 * m1 + 0.1 * g[i].double()
            x = u / (u.norm() + 1e-7)
            x = x.t().contiguous() if rows > cols else x
            norms = [float(x.norm())]
            a, b, c = ref.NS
            for _ in range(steps):
                A = x @ x.t().contiguous()
                x = a * x + (b * A + c * (A @ A)) @ x
                norms.append(float(x.norm()))
            x = x.t() if rows > cols else x
            want = 0.9 * p0 - 0.3 * x
            size = 0.9 * m0.abs() + 0.1 * g[i].double().abs()
            assert ((m[i].double() - m1).abs() <= 4 * U * size).all()
            off = float((p[i].double() - want).norm())
            bound = 0.3 * (muon_bound(norms, max(rows, cols), steps)
                           + 8 * U * float(size.norm() / u.norm()) * 3.9 ** steps) \
                + (4 * U + LAST[io]) * float(p0.norm() + want.norm())
            print(f"ERR {rows}x{cols} steps {steps}: {off / bound:.4f} of its bound, which is "
                  f"{bound / 0.3 / norms[-1]:.1e} of x", flush=True)
            assert off <= bound, (rows, cols)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_muon_unaligned(rb, io, offset):
    """Matrices that start anywhere."""
    shapes = [(33, 40), (128, 128), (40, 33), (140, 260), (261, 140)]
    c = muon_case(io, shapes, seed=7)
    for name, t in (("p", io), ("g", io), ("m", "f32")):
        c[name] = [put(a, t, offset)[0] for a in c[name + "_"]]
    check_muon(rb, c)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_muon_list(rb, io):
    """Many matrices of all sizes in one call, more than a launch takes of either kind."""
    shapes = [MUON[i % len(MUON)] for i in range(100)] + [(7 + i, 5) for i in range(60)]
    check_muon(rb, muon_case(io, shapes, seed=1))


@pytest.mark.parametrize("kind", ["random", "low"])
@pytest.mark.parametrize("shape", [(60, 100), (128, 128), (140, 260), (520, 390)])
def test_muon_update_itself(rb, kind, shape):
    """Parameters of zero, no decay and a rate of one: the update as it is."""
    import torch
    c = muon_case("f32", [shape], seed=2, kind=kind, momenta=False)
    c["p"] = [torch.zeros_like(c["p"][0])]
    c["p_"] = [np.zeros(shape)]
    for nesterov in (False, True):
        for steps in (1, 2, 5, 7):
            c["p"][0].zero_()
            c["m"][0].zero_()
            check_muon(rb, c, lr=1.0, wd=0.0, nesterov=nesterov, steps=steps, scale=0.25)


def test_muon_zero_and_nan(rb):
    """Zeros leave X = 0; a NaN or an infinity spoils its own matrix and no other."""
    import torch
    shapes = [(40, 50), (200, 300), (40, 50), (200, 300), (40, 50), (200, 300)]
    c = muon_case("f32", shapes, seed=3)
    for i in (0, 1):
        c["g"][i].zero_(), c["m"][i].zero_()
    c["g"][2][3, 4] = math.nan
    c["g"][3][100, 7] = math.inf
    opt = rb.Muon(c["p"], lr=0.1, weight_decay=0.5, state=c["m"])
    opt.step(c["g"])
    for i in (0, 1):
        assert np.allclose(host(c["p"][i]), c["p_"][i] * 0.95, rtol=1e-6)
    assert torch.isnan(c["p"][2]).all() and torch.isnan(c["p"][3]).all()
    assert all(torch.isfinite(c["p"][i]).all() for i in (4, 5))


@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-12, 1e12, 1e30, 5e37])
def test_muon_scales(rb, size):
    """The update hangs on the gradient's direction alone, as far as eps lets it: its norm is
    formed in 64 bits, so no square over- or underflows."""
    c = muon_case("f32", [(40, 50), (200, 150)], seed=4, momenta=False)
    for i in range(2):
        c["g"][i], c["g_"][i] = put(c["g_"][i] * size)
    opt = rb.Muon(c["p"], lr=1.0, momentum=0.0, nesterov=False, eps=1e-300, state=c["m"])
    opt.step(c["g"])
    for i in range(2):
        x, norms = ref.newton_schulz(c["g_"][i] / np.linalg.norm(c["g_"][i]), 5)
        rows, cols = c["shapes"][i]
        off = np.linalg.norm(c["p_"][i] - host(c["p"][i]) - max(1, rows / cols) ** 0.5 * x)
        assert off <= max(1, rows / cols) ** 0.5 * (muon_bound(norms, 200, 5) + 8 * U * 3.9 ** 5) \
            + 4 * U * np.linalg.norm(c["p_"][i])


def test_muon_writes_its_matrices_only(rb):
    import torch
    for io in ("f32", "bf16"):
        for shape in ((5, 9), (45, 33), (129, 131), (300, 129)):
            p, p_ok = poisoned(shape, dtype_of(io))
            m, m_ok = poisoned(shape, torch.float32)
            p.normal_(), m.zero_()
            g = torch.randn(shape, device="cuda").to(dtype_of(io))
            before = g.clone()
            rb.Muon([p], state=[m]).step([g])
            torch.cuda.synchronize()
            assert p_ok() and m_ok() and torch.equal(g, before)
            assert torch.isfinite(p).all()


def test_muon_shared_gradient(rb):
    """One gradient for two matrices, small and large ones."""
    import torch
    for shape in ((50, 40), (300, 200)):
        p = [torch.randn(shape, device="cuda")]
        p.append(p[0].clone())
        g = torch.randn(shape, device="cuda")
        before = p[0].clone()
        rb.Muon(p).step([g, g])
        assert torch.equal(p[0], p[1]) and not torch.equal(p[0], before)


def test_muon_binding(rb):
    """States that are made, rates of a step, memory that was replaced, refusals."""
    import torch
    p = [torch.randn(6, 8, device="cuda"), torch.randn(200, 40, device="cuda")]
    g = [torch.randn_like(x) for x in p]
    q = [x.clone() for x in p]
    opt, two = rb.Muon(p, lr=0.1), rb.Muon(q, lr=0.3)
    for k in range(3):
        opt.step(g)
        if k == 1:  # other memory with the same values
            two.m[1] = two.m[1].clone()
            q[0].data = q[0].data.clone()
        two.step(g, lr=0.1)
    assert all(torch.equal(a, b) for a, b in zip(p, q))
    with pytest.raises(ValueError):
        opt.step(g[:1])
    with pytest.raises(ValueError):
        opt.step([g[0], g[1].t().contiguous()])
    with pytest.raises(ValueError):
        opt.step([g[0], g[1].bfloat16()])
    with pytest.raises(ValueError):
        rb.Muon([torch.randn(5, device="cuda")])
    with pytest.raises(ValueError):
        rb.Muon(p, state=[opt.m[0]])
    with pytest.raises(ValueError):
        rb.Muon([p[1].t()])
    with pytest.raises(ValueError):
        rb.Muon(p, weight_decay=[0.1])
    with pytest.raises(rb.RecblrError):
        rb.Muon([p[0], p[0]]).step([g[0], g[0]])
    rb.Muon([torch.empty(0, 5, device="cuda")]).step([torch.empty(0, 5, device="cuda")])


# ------------------------------------------------------------------ streams, graphs, devices

def passes(rb, io, seed=0):
    """name -> (call, its outputs' clones): one pass of every operator, few and many rows."""
    import torch
    out = {}
    for N in (100, 3000, 12000):
        c = embed_case(io, N, 300, 64, seed=seed)
        ids = ints(c["ids"])
        out[f"embed {N}"] = lambda c=c, ids=ids: [
            rb.embed(c["table"], ids, scale=2.0, pad_id=0),
            rb.embed_backward(ids, c["dout"], 300, pad_id=0)]
    for D in (64, 33):
        c = qk_case(io, (5, 40), 2, 1, D, D // 2 * 2, far=100, seed=seed)
        pos = ints(c["pos"])
        how = lambda c=c, pos=pos: dict(wq=c["wq"], wk=c["wk"], positions=pos)  # noqa: E731
        out[f"qk {D}"] = lambda c=c, how=how: [
            *rb.qk_norm(c["q"], c["k"], **how()),
            *rb.qk_norm_backward(c["q"], c["k"], c["dq"], c["dk"], **how()).values()]
    for size in ((40, 50), (130, 3000), (3, 30000), (3, 140000)):
        c = policy_case(io, *size, seed=seed)
        ids = ints(c["ids"])
        out[f"policy {size}"] = lambda c=c, ids=ids: list(rb.policy_loss(
            c["logits"], ids, c["old_logp"], c["advantage"], ref_logp=c["ref_logp"], kl=0.1))
    c = muon_case(io, [(40, 50), (200, 300), (300, 140)], seed=seed)
    start = [t.clone() for t in c["p"] + c["m"]]
    opt = rb.Muon(c["p"], state=c["m"])

    def muon():
        for t, s in zip(c["p"] + c["m"], start):
            t.copy_(s)
        opt.step(c["g"])
        return c["p"] + c["m"]
    out["muon"] = muon
    return out


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_repeats_and_graphs(rb, io):
    """Bitwise repeatable; captured graphs, two in one pool, give the eager results on every
    replay, with other work in between."""
    import torch
    for name, run in passes(rb, io).items():
        print(name, flush=True)
        want = [t.clone() for t in run()]
        assert all(torch.equal(a, b) for a, b in zip(want, run())), name
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        with torch.cuda.graph(other, pool=graph.pool()):
            run()
        for _ in range(3):
            for t in got:
                t.fill_(7.0)
            torch.cuda.synchronize()
            other.replay()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), name
            run()
            torch.cuda.synchronize()


def test_two_streams(rb):
    """Calls on two streams at once, and through the stream argument, give what one alone gives."""
    import torch
    runs = passes(rb, "f32"), passes(rb, "f32", seed=1)
    want = [{n: [t.clone() for t in f()] for n, f in r.items()} for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = [{}, {}]
    for name in runs[0]:
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k][name] = runs[k][name]()
    torch.cuda.synchronize()
    for k in range(2):
        for name, ts in want[k].items():
            assert all(torch.equal(a, b) for a, b in zip(ts, got[k][name])), name
    c = embed_case("f32", 6000, 300, 64)
    ids, s = ints(c["ids"]), torch.cuda.Stream()
    torch.cuda.synchronize()
    d = rb.embed_backward(ids, c["dout"], 300, stream=s)
    s.synchronize()
    assert torch.equal(d, rb.embed_backward(ids, c["dout"], 300))


# ------------------------------------------------------------------ large tensors

def test_embed_beyond_31_bits(rb):
    """A table of more than 2^31 elements: rows at its end, looked up and added to."""
    import torch
    V, D = 9_000_001, 256
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    ids = np.array([0, V - 1, 8_500_000, V - 1, 8_388_608, 8_388_607] + [V - 2] * 1500)
    vals = torch.arange(1, 7, device="cuda")
    for i, v in zip(ids[:6], vals):
        table[int(i)] = v
    out = rb.embed(table, ints(ids))
    want = [1, 4, 3, 4, 5, 6]
    assert [float(x) for x in out[:6, 200]] == want
    dout = torch.ones(len(ids), D, dtype=torch.bfloat16, device="cuda")
    d = rb.embed_backward(ints(ids), dout, V, into=table)
    assert float(d[V - 1, 255]) == 6 and float(d[8_500_000, 0]) == 4 and float(d[V - 2, 9]) == 1504  # 1500 as bf16
    assert float(d[8_388_606].abs().max()) == 0
    many = np.concatenate([ids, [V - 3] * 5000])      # sorted
    d = rb.embed_backward(ints(many), torch.ones(len(many), D, dtype=torch.bfloat16,
                                                 device="cuda"), V)
    assert float(d[V - 1, 255]) == 2 and float(d[V - 3, 7]) == 4992  # 5000 as bf16
    assert float(d[8_500_000, 0]) == 1 and float(d[8_388_606].abs().max()) == 0
    few = rb.embed_backward(ints(ids[:6]), dout[:6], V)
    assert float(few[V - 1, 3]) == 2 and float(few.float().sum()) == 6 * D


def test_policy_beyond_31_bits(rb):
    """Rows that start behind 2^31 elements, each way of taking a row."""
    import torch
    for N, V in ((40000, 60000), (2200000, 1000), (140, 16000000)):
        x = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
        ids = torch.full((N,), -1, dtype=torch.int32, device="cuda")
        ids[-1], x[-1, V // 2] = V // 2, 4.0
        z = torch.zeros(N, device="cuda")
        one = torch.ones(N, device="cuda")
        loss, logp, grad = rb.policy_loss(x, ids, z, one)
        p = math.exp(4.0) / (math.exp(4.0) + V - 1)
        assert abs(float(logp[-1]) - math.log(p)) < 1e-4 and abs(float(loss) + p) < 1e-4 * p
        g = grad[-1].float()
        assert abs(float(g[V // 2]) + p * (1 - p)) <= 0.01 * p  # bf16
        assert abs(float(g.double().sum())) <= 0.01 * p and not grad[0].any()
        del x, grad, g


# ------------------------------------------------------------------ together

def test_training_step_of_a_delta_rule_model(rb):
    """A step of a one-layer model: items looked up, projected, queries and keys normalised and
    rotated, the gated delta rule, logits by the item table, an item sampled, the policy loss, all
    gradients, the table's from both of its uses, and both optimisers.  Gradients against autograd
    in 64 bits of the same formulas.

    Eight stages stand behind one another, each off by at most 6 (D + 64) U of its size (the
    delta rule's own bar, the largest of them): 48 * 128 U."""
    import torch
    from helpers import floored_rel_err
    torch.manual_seed(0)
    B, L, V, D, H = 6, 70, 90, 64, 2
    Dk = Dv = D // H
    dev = "cuda"
    table = 0.5 * torch.randn(V, D, device=dev)
    ws = [torch.randn(D, D, device=dev) * D ** -0.5 for _ in range(3)]
    wq, wk = 0.5 + torch.rand(Dk, device=dev), 0.5 + torch.rand(Dk, device=dev)
    ids = ints(np.random.default_rng(1).integers(1, V, (B, L)))
    ids[0, :20] = 0                                   # padding
    g = (-0.2 * torch.rand(B, L, H, device=dev)).masked_fill((ids == 0)[..., None], 0)
    beta = torch.rand(B, L, H, device=dev).masked_fill((ids == 0)[..., None], 0)
    how = dict(wq=wq, wk=wk, norm="rms", eps=1e-5)

    x = rb.embed(table, ids, scale=2.0, pad_id=0)
    q, k, v = ((x @ w).view(B, L, H, Dk) for w in ws)
    qn, kn = rb.qk_norm(q, k, **how)
    kn = kn * 0.1                                     # keys shorter than one, as the rule needs
    o, _, states = rb.delta_forward(qn, kn, v.contiguous(), g, beta, keep_states=True)
    h = o[:, -1].reshape(B, D)
    logits = h @ table.t()
    logits[:, 0] = -math.inf
    u = torch.rand(B, device=dev)
    chosen, prob = rb.sample(logits, u)
    A = torch.randn(B, device=dev)
    old = torch.log(prob) - 0.1
    loss, logp, dl = rb.policy_loss(logits, chosen, old, A, ref_logp=old, kl=0.1)
    dh = dl @ table
    dtable = dl.t() @ h
    do = torch.zeros_like(o)
    do[:, -1] = dh.view(B, H, Dv)
    d = rb.delta_backward(qn, kn, v.contiguous(), g, beta, states, do, need_dh0=False)
    n = rb.qk_norm_backward(q, k, d["dq"], d["dk"] * 0.1, **how)
    flat = lambda t: t.reshape(B * L, D)  # noqa: E731
    dws = [flat(x).t() @ flat(t) for t in (n["dq"], n["dk"], d["dv"])]
    dx = sum(flat(t) @ w.t() for t, w in zip((n["dq"], n["dk"], d["dv"]), ws)).view(B, L, D)
    rb.embed_backward(ids, dx, V, scale=2.0, pad_id=0, into=dtable)

    # The same in 64 bits, on the CPU, step by step.
    leaf = lambda t: t.detach().double().cpu().requires_grad_()  # noqa: E731
    T_, W_, wq_, wk_ = leaf(table), [leaf(w) for w in ws], leaf(wq), leaf(wk)
    i_, g_, b_ = ids.cpu().long(), g.double().cpu(), beta.double().cpu()
    x_ = 2.0 * T_[i_] * (i_ != 0)[..., None]
    q_, k_, v_ = ((x_ @ w).view(B, L, H, Dk) for w in W_)
    t = torch.arange(L, dtype=torch.float64)[None, :, None, None] * (
        10000.0 ** (-2.0 * torch.arange(Dk // 2, dtype=torch.float64) / Dk))

    def normed(y, w):
        y = w * y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5)
        a, b = y[..., :Dk // 2], y[..., Dk // 2:]
        return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], -1)
    q_, k_ = normed(q_, wq_), 0.1 * normed(k_, wk_)
    S = torch.zeros(B, H, Dk, Dv, dtype=torch.float64)
    for s in range(L):
        S = S * g_[:, s].exp()[..., None, None]
        e = v_[:, s] - (S * k_[:, s, :, :, None]).sum(2)
        S = S + k_[:, s, :, :, None] * (b_[:, s, :, None] * e)[:, :, None]
    o_ = (S * q_[:, -1, :, :, None]).sum(2) * Dk ** -0.5
    l_ = o_.reshape(B, D) @ T_.t()
    l_ = l_.masked_fill(torch.arange(V) == 0, -math.inf)
    lp = torch.log_softmax(l_, 1).gather(1, chosen.cpu().long()[:, None])[:, 0]
    r, dd = torch.exp(lp - old.double().cpu()), old.double().cpu() - lp
    A_ = A.double().cpu()
    loss_ = (-torch.minimum(r * A_, r.clamp(0.8, 1.2) * A_) + 0.1 * (dd.exp() - dd - 1)).sum()
    loss_.backward()
    bar = 48 * 128 * U
    for name, got, want in (("loss", loss, loss_.detach().reshape(1)), ("logp", logp, lp.detach()),
                            ("table", dtable, T_.grad), ("wq", n["dwq"], wq_.grad),
                            ("wk", n["dwk"], wk_.grad),
                            *((f"W{j}", dws[j], W_[j].grad) for j in range(3))):
        err = floored_rel_err(host(got), want.numpy())
        print(f"ERR {name}: {err:.2e} of {bar:.2e}", flush=True)
        assert err <= bar, name

    before = [w.clone() for w in ws]
    muon, adam = rb.Muon(ws, lr=0.02, weight_decay=0.1), rb.AdamW([table, wq, wk])
    muon.step(dws)
    adam.step([dtable, n["dwq"], n["dwk"]])
    for w, b, dw in zip(ws, before, dws):
        want, _, _, norms = ref.muon(host(b), host(dw), np.zeros((D, D)), 0.02, 0.95, True, 0.1, 1.0)
        off = np.linalg.norm(host(w) - want)
        assert off <= 0.02 * (muon_bound(norms, D, 5) + 8 * U * 3.9 ** 5) + 8 * U * np.linalg.norm(
            want)
