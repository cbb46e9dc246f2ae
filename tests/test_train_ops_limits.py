"""What the operators around the layer ask of memory and of torch, without a GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rb():
    from paper_2406_12580_amd import recblr
    return recblr


def muon_bytes(rb, shapes, io=0):
    t = (rb.MuonTensor * len(shapes))()
    for entry, (rows, cols) in zip(t, shapes):
        entry.rows, entry.cols = rows, cols
    return rb.recblr_muon_workspace_size(t, len(shapes), io)


def test_muon_workspace_is_that_of_matrices_worked_on_together(rb):
    """Sixteen at most: a longer list needs the most that sixteen in a row need of those that need
    any, and does not grow."""
    big = (4096, 4096)
    assert muon_bytes(rb, [big] * 100) == muon_bytes(rb, [big] * 16) == 16 * muon_bytes(rb, [big])
    shapes = [(300 + 10 * i, 500) for i in range(40)]
    each = [muon_bytes(rb, [s]) for s in shapes]
    want = max(sum(each[i:i + 16]) for i in (0, 16, 32))
    assert muon_bytes(rb, shapes) == want
    mixed = [s for x in shapes for s in (x, (64, 64), (0, 5000))]  # and those between need none
    assert muon_bytes(rb, mixed) == want


def test_import_under_a_torch_without_the_stream_call():
    """A torch built without GPUs lacks the call that gives a device's stream: the module is there all
    the same, for entry points that take addresses, and wrappers say that tensors are not on a GPU."""
    code = ("import torch\n"
            "if hasattr(torch._C, '_cuda_getCurrentRawStream'):\n"
            "    del torch._C._cuda_getCurrentRawStream\n"
            "from paper_2406_12580_amd import recblr\n"
            "assert recblr.recblr_status_string(0)\n"
            "try:\n"
            "    recblr.embed(torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32))\n"
            "except ValueError as e:\n"
            "    assert 'on the GPU' in str(e)\n"
            "else:\n"
            "    raise AssertionError\n")
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                         cwd=ROOT)
    assert res.returncode == 0, res.stderr
