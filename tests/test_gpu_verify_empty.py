"""agzo_verify_drafts where no sequence has a row: what is counted is zero all the same, as for a sequence without rows beside others."""
import pytest
import torch

from paper_2601_17261_amd import binding
from test_gpu_cache import ints

pytestmark = pytest.mark.gpu


def nothing(dtype=torch.float32):
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    return torch.empty(0, 300, dtype=dtype, device="cuda"), e, torch.empty(0, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_seq", [1, 3, 256, 257, 65535])
def test_no_rows_at_all(n_seq, dtype):
    p, e, u = nothing(dtype)
    cu, counts = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda"), torch.full((n_seq + 5,), 77, dtype=torch.int32, device="cuda")
    ctx = binding.Context()
    for q, parents in ((None, None), (p, None), (None, e)):
        counts.fill_(77)
        ctx.verify_drafts(p, q, e, u, cu, e, e.clone(), counts[:n_seq], parents=parents)
        assert (counts[:n_seq] == 0).all() and (counts[n_seq:] == 77).all()
    # offsets that are none of a list without rows
    counts.fill_(77)
    ctx.verify_drafts(p, None, e, u, cu + 3, e, e.clone(), counts[:n_seq])
    assert (counts[:n_seq] == 0).all() and (counts[n_seq:] == 77).all()
    ctx.check()


def test_no_sequences():
    p, e, u = nothing()
    ctx = binding.Context()
    ctx.verify_drafts(p, None, e, u, ints([0]), e, e.clone(), e.clone())
    out = [torch.full((2,), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
    ctx.verify_drafts(torch.rand(2, 300, device="cuda"), None, ints([1, 2]), torch.rand(2, device="cuda"), ints([0]), *out, e.clone())
    assert all(o.tolist() == [77, 77] for o in out)                  # rows of no sequence
    ctx.check()


def test_captured_and_replayed():
    """by a context that has no workspace yet"""
    side = torch.cuda.Stream()
    ctx = binding.Context(side)
    p, e, u = nothing()
    cu, counts, rows = ints([0] * 4), ints([77] * 3), e.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.verify_drafts(p, None, e, u, cu, e, rows, counts)
    for i in range(3):
        counts.fill_(5 + i)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert counts.tolist() == [0, 0, 0]
