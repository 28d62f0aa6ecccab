"""The head's gradient on the ways that sum in shares and in pieces: weights' gradients in shares of the tokens, ragged tiles of the inputs' gradients that are
added to for a further piece of the outputs (the last of them smaller), each against 64 bits with the bounds of test_gpu_ce_gradient."""
import pytest
import torch

from paper_2601_17261_amd import binding
from test_gpu_ce_gradient import check, exact, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d,v", [(2048, 512, 1000), (1500, 264, 4001), (1100, 256, 300), (4096, 1024, 2000), (961, 256, 256), (1500, 256, 4000)])
def test_weights_gradients_in_shares_of_the_tokens(n, d, v):
    w, x, ids = make(n + v, n, d, v)
    check(run(binding.Context(), w, x, ids), exact(w, x, ids))


@pytest.mark.parametrize("n,d,v", [(300, 16384, 17003), (257, 8200, 33001), (700, 16392, 16500)])
def test_inputs_gradients_of_several_pieces_in_ragged_tiles(n, d, v):
    w, x, ids = make(n + v, n, d, v)
    got = run(binding.Context(), w, x, ids)
    check(got, exact(w, x, ids))
    one = run(binding.Context(), w, x, ids, dw=False)
    assert torch.equal(one["dx"], got["dx"])


@pytest.mark.parametrize("n,d,v", [(7, 64, 500), (31, 264, 3001), (50, 128, 900), (120, 512, 2000), (200, 256, 5000), (70, 256, 30000), (600, 200, 700), (1500, 264, 4001)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_that_are_not_counted_have_no_part_on_any_way(n, d, v, value):
    ctx = binding.Context()
    w, x, ids = make(n, n, d, v)
    ids[2], ids[n - 1] = -1, v
    clean = run(ctx, w, x, ids)
    y = x.clone()
    y[2], y[n - 1] = value, value
    got = run(ctx, w, y, ids)
    assert not got["dx"][2].any() and not got["dx"][n - 1].any() and all(torch.equal(got[name], clean[name]) for name in ("dx", "dw", "loss"))
