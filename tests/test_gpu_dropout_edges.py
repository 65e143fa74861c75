"""The dropout mask at its edges against the oracle: a rate that rounds to 2^32 steps, above every word."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_14806_amd import dropout as D
from tests.gpu_util import host, needs_gpu

# with seed 1 and offset 0 the word of this element is 2^32 - 1 (the largest; one in 2^32 is)
SEED, LAST = 1, 6845800136


def place_of(channels, n_cols, rows, cols):
    """A tile around that element: (row0, col0) and the element's index in it."""
    r, rest = divmod(LAST, n_cols * channels)
    j, c = divmod(rest, channels)
    row0, col0 = r - rows // 2, max(0, min(j - cols // 2, n_cols - cols))
    return dict(row0=row0, col0=col0, n_cols=n_cols), (r - row0, j - col0, c)


@pytest.mark.parametrize("channels,n_cols", [(8, 1000), (12, 97), (7, 101), (1, 5)])
def test_the_largest_word(channels, n_cols):
    place, at = place_of(channels, n_cols, 3, 5)
    m = oracle.keep(3, 5, channels, 1 - 2.0 ** -32, SEED, 0, "none", **place)
    assert m[at] and m.sum() == 1
    assert not oracle.keep(3, 5, channels, 1 - 2.0 ** -40, SEED, 0, "none", **place).any()


@pytest.mark.gpu
@needs_gpu
@pytest.mark.parametrize("channels,n_cols", [(8, 1000), (12, 97), (7, 101), (1, 5)])
@pytest.mark.parametrize("p", [0.0, 1 - 2.0 ** -32, 1 - 2.0 ** -33, 1 - 2.0 ** -40, 1 - 2.0 ** -53])
def test_rates_next_to_one(p, channels, n_cols):
    """2^32 p rounds to 2^32 - 1 (kept: the largest word alone) or to 2^32 (nothing)."""
    place, at = place_of(channels, n_cols, 3, 5)
    x = torch.full((3, 5, channels), 0.5, device="cuda")
    z = torch.ones_like(x)
    keep = oracle.keep(3, 5, channels, p, SEED, 0, "none", **place)
    assert bool(keep[at]) == (round(p * 2 ** 32) < 2 ** 32)
    term = np.where(keep, 0.5 / (1 - p), 0.0)
    # powers of two: exact but for the sum's own rounding
    assert np.abs(host(D.dropout_add(x, z, p, SEED, 0, **place)) - (1 + term)).max() <= 2.0 ** -24 * (1 + term.max())
    assert np.array_equal(host(D.dropout_backward(x, p, SEED, 0, **place)), term)


@pytest.mark.gpu
@needs_gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_residual_rows_of_a_larger_tensor(dtype):
    """x and residual both tiles of larger tensors, with and without an out: the result of contiguous copies."""
    g = torch.Generator().manual_seed(4)
    big, wide = (torch.randn((9, n, 16), generator=g).to(dtype).cuda() for n in (20, 31))
    x, z = big[2:7, 4:15], wide[1:6, 7:18]
    before = wide.clone()
    place = dict(row0=2, col0=4, n_cols=20)
    want = D.dropout_add(x.contiguous(), z.contiguous(), 0.3, 5, 1, "columns", **place)
    got = D.dropout_add(x, z, 0.3, 5, 1, "columns", **place)
    assert got.is_contiguous() and torch.equal(got, want) and torch.equal(wide, before)
    assert D.dropout_add(x, z, 0.3, 5, 1, "columns", out=z, **place) is z and torch.equal(z, want)
    before[1:6, 7:18] = want
    assert torch.equal(wide, before)                           # and nothing around it
    with pytest.raises(ValueError, match="row stride"):
        D.dropout_add(x, z, 0.3, out=torch.empty_like(want))
    one = wide[3:4, 7:18]                                      # a single row has no stride
    assert torch.equal(D.dropout_add(big[3:4, 4:15], one, 0.3, 5), D.dropout_add(big[3:4, 4:15].contiguous(), one.contiguous(), 0.3, 5))


@pytest.mark.gpu
@needs_gpu
def test_replays_keep_the_captured_mask():
    """Seed and offset are the captured call's own, as documented."""
    x = torch.ones((30, 30, 128), device="cuda")
    D.dropout_add(x, None, 0.5, 1, 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = D.dropout_add(x, None, 0.5, 1, 2)
    for i in range(3):
        graph.replay()
        other = D.dropout_add(x, None, 0.5, 1, 3 + i)
        torch.cuda.synchronize()
        assert torch.equal(y, D.dropout_add(x, None, 0.5, 1, 2)) and not torch.equal(y, other)
