"""Sizes and shapes of the training operators at which a launch, a loop or a sum behaves in another way (needs an MI355X)."""
import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import BF16, DEV, F16, F32, count

pytestmark = pytest.mark.gpu


def test_gradient_of_more_than_2_30_ids():
    """The blocks that add up take three launches.  2^20 ones to a row: every sum is exact; the last row has 77."""
    each, last = 2 ** 20, 77
    n = 2 ** 30 + 5 * each + last
    rows = n // each + 1
    ids = torch.arange(n - 1, -1, -1, device=DEV).div_(each, rounding_mode="floor").to(torch.int32)
    dy = torch.ones((n, 1), dtype=F16, device=DEV)
    want = torch.full((rows, 1), float(each), device=DEV)
    want[rows - 1] = last
    ws = smfg.embedding_grad_workspace(n, rows, 1)
    g = torch.full((rows, 1), 9.0, device=DEV)
    smfg.embedding_grad(ids, count(n), n, dy, g, ws)
    assert torch.equal(g, want)
    smfg.embedding_grad(ids, count(n), n, dy, g, ws, scale=2.0, accumulate=True)
    assert torch.equal(g, 3 * want)
    row_ids, num = torch.full((n,), -7, dtype=torch.int32, device=DEV), count(-1)
    c = torch.full((n, 1), 5.0, dtype=F16, device=DEV)
    smfg.embedding_grad_rows(ids, count(n), n, dy, rows, row_ids, num, c, ws, scale=2.0 ** -12)
    assert int(num) == rows and torch.equal(row_ids[:rows].cpu(), torch.arange(rows, dtype=torch.int32)) and bool((row_ids[rows:] == -7).all())
    assert torch.equal(c[:rows], (want * 2.0 ** -12).half()) and bool((c[rows:] == 5).all())


@pytest.mark.parametrize("n", [0, 3, 300])
def test_gradient_of_a_table_of_2_31_rows(n):
    """All rows that no id names become zeros, beside up to 256 ids by more blocks than a launch has."""
    rows, dim = 2 ** 31 - 1, 2
    at = torch.tensor([0, 2 ** 30 + 1, rows - 1], device=DEV)
    g = torch.ones((rows, dim), dtype=F16, device=DEV)
    ids = at[torch.arange(max(1, n), device=DEV) % 3]
    dy = torch.ones((max(1, n), dim), dtype=F16, device=DEV)
    smfg.embedding_grad(ids, count(n), n, dy, g, smfg.embedding_grad_workspace(n, rows, dim))
    assert torch.equal(g[at], torch.full((3, dim), n / 3, dtype=F16, device=DEV))
    g[at] = 0
    for piece in g.split(2 ** 28):
        assert int(torch.count_nonzero(piece)) == 0
