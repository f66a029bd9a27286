"""qdec_argmax_rows: every row as qdec_argmax gives it."""

import pytest
import torch

from oracle import qmatmul_oracle as O
from paper_2607_00501_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n", [(1, 1), (3, 1), (2, 63), (300, 255), (7, 4096), (5, 4097), (33, 32001),
                                    (64, 151936), (2, 1500000), (32768, 3)])
def test_rows_match_the_oracle(rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    x = torch.randint(-40, 40, (rows, n), generator=g, device="cuda").float()     # ties in every row
    got = B.qdec_argmax_rows(x)
    top = x.amax(1, keepdim=True)
    want = torch.where(x == top, torch.arange(n, device="cuda"), n).amin(1)
    assert torch.equal(got.long(), want)
    for r in range(min(rows, 3)):
        assert got[r].item() == B.qdec_argmax(x[r].contiguous()).item()


def test_odd_values():
    inf, nan = float("inf"), float("nan")
    rows = [[nan] * 6, [nan, -inf, nan, -inf, nan, nan], [-inf] * 6, [1, inf, nan, inf, 2, 3], [0.0, -0.0, -1, 0, 0, -2],
            [-0.0, 0.0, -1, 0, 0, -2], [-1, nan, -2, -1, -3, -1], [-3.4e38, -3.4028235e38, nan, nan, nan, nan]]
    x = torch.tensor(rows, device="cuda")
    assert B.qdec_argmax_rows(x).tolist() == [O.greedy_token(r) for r in x.cpu().numpy()]
    wide = torch.full((8, 9000), nan, device="cuda")      # the same over several workgroups of a row
    wide[:, 8000:8006] = x
    assert B.qdec_argmax_rows(wide).tolist() == [O.greedy_token(r) for r in wide.cpu().numpy()]


def test_rows_past_32_bits():
    x = torch.zeros((16400, 262147), dtype=torch.float32, device="cuda")          # 4.3e9 logits
    x[-1, 262146], x[0, 5], x[16390, 70000] = 1, 1, 1
    got = B.qdec_argmax_rows(x)
    assert got[-1].item() == 262146 and got[0].item() == 5 and got[16390].item() == 70000 and got[1].item() == 0


@pytest.mark.parametrize("rows", [1, 102, 103])
@pytest.mark.parametrize("n", [49152, 49153, 60001])
def test_both_ways_at_their_border(rows, n):
    """Rows that begin at every place of 16 bytes, ties, NaNs and infinities at the ends."""
    g = torch.Generator(device="cuda").manual_seed(n + rows)
    inf, nan = float("inf"), float("nan")
    for shift in range(4):
        x = torch.randint(-900, 900, (rows * n + shift,), generator=g, device="cuda").float()[shift:].view(rows, n)
        x[0, :], x[0, n - 1], x[-1, 0] = nan, -inf, inf
        got = B.qdec_argmax_rows(x)
        clean = torch.where(x.isnan(), -inf, x)
        best = (clean == clean.amax(1, keepdim=True)) & ~x.isnan()
        assert torch.equal(got.long(), torch.where(best, torch.arange(n, device="cuda"), n).amin(1))
