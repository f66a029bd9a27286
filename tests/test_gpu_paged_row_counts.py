"""qattn_paged_f16 over tiles whose last wavefronts have few rows or none, with
NaN in every row of the queries that is no token of the batch."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2607_00501_amd import binding as B
from tests.paged_cases import assert_close, batch, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 1), (128, 6, 2)])
@pytest.mark.parametrize("prefix_pages", [0, 5])
@pytest.mark.parametrize("rows", [17, 31, 32, 33, 48, 63, 65, 96, 97, 127, 129, 160, 161, 255])
def test_rows_of_the_last_tile(rows, prefix_pages, d, hq, hkv):
    """rows of a KV head in the batch's first request (rounded up to whole tokens),
    after a cache of some blocks, beside a single token and one row more."""
    group = hq // hkv
    new = [-(-rows // group), 1, 2]
    kv = [16 * prefix_pages + 200 + new[0], 16 * prefix_pages + 90, 16 * prefix_pages + 2]
    args = batch(rows + d, hq, hkv, d, 16, kv, new, prefix_pages=prefix_pages, pad=5)
    n = sum(new)
    args[0][n:] = np.nan
    q, k, v, tables, offsets, lens, prefix = on_gpu(*args)
    scale = np.float32(1 / np.sqrt(d))
    out = B.qattn_paged_f16(q, k, v, tables, offsets, lens, float(scale), prefix=prefix,
                            out=torch.full((n + 5, hq * d), 5.0, dtype=torch.float16, device="cuda")).cpu().numpy()
    ref, size = PO.paged_attention(args[0][:n], *args[1:6], scale, args[6])
    assert_close(out[:n].reshape(n, hq, d), ref, size, d)
    assert (out[n:] == 5.0).all()
