"""qattn_paged_f16: infinite and NaN values at keys that rows see, wherever they lie."""

import numpy as np
import pytest

from oracle import paged_oracle as PO
from paper_2607_00501_amd import binding as B
from tests.paged_cases import batch, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("d,hq,hkv,new,prefix_pages", [
    (64, 4, 1, 1, 0), (128, 16, 8, 1, 0), (64, 4, 1, 40, 0), (128, 6, 2, 90, 0), (64, 40, 2, 1, 0), (128, 16, 8, 1, 6),
    (64, 8, 2, 50, 6)])
def test_infinite_values_that_rows_see(value, d, hq, hkv, new, prefix_pages):
    """The first key, the borders and the middle of the blocks that every row sees, the
    last blocks: with a weight like the others' the dimension is as in 64 bits, with one
    of 2^-40 of them and less it is infinite or NaN; all else is as without it."""
    kv, group = [200 + new, 100 + 16 * prefix_pages], hq // hkv
    for key in (0, 31, 32, 63, 64, 100, 130, 191, 192, 199):
        for small in (False, True):
            args = list(batch(d + key, hq, hkv, d, 16, kv, [new, 1], prefix_pages=prefix_pages, poison=np.nan))
            q, k, v, tables = args[:4]
            page, at = tables[0, key // 16], key % 16
            if small:                                    # scores of -75, the others within +-6
                q[:, :group, 0] = 1
                k[page, 0, at] = 0
                k[page, 0, at, 0] = -600
            want, size = PO.paged_attention(*args[:6], np.float32(0.125), args[6])
            v[page, 0, at, 7] = value
            dev = on_gpu(*args)
            out = B.qattn_paged_f16(*dev[:6], 0.125, prefix=dev[6]).cpu().numpy().reshape(q.shape)
            # Rows of both requests see a key of the prefix, else those of the first do.
            hit = np.zeros(out.shape, bool)
            hit[:new + (key < 16 * prefix_pages), :group, 7] = True
            odd = out[hit]
            if np.isnan(value):
                assert np.isnan(odd).all(), (key, small)
            elif small:
                assert not np.isfinite(odd).any() and not (odd == -value).any(), key
            else:
                assert (odd == value).all(), key
            # Half a step of fp16 of the result and of each weight, scores in fp32 (below 2^-12 of size).
            bound = 2.0 ** -11 * np.abs(want) + (2.0 ** -11 + 2.0 ** -12) * size + 2.0 ** -25
            assert (np.abs(out - want)[~hit] <= bound[~hit]).all(), (key, small)
