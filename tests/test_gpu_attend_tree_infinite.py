"""maskkv_attend_tree over cached rows with infinite values (needs an MI355X): a result with a row of infinity is infinite, also where that row is the last
one of a head and the places of a tile behind it are filled with what is no row.  The rows' own probabilities are far from underflow."""
import numpy as np
import pytest
import torch

from tests import helpers as hp
from tests import mx_helpers as mh
from tests.test_gpu_attend_tree import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,g,lens", [(5, 1, [1, 33, 64, 70]), (1, 7, [9000, 31, 32, 4001]), (40, 2, [100, 63, 65, 300]), (256, 2, [4000, 3999, 65, 1]),
                                      (64, 7, [130, 127, 128, 1])])
def test_an_infinite_value_in_the_last_cached_row(dtype, d, n, g, lens):
    c = Case(70 + n, 1, 4, d, n, lens, g=g, dtype=dtype)
    last = c.cu[1:] - 1
    for h, row in enumerate(last):
        c.v[row, h % 2::2] = np.inf if h < 2 else -np.inf
    c.upload()
    c.run().check()
    O = c.O.float().cpu().numpy().reshape(4, g * n, d)
    for h in range(4):
        assert np.all(O[h, :, h % 2::2] == (np.inf if h < 2 else -np.inf)) and np.all(np.isfinite(O[h, :, 1 - h % 2::2]))


@pytest.mark.parametrize("n,g", [(5, 1), (256, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_key_in_the_last_cached_row_of_another_head(dtype, n, g):
    """What follows a head in the cache, and is infinite or NaN, is another head's."""
    c = Case(80 + n, 1, 3, 64, n, [70, 40, 3], g=g, dtype=dtype)
    c.k[70:110], c.v[70:110] = np.inf, np.nan
    c.upload()
    c.run().check(heads=(0, 2))
    assert bool(torch.isfinite(c.O[:, :g]).all()) and bool(torch.isfinite(c.O[:, 2 * g:]).all())
