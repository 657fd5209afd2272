"""GPU tests of the row that gva_append_rows and gqa_append name: its number up to 2^23 - 1, and 2^23 - 1 for it and all rows behind it
(a status word has 23 bits for it).  Whole numbers: exact."""
import numpy as np
import pytest
import torch

from paper_2609_13285_b200 import binding as gb
from paper_2609_13285_b200 import workloads as wl
from tests.test_gpu_compact import G1, Cache, Handle
from tests.test_gpu_draft import code, zeros

pytestmark = pytest.mark.gpu
LAST = 2 ** 23 - 1


@pytest.fixture(scope="module", autouse=True)
def _built():
    from tests import gpu_util
    gpu_util.ensure_built()


@pytest.mark.parametrize("row", [0, 3, LAST - 1, LAST, LAST + 1, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 2])
@pytest.mark.parametrize("error", [gb.GVA_ERR_BAD_PAGE, gb.GVA_ERR_SEQ_LEN])
def test_the_row_that_is_named(row, error):
    n, d = row + 1, 64
    c = Cache(G1, [100], kind="bf16", seed=1)
    pos, slots = zeros(n), zeros(n) - 1                             # padded rows, and one that is wrong
    if error == gb.GVA_ERR_BAD_PAGE:
        slots[row] = c.num_pages * c.page
    else:
        slots[row], pos[row] = 5, -1
    x = torch.zeros(n, d, device="cuda")                            # (4 GB of rows where they are most)
    with Handle(G1) as h:
        status = zeros(1)
        gb.gva_append_rows(h.h, c.c, x, torch.zeros(n, 16, device="cuda"), pos, slots, n, status)
        assert code(status) == (error, min(row, LAST))
        status = zeros(1)
        gb.gqa_append(h.h, gb.make_gqa_cache(c.d[0], c.d[0], None, c.num_pages, 1), None, 0, x, d, x, d, pos, slots, None, n, status)
        assert code(status) == (error, min(row, LAST))
        for old, new in zip(c.pools, c.download()):
            assert np.array_equal(old.view(np.uint8), new.view(np.uint8))
