"""Page operations whose tables are larger than 32-bit counts, through the C ABI."""
import pytest
import torch

from paper_2504_11816_b200 import binding as B

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_rows_that_ask_for_more_than_two_to_the_31_pages():
    """17 rows grow by 2^27 - 1 blocks each: 2.28e9 entries are wanted, and a few hundred pages are free.  The first row gets
    them, in order; every other entry becomes ISV_BLOCK_NONE."""
    rows, most, n_pages = 17, 2 ** 27 - 1, 1000
    table = torch.zeros((rows, most), dtype=torch.int32, device="cuda")
    table[16, :7] = torch.arange(100, 107, dtype=torch.int32, device="cuda")
    old, new = _dev([0] * 16 + [7 * 16]), _dev([16 * most] * rows)
    status = _dev([0])
    B.isv_pages_resize(table, old, new, rows, most, most, 1, n_pages, status)
    assert status.item() == B.ISV_STATUS_NO_PAGES
    free = [i for i in range(n_pages) if not 100 <= i < 107]
    assert table[0, :len(free)].tolist() == free and table[16, :7].tolist() == list(range(100, 107))
    assert bool((table[0, len(free):] == B.ISV_BLOCK_NONE).all()) and bool((table[16, 7:] == B.ISV_BLOCK_NONE).all())
    for r in range(1, 16):
        assert bool((table[r] == B.ISV_BLOCK_NONE).all())
