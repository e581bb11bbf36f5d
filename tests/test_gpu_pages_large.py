"""Page operations whose tables are larger than 32-bit counts, through the C ABI."""
import pytest
import torch

from paper_2504_11816_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _return_the_memory():
    yield
    torch.cuda.empty_cache()


def _needs(gb):
    free, _ = torch.cuda.mem_get_info()
    if free < gb << 30:
        pytest.skip(f"{gb} GB of device memory are not free")


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_rows_that_ask_for_more_than_two_to_the_31_pages():
    """17 rows grow by 2^27 - 1 blocks each: 2.28e9 entries are wanted, and a few hundred pages are free.  The first row gets
    them, in order; every other entry becomes ISV_BLOCK_NONE."""
    _needs(12)
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


def test_as_many_layers_as_an_int_holds():
    """2^31 - 1 layers of two 16-byte pages: the step from layer to layer passes 2^31 at the end."""
    _needs(76)
    layers = 2 ** 31 - 1
    pool = torch.zeros((layers, 2, 2), dtype=torch.int64, device="cuda")
    for at in range(0, layers, 1 << 28):
        part = pool[at:at + (1 << 28), 0, 0]
        part.copy_(torch.arange(at, at + part.shape[0], device="cuda"))
    status = _dev([0])
    B.isv_pages_copy(pool, 2, pool, 2, 16, layers, 32, 32, _dev([0]), _dev([1]), 1, None, status)
    assert status.item() == 0
    for at in range(0, layers, 1 << 28):
        part = pool[at:at + (1 << 28)]
        assert bool((part[:, 1, 0] == part[:, 0, 0]).all()) and bool((part[:, 1, 1] == 0).all())
    assert pool[layers - 1, 1, 0].item() == layers - 1


def test_as_many_moves_as_an_int_holds():
    """Lists of 2^31 - 1 moves: the step that fills them up passes 2^31 at the end."""
    _needs(24)
    m = 2 ** 31 - 1
    table, out = _dev([[5, 0]]), _dev([[9, 9]])
    src, dst = (torch.full((m,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    counts, status = _dev([0, 0]), _dev([0])
    B.isv_pages_compact(table, _dev([32]), 1, 2, 2, 1, 8, out, src, dst, m, counts, status)
    assert out.tolist() == [[1, 0]] and counts.tolist() == [2, 1] and status.item() == 0
    for x, first in ((src, 5), (dst, 1)):
        assert x[0].item() == first
        for at in range(1, m, 1 << 28):
            assert bool((x[at:at + (1 << 28)] == B.ISV_BLOCK_NONE).all())
