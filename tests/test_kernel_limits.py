"""Calls at the far end of what the arguments' types hold are refused before anything reaches a GPU.  CPU only: the
addresses given here are never followed."""
import pytest

from paper_2504_11816_b200 import binding as B

A = 1 << 20        # an aligned address


def _refused(text, fn, *a, **kw):
    with pytest.raises(B.IsvError) as ei:
        fn(*a, **kw)
    assert ei.value.code == B.ISV_EINVAL and text in ei.value.message, ei.value


@pytest.mark.parametrize("n,page_bytes", [(2 ** 31 - 1, 32 << 10), (2 ** 31 - 1, 17 << 10), (2 ** 20 - 76, 1 << 26)])
def test_copies_whose_item_counter_would_wrap(n, page_bytes):
    """A CTA of the copy kernel steps from item to item by the grid's size in 32 bits: where that can pass 2^32 the walk
    would begin anew and never end."""
    pieces = (page_bytes + (16 << 10) - 1) >> 14
    assert 2 ** 32 - (1 << 20) <= n * pieces < 2 ** 32
    _refused("too large", B.isv_pages_copy, A, 4, 2 * A, 4, page_bytes, 1, 0, 0, 3 * A, None, n)
