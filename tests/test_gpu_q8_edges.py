"""The 8-bit KV cache at the edges of its ranges, through the C ABI, against the fp64 reference."""
import pytest
import torch

from paper_2504_11816_b200 import binding as B
from test_gpu_q8 import Cache

pytestmark = pytest.mark.gpu


def test_rows_longer_than_32_bit_lengths_are_refused():
    """16 * max_blocks + 15 tokens, the longest length of a row, is rounded up to blocks in 32 bits: 2^27 - 2 is the most."""
    with Cache([16], 2, 2, 64) as c:
        c.fill()
        lens = torch.tensor([16], dtype=torch.int32, device="cuda")
        out = torch.zeros_like(c.q)
        for most, fine in ((2 ** 27 - 2, True), (2 ** 27 - 1, False)):
            attn = (c.h, c.pool, c.n_pages, c.tails, c.table, most, most, lens, c.q, out, None, 1)
            write = (c.h, c.pool, c.n_pages, c.tails, c.table, most, most, lens, None, *c.kept[:2], 16 * 128, 128, 1, 16)
            for fn, args in ((B.isv_q8_attn, attn), (B.isv_q8_write, write)):
                if fine:
                    fn(*args)
                    continue
                with pytest.raises(B.IsvError) as ei:
                    fn(*args)
                assert ei.value.code == B.ISV_EINVAL and "table row" in ei.value.message
        torch.cuda.synchronize()
        c.check(out, None)
        c.check_bytes()
