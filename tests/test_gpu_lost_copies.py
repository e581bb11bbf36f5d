"""Copies that never arrive in the kernels of the 4-bit layers and of the 8-bit cache: the wait runs out after the polls
that were set, the launch ends, the status says so once, and the handle works as before.  Nothing faults or hangs: one warp
arms a barrier without issuing the copy."""
import pytest
import torch

from paper_2504_11816_b200 import binding as B
from test_gpu_linear4 import _case, _check
from test_gpu_q8 import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,group", [
    (1, 4096, 4096, 128),       # a cluster of CTAs shares K
    (1, 40, 256, 32),           # fewer steps than the ring holds
    (1, 40000, 1024, 64),       # a warp walks many row tiles
    (6, 20000, 2048, 128),      # four row blocks a CTA
    (20, 4096, 4096, 64), (40, 300, 640, 64)])
def test_a_lost_copy_of_weights_ends_in_a_status(M, N, K, group):
    x, w4, scales = _case(M, N, K, group, "f16", seed=N)
    l = B.isv_linear4_create(w4.cuda(), scales.cuda(), N, K, group, B.ISV_F16, M)
    try:
        xd = x.cuda()
        before, y = (torch.zeros((M, N), device="cuda") for _ in range(2))
        B.isv_linear4_forward(l, xd, None, before, M)
        _check(None, before, x, w4, scales, group, "f16")
        for polls, launches in ((2000, 1), (1, 2)):
            B.isv_linear4_set_wait_limit(l, polls)
            B.isv_linear4_inject_lost_copy(l, launches)
            for _ in range(launches):
                B.isv_linear4_forward(l, xd, None, y, M)
                with pytest.raises(B.IsvError) as ei:
                    B.isv_linear4_status(l)
                assert ei.value.code == B.ISV_EDEVICE_STATUS and "0x2" in ei.value.message
                assert B.isv_linear4_status(l) == 0                     # reported once
            B.isv_linear4_set_wait_limit(l, 0)
            for _ in range(2):
                y.zero_()
                B.isv_linear4_forward(l, xd, None, y, M)
                assert B.isv_linear4_status(l) == 0 and torch.equal(y, before)
    finally:
        B.isv_linear4_free(l)


@pytest.mark.parametrize("lens,hq,hkv,d,fmt", [
    ([4000], 8, 2, 128, B.ISV_Q8_E4M3),                 # one sequence over many CTAs
    ([40, 0, 17], 4, 4, 64, B.ISV_Q8_INT8),             # fewer visits than the ring holds
    ([900] * 40, 16, 4, 80, B.ISV_Q8_INT8), ([2000, 5, 700], 12, 1, 64, B.ISV_Q8_E4M3), ([3000, 100], 32, 2, 128, B.ISV_Q8_INT8)])
def test_a_lost_copy_of_a_block_ends_in_a_status(lens, hq, hkv, d, fmt):
    with Cache(lens, hq, hkv, d, "f16", fmt, seed=23) as c:
        c.fill()
        before = c.attend()
        c.check(*before, rows=range(0, len(lens), 8) if len(lens) > 8 else None)
        for polls, launches in ((2000, 1), (1, 2)):
            B.isv_q8_set_wait_limit(c.h, polls)
            B.isv_q8_inject_lost_copy(c.h, launches)
            for _ in range(launches):
                c.attend()
                with pytest.raises(B.IsvError) as ei:
                    B.isv_q8_status(c.h)
                assert ei.value.code == B.ISV_EDEVICE_STATUS and "0x2" in ei.value.message
                assert B.isv_q8_status(c.h) == 0                        # reported once
            B.isv_q8_set_wait_limit(c.h, 0)
            for _ in range(2):                                          # scratch and tickets are as they were
                again = c.attend()
                assert B.isv_q8_status(c.h) == 0
                assert torch.equal(again[0], before[0]) and torch.equal(again[1], before[1])


def test_bad_arguments_of_the_failure_calls():
    with Cache([16], 2, 2, 64) as c:
        for fn, args in ((B.isv_q8_inject_lost_copy, (c.h, -1)), (B.isv_q8_inject_lost_copy, (None, 1)),
                         (B.isv_q8_set_wait_limit, (None, 1))):
            with pytest.raises(B.IsvError) as ei:
                fn(*args)
            assert ei.value.code == B.ISV_EINVAL
    x, w4, scales = _case(1, 32, 64, 32, "f16")
    l = B.isv_linear4_create(w4.cuda(), scales.cuda(), 32, 64, 32, B.ISV_F16, 1)
    try:
        for fn, args in ((B.isv_linear4_inject_lost_copy, (l, -1)), (B.isv_linear4_inject_lost_copy, (None, 1)),
                         (B.isv_linear4_set_wait_limit, (None, 1))):
            with pytest.raises(B.IsvError) as ei:
                fn(*args)
            assert ei.value.code == B.ISV_EINVAL
    finally:
        B.isv_linear4_free(l)
