"""4-bit linear layers keep fp32 sums (oracle.linear.linear4_typical), and calls that overlap do not disturb each other."""
import numpy as np
import pytest
import torch

from oracle import linear as ol
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W
from test_gpu_linear4 import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("N,K,group", [(17, 96, 32), (128, 4096, 128), (48, 12800, 64), (257, 11008, 32), (1000, 2560, 128)])
def test_sums_are_as_exact_as_fp32(N, K, group, dtype):
    for M in (1, 5, 9, 24, 40):
        x, w4, scales = _case(M, N, K, group, dtype, seed=N + K + M)
        y = torch.zeros((M, N), device="cuda")
        l = B.isv_linear4_create(w4.cuda(), scales.cuda(), N, K, group, B.ISV_F16 if dtype == "f16" else B.ISV_BF16, M)
        try:
            B.isv_linear4_forward(l, x.cuda(), None, y, M)
            off = np.abs(y.double().cpu().numpy() - ol.linear4(x, w4.numpy(), scales, group))
            assert np.all(off <= ol.linear4_typical(x, w4.numpy(), scales, group)), M
        finally:
            B.isv_linear4_free(l)


@pytest.mark.parametrize("N,K,Ms", [(4096, 4096, (1, 3)), (3000, 2048, (8, 20)), (40, 11008, (2, 64))])
def test_calls_on_two_streams_may_overlap(N, K, Ms):
    """One handle, two streams, many calls in flight: every output is what a call alone gives."""
    g = torch.Generator().manual_seed(N)
    _, w4, scales = _case(1, N, K, 128, "bf16", seed=N)
    xs = [torch.randn((M, K), generator=g).to(W.torch_dtype("bf16")).cuda() for M in Ms]
    l = B.isv_linear4_create(w4.cuda(), scales.cuda(), N, K, 128, B.ISV_BF16, max(Ms))
    try:
        alone = [torch.zeros((M, N), device="cuda") for M in Ms]
        for x, y, M in zip(xs, alone, Ms):
            B.isv_linear4_forward(l, x, None, y, M)
            torch.cuda.synchronize()
            _check(None, y, x.cpu(), w4, scales, 128, "bf16")
        streams = [torch.cuda.Stream() for _ in Ms]
        outs = [[torch.zeros((M, N), device="cuda") for _ in range(40)] for M in Ms]
        torch.cuda.synchronize()
        for i in range(40):
            for x, o, M, st in zip(xs, outs, Ms, streams):
                B.isv_linear4_forward(l, x, None, o[i], M, st.cuda_stream)
        torch.cuda.synchronize()
        for o, y in zip(outs, alone):
            assert all(torch.equal(z, y) for z in o)
        assert B.isv_linear4_status(l) == 0
    finally:
        B.isv_linear4_free(l)
