"""4-bit linear layers against the fp64 reference, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import linear as ol
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W

pytestmark = pytest.mark.gpu

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _case(M, N, K, group, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g).to(W.torch_dtype(dtype))
    w4 = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    scales = (torch.randn((N, K // group), generator=g) / np.sqrt(K)).to(W.torch_dtype(dtype))
    return x, w4, scales


def _check(y16, y32, x, w4, scales, group, dtype):
    want, tol = ol.linear4(x, w4.numpy(), scales, group), ol.linear4_error(x, w4.numpy(), scales, group)
    if y32 is not None:
        assert np.all(np.abs(y32.double().cpu().numpy() - want) <= tol)
    if y16 is not None:
        room = HALF_STEP[dtype] * (np.abs(want) + tol) + 2.0 ** -25      # and half a step of the smallest fp16 numbers
        assert np.all(np.abs(y16.double().cpu().numpy() - want) <= tol + room)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("N,K,group", [
    (1, 32, 32), (15, 64, 64), (16, 128, 128), (17, 96, 32), (33, 640, 128), (100, 1056, 32), (128, 4096, 128), (257, 320, 64),
    (1000, 2560, 64), (4097, 352, 32), (640, 10240, 128), (48, 12800, 64)])
def test_matches_the_reference(N, K, group, dtype):
    for M in (1, 2, 3, 7, 8, 9, 16, 17, 31, 32, 33, 64):
        x, w4, scales = _case(M, N, K, group, dtype, seed=N + K + M)
        xd = x.cuda()
        y16 = torch.full((M, N), float("nan"), dtype=x.dtype, device="cuda")
        y32 = torch.full((M, N), float("nan"), device="cuda")
        l = B.isv_linear4_create(w4.cuda(), scales.cuda(), N, K, group, B.ISV_F16 if dtype == "f16" else B.ISV_BF16, M)
        try:
            B.isv_linear4_forward(l, xd, y16, y32, M)
            _check(y16, y32, x, w4, scales, group, dtype)
            again = torch.zeros_like(y32)
            B.isv_linear4_forward(l, xd, None, again, M)
            assert torch.equal(again, y32)                              # the same bits every time
            only = torch.zeros_like(y16)
            B.isv_linear4_forward(l, xd, only, None, M)
            assert torch.equal(only, y16)
            assert B.isv_linear4_status(l) == 0
        finally:
            B.isv_linear4_free(l)


def test_large_layers_and_fewer_tokens_than_max():
    for N, K, group, dtype in ((4096, 4096, 128, "bf16"), (22016, 4096, 64, "f16"), (4096, 11008, 32, "bf16")):
        x, w4, scales = _case(20, N, K, group, dtype)
        l = B.isv_linear4_create(w4.cuda(), scales.cuda(), N, K, group, B.ISV_F16 if dtype == "f16" else B.ISV_BF16, 64)
        try:
            for M in (1, 5, 20):
                y = torch.zeros((M + 1, N), device="cuda")
                B.isv_linear4_forward(l, x[:M].cuda().contiguous(), None, y, M)
                _check(None, y[:M], x[:M], w4, scales, group, dtype)
                assert (y[M] == 0).all()                                # nothing behind the last token
        finally:
            B.isv_linear4_free(l)


def test_extreme_inputs_stay_where_they_are():
    """Large and tiny activations, scales of zero and of any sign; an infinity reaches its own token only."""
    x, w4, scales = _case(4, 40, 256, 64, "bf16")
    x[0] *= 1e30
    x[1] *= 1e-30
    scales[3] = 0
    scales[5] *= -1e4
    l = B.isv_linear4_create(w4.cuda(), scales.cuda(), 40, 256, 64, B.ISV_BF16, 4)
    try:
        y = torch.zeros((4, 40), device="cuda")
        B.isv_linear4_forward(l, x.cuda(), None, y, 4)
        _check(None, y, x, w4, scales, 64, "bf16")
        bad = x.clone()
        bad[2, 17] = float("inf")
        z = torch.zeros_like(y)
        B.isv_linear4_forward(l, bad.cuda(), None, z, 4)
        assert torch.equal(z[[0, 1, 3]], y[[0, 1, 3]]) and not torch.isfinite(z[2][w4[:, 8] >> 4 != 8]).any()
    finally:
        B.isv_linear4_free(l)


def test_streams_graphs_unaligned_outputs_and_freed_weights():
    M, N, K = 3, 200, 512
    x, w4, scales = _case(M, N, K, 128, "f16")
    wd, sd = w4.cuda(), scales.cuda()
    l = B.isv_linear4_create(wd, sd, N, K, 128, B.ISV_F16, 8)
    wd.zero_(), sd.zero_()                                              # the handle has its own copy
    try:
        xd, side = x.cuda(), torch.cuda.Stream()
        y = torch.zeros((M * N + 1,), dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        B.isv_linear4_forward(l, xd, y.data_ptr() + 2, None, M, side.cuda_stream)     # aligned to its elements only
        side.synchronize()
        _check(y[1:].view(M, N), None, x, w4, scales, 128, "f16")
        assert y[0] == 0
        out = torch.zeros((M, N), device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.isv_linear4_forward(l, xd, None, out, M, torch.cuda.current_stream().cuda_stream)
        x2 = torch.randn(x.shape).half()
        xd.copy_(x2)
        graph.replay()
        torch.cuda.synchronize()
        _check(None, out, x2, w4, scales, 128, "f16")
    finally:
        B.isv_linear4_free(l)


def test_forward_refuses_bad_arguments():
    x, w4, scales = _case(4, 32, 64, 32, "f16")
    l = B.isv_linear4_create(w4.cuda(), scales.cuda(), 32, 64, 32, B.ISV_F16, 4)
    try:
        xd, y = x.cuda(), torch.zeros((4, 32), device="cuda")
        for args in ((None, y, y, 1), (xd, None, None, 1), (xd, None, y, 0), (xd, None, y, 5), (xd.data_ptr() + 2, None, y, 1),
                     (xd, y.data_ptr() + 1, None, 1), (xd, None, y.data_ptr() + 2, 1)):
            with pytest.raises(B.IsvError) as ei:
                B.isv_linear4_forward(l, *args)
            assert ei.value.code == B.ISV_EINVAL
    finally:
        B.isv_linear4_free(l)
