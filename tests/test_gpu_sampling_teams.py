"""Rows that several blocks share: more than 32 KB of logits, in calls of few rows.  Filters, masks and extreme parameters as in
test_gpu_sampling.py, whose shorter rows one block takes whole."""
import numpy as np
import pytest
import torch

from test_gpu_sampling import DT, FILTERS, check, dev, hb, logits  # noqa: F401

pytestmark = pytest.mark.gpu
V_OF = {"f32": 8209, "f16": 16421, "bf16": 20011}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 5])
def test_filters_over_several_blocks(hb, dtype, rows):                                 # noqa: F811
    x, u = logits(71, DT[dtype], rows, 1, V_OF[dtype])
    for kw in FILTERS:
        check(hb, x, u, **{n: [v] * rows for n, v in kw.items()}, what=str(kw))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masks_infinities_and_nan_over_several_blocks(hb, dtype):                      # noqa: F811
    dt, V, inf, nan = DT[dtype], V_OF[dtype], float("inf"), float("nan")
    x = torch.randn((10, 1, V), generator=torch.Generator().manual_seed(72))
    x[0] = nan
    x[1] = -inf
    x[2, 0], x[2, 0, V - 40:] = nan, -inf                                               # all but the last block's tokens are NaN
    x[3, 0, ::3] = nan
    x[4, 0, :V - 700] = -inf                                                            # blocks without a token
    x[5, 0, 100], x[5, 0, V - 2] = inf, inf
    x[6, 0, 5:] = torch.finfo(dt).min
    x[7] = torch.finfo(dt).min
    x[8, 0, 700:] = -inf
    x[9, 0], x[9, 0, V - 1] = -inf, 0.0
    x = x.to(dt).cuda()
    for seed in range(2):
        u = np.random.default_rng(seed).random((10, 1)).astype(np.float32)
        for kw in (dict(), dict(k=[600] * 10), dict(k=[3] * 10), dict(p=[0.7] * 10), dict(T=[0.0] * 10), dict(m=[0.3] * 10), dict(k=[20] * 10, p=[0.9] * 10)):
            check(hb, x, u, **kw, what=str(kw))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_extreme_parameters_over_several_blocks(hb, dtype):                            # noqa: F811
    V = V_OF[dtype]
    x, u = logits(73, DT[dtype], 8, 1, V)
    check(hb, x, u, T=[1e-30, 1e-38, 1e-3, 1e3, 1e10, 1e30, 1.0, 1.0])
    check(hb, x, u, T=[1e-30, 1e-3, 1e3, 1e10] * 2, p=[0.5] * 8)
    check(hb, x, u, k=[V - 1, V, V + 1, 2 ** 31 - 1, -(2 ** 31), 512, 513, 1])
    check(hb, x, u, p=[1e-30, 1e-6, 0.9999999, 1.0, 2.0, 0.0, -1.0, 1.0], m=[0, 0, 0, 1.0, 0.999, 1e-30, 0.5, -3.0])
    for end in (0.0, 1.0):
        check(hb, x, np.full((8, 1), end, np.float32), p=[0.9] * 8, k=[0, 40, 700, 300, 256, 257, 128, 2000])


def test_many_rows_captured_and_replayed_with_new_numbers(hb):                         # noqa: F811
    """The check ahead of the call is part of the graph."""
    N, V = 2100, 30
    x, u = logits(74, torch.float32, 2, N, V)
    ud, token = dev(u), torch.empty((2, N), dtype=torch.int32, device="cuda")
    hb.sample(x, ud, token=token)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _, st = hb.sample(x, ud, token=token)
    for bad in (False, True, False):
        ud.copy_(torch.rand_like(ud))
        if bad:
            ud[1, 7] = 2.0
        graph.replay()
        torch.cuda.synchronize()
        want, wst = hb.sample(x, ud)
        assert st.tolist() == [0, 7 if bad else 0] == wst.tolist() and torch.equal(token, want)
        assert ((token[1] == -1).all() == bad).item() and (token[0] >= 0).all()
