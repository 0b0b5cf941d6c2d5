"""Weights in 4 bits and the choice of tokens: buffers that are written again between calls, numbers at the ends of their types, rows
and requests that differ in kind (run with -m gpu on a B200)."""
import numpy as np
import pytest

from oracle import tokens as tk

pytestmark = pytest.mark.gpu
INF, NAN = np.inf, np.nan


@pytest.fixture(scope="module")
def T():
    import torch
    from paper_2605_25655_b200 import thinfer
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    thinfer.lib("f16"), thinfer.lib("bf16")
    return torch, thinfer


# ------------------------------------------------------------------ chains of calls
@pytest.mark.parametrize("t", ["float16", "bfloat16"])
@pytest.mark.parametrize("rows,group", [(17, 128), (40, 128), (64, 128), (32, 64), (64, 64), (24, 32), (64, 32), (5, 128)])
def test_weights_quantised_anew_between_products(T, t, rows, group):
    """One buffer of packed weights, written again in front of every product and without a pause: codes, scales and zero points all
    change (weights of -15 .. 0, then of 0 .. 30 in steps of two), and whole numbers leave nothing to round."""
    torch, thinfer = T
    n, k, tt = 2600, 8200, getattr(torch, t)
    gen = torch.Generator(device="cuda").manual_seed(rows + group)
    low = torch.randint(-15, 1, (n, k), device="cuda", generator=gen)
    high = torch.randint(0, 16, (n, k), device="cuda", generator=gen) * 2
    low[:, ::8], low[:, 1::8], high[:, ::8], high[:, 1::8] = -15, 0, 0, 30      # every group spans 15 steps
    w = [low.to(tt), high.to(tt)]
    x = torch.randint(-2, 3, (rows, k), device="cuda", generator=gen).to(tt)
    want = [x.double() @ a.double().T for a in w]     # whole numbers below 2^19
    packed = thinfer.op_w4_quantize(w[0], group)
    torch.cuda.synchronize()
    got = []
    for i in range(24):
        thinfer.op_w4_quantize(w[i % 2], group, packed=packed)
        got.append(thinfer.op_w4_linear(x, packed, n, group, out_fp32=True))
    assert all(torch.equal(y.double(), want[i % 2]) for i, y in enumerate(got))
