"""The 4-bit paged cache and the norm with rotation where numbers reach the ends of their type, calls their limits, and
tables the sizes that are walked in another way (run with -m gpu on a B200).  Definitions: oracle/kv4.py, float64.

Tolerances as in test_gpu_kv4.py: a stored result is rounded to the storage type once, EPS * |value|; what FP32 arithmetic
adds before that is written at each test.
"""
import numpy as np
import pytest

from oracle import kv4

pytestmark = pytest.mark.gpu
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
DT = {"f16": np.float16, "bf16": "bf16"}


@pytest.fixture(scope="module")
def T():
    import torch
    from paper_2605_25655_b200 import thinfer
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    thinfer.lib("f16"), thinfer.lib("bf16")
    return torch, thinfer


def _tt(torch, t):
    return {"f16": torch.float16, "bf16": torch.bfloat16}[t]


def _dev(torch, x, t):
    return torch.from_numpy(np.ascontiguousarray(x)).to(_tt(torch, t)).cuda()


def _host(x):
    return x.double().cpu().numpy()


def _int(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _one_row(torch, thinfer, k, v, t, page):
    """A pool of one table row that holds k, v [tokens][hkv][d], its table, and the same bytes for the oracle."""
    n, hkv, d = k.shape
    pages = -(-n // page)
    pool = torch.full((pages, hkv * page * (d + 8)), 255, dtype=torch.uint8, device="cuda")
    table = [list(range(pages))[::-1]]
    rows, pos = _int(torch, [0] * n), _int(torch, list(range(n)))
    thinfer.op_kv4_append(pool, _int(torch, table), _dev(torch, k, t), _dev(torch, v, t), rows, pos, page)
    return pool, table, rows, pos, kv4.Pool(pool.cpu().numpy(), hkv, d, page, DT[t])


# ------------------------------------------------------------------ read
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_read_of_rows_with_large_scales(T, d, page):
    """BF16 rows of 1e28 to 3e37: 2^24 times their scale is on either side of FP32's largest value."""
    torch, thinfer = T
    rng = np.random.default_rng(d)
    sizes = np.array([1e28, 1e31, 1.2e32, 2e32, 2e33, 1e35, 1e37, 3e37])
    x = kv4.round_to(np.clip(rng.standard_normal((8, 2, d)), -4, 4) * sizes[:, None, None], "bf16")
    x[3, 0, :] = kv4.round_to(2e32 * np.where(np.arange(d) % 2, 1.0, -1.0), "bf16")
    pool, table, rows, pos, ref = _one_row(torch, thinfer, x, -x, "bf16", page)
    got = thinfer.op_kv4_read(pool, _int(torch, table), rows, pos, page, d, torch.bfloat16)
    for which in (0, 1):
        want = np.stack([[ref.read(table[0][i // page], i % page, h, which) for h in (0, 1)] for i in range(8)])
        assert np.all(np.isfinite(want))
        # one FP32 rounding (2^-24) before the stored one
        assert np.all(np.abs(_host(got[which]) - want) <= EPS["bf16"] * np.abs(want) * 1.001)
