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


# ------------------------------------------------------------------ attention
def _attend(T, rng, q, k, v, queries=1, page=16, with_mag=True):
    """BF16 attention of one request whose last tokens are q [queries][hq][d], against the float64 definition over the
    stored bytes; the tolerance of test_gpu_kv4.test_attention (without the part for scores where they decide by far)."""
    torch, thinfer = T
    n, hkv, d = k.shape
    q, k, v = (kv4.round_to(x, "bf16") for x in (q, k, v))
    pool, table, _, _, ref = _one_row(torch, thinfer, k, v, "bf16", page)
    got = _host(thinfer.op_kv4_attention(_dev(torch, q[None], "bf16"), pool, _int(torch, table), _int(torch, [n]), page))[0]
    kv = kv4.keys_values(ref, table[0], n)
    assert np.all(np.isfinite(kv))
    for i in range(queries):
        want, spread, mag = kv4.attention(q[i], kv, n, queries - 1 - i)
        far = spread + np.abs(want) + kv4.attention(q[i], (kv[0], np.abs(kv[1])), n, queries - 1 - i)[0]
        tol = EPS["bf16"] * np.abs(want) + 2.0 ** -10 * spread + (2.0 ** -19 * (1 + 16 * mag) * far if with_mag else 0)
        assert np.all(np.isfinite(got[i])) and np.all(np.abs(got[i] - want) <= tol), (i, np.max(np.abs(got[i] - want) / tol))


@pytest.mark.parametrize("n,hq,hkv,d,queries", [(1, 2, 1, 64, 1), (50, 4, 2, 64, 1), (70, 4, 1, 128, 5), (700, 2, 1, 128, 1)])
def test_attention_of_queries_near_the_largest_value(T, n, hq, hkv, d, queries):
    """Queries on either side of 2^116 (8.3e34) and up to 1.5e38 over small keys: scores of ordinary size."""
    rng = np.random.default_rng(n)
    for q_size, k_size in ((5e34, 1e-34), (1e35, 1e-34), (1e37, 1e-36), (4e37, 1e-37), (1e-33, 1e33), (1e-37, 1e37)):
        q = np.clip(rng.standard_normal((queries, hq, d)), -3.5, 3.5) * q_size
        _attend(T, rng, q, rng.standard_normal((n, hkv, d)) * k_size / 4, rng.standard_normal((n, hkv, d)), queries)
    same = 1.5e38 * (1 - 0.2 * rng.random((queries, hq, d)))      # of one sign: their sum is beyond FP32
    _attend(T, rng, same, (rng.standard_normal((n, hkv, d)) + 3) * 1e-38 / 4, rng.standard_normal((n, hkv, d)), queries)


@pytest.mark.parametrize("n,hq,hkv,d,queries", [(1, 2, 1, 64, 1), (3, 4, 2, 64, 1), (40, 4, 1, 128, 4), (700, 2, 1, 128, 1)])
def test_attention_where_every_score_is_far_below_zero(T, n, hq, hkv, d, queries):
    """Scores of -1e32 to -2e38.  Keys grow smaller towards the last one, in steps of 5 % of its size, far more than the values
    of a key differ: the last key that a query sees takes all the weight."""
    rng = np.random.default_rng(n + d)
    for q_size, k_size in ((1e16, 1e16), (1e18, 1e18), (-1e20, -1e16), (5e18, 1e19)):
        q = q_size * (1 + 0.1 * rng.random((queries, hq, d)))
        far = np.minimum(np.arange(n)[::-1], 20)[:, None, None]
        k = -k_size / 8 * (1 + 0.05 * far) * (1 + 0.005 * rng.random((n, hkv, d)))
        _attend(T, rng, q, k, rng.standard_normal((n, hkv, d)), queries, with_mag=False)
