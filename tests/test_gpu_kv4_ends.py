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


# ------------------------------------------------------------------ append
def _written_bytes_are_the_definitions(T, x, t, page=16):
    """Appends x [tokens][d] as K and, in reverse order, as V of one head; every byte against the float64 definition."""
    torch, thinfer = T
    n, d = x.shape
    pages = -(-n // page)
    pool = torch.zeros(pages, page * (d + 8), dtype=torch.uint8, device="cuda")
    ref = kv4.Pool(pool.cpu().numpy(), 1, d, page, DT[t])
    k, v = x[:, None], x[::-1][:, None]
    tab, rows, pos = _int(torch, [list(range(pages))]), _int(torch, [0] * n), _int(torch, list(range(n)))
    thinfer.op_kv4_append(pool, tab, _dev(torch, k, t), _dev(torch, v, t), rows, pos, page)
    for i in range(n):
        ref.write(i // page, i % page, 0, 0, k[i, 0])
        ref.write(i // page, i % page, 0, 1, v[i, 0])
    got = pool.cpu().numpy()
    bad = np.argwhere(got != ref.data)
    assert len(bad) == 0, (len(bad), bad[:3], got[got != ref.data][:3], ref.data[got != ref.data][:3])


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_rows_of_wide_spread(T, t, d):
    """Rows whose values differ by many powers of two: x - offset takes more bits than FP32 has."""
    rng = np.random.default_rng(d)
    rows = []
    for sigma in (1.0, 3.0, 6.0):
        x = rng.choice([-1.0, 1.0], (1200, d)) * np.exp(sigma * rng.standard_normal((1200, d)))
        x /= np.maximum(1, np.abs(x).max(-1, keepdims=True) / 30000.0)        # inside FP16
        rows.append(x)
    _written_bytes_are_the_definitions(T, kv4.round_to(np.concatenate(rows), DT[t]), t)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_codes_beside_the_middle_of_two(T, t):
    """Rows from -7.5 m to 7.5 m and from 0 to 15 m, of scale m, with values that are 0 or tiny or a half step with both signs of
    tiny beside it: as far from the half step as the type can say."""
    rows = []
    tiny = [0.0] + [s * 2.0 ** -e for e in range(2, 25) for s in (1, -1)]
    for m in (1.0, 0.125, 64.0, 2.0 ** -8):
        x = np.resize(np.array(tiny), 64) * m
        x[0], x[1] = -7.5 * m, 7.5 * m
        rows.append(x)
        x = np.resize(np.concatenate([np.arange(0.5, 15), np.abs(tiny)]), 64) * m
        x[0], x[1] = 15 * m, 0.0
        rows.append(x)
        rows.append(np.where(np.arange(64) % 9 == 0, 0.0, rows[-1]) - 2.0 ** -20)   # the offset is the tiny one
        x = np.resize((np.arange(0.5, 15)[:, None] * (1 + np.array([0, 1, -1, 2, -2]) * 2.0 ** -9)).ravel(), 64) * m
        x[0], x[1] = 15 * m, 0.0
        rows.append(x)
    _written_bytes_are_the_definitions(T, kv4.round_to(np.array(rows), DT[t]), t)


def test_rows_that_span_more_than_the_largest_value(T):
    """BF16 rows from -3.3e38 to 3.3e38: max - min is beyond FP32, scale and codes are not."""
    torch, thinfer = T
    rng = np.random.default_rng(8)
    x = rng.uniform(-1, 1, (40, 64)) * np.array([1.6e38, 1.75e38, 2.5e38, 3.35e38])[np.arange(40) % 4][:, None]
    x[::3] *= 10.0 ** rng.integers(-50, 1, (14, 64))
    x[:, 0], x[:, 1] = -np.abs(x).max(-1) * 0.99, np.abs(x).max(-1)
    x = kv4.round_to(x, "bf16")
    assert np.all(np.isfinite(x)) and np.sum(x[:, 1] - x[:, 0] > 3.5e38) == 15
    _written_bytes_are_the_definitions(T, x, "bf16")
    pool, table, rows, pos, ref = _one_row(torch, thinfer, x[:, None], x[:, None], "bf16", 16)
    want = kv4.round_to(np.stack([ref.read(table[0][i // 16], i % 16, 0, 0) for i in range(40)]), "bf16")
    for got in thinfer.op_kv4_read(pool, _int(torch, table), rows, pos, 16, 64, torch.bfloat16):
        got = _host(got)[:, 0]
        near = np.isfinite(want)
        assert near.mean() > 0.9 and np.array_equal(got[~near], want[~near])
        assert np.all(np.abs(got - want)[near] <= 2 * EPS["bf16"] * np.abs(want)[near] * 1.001)     # FP32's rounding beside a tie


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_codes_of_rows_of_tiny_values(T, t):
    """Rows whose scale is subnormal, or so small that it rounds to 0."""
    rng = np.random.default_rng(9)
    sizes = 2.0 ** -np.arange(8, 25) if t == "f16" else 2.0 ** -np.arange(96, 134)
    x = rng.standard_normal((4 * len(sizes), 64)) * np.repeat(sizes, 4)[:, None]
    _written_bytes_are_the_definitions(T, kv4.round_to(x, DT[t]), t)


# ------------------------------------------------------------------ page tables
_POOL_SIZES = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2605_25655_b200 import thinfer
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
for call, sizes in (("reserve", {reserve}), ("fork", {fork}), ("compact", {compact})):
    for n in sizes:
        tab, lens = i32([[n - 1, -1], [n - 2, -1]]), i32([16, 5])
        if call == "reserve":
            out, refused = thinfer.op_kv4_reserve(tab, lens, i32([16, 0]), n, 16)
            ok = tab.tolist() == [[n - 1, 0], [n - 2, -1]] and out.tolist() == [32, 5]
            out, refused = thinfer.op_kv4_reserve(tab, lens, i32([0, 1]), n, 16)
            ok = ok and out.tolist() == [16, 6] and refused.item() == 0
        else:
            pool = torch.zeros(1, n, 16 * 72, dtype=torch.uint8, device="cuda")
            pool[0, n - 2] = 7
            if call == "fork":
                t, l, bad = thinfer.op_kv4_fork(pool, tab[1:], lens[1:], i32([0]), 16, 64)
                ok = t.tolist() == [[n - 2, -1]] and l.tolist() == [5] and bad.item() == 0
            else:
                t, live = thinfer.op_kv4_compact(pool, tab, lens, 16, 64)
                ok = t.tolist() == [[1, -1], [0, -1]] and live.item() == 2 and bool((pool[0, 0] == 7).all())
        assert ok, (call, n)
print("all right")
"""


def test_page_calls_of_pools_of_every_size_in_a_fresh_process(T):
    """Pools whose bitmap is just below 48 KB, or goes above it with what a kernel holds of its own: nothing has been asked of
    the device before, as the tests of a larger pool in this process have."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = _POOL_SIZES.format(root=root, reserve=[40, 146000, 146896, 146912, 160000, 196608, 196640, 1 << 18],
                              fork=[196480, 196512, 196544, 196576, 196608], compact=[195000, 196096, 196576, 196608, 196640])
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "all right" in got.stdout, got.stdout[-500:] + got.stderr[-1500:]


def test_read_into_every_layout_that_does_not_overlap(T):
    """Strides and distances of the outputs at random: refused exactly where two rows share an element (counted here element by
    element), and elsewhere the same values."""
    import ctypes as C
    torch, thinfer = T
    rng = np.random.default_rng(12)
    d, page, most = 64, 16, 6
    x = kv4.round_to(rng.standard_normal((most, 5, d)), np.float16)
    seen = {True: 0, False: 0}
    buf = torch.zeros(1 << 17, dtype=torch.float16, device="cuda")
    for trial in range(400):
        n, hkv = int(rng.integers(1, most + 1)), int(rng.integers(1, 6))
        pool, table, rows, pos, _ = _one_row(torch, thinfer, x[:n, :hkv], -x[:n, :hkv], "f16", page)
        if trial % 4 == 0:                                   # K and V side by side in a token, or in a head
            ts, hs, apart = [(2 * hkv * d, d, hkv * d), (2 * hkv * d, 2 * d, d)][trial // 4 % 2]
        else:
            ts, hs = (int(d + 8 * rng.integers(0, 40)) if rng.random() < 0.5 else d * int(rng.integers(1, 8)) for _ in range(2))
            apart = int(rng.integers(-200, 200)) * 8 if rng.random() < 0.7 else int(rng.integers(-8, 8)) * d
        at = (1 << 16) + np.arange(d) + ts * np.arange(n)[:, None, None] + hs * np.arange(hkv)[:, None]
        want = np.concatenate([at.ravel(), at.ravel() + apart])
        clash = len(np.unique(want)) < len(want)
        seen[clash] += 1
        buf.fill_(7.0)
        tab = _int(torch, table)
        rc = thinfer.lib().thinfer_op_kv4_read(C.c_void_p(pool.data_ptr()), pool.shape[0], C.c_void_p(tab.data_ptr()), 1, tab.shape[1],
                                               C.c_void_p(buf.data_ptr() + (2 << 16)), C.c_void_p(buf.data_ptr() + (2 << 16) + 2 * apart), ts, hs,
                                               C.c_void_p(rows.data_ptr()), C.c_void_p(pos.data_ptr()), n, hkv, d, page,
                                               C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == (thinfer.EINVAL if clash else thinfer.OK), (n, hkv, ts, hs, apart)
        if not clash:
            k, v = thinfer.op_kv4_read(pool, tab, rows, pos, page, d, torch.float16)
            assert torch.equal(buf[torch.from_numpy(at)], k) and torch.equal(buf[torch.from_numpy(at + apart)], v)
            assert torch.sum(buf == 7.0).item() >= len(buf) - len(want)
    assert min(seen.values()) > 100, seen


def test_norm_with_small_tensors_between_the_rows_of_an_output(T):
    """Gains, turns and positions in the gaps of a strided output are no overlap."""
    torch, thinfer = T
    g = torch.Generator(device="cuda").manual_seed(3)
    buf = torch.zeros(4, 1024, dtype=torch.float16, device="cuda")       # rows of 4 x 64 values for q_out, then gaps
    q, k = (torch.randn(4, h, 64, generator=g, device="cuda").half() for h in (4, 1))
    qg, kg, turns = torch.randn(64, generator=g, device="cuda").half(), torch.randn(64, generator=g, device="cuda").half(), thinfer.rope_turns(1e4, 64)
    pos = _int(torch, [3, 0, 700, 12])
    want = thinfer.op_qk_norm_rope(q, k, qg, kg, 1e-6, turns, pos)
    in_gap = [buf[0, 256:320], buf[1, 256:320], buf[2, 256:384].view(torch.float64), buf[0, 512:520].view(torch.int32)]
    for dst, src in zip(in_gap, (qg, kg, turns, pos)):
        dst.copy_(src)
    got = thinfer.op_qk_norm_rope(q, k, in_gap[0], in_gap[1], 1e-6, in_gap[2], in_gap[3], q_out=buf[:, :256].unflatten(1, (4, 64)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------ calls from Python
def test_other_threads_go_on_while_a_call_waits(T, tmp_path):
    """A call that has to wait in the driver (here: an entry point that sleeps half a second) does not hold the interpreter."""
    import ctypes as C
    import subprocess
    import threading
    import time
    torch, thinfer = T
    (tmp_path / "slow.c").write_text("#include <unistd.h>\nint slow(void) { usleep(500000); return 0; }\n")
    subprocess.run(["gcc", "-shared", "-fPIC", str(tmp_path / "slow.c"), "-o", str(tmp_path / "slow.so")], check=True, timeout=120)
    slow = C.cast(C.CDLL(str(tmp_path / "slow.so")).slow, C.c_void_p).value
    ops = thinfer._load_fast()
    real = [[C.cast(getattr(thinfer.lib(s), n), C.c_void_p).value for n in thinfer._FAST_NAMES] for s in ("f16", "bf16")]
    quick = ("thinfer_kv4_attention_workspace", "thinfer_kv4_pages_workspace", "thinfer_last_error")
    z = _int(torch, [0])
    pool, kv = torch.zeros(1, 16 * 72, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
    gain, turns = kv[0, 0], thinfer.rope_turns(1e4, 64)
    calls = (lambda: thinfer.op_qk_norm_rope(kv, kv, gain, gain, 1e-6, turns, z), lambda: thinfer.op_kv4_reserve(z.view(1, 1), z, z, 1, 16),
             lambda: thinfer.op_kv4_append(pool, z.view(1, 1), kv, kv, z, z, 16), lambda: thinfer.op_kv4_read(pool, z.view(1, 1), z, z, 16, 64, kv.dtype),
             lambda: thinfer.op_kv4_attention(kv.view(1, 1, 1, 64), pool, z.view(1, 1), z, 16),
             lambda: thinfer.op_kv4_fork(pool[None], z.view(1, 1), z, z, 16, 64), lambda: thinfer.op_kv4_compact(pool[None], z.view(1, 1), z, 16, 64))
    ops.bind(thinfer.ThinferError, *([a if n in quick else slow for a, n in zip(r, thinfer._FAST_NAMES)] for r in real))
    try:
        for call in calls:
            turns_taken, stop = [0], threading.Event()

            def other():
                while not stop.is_set():
                    time.sleep(0.01)
                    turns_taken[0] += 1
            t = threading.Thread(target=other)
            t.start()
            begun, before = time.monotonic(), turns_taken[0]
            call()
            during, took = turns_taken[0] - before, time.monotonic() - begun
            stop.set()
            t.join()
            assert took > 0.4 and during >= 10, (took, during)
    finally:
        ops.bind(thinfer.ThinferError, *real)
    _, refused = thinfer.op_kv4_reserve(_int(torch, [[-1]]), z, _int(torch, [1]), 1, 16)      # the library's own again
    assert refused.item() == 0


def test_a_truth_value_that_is_none_is_refused(T):
    torch, thinfer = T
    z, kv = _int(torch, [0]), torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
    for bad in (np.zeros(2), torch.zeros(2)):
        with pytest.raises(thinfer.ThinferError) as e:
            thinfer.op_qk_norm_rope(kv, kv, kv[0, 0], kv[0, 0], 1e-6, thinfer.rope_turns(1e4, 64), z, halves=bad)
        assert e.value.code == thinfer.EINVAL and "halves" in str(e.value)


# ------------------------------------------------------------------ norm with rotation
@pytest.mark.parametrize("d,rot,halves", [(64, 64, False), (128, 64, True)])
def test_norm_of_rows_whose_squares_leave_fp32(T, d, rot, halves):
    """BF16 rows of 1e16 to 3e38, and of 1e-16 to 1e-38 with an eps of 0 or small beside their squares."""
    torch, thinfer = T
    rng = np.random.default_rng(d)
    sizes = np.array([1e16, 1e18, 1e19, 3e20, 1e30, 1e37, 9e37, 1.0, 1e-12, 1e-16, 1e-19, 1e-22, 1e-30, 1e-36])
    n = len(sizes)
    x = kv4.round_to(np.clip(rng.standard_normal((n, 3, d)), -3.5, 3.5) * sizes[:, None, None], "bf16")
    gain = kv4.round_to(1 + 0.1 * rng.standard_normal(d), "bf16")
    turns = 10000.0 ** (-2 * np.arange(rot // 2) / rot) / (2 * np.pi)
    pos = rng.integers(0, 5000, n)
    for eps in (0.0, 1e-40, 1e-30, 1e-24, 1e-6):
        got = thinfer.op_qk_norm_rope(_dev(torch, x[:, :2], "bf16"), _dev(torch, x[:, 2:], "bf16"), _dev(torch, gain, "bf16"), _dev(torch, gain, "bf16"), eps,
                                      torch.tensor(turns, device="cuda"), _int(torch, pos.tolist()), halves=halves)
        # eps is FP32 in the call
        want = kv4.qk_norm_rope(x, gain, float(np.float32(eps)), turns, pos, halves)
        got = np.concatenate([_host(g) for g in got], 1)
        big = np.max(np.abs(want), axis=-1, keepdims=True)
        # as in test_norm_and_rotation; results below the smallest normal number are on BF16's grid of 2^-133
        assert np.all(np.abs(got - want) <= EPS["bf16"] * np.abs(want) + 2.0 ** -18 * big + 2.0 ** -133), eps


def test_norm_of_many_rows_with_such_rows_among_them(T):
    """Lane groups that walk several heads of a token; gains so large that a finished row looks like one of those rows, in place
    too."""
    torch, thinfer = T
    g = torch.Generator(device="cuda").manual_seed(7)
    n, hq, hkv, d = 2400, 30, 10, 128
    x = torch.randn(n, hq + hkv, d, generator=g, device="cuda", dtype=torch.float64)
    x *= torch.where(torch.rand(n, hq + hkv, 1, generator=g, device="cuda") < 0.1, 1e25, 1.0)
    x = x.bfloat16()
    gain = (1e20 * (1 + 0.1 * torch.randn(d, generator=g, device="cuda", dtype=torch.float64))).bfloat16()
    turns, pos = thinfer.rope_turns(1e4, d), torch.randint(0, 4000, (n,), generator=g, device="cuda").to(torch.int32)
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + float(np.float32(1e-6))) * gain.double()
    angle = 2 * np.pi * torch.remainder(pos.double()[:, None] * turns, 1.0)[:, None]
    a, b = y[..., 0::2], y[..., 1::2]
    want = torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).flatten(-2)
    q, k = thinfer.op_qk_norm_rope(x[:, :hq], x[:, hq:], gain, gain, 1e-6, turns, pos)
    tol = EPS["bf16"] * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)
    assert torch.all((torch.cat([q, k], 1).double() - want).abs() <= tol)
    thinfer.op_qk_norm_rope(x[:, :hq], x[:, hq:], gain, gain, 1e-6, turns, pos, q_out=x[:, :hq], k_out=x[:, hq:])
    assert torch.equal(x, torch.cat([q, k], 1))


# ------------------------------------------------------------------ the same bits every time
@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("hq,hkv,d,page,lens,queries", [
    (8, 8, 128, 64, [1500, 3, 0, 700], 1), (16, 4, 64, 16, [9000, 1, 4000], 1), (64, 8, 128, 16, [2100, 1999, 4001], 4), (40, 40, 128, 64, [640, 1279, 1000], 1),
    (2, 1, 64, 32, [33000], 1)])
def test_attention_repeats_itself_bit_by_bit(T, t, hq, hkv, d, page, lens, queries):
    """Pairs that are cut across warps and CTAs are merged in a fixed order: twenty calls, some of them beside other work, give
    the same bits, NaN and all."""
    torch, thinfer = T
    g = torch.Generator(device="cuda").manual_seed(hq + d)
    width = max(-(-n // page) for n in lens) + 1
    n_pages = len(lens) * width
    pool = torch.randint(0, 256, (n_pages, hkv * page * (d + 8)), dtype=torch.uint8, device="cuda", generator=g)
    params = torch.rand(n_pages, hkv, 2 * page, 2, generator=g, device="cuda") * 0.2 + 0.2
    params[..., 1] *= -7
    pool.view(n_pages, hkv, -1)[..., page * d:] = params.to(_tt(torch, t)).view(torch.uint8).reshape(n_pages, hkv, -1)
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(len(lens), width)
    q = torch.randn(len(lens), queries, hq, d, generator=g, device="cuda").to(_tt(torch, t))
    q[-1, 0, 0, 0] = float("nan")                           # one query column that is NaN throughout
    lens, side = _int(torch, lens), torch.cuda.Stream()
    first = thinfer.op_kv4_attention(q, pool, table, lens, page)
    assert first[-1, 0, 0].isnan().all() and first.isfinite().sum() == first.numel() - d
    busy = torch.randn(2048, 2048, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for i in range(20):
        if i % 3 == 1:
            with torch.cuda.stream(side):
                busy = busy @ busy * 1e-3                   # takes SMs, so that CTAs begin at other times
        again = thinfer.op_kv4_attention(q, pool, table, lens, page)
        assert torch.equal(again.view(torch.int16), first.view(torch.int16)), i
    torch.cuda.synchronize()


def test_attention_with_the_callers_workspace(T):
    """One workspace for calls in a row, full of NaN at first, of the least size and of a larger one; a smaller one is refused."""
    import ctypes as C
    torch, thinfer = T
    rng = np.random.default_rng(4)
    x = kv4.round_to(rng.standard_normal((700, 2, 64)), np.float16)
    pool, table, _, _, _ = _one_row(torch, thinfer, x, x[::-1], "f16", 16)
    tab, lens = _int(torch, table), _int(torch, [700])
    need = C.c_size_t(0)
    assert thinfer.lib().thinfer_kv4_attention_workspace(1, 3, 8, 2, 64, C.byref(need)) == thinfer.OK
    for extra in (0, 4096):
        ws = torch.full((need.value + extra,), 255, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            q = torch.randn(1, 3, 8, 64, device="cuda").half()
            assert torch.equal(thinfer.op_kv4_attention(q, pool, tab, lens, 16, workspace=ws), thinfer.op_kv4_attention(q, pool, tab, lens, 16))
        assert torch.all(ws[need.value:] == 255)
    with pytest.raises(thinfer.ThinferError) as e:
        thinfer.op_kv4_attention(q, pool, tab, lens, 16, workspace=ws[:need.value - 1])
    assert e.value.code == thinfer.ECAPACITY


@pytest.mark.parametrize("n", [1, 50, 700])
def test_attention_of_large_values(T, n):
    """V rows of 1e31 to 1e34, and K rows of scales on either side of 2^104 under queries as small."""
    rng = np.random.default_rng(n)
    for q_size, k_size, v_size in ((1.0, 1.0, 1e31), (1.0, 1.0, 1e33), (1.0, 1.0, 1e34), (1e-31, 1e31, 1e32), (1e-33, 1e33, 1e33)):
        _attend(T, rng, rng.standard_normal((1, 4, 64)) * q_size, rng.standard_normal((n, 2, 64)) * k_size, rng.standard_normal((n, 2, 64)) * v_size)


# ------------------------------------------------------------------ tables of more than 65536 entries
def _long_tables(rng, rows, width, n_pages, page, fill):
    counts = rng.multinomial(int(n_pages * fill), [1 / rows] * rows).clip(0, width)
    lens = [int(max(0, c * page - rng.integers(0, page))) if c else 0 for c in counts]
    ids, table, at = rng.permutation(n_pages), [], 0
    for c in counts:
        table.append([int(i) for i in ids[at:at + c]] + [int(i) for i in rng.integers(-3, n_pages, width - c)])    # stale entries behind
        at += c
    return table, lens


@pytest.mark.parametrize("rows,width,n_pages,page,fill", [(64, 2048, 7000, 16, 0.7), (3, 30000, 9000, 16, 0.6), (4096, 17, 9000, 32, 0.8), (300, 257, 7000, 128, 0.95)])
def test_page_calls_over_long_tables(T, rows, width, n_pages, page, fill):
    torch, thinfer = T
    assert rows * width > 65536
    rng = np.random.default_rng(rows)
    table, lens = _long_tables(rng, rows, width, n_pages, page, fill)
    t_in, l_in = _int(torch, table), _int(torch, lens)
    add = [int(x) for x in rng.integers(-2, 3 * page, rows)]
    want = kv4.reserve(table, lens, add, n_pages, page)
    tab = t_in.clone()
    out, refused = thinfer.op_kv4_reserve(tab, l_in, _int(torch, add), n_pages, page)
    assert tab.tolist() == want[0] and out.tolist() == want[1] and refused.item() == want[2]
    g = torch.Generator(device="cuda").manual_seed(rows)
    start = torch.randint(0, 256, (1, n_pages, page * 72), dtype=torch.uint8, device="cuda", generator=g)
    # the oracle's fork looks through all rows for every row: take few distinct sources where there are many rows
    source = [int(x) for x in (rng.integers(-1, rows, rows) if rows <= 300 else np.repeat(rng.integers(-1, rows, 16), rows // 16))]
    tab, l, refused, moves = kv4.fork(table, lens, source, n_pages, page)
    pool = start.clone()
    t_out, l_out, bad = thinfer.op_kv4_fork(pool, t_in, l_in, _int(torch, source), page, 64)
    assert t_out.tolist() == tab and l_out.tolist() == l and bad.item() == refused
    assert np.array_equal(pool.cpu().numpy(), kv4.copied(start.cpu().numpy(), moves, 1, 64, page))
    tab, live, moves = kv4.compact(table, lens, n_pages, page)
    pool = start.clone()
    t_out, count = thinfer.op_kv4_compact(pool, t_in, l_in, page, 64)
    assert t_out.tolist() == tab and count.item() == live and t_in.tolist() == table
    assert np.array_equal(pool.cpu().numpy(), kv4.copied(start.cpu().numpy(), moves, 1, 64, page))


def test_calls_with_nothing_to_do_are_refused(T):
    torch, thinfer = T
    pool = torch.zeros(2, 16 * 72, dtype=torch.uint8, device="cuda")
    kv, z, none = torch.zeros(0, 1, 64, dtype=torch.float16, device="cuda"), _int(torch, [0]), torch.zeros(0, dtype=torch.int32, device="cuda")
    gain, tab, no_rows = torch.ones(64, dtype=torch.float16, device="cuda"), _int(torch, [[0]]), torch.zeros(0, 1, dtype=torch.int32, device="cuda")
    for call in (lambda: thinfer.op_qk_norm_rope(kv, kv, gain, gain, 1e-6, thinfer.rope_turns(1e4, 64), none),
                 lambda: thinfer.op_kv4_append(pool, tab, kv, kv, none, none, 16), lambda: thinfer.op_kv4_read(pool, tab, none, none, 16, 64, kv.dtype),
                 lambda: thinfer.op_kv4_attention(kv.view(0, 1, 1, 64), pool, no_rows, none, 16), lambda: thinfer.op_kv4_reserve(no_rows, none, none, 2, 16),
                 lambda: thinfer.op_kv4_fork(pool[None], no_rows, none, none, 16, 64), lambda: thinfer.op_kv4_compact(pool[None], no_rows, none, 16, 64),
                 lambda: thinfer.op_kv4_reserve(torch.zeros(1, 0, dtype=torch.int32, device="cuda"), z, z, 2, 16),
                 lambda: thinfer.op_kv4_append(pool[:0], tab, kv, kv, none, none, 16)):
        with pytest.raises(thinfer.ThinferError) as e:
            call()
        assert e.value.code == thinfer.EINVAL


@pytest.mark.parametrize("n,hkv", [(1, 3), (4, 1), (1, 1)])
def test_read_into_outputs_whose_strides_differ_where_there_is_one(T, n, hkv):
    torch, thinfer = T
    x = kv4.round_to(np.random.default_rng(n).standard_normal((n, hkv, 64)), np.float16)
    pool, table, rows, pos, _ = _one_row(torch, thinfer, x, -x, "f16", 16)
    want = thinfer.op_kv4_read(pool, _int(torch, table), rows, pos, 16, 64, torch.float16)
    k = torch.empty_strided((n, hkv, 64), (64 * hkv if n > 1 else 3, 64 if hkv > 1 else 0, 1), dtype=torch.float16, device="cuda")
    v = torch.empty_strided((n, hkv, 64), (64 * hkv if n > 1 else 4096, 64 if hkv > 1 else 8, 1), dtype=torch.float16, device="cuda")
    thinfer.op_kv4_read(pool, _int(torch, table), rows, pos, 16, 64, torch.float16, k_out=k, v_out=v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    with pytest.raises(thinfer.ThinferError):
        thinfer.op_kv4_read(pool, _int(torch, table), rows, pos, 16, 64, torch.float16, k_out=k, v_out=torch.empty(n, hkv, 128, dtype=k.dtype, device="cuda")[..., ::2])


@pytest.mark.parametrize("n", [1, 50, 700])
def test_attention_of_tiny_values(T, n):
    """V rows of 1e-28 to 1e-36, some of them constant (scale 0)."""
    rng = np.random.default_rng(n + 1)
    for v_size in (1e-28, 1e-31, 1e-33, 1e-35, 1e-36):
        v = rng.standard_normal((n, 2, 64)) * v_size
        v[::3, 0] = v[::3, 0, :1]
        _attend(T, rng, rng.standard_normal((1, 4, 64)), rng.standard_normal((n, 2, 64)), v)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_scales_beside_the_middle_of_two(T, t):
    """Rows whose max - min is 15 times the middle of two values of the type, or just beside that: by less than FP32 can tell."""
    rng = np.random.default_rng(15)
    bits, rows = {"f16": 11, "bf16": 8}[t], []
    while len(rows) < 600:
        e = int(rng.integers(-6, 3)) if t == "f16" else int(rng.integers(-40, 40))
        far = 15.0 * (2 * int(rng.integers(2 ** (bits - 1), 2 ** bits)) + 1) * 2.0 ** e       # 15 times a middle
        high = float(kv4.round_to(far, DT[t]))
        low = -(far - high)
        if not 0 < abs(high) < 65504 or low >= 0:
            continue
        low = float(kv4.round_to(low, DT[t]))
        step = 2.0 ** (np.floor(np.log2(-low)) - bits + 1)
        low += step * int(rng.integers(-2, 3))                                                # 0: on the middle itself
        x = rng.uniform(low, high, 64)
        x[0], x[1] = high, low
        rows.append(x)
    _written_bytes_are_the_definitions(T, kv4.round_to(np.array(rows), DT[t]), t)


def test_reserve_behind_a_row_whose_length_is_beyond_its_table(T):
    """It is refused, and the rows behind it get the pages that its length, as it stands, leaves them."""
    torch, thinfer = T
    for lens, add in (([33, 5, 16], [10, 20, 1]), ([33, 5, 16], [20, 20, 1]), ([48, 0, 0], [0, 3, 4]), ([47, 1, 1], [2, 40, 20])):
        table = [[7, 8], [9, -1], [3, -1]]
        want = kv4.reserve(table, lens, add, 10, 16)
        tab = _int(torch, table)
        out, refused = thinfer.op_kv4_reserve(tab, _int(torch, lens), _int(torch, add), 10, 16)
        assert tab.tolist() == want[0] and out.tolist() == want[1] and refused.item() == want[2], (lens, add)


def test_calls_from_several_threads(T):
    """Four threads, each with its own stream, sizes, results and refusals."""
    import threading
    torch, thinfer = T
    rng = np.random.default_rng(3)
    jobs = []
    for i in range(4):
        n, t = (900, 33, 2500, 300)[i], ("f16", "bf16")[i % 2]
        k, v = (kv4.round_to(rng.standard_normal((n, 2, 64)), DT[t]) for _ in range(2))
        pool, table, rows, pos, _ = _one_row(torch, thinfer, k, v, t, 16)
        q = torch.from_numpy(rng.standard_normal((1, 1, 8, 64))).to(_tt(torch, t)).cuda()
        tab, lens = _int(torch, table), _int(torch, [n])
        jobs.append((pool, tab, rows, pos, _dev(torch, k, t), _dev(torch, v, t), q, lens, thinfer.op_kv4_attention(q, pool, tab, lens, 16)))
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        pool, tab, rows, pos, k, v, q, lens, want = jobs[i]
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for j in range(60):
                    mine = torch.full_like(pool, 255)
                    thinfer.op_kv4_append(mine, tab, k, v, rows, pos, 16)
                    out = thinfer.op_kv4_attention(q, mine, tab, lens, 16)
                    _, refused = thinfer.op_kv4_reserve(tab.clone(), lens, lens * 0, 1000 + 50 * i, 16)
                    try:
                        thinfer.op_kv4_attention(q, mine, tab, lens, 17 + i)
                        wrong.append((i, j, "not refused"))
                    except thinfer.ThinferError as e:
                        if f"multiple of {(17 + i) * 72} bytes" not in str(e):
                            wrong.append((i, j, str(e)))
                    torch.cuda.current_stream().synchronize()
                    if not (torch.equal(mine, pool) and torch.equal(out, want) and refused.item() == 0):
                        wrong.append((i, j))
        except Exception as e:  # noqa: BLE001  (told by the test)
            wrong.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not wrong, wrong[:3]
