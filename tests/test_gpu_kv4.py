"""Per-head norm with rotation and the 4-bit paged cache against their float64 definitions (run with -m gpu on a B200).

Tolerances.  A stored result is rounded to the storage type once: half a unit in the last place, EPS * |value| with
EPS = 2^-11 (FP16) or 2^-8 (BF16), and 2^-25 at the bottom of FP16's subnormals.  What the FP32 arithmetic before it
may add is written at each test.
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
    """float64 values of the storage type -> CUDA tensor."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(_tt(torch, t)).cuda()


def _host(x):
    return x.double().cpu().numpy()


def _int(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _values(rng, shape, t, std=1.0):
    return kv4.round_to(rng.standard_normal(shape) * std, DT[t])


# ------------------------------------------------------------------ norm + rotation
@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("tokens,hq,hkv,d,rot,halves", [
    (1, 64, 8, 128, 128, False), (1, 4, 4, 64, 64, True), (3, 5, 1, 128, 64, True), (33, 8, 2, 64, 32, False), (130, 4, 2, 128, 128, True),
    (17, 12, 12, 128, 16, True), (9, 3, 3, 64, 0, False), (2, 1, 1, 128, 112, True), (700, 8, 8, 64, 64, False), (65, 40, 40, 128, 128, False)])
def test_norm_and_rotation(T, t, tokens, hq, hkv, d, rot, halves):
    torch, thinfer = T
    rng = np.random.default_rng(tokens * 31 + d + rot)
    x = _values(rng, (tokens, hq + 2 * hkv, d), t, 2.0)
    gains = [kv4.round_to(1 + 0.1 * rng.standard_normal(d), DT[t]) for _ in range(2)]
    pos = rng.integers(0, [1, 5000, 2 ** 31 - 1][tokens % 3], tokens)
    pos[0] = 0
    if tokens > 2:
        pos[1] = -1                               # padding: left as it was
    turns = 10000.0 ** (-2 * np.arange(rot // 2) / max(rot, 1)) / (2 * np.pi)
    qkv = _dev(torch, x, t).view(tokens, -1)      # q and k lie inside one fused row
    q, k = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    before = qkv.clone()
    tu = torch.tensor(turns, dtype=torch.float64, device="cuda")
    qo = torch.full((tokens, hq, d), 7.0, dtype=_tt(torch, t), device="cuda")
    ko = torch.full((tokens, hkv + 1, d), 7.0, dtype=_tt(torch, t), device="cuda")[:, :hkv]      # a strided output
    args = (_dev(torch, gains[0], t), _dev(torch, gains[1], t), 1e-6, tu, _int(torch, pos.tolist()))
    thinfer.op_qk_norm_rope(q, k, *args, halves=halves, q_out=qo, k_out=ko)
    assert torch.equal(qkv, before)
    for got, part, gain in ((_host(qo), x[:, :hq], gains[0]), (_host(ko), x[:, hq:hq + hkv], gains[1])):
        want = kv4.qk_norm_rope(part, gain, 1e-6, turns, pos, halves)
        # FP32 before the rounding: norm, gain and rotation are ~8 roundings of 2^-24 of the pair's length, rsqrt, sine
        # and cosine 2 units each, the angle 2 pi 2^-25: below 2^-19 of the pair's length, itself <= sqrt(2) * max
        big = np.max(np.abs(want), axis=-1, keepdims=True)
        tol = EPS[t] * np.abs(want) + 2.0 ** -18 * big + 2.0 ** -25
        live = pos >= 0
        assert np.all(np.abs(got - want)[live] <= tol[live])
        assert np.all(got[~live] == 7.0)
    # in place: the same bits
    thinfer.op_qk_norm_rope(q, k, *args, halves=halves, q_out=q, k_out=k)
    live = torch.tensor(pos >= 0)
    assert torch.equal(q.cpu()[live], qo.cpu()[live]) and torch.equal(k.cpu()[live], ko.cpu()[live])
    assert torch.equal(qkv[~live.cuda()], before[~live.cuda()]) and torch.equal(qkv[:, (hq + hkv) * d:], before[:, (hq + hkv) * d:])


def test_norm_of_zero_and_nonfinite_rows(T):
    torch, thinfer = T
    q = torch.zeros(1, 3, 64, dtype=torch.float16, device="cuda")
    q[0, 1] = 1.0
    q[0, 2, 5] = float("nan")
    one = torch.ones(64, dtype=torch.float16, device="cuda")
    tu = thinfer.rope_turns(10000.0, 64)
    out, _ = thinfer.op_qk_norm_rope(q, q[:, :1], one, one, 1e-6, tu, _int(torch, [0]))
    assert torch.all(out[0, 0] == 0) and torch.all((out[0, 1] - 1).abs() <= 2 ** -10) and torch.all(out[0, 2].isnan())


# ------------------------------------------------------------------ append and read
def _fresh_pool(torch, n_pages, hkv, d, page, layers=None):
    """0xFF bytes: params are NaN wherever nothing has been written."""
    shape = (n_pages, hkv * page * (d + 8)) if layers is None else (layers, n_pages, hkv * page * (d + 8))
    return torch.full(shape, 255, dtype=torch.uint8, device="cuda")


def _grid(rng, shape):
    """Multiples of 2^-9 below 4: x - min and the codes' quotients are then exact enough in FP32 that no code can differ
    (2 (x - min) - (2k + 1) scale is a multiple of 2^-14, so a quotient that is no tie is 2^-14 away from one)."""
    return np.clip(np.rint(rng.standard_normal(shape) * 512), -2000, 2000) / 512


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("hkv,d,page", [(1, 64, 16), (3, 128, 16), (2, 64, 128), (2, 128, 64), (5, 64, 32)])
def test_append_and_read(T, t, hkv, d, page):
    torch, thinfer = T
    rng = np.random.default_rng(hkv * 100 + d + page)
    n_pages, width = 12, 4
    ids = rng.permutation(n_pages)[:8]
    table = [[int(i) for i in ids[:4]], [int(i) for i in ids[4:7]] + [-1], [int(ids[7]), n_pages, -5, -1]]
    spots = [(0, p) for p in range(3, min(4 * page, 90))] + [(1, p) for p in (0, 1, page - 1, page, 3 * page - 1)] + [(2, 0)]
    spots = [spots[i] for i in rng.permutation(len(spots))]
    # skipped (negative), no page of the pool, behind the table, a row that is none: nothing is written for these
    bad = [(-1, 3), (0, -2), (2, page), (2, 2 * page + 1), (1, 3 * page), (0, 4 * page), (3, 0), (2, 3 * page)]
    every = spots[:5] + bad + spots[5:]
    n = len(every)
    k, v = _grid(rng, (n, hkv, d)), _grid(rng, (n, hkv, d))
    k, v = kv4.round_to(k, DT[t]), kv4.round_to(v, DT[t])
    k[0], v[1, 0] = 2.5, -0.375                       # constant rows: scale 0
    pool = _fresh_pool(torch, n_pages, hkv, d, page)
    ref = kv4.Pool(pool.cpu().numpy().copy(), hkv, d, page, DT[t])
    both = _dev(torch, np.stack([k, v], 1), t).view(n, -1)      # k and v side by side in one row: strided inputs
    kd, vd = both[:, :hkv * d].unflatten(1, (hkv, d)), both[:, hkv * d:].unflatten(1, (hkv, d))
    tab, rows, pos = _int(torch, table), _int(torch, [s[0] for s in every]), _int(torch, [s[1] for s in every])
    thinfer.op_kv4_append(pool, tab, kd, vd, rows, pos, page)
    for i, (r, p) in enumerate(every):
        if (r, p) in spots:
            for h in range(hkv):
                ref.write(table[r][p // page], p % page, h, 0, k[i, h])
                ref.write(table[r][p // page], p % page, h, 1, v[i, h])
    assert np.array_equal(pool.cpu().numpy(), ref.data)
    # read back: the values, NaN where there is no page, padding left alone
    ko = torch.full((hkv, n, d), 7.0, dtype=_tt(torch, t), device="cuda").transpose(0, 1)
    vo = torch.full((hkv, n, d), 7.0, dtype=_tt(torch, t), device="cuda").transpose(0, 1)
    thinfer.op_kv4_read(pool, tab, rows, pos, page, d, _tt(torch, t), k_out=ko, v_out=vo)
    ko, vo = _host(ko), _host(vo)
    for i, (r, p) in enumerate(every):
        for h in range(hkv):
            for which, got in ((0, ko[i, h]), (1, vo[i, h])):
                if r < 0 or p < 0:
                    assert np.all(got == 7.0)
                elif (r, p) in bad:
                    assert np.all(np.isnan(got))
                else:
                    want = ref.read(table[r][p // page], p % page, h, which)
                    # one FP32 rounding (2^-24) before the stored one
                    assert np.all(np.abs(got - want) <= EPS[t] * np.abs(want) * 1.001 + 2.0 ** -25)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_rows_with_nan_or_infinity_read_as_nan_and_touch_nobody_else(T, t):
    torch, thinfer = T
    pool, tab = _fresh_pool(torch, 1, 2, 64, 16), _int(torch, [[0]])
    k = torch.ones(4, 2, 64, dtype=_tt(torch, t), device="cuda")
    k[0, 0, 3], k[1, 1, 60], k[2, 0, 0] = float("nan"), float("inf"), float("-inf")
    rows, pos = _int(torch, [0] * 4), _int(torch, [0, 1, 2, 3])
    thinfer.op_kv4_append(pool, tab, k, k, rows, pos, 16)
    ko, vo = thinfer.op_kv4_read(pool, tab, rows, pos, 16, 64, k.dtype)
    nan = torch.zeros(4, 2, dtype=torch.bool, device="cuda")
    nan[0, 0] = nan[1, 1] = nan[2, 0] = True
    for o in (ko, vo):
        assert torch.equal(o.isnan(), nan[:, :, None].expand_as(o)) and torch.all(o[~nan] == 1)


def test_largest_values_and_tiny_ranges(T):
    torch, thinfer = T
    pool, tab = _fresh_pool(torch, 1, 1, 64, 16), _int(torch, [[0]])
    k = torch.zeros(3, 1, 64, dtype=torch.float16, device="cuda")
    k[0, 0, 0], k[0, 0, 1] = 65504, -65504
    k[1] = torch.arange(64, device="cuda").half().view(1, 64) * 2.0 ** -24      # subnormal values
    k[2] = 2048 + torch.arange(64, device="cuda").half().view(1, 64) * 2
    rows, pos = _int(torch, [0, 0, 0]), _int(torch, [5, 6, 7])
    thinfer.op_kv4_append(pool, tab, k, k, rows, pos, 16)
    ref = kv4.Pool(np.full((1, 16 * 72), 255, np.uint8), 1, 64, 16, np.float16)
    for i in range(3):
        for w in (0, 1):
            ref.write(0, 5 + i, 0, w, _host(k)[i, 0])
    assert np.array_equal(pool.cpu().numpy(), ref.data)


@pytest.mark.parametrize("t,tokens,hkv,d,page", [("f16", 900, 40, 128, 64), ("bf16", 4100, 8, 128, 16), ("bf16", 9001, 1, 128, 128),
                                                 ("f16", 2500, 24, 64, 32), ("bf16", 7000, 6, 64, 16), ("f16", 333, 33, 128, 16)])
def test_many_tokens_in_one_call_and_in_small_ones(T, t, tokens, hkv, d, page):
    """How the rows of a call are shared out depends on its size; the bytes and values do not."""
    torch, thinfer = T
    g = torch.Generator(device="cuda").manual_seed(tokens)
    width, rows_n = -(-tokens // 5 // page) + 2, 5
    n_pages = rows_n * width
    tab = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(rows_n, width)
    rows = (torch.arange(tokens, device="cuda") % rows_n).to(torch.int32)
    pos = (torch.arange(tokens, device="cuda") // rows_n + 3).to(torch.int32)
    rows[::17], pos[5::23] = -1, -4                                       # padding
    k, v = (torch.randn(tokens, hkv, d, generator=g, device="cuda").to(_tt(torch, t)) for _ in range(2))
    one, many = _fresh_pool(torch, n_pages, hkv, d, page), _fresh_pool(torch, n_pages, hkv, d, page)
    thinfer.op_kv4_append(one, tab, k, v, rows, pos, page)
    for i in range(0, tokens, 61):
        s = slice(i, i + 61)
        thinfer.op_kv4_append(many, tab, k[s], v[s], rows[s], pos[s], page)
    assert torch.equal(one, many)
    out = [torch.full_like(k, 7.0) for _ in range(4)]
    thinfer.op_kv4_read(one, tab, rows, pos, page, d, k.dtype, k_out=out[0], v_out=out[1])
    for i in range(0, tokens, 61):
        s = slice(i, i + 61)
        thinfer.op_kv4_read(one, tab, rows[s], pos[s], page, d, k.dtype, k_out=out[2][s], v_out=out[3][s])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    skip = (rows < 0) | (pos < 0)
    assert torch.all(out[0][skip] == 7.0)
    # half a step is span / 30; the rounding of the scale moves the step by EPS of itself, 15 of them by EPS of the span; the
    # value read is rounded once
    for x, y in ((k, out[0]), (v, out[1])):
        x, y = x[~skip].double(), y[~skip].double()
        span = x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)
        assert torch.all((x - y).abs() <= span * (1 / 30 + 2 * EPS[t]) + y.abs() * EPS[t])


def test_a_block_far_into_a_large_pool(T):
    """Byte offsets beyond 2^32."""
    torch, thinfer = T
    hkv, d, page = 40, 128, 128
    n_pages = (5 << 30) // (hkv * page * (d + 8))
    pool = torch.zeros(n_pages, hkv * page * (d + 8), dtype=torch.uint8, device="cuda")
    tab = _int(torch, [[n_pages - 1, 2]])
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(200, hkv, d, generator=g, device="cuda").half()
    rows, pos = torch.zeros(200, dtype=torch.int32, device="cuda"), torch.arange(200, device="cuda", dtype=torch.int32)
    thinfer.op_kv4_append(pool, tab, k, -k, rows, pos, page)
    ko, vo = thinfer.op_kv4_read(pool, tab, rows, pos, page, d, torch.float16)
    step = (k.float().amax(-1) - k.float().amin(-1)) / 15
    # half a step, the rounding of the scale (15 * 2^-11 of a step) and of the stored value (|x| < 6: 2^-9)
    assert torch.all((ko.float() - k.float()).abs() <= step[..., None] * 0.51 + 2.0 ** -9)
    assert torch.all((vo.float() + k.float()).abs() <= step[..., None] * 0.51 + 2.0 ** -9)
    q = torch.randn(1, 1, 2 * hkv, d, generator=g, device="cuda").half()
    out = thinfer.op_kv4_attention(q, pool, tab, _int(torch, [200]), page).double()
    kd, vd = (x.double().permute(1, 0, 2) for x in (ko, vo))
    p = torch.softmax(q.double().view(hkv, 2, d) @ kd.transpose(1, 2) / d ** 0.5, -1)
    want = (p @ vd).view(1, 1, 2 * hkv, d)
    # the reference uses the rounded values: EPS of K moves scores by <= 2^-11 * |q|.|k| / sqrt(d) ~ 0.05, in effect an
    # average over 200 keys; a wrong page would be off by the size of the output
    assert (out - want).norm() / want.norm() < 0.02
    del pool
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ attention
def _filled(T, rng, t, hkv, d, page, lens, extra=3, k_std=1.0, v_std=1.0, spread=0.0):
    """A pool whose rows hold random tokens on scattered pages; everything else has NaN params."""
    torch, thinfer = T
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + extra
    width = max(counts + [1]) + 1
    ids = rng.permutation(n_pages)
    table, at = [], 0
    for c in counts:
        table.append([int(i) for i in ids[at:at + c]] + [-1] * (width - c))
        at += c
    pool = _fresh_pool(torch, n_pages, hkv, d, page)
    tab = _int(torch, table)
    total = sum(lens)
    if total:
        k, v = _values(rng, (total, hkv, d), t, k_std), rng.standard_normal((total, hkv, d)) * v_std
        if spread:                                      # V rows whose sizes differ by powers of two
            v = v * 2.0 ** rng.integers(-spread, spread, (total, hkv, 1))
        v = kv4.round_to(v, DT[t])
        rows = np.repeat(np.arange(len(lens)), lens)
        pos = np.concatenate([np.arange(n) for n in lens])
        thinfer.op_kv4_append(pool, tab, _dev(torch, k, t), _dev(torch, v, t), _int(torch, rows.tolist()), _int(torch, pos.tolist()), page)
    return pool, tab, table


def kv4_abs(kv, q, n, shift):
    """sum_t p_t |v_t| of every head."""
    return kv4.attention(q, (kv[0], np.abs(kv[1])), n, shift)[0]


def _check_attention(T, rng, t, hq, hkv, d, page, lens, queries, pool, tab, table, q_std=1.0, strided=False, lens_dev=None):
    torch, thinfer = T
    b = len(lens)
    q = _values(rng, (b, queries, hq, d), t, q_std)
    if strided:                                         # q inside a wider fused row
        wide = torch.zeros(b, queries, (hq + 2 * hkv) * d, dtype=_tt(torch, t), device="cuda")
        wide[..., :hq * d] = _dev(torch, q, t).view(b, queries, -1)
        qd = wide[..., :hq * d].unflatten(2, (hq, d))
    else:
        qd = _dev(torch, q, t)
    out = thinfer.op_kv4_attention(qd, pool, tab, _int(torch, lens) if lens_dev is None else lens_dev, page)
    again = thinfer.op_kv4_attention(qd, pool, tab, _int(torch, lens) if lens_dev is None else lens_dev, page)
    assert torch.equal(out, again) or torch.equal(out.isnan(), again.isnan())
    got = _host(out)
    ref = kv4.Pool(pool.cpu().numpy(), hkv, d, page, DT[t])
    for i in range(b):
        kv = kv4.keys_values(ref, table[i], lens[i])
        for n in range(queries):
            want, spread, mag = kv4.attention(q[i, n], kv, lens[i], queries - 1 - n)
            # v = mid + scale (code - 8) with mid = offset + 8 scale: sum p mid is FP32, and the weights p scale of the second
            # part are rounded to 11 bits, so that each rounding moves the result by at most
            # 2^-11 p scale |code - 8| = 2^-11 p |v - mid|.  mid is half a step above the middle of the row's range, or a
            # whole one where no code is 15 (then 14 is the largest): |v - mid| <= |v - middle| + range / 14, which is less
            # than twice a term of `spread`
            # Scores in FP32 from exact products: the code part sums terms of up to 15 steps of a row, about four times |k|,
            # in eight accumulation steps of 2^-22: 8 * 4 * 2^-22 = 2^-17 of the largest sum |q k| / sqrt(d) in the exponent
            # of numerator and denominator, 2^-16 in all (2^-15 with the offset part), times the distance of a key's value
            # from the result, at most spread + |want| + sum p |v|
            far = spread + np.abs(want) + kv4_abs(kv, q[i, n], lens[i], queries - 1 - n)
            tol = EPS[t] * np.abs(want) + 2.0 ** -10 * spread + 2.0 ** -19 * (1 + 16 * mag) * far + 2.0 ** -25
            bad = np.abs(got[i, n] - want) > tol
            assert not bad.any(), (i, n, lens[i], np.argwhere(bad)[:3], np.max(np.abs(got[i, n] - want) / tol))


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("hq,hkv,d,page,lens,queries", [
    (8, 1, 128, 64, [1], 1), (4, 4, 64, 16, [0], 1), (2, 1, 64, 16, [15, 16, 17, 0, 31, 32, 33], 1), (8, 2, 128, 16, [257, 1, 64, 65, 63], 1),
    (5, 5, 128, 64, [130, 7, 300], 1), (6, 2, 64, 32, [95, 500], 1), (16, 1, 128, 64, [511, 40], 1), (24, 2, 64, 128, [129, 400, 128], 1),
    (10, 2, 128, 64, [77, 0, 1000], 1), (8, 2, 128, 16, [3, 1, 0, 90], 4), (4, 4, 64, 64, [70, 2, 129], 3), (16, 2, 128, 32, [45, 200], 2),
    (8, 1, 64, 16, [33, 5], 7), (3, 1, 128, 128, [129, 31], 5), (64, 2, 64, 64, [65, 7], 1), (2, 2, 128, 64, [66, 12, 13, 11, 10], 12), (1, 1, 64, 16, [2500], 1), (8, 8, 128, 128, [1500, 3], 1)])
def test_attention(T, t, hq, hkv, d, page, lens, queries):
    rng = np.random.default_rng(hq * 1000 + d + sum(lens) + queries)
    pool, tab, table = _filled(T, rng, t, hkv, d, page, lens)
    _check_attention(T, rng, t, hq, hkv, d, page, lens, queries, pool, tab, table, strided=len(lens) % 2 == 1)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_attention_with_sharp_and_uneven_rows(T, t):
    """Scores of hundreds (one key takes all the weight), V rows whose scales differ by up to 2^16, tiny queries."""
    rng = np.random.default_rng(11)
    lens = [200, 61]
    for q_std, k_std, spread in ((12.0, 6.0, 0), (1.0, 1.0, 8), (1e-3, 1.0, 0), (200.0, 0.01, 8)):
        pool, tab, table = _filled(T, rng, t, 2, 128, 16, lens, k_std=k_std, spread=spread)
        _check_attention(T, rng, t, 8, 2, 128, 16, lens, 1, pool, tab, table, q_std=q_std)


@pytest.mark.parametrize("batch,n", [(40, 37), (3, 9000), (130, 5)])
def test_attention_over_many_and_long_rows(T, batch, n):
    """Work that is cut across many CTAs at uneven places, against float64 on the device."""
    torch, thinfer = T
    hq, hkv, d, page = 16, 4, 64, 64
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, n + 1, batch)]
    lens[0] = n
    pool, tab, _ = _filled(T, rng, "f16", hkv, d, page, lens)
    q = torch.from_numpy(rng.standard_normal((batch, 1, hq, d))).half().cuda()
    got = thinfer.op_kv4_attention(q, pool, tab, _int(torch, lens), page).double()
    for i, m in enumerate(lens):
        if m == 0:
            assert torch.all(got[i] == 0)
            continue
        pos = torch.arange(m, dtype=torch.int32, device="cuda")
        kk, vv = _exact_rows(torch, pool, tab[i], m, hkv, d, page)
        s = torch.einsum("hgd,thd->hgt", q[i, 0].double().view(hkv, 4, d), kk) / 8.0
        p = torch.softmax(s, -1)
        want = torch.einsum("hgt,thd->hgd", p, vv).reshape(hq, d)
        low, high = vv.amin(-1, keepdim=True), vv.amax(-1, keepdim=True)
        spread = torch.einsum("hgt,thd->hgd", p, (vv - (low + high) / 2).abs() + (high - low) / 28).reshape(hq, d)
        mag = torch.einsum("hgd,thd->hgt", q[i, 0].double().view(hkv, 4, d).abs(), kk.abs()).amax(-1).reshape(hq, 1) / 8.0      # as above
        far = spread + want.abs() + torch.einsum("hgt,thd->hgd", p, vv.abs()).reshape(hq, d)
        tol = EPS["f16"] * want.abs() + 2.0 ** -10 * spread + 2.0 ** -19 * (1 + 16 * mag) * far + 2.0 ** -25
        assert torch.all((got[i, 0] - want).abs() <= tol)
        del pos


def test_attention_of_a_batch_of_rows_without_keys(T):
    torch, thinfer = T
    pool = _fresh_pool(torch, 3, 2, 64, 16)
    q = torch.randn(5, 2, 4, 64, device="cuda").half()
    for lens in ([0] * 5, [-3, 0, 0, -1, 0]):
        out = torch.full((5, 2, 4, 64), 7.0, dtype=torch.float16, device="cuda")
        thinfer.op_kv4_attention(q, pool, torch.full((5, 2), -1, dtype=torch.int32, device="cuda"), _int(torch, lens), 16, out=out)
        assert torch.all(out == 0)


def test_attention_of_2048_rows(T):
    """The most a call takes; every seventh row is empty, the last rows too."""
    torch, thinfer = T
    rng = np.random.default_rng(2048)
    lens = [0 if b % 7 == 0 or b >= 2040 else 1 + int(rng.integers(0, 70)) for b in range(2048)]
    pool, tab, table = _filled(T, rng, "f16", 1, 64, 16, lens)
    q = _values(rng, (2048, 1, 3, 64), "f16")
    out = _host(thinfer.op_kv4_attention(_dev(torch, q, "f16"), pool, tab, _int(torch, lens), 16))
    ref = kv4.Pool(pool.cpu().numpy(), 1, 64, 16, np.float16)
    for i in list(range(0, 2048, 97)) + list(range(2030, 2048)):
        kv = kv4.keys_values(ref, table[i], lens[i])
        want, spread, mag = kv4.attention(q[i, 0], kv, lens[i], 0)
        far = spread + np.abs(want) + kv4_abs(kv, q[i, 0], lens[i], 0)
        assert np.all(np.abs(out[i, 0] - want) <= EPS["f16"] * np.abs(want) + 2.0 ** -10 * spread + 2.0 ** -19 * (1 + 16 * mag) * far + 2.0 ** -25)
    assert np.all(out[::7] == 0) and np.all(out[2040:] == 0)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_attention_with_many_query_columns(T, t):
    """40 query tokens of 8 heads: 20 column tiles; some queries come before the first key."""
    rng = np.random.default_rng(40)
    lens = [39, 100, 12]
    pool, tab, table = _filled(T, rng, t, 1, 64, 16, lens)
    _check_attention(T, rng, t, 8, 1, 64, 16, lens, 40, pool, tab, table)


def test_attention_with_the_ends_of_bf16(T):
    """Values of 1e30 and of 1e-25 side by side with ordinary ones, and queries of 1e-20 and 1e10."""
    torch, thinfer = T
    rng = np.random.default_rng(30)
    for v_std, q_std, k_std in ((1e30, 1.0, 1.0), (1e-25, 1.0, 1.0), (1.0, 1e10, 1e-9), (1.0, 1e-20, 1e18)):
        pool, tab, table = _filled(T, rng, "bf16", 2, 64, 16, [50, 3], k_std=k_std, v_std=v_std)
        q = _values(rng, (2, 1, 4, 64), "bf16", q_std)
        out = _host(thinfer.op_kv4_attention(_dev(torch, q, "bf16"), pool, tab, _int(torch, [50, 3]), 16))
        ref = kv4.Pool(pool.cpu().numpy(), 2, 64, 16, "bf16")
        for i, n in enumerate((50, 3)):
            kv = kv4.keys_values(ref, table[i], n)
            want, spread, mag = kv4.attention(q[i, 0], kv, n, 0)
            far = spread + np.abs(want) + kv4_abs(kv, q[i, 0], n, 0)
            assert np.all(np.abs(out[i, 0] - want) <= EPS["bf16"] * np.abs(want) + 2.0 ** -10 * spread + 2.0 ** -19 * (1 + 16 * mag) * far)


def test_attention_of_queries_that_end_at_the_tables_edge(T):
    """A length one beyond the table: only the queries that see the key that has no page give NaN."""
    torch, thinfer = T
    rng = np.random.default_rng(31)
    pool, tab, table = _filled(T, rng, "f16", 1, 64, 16, [32])
    tab = tab[:, :2].contiguous()
    q = torch.randn(1, 3, 2, 64, device="cuda").half()
    out = thinfer.op_kv4_attention(q, pool, tab, _int(torch, [33]), 16)
    assert torch.all(out[0, :2].isfinite()) and torch.all(out[0, 2].isnan())
    same = thinfer.op_kv4_attention(q[:, :2].contiguous(), pool, tab, _int(torch, [32]), 16)
    assert torch.equal(out[:, :2], same)


def _exact_rows(torch, pool, row, m, hkv, d, page):
    """K, V [m][hkv][d] in float64 from the bytes of a pool (FP16 params)."""
    p = pool.view(pool.shape[0], hkv, page * (d + 8))[row[:-(-m // page)].long()]
    kb = p[..., :page * d // 2].reshape(-1, hkv, page, d // 2)
    vb = p[..., page * d // 2:page * d].reshape(-1, hkv, page // 2, d // 4, 2, 2).transpose(3, 4).reshape(-1, hkv, page, d // 2)
    par = p[..., page * d:].contiguous().view(torch.float16).double().view(-1, hkv, 2, page, 2)
    out = []
    for w, b in ((0, kb), (1, vb)):
        c = torch.stack([b & 15, b >> 4], -1).flatten(-2).double()
        x = par[:, :, w, :, 1:] + par[:, :, w, :, :1] * c
        out.append(x.transpose(1, 2).reshape(-1, hkv, d)[:m])
    return out


def test_attention_over_shared_and_missing_pages(T):
    torch, thinfer = T
    rng = np.random.default_rng(21)
    pool, tab, table = _filled(T, rng, "f16", 2, 128, 16, [64, 40])
    shared = [table[0][:2] + table[1][:2] + [-1], table[0][:4] + [-1], table[0][:1] + table[0][:1] + [-1] * 3]
    _check_attention(T, rng, "f16", 8, 2, 128, 16, [50, 64, 32], 1, pool, _int(torch, shared), shared)
    # a page number outside the pool, or more tokens than the table names: NaN for that request, nothing for the others
    missing = [table[0][:1] + [10 ** 6] + table[0][2:4] + [-1], table[0][:4] + [-1], table[1][:3] + [-1, -1]]
    q = torch.randn(3, 1, 8, 128, device="cuda").half()
    out = thinfer.op_kv4_attention(q, pool, _int(torch, missing), _int(torch, [64, 64, 500]), 16)
    assert torch.all(out[0].isnan()) and torch.all(out[1].isfinite()) and torch.all(out[2].isnan())
    lone = thinfer.op_kv4_attention(q[1:2].contiguous(), pool, _int(torch, missing)[1:2], _int(torch, [64]), 16)
    assert torch.allclose(lone.float(), out[1:2].float(), atol=2e-3)
    # a negative length is an empty row
    assert torch.all(thinfer.op_kv4_attention(q[:1], pool, _int(torch, shared)[:1], _int(torch, [-4]), 16) == 0)


def test_attention_passes_nan_on_from_a_key_that_is_seen_only(T):
    torch, thinfer = T
    rng = np.random.default_rng(22)
    pool, tab, table = _filled(T, rng, "f16", 2, 64, 16, [40, 40])
    bad = torch.ones(1, 2, 64, dtype=torch.float16, device="cuda")
    bad[0, 1, 7] = float("nan")
    good = torch.ones_like(bad)
    thinfer.op_kv4_append(pool, tab, good, bad, _int(torch, [0]), _int(torch, [38]), 16)      # V of token 38, head 1
    q = torch.randn(2, 3, 4, 64, device="cuda").half()
    out = thinfer.op_kv4_attention(q, pool, tab, _int(torch, [40, 40]), 16)
    # three queries see 38, 39 and 40 keys
    assert torch.all(out[0, 0].isfinite()) and torch.all(out[0, 1:, 2:].isnan()) and torch.all(out[0, :, :2].isfinite()) and torch.all(out[1].isfinite())


# ------------------------------------------------------------------ page tables
def _random_tables(rng, rows, width, n_pages, page, fill):
    counts = rng.multinomial(int(n_pages * fill), [1 / rows] * rows).clip(0, width)
    lens = [int(max(0, c * page - rng.integers(0, page))) if c else 0 for c in counts]
    ids = rng.permutation(n_pages)
    table, at = [], 0
    for c in counts:
        table.append([int(i) for i in ids[at:at + c]] + [int(rng.integers(-3, n_pages)) for _ in range(width - c)])   # stale entries behind
        at += c
    return table, lens


@pytest.mark.parametrize("rows,width,n_pages,page,fill", [(1, 1, 1, 16, 0.0), (3, 4, 10, 16, 0.5), (7, 300, 700, 64, 0.6), (64, 20, 900, 16, 0.9),
                                                          (1500, 3, 4000, 32, 0.4), (5, 9, 33, 128, 1.0), (2, 5000, 9000, 16, 0.8)])
def test_reserve(T, rows, width, n_pages, page, fill):
    torch, thinfer = T
    rng = np.random.default_rng(rows + width)
    table, lens = _random_tables(rng, rows, width, n_pages, page, fill)
    for add in ([1] * rows, [int(x) for x in rng.integers(-2, 3 * page, rows)], [0] * rows, [int(x) for x in rng.integers(0, page * width, rows)]):
        want = kv4.reserve(table, lens, add, n_pages, page)
        tab, l = _int(torch, table), _int(torch, lens)
        out, refused = thinfer.op_kv4_reserve(tab, l, _int(torch, add), n_pages, page)
        assert tab.tolist() == want[0] and out.tolist() == want[1] and refused.item() == want[2]
        assert l.tolist() == lens
        thinfer.op_kv4_reserve(_int(torch, table), l, _int(torch, add), n_pages, page, lens_out=l)      # in place
        assert l.tolist() == want[1]


def test_reserve_of_lengths_beyond_the_table(T):
    torch, thinfer = T
    tab = _int(torch, [[0, 1], [2, -1]])
    out, refused = thinfer.op_kv4_reserve(tab, _int(torch, [40, 2 ** 31 - 1]), _int(torch, [0, 2 ** 31 - 1]), 8, 16)
    assert out.tolist() == [40, 2 ** 31 - 1] and refused.item() == 2 and tab.tolist() == [[0, 1], [2, -1]]


@pytest.mark.parametrize("rows,width,n_pages,page,fill,hkv,d,layers", [
    (1, 1, 2, 16, 0.5, 1, 64, 1), (4, 5, 14, 16, 0.8, 2, 64, 3), (6, 3, 9, 64, 0.8, 1, 128, 2), (64, 4, 250, 16, 0.7, 1, 64, 2), (1100, 2, 2000, 16, 0.5, 1, 64, 1),
    (9, 6, 40, 128, 0.7, 2, 128, 2)])
def test_fork(T, rows, width, n_pages, page, fill, hkv, d, layers):
    torch, thinfer = T
    rng = np.random.default_rng(rows * 3 + page)
    table, lens = _random_tables(rng, rows, width, n_pages, page, fill)
    g = torch.Generator(device="cuda").manual_seed(rows)
    start = torch.randint(0, 256, (layers, n_pages, hkv * page * (d + 8)), dtype=torch.uint8, device="cuda", generator=g)
    for source in (list(range(rows)), [0] * rows, [int(x) for x in rng.integers(-1, rows, rows)], [rows - 1 - r for r in range(rows)], [-1] * rows,
                   [rows if r % 3 == 0 else r for r in range(rows)]):
        pool = start.clone()
        tab, l, refused, moves = kv4.fork(table, lens, source, n_pages, page)
        t_in, l_in = _int(torch, table), _int(torch, lens)
        t_out, l_out, bad = thinfer.op_kv4_fork(pool, t_in, l_in, _int(torch, source), page, d)
        assert t_out.tolist() == tab and l_out.tolist() == l and bad.item() == refused
        assert t_in.tolist() == table and l_in.tolist() == lens
        assert np.array_equal(pool.cpu().numpy(), kv4.copied(start.cpu().numpy(), moves, hkv, d, page))


@pytest.mark.parametrize("rows,width,n_pages,page,fill,hkv,d,layers", [
    (1, 1, 1, 16, 0.0, 1, 64, 1), (1, 2, 2, 16, 0.5, 1, 64, 1), (3, 5, 30, 16, 0.4, 2, 64, 3), (6, 20, 200, 64, 0.5, 1, 128, 2),
    (40, 30, 1000, 16, 0.9, 1, 64, 2), (5, 8, 33, 32, 1.0, 2, 128, 2), (1200, 2, 3000, 16, 0.3, 1, 64, 1)])
def test_compact(T, rows, width, n_pages, page, fill, hkv, d, layers):
    torch, thinfer = T
    rng = np.random.default_rng(rows * 5 + page)
    table, lens = _random_tables(rng, rows, width, n_pages, page, fill)
    if rows > 2:
        k = -(-lens[0] // page)                       # a row that shares all its pages and ends earlier on the last
        table[1][:k], lens[1] = table[0][:k], max(0, lens[0] - 3)
    g = torch.Generator(device="cuda").manual_seed(rows)
    start = torch.randint(0, 256, (layers, n_pages, hkv * page * (d + 8)), dtype=torch.uint8, device="cuda", generator=g)
    pool = start.clone()
    tab, live, moves = kv4.compact(table, lens, n_pages, page)
    t_in = _int(torch, table)
    t_out, count = thinfer.op_kv4_compact(pool, t_in, _int(torch, lens), page, d)
    assert t_out.tolist() == tab and count.item() == live and t_in.tolist() == table
    assert np.array_equal(pool.cpu().numpy(), kv4.copied(start.cpu().numpy(), moves, hkv, d, page))


def test_largest_pool_of_pages(T):
    """262144 pages, the most a plan covers: one page in use at the far end moves to the front."""
    torch, thinfer = T
    n_pages = 1 << 18
    pool = torch.zeros(1, n_pages, 16 * 72, dtype=torch.uint8, device="cuda")
    pool[0, n_pages - 1] = torch.arange(16 * 72, device="cuda").to(torch.uint8)
    tab = _int(torch, [[n_pages - 1, 5]])
    t_out, live = thinfer.op_kv4_compact(pool, tab, _int(torch, [16]), 16, 64)
    assert t_out.tolist() == [[0, -1]] and live.item() == 1 and torch.equal(pool[0, 0], pool[0, n_pages - 1])
    out, refused = thinfer.op_kv4_reserve(tab, _int(torch, [16]), _int(torch, [16]), n_pages, 16)
    assert tab.tolist() == [[n_pages - 1, 0]] and refused.item() == 0


# ------------------------------------------------------------------ together, as a decoder uses them
@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_a_run_of_them_together(T, t):
    """Prompts, a beam fork, captured and replayed decode steps across page borders, a released row, a compaction:
    after every step the attention output follows the float64 attention over values read back from float64 rows."""
    torch, thinfer = T
    rng = np.random.default_rng(77)
    hq, hkv, d, page, rows, width, n_pages, layers = 8, 2, 64, 16, 4, 6, 20, 2
    tt = _tt(torch, t)
    pool = _fresh_pool(torch, n_pages, hkv, d, page, layers)
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    gain = torch.ones(d, dtype=tt, device="cuda")
    turns = thinfer.rope_turns(10000.0, d)
    row_ids = torch.arange(rows, dtype=torch.int32, device="cuda")
    history = [[] for _ in range(rows)]               # per row: (k, v) of the tokens it holds, [hkv][d], per layer
    # -- prompts of 29, 16 and 5 tokens; row 3 stays empty
    news = [29, 16, 5, 0]
    lens, refused = thinfer.op_kv4_reserve(table, lens, _int(torch, news), n_pages, page)
    assert refused.item() == 0
    r_of = np.repeat(np.arange(rows), news)
    pos = np.concatenate([np.arange(n) for n in news])

    def tokens(n):
        return torch.from_numpy(rng.standard_normal((n, (hq + 2 * hkv) * d))).to(tt).cuda()

    def heads(x):
        n = x.shape[0]
        return (x[:, :hq * d].unflatten(1, (hq, d)), x[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)), x[:, (hq + hkv) * d:].unflatten(1, (hkv, d)))

    for layer in range(layers):
        q, k, v = heads(tokens(sum(news)))
        _, k = thinfer.op_qk_norm_rope(q, k, gain, gain, 1e-6, turns, _int(torch, pos.tolist()))
        thinfer.op_kv4_append(pool[layer], table, k, v, _int(torch, r_of.tolist()), _int(torch, pos.tolist()), page)
        for i, r in enumerate(r_of):
            if layer == 0:
                history[r].append([])
            history[r][pos[i]].append((_host(k[i]), _host(v[i])))

    def check(out, q, layer):
        # the same tolerance as the attention tests, from the float64 quantisation of what was appended: a code may differ
        # from it only where FP32 meets a tie, which these draws do not
        for r in range(rows):
            n = len(history[r])
            if n == 0:
                assert torch.all(out[r] == 0)
                continue
            kv = np.zeros((2, n, hkv, d))
            for i, tok in enumerate(history[r]):
                for w in (0, 1):
                    for h in range(hkv):
                        c, s, o = kv4.quantise(tok[layer][w][h], DT[t])
                        kv[w, i, h] = o + s * c
            want, spread, mag = kv4.attention(_host(q[r]), kv, n, 0)
            tol = EPS[t] * np.abs(want) + (2.0 ** -11 + 2.0 ** -19 * (1 + 16 * mag)) * spread + 2.0 ** -25
            assert np.all(np.abs(_host(out[r, 0]) - want) <= tol), (r, n, layer)

    # -- fork: rows 0, 2 and 3 continue row 0, row 1 keeps its own (row 2's old tokens are given up)
    table, lens, refused = thinfer.op_kv4_fork(pool, table, lens, _int(torch, [0, 1, 0, 0]), page, d)
    assert refused.item() == 0 and lens.tolist() == [29, 16, 29, 29]
    history = [list(history[0]), list(history[1]), list(history[0]), list(history[0])]
    # -- decode: one captured step, replayed; it follows lens and table on the device
    one = torch.ones(rows, dtype=torch.int32, device="cuda")
    fresh = torch.zeros(layers, rows, (hq + 2 * hkv) * d, dtype=tt, device="cuda")
    outs, qs = torch.zeros(layers, rows, 1, hq, d, dtype=tt, device="cuda"), torch.zeros(layers, rows, hq, d, dtype=tt, device="cuda")
    ks = torch.zeros(layers, rows, hkv, d, dtype=tt, device="cuda")
    bad = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        at = lens.clone()
        thinfer.op_kv4_reserve(table, lens, one, n_pages, page, lens_out=lens, refused=bad)
        for layer in range(layers):
            q, k, v = heads(fresh[layer])
            thinfer.op_qk_norm_rope(q, k, gain, gain, 1e-6, turns, at, q_out=qs[layer], k_out=ks[layer])
            thinfer.op_kv4_append(pool[layer], table, ks[layer], v, row_ids, at, page)
            thinfer.op_kv4_attention(qs[layer].view(rows, 1, hq, d), pool[layer], table, lens, page, out=outs[layer])

    saved = (table.clone(), lens.clone(), pool.clone())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()                                          # warm-up outside the capture
    torch.cuda.current_stream().wait_stream(stream)
    for dst, src in zip((table, lens, pool), saved):
        dst.copy_(src)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for dst, src in zip((table, lens, pool), saved):
        dst.copy_(src)
    for _ in range(21):                                 # past two page borders of every row
        for layer in range(layers):
            fresh[layer] = tokens(rows)
        graph.replay()
        assert bad.item() == 0
        for r in range(rows):
            history[r].append([(_host(ks[layer][r]), _host(heads(fresh[layer])[2][r])) for layer in range(layers)])
        for layer in range(layers):
            check(outs[layer], qs[layer], layer)
    # -- row 1 ends, the pool is compacted, and one more step runs on the moved pages
    lens[1] = 0
    history[1] = []
    moved, live = thinfer.op_kv4_compact(pool, table, lens, page, d)
    table.copy_(moved)
    assert live.item() == len({p for r in moved.tolist() for p in r if p >= 0}) and moved.max().item() < live.item()
    for layer in range(layers):
        out = thinfer.op_kv4_attention(qs[layer].view(rows, 1, hq, d), pool[layer], table, lens, page)
        check(out, qs[layer], layer)
    # -- and the read-back of a whole row feeds the prefill attention's layout
    n = len(history[3])
    kk = torch.empty(1, hkv, n, d, dtype=tt, device="cuda")
    vv = torch.empty_like(kk)
    thinfer.op_kv4_read(pool[0], table, torch.full((n,), 3, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda"), page, d,
                        tt, k_out=kk[0].transpose(0, 1), v_out=vv[0].transpose(0, 1))
    qq = torch.randn(1, hq, n, d, device="cuda").to(tt)
    pre = thinfer.op_attention_prefill(qq, kk, vv)[0, -1].view(hq, d)
    dec = thinfer.op_kv4_attention(qq[0, :, -1].contiguous().view(1, 1, hq, d), pool[0], table[3:4].contiguous(), lens[3:4].contiguous(), page)[0, 0]
    # the prefill kernel reads K and V rounded once more: EPS of |v| and of the scores (|q k| / sqrt(d) < 16)
    assert torch.all((pre.double() - dec.double()).abs() <= EPS[t] * 40 * (1 + dec.double().abs()))


def test_calls_on_a_side_stream_and_two_at_once(T):
    torch, thinfer = T
    rng = np.random.default_rng(5)
    pool, tab, _ = _filled(T, rng, "f16", 4, 128, 64, [900, 1200, 40])
    lens = _int(torch, [900, 1200, 40])
    q = [torch.randn(3, 1, 16, 128, device="cuda").half() for _ in range(2)]
    want = [thinfer.op_kv4_attention(x, pool, tab, lens, 64) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):         # each call's workspace is its own
                got[i].append(thinfer.op_kv4_attention(q[i], pool, tab, lens, 64))
    torch.cuda.synchronize()
    explicit = thinfer.op_kv4_attention(q[0], pool, tab, lens, 64, stream=streams[0])
    streams[0].synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])
    assert torch.equal(explicit, want[0])


def test_workspaces_of_a_call_on_an_explicit_stream_belong_to_that_stream(T):
    """The call's workspace is given back when it returns; memory taken on the current stream meanwhile must not be it."""
    torch, thinfer = T
    rng = np.random.default_rng(6)
    pool, tab, _ = _filled(T, rng, "f16", 4, 128, 64, [3000, 2000])
    lens, q = _int(torch, [3000, 2000]), torch.randn(2, 1, 16, 128, device="cuda").half()
    want = thinfer.op_kv4_attention(q, pool, tab, lens, 64)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                    # some 10 ms: the call below waits in line
    out = thinfer.op_kv4_attention(q, pool, tab, lens, 64, stream=side)
    taken = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(taken) == 64
    with pytest.raises(thinfer.ThinferError):
        thinfer.op_kv4_attention(q.cpu(), pool, tab, lens, 64, stream=side)
