"""Pins of the float64 definitions of the 4-bit paged cache, and the refusals of its entry points (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv4
from oracle import oracle as O
from paper_2605_25655_b200 import _build, thinfer


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return thinfer.lib()


# ------------------------------------------------------------------ the oracle
def test_round_to_bf16_matches_torch():
    import torch
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(2000) * 10.0 ** rng.integers(-6, 6, 2000), [0.0, -0.0, 1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8]])
    assert np.array_equal(kv4.round_to(x, "bf16"), torch.from_numpy(x).to(torch.bfloat16).double().numpy())
    # just above a tie in float64 that float32 rounds onto the tie
    assert kv4.round_to(1 + 2.0 ** -8 + 2.0 ** -40, "bf16") == 1 + 2.0 ** -7


@pytest.mark.parametrize("dt", [np.float16, "bf16"])
def test_quantised_rows_are_within_half_a_step(dt):
    rng = np.random.default_rng(1)
    eps = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11      # half a unit in the last place, relative
    for _ in range(50):
        x = kv4.round_to(rng.standard_normal(64) * 10.0 ** rng.integers(-2, 3), dt)
        c, s, o = kv4.quantise(x, dt)
        assert c.min() == 0 and c.max() >= 14
        # half a step, or at the top the range that the rounding of the scale cut off
        assert np.max(np.abs(o + s * c - x)) <= s * (0.5 + 15 * eps)
    assert kv4.quantise(np.full(64, 1.5), dt)[1:] == (0.0, 1.5)
    assert np.isnan(kv4.quantise(np.array([1.0, np.inf] * 32), dt)[1])


@pytest.mark.parametrize("page,d", [(16, 64), (64, 128)])
def test_every_code_of_a_page_has_its_own_nibble(page, d):
    p = kv4.Pool(np.zeros((1, 2 * page * (d + 8)), np.uint8), 2, d, page, np.float16)
    at = {(w, *p._code_at(w, s, e)) for w in (0, 1) for s in range(page) for e in range(d)}
    assert len({a[1:] for a in at}) == 2 * page * d and max(a[1] for a in at) == page * d - 1
    rng = np.random.default_rng(2)
    rows = {(s, h, w): kv4.round_to(rng.standard_normal(d), np.float16) for s in (0, 1, page - 1) for h in (0, 1) for w in (0, 1)}
    for (s, h, w), x in rows.items():
        p.write(0, s, h, w, x)
    for (s, h, w), x in rows.items():
        c, sc, o = kv4.quantise(x, np.float16)
        assert np.array_equal(p.read(0, s, h, w), o + sc * c)


def test_attention_is_the_oracles_attention():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    q = rng.standard_normal((9, 4, 64))
    want = O.causal_attention(q.transpose(1, 0, 2), k.transpose(1, 0, 2), v.transpose(1, 0, 2))
    got = np.stack([kv4.attention(q[i], (k, v), 9, 8 - i)[0] for i in range(9)])
    assert np.allclose(want, got.reshape(9, -1), atol=1e-12)


def test_rotation_matches_the_oracles_rope_after_the_norm():
    rng = np.random.default_rng(4)
    x, gain = rng.standard_normal((5, 3, 64)), 1 + 0.1 * rng.standard_normal(64)
    turns = 10000.0 ** (-2 * np.arange(32) / 64) / (2 * np.pi)
    pos = np.array([0, 1, 7, 100, 4095])
    got = kv4.qk_norm_rope(x, gain, 1e-5, turns, pos, False)
    normed = O.rmsnorm(x, gain, 1e-5)
    for t in range(5):
        assert np.allclose(got[t], O.rope(normed[t], pos[t], 10000.0), atol=1e-9)
    # halves: the same rotation of permuted dimensions
    perm = np.r_[0:64:2, 1:64:2]
    half = kv4.qk_norm_rope(x[..., perm], gain[perm], 1e-5, turns, pos, True)
    assert np.allclose(half, got[..., perm], atol=1e-12)


def test_fork_and_compact_keep_every_rows_contents():
    rng = np.random.default_rng(5)
    page, width, n_pages = 16, 4, 40
    ids = rng.permutation(n_pages)
    lens = [33, 0, 16, 50, 7]
    table, at = [], 0
    for n in lens:
        k = -(-n // page)
        table.append([int(x) for x in ids[at:at + k]] + [-1] * (width - k))
        at += k
    data = rng.integers(0, 256, (2, n_pages, page * 72), dtype=np.uint8)
    source = [0, 3, 3, 0, -1]
    t2, l2, refused, moves = kv4.fork(table, lens, source, n_pages, page)
    assert refused == 0 and l2 == [33, 50, 50, 33, 0] and len(moves) == 2
    assert t2[0] == table[0] and t2[1] == table[3] and t2[2][:3] == table[3][:3] and t2[2][3] not in ids[:at]
    d2 = kv4.copied(data, moves, 1, 64, page)
    p = lambda dd, i: kv4.Pool(dd[i], 1, 64, page, np.float16)   # noqa: E731
    for r, s in enumerate(source):
        if s >= 0:
            assert np.array_equal(kv4.keys_values(p(d2, 1), t2[r], lens[s]), kv4.keys_values(p(data, 1), table[s], lens[s]), equal_nan=True)
    t3, live, moves = kv4.compact(t2, l2, n_pages, page)
    assert live == len({x for row in t2 for x in row if x >= 0}) and max(max(r) for r in t3) < live
    d3 = kv4.copied(d2, moves, 1, 64, page)
    for r in range(5):
        assert np.array_equal(kv4.keys_values(p(d3, 0), t3[r], l2[r]), kv4.keys_values(p(d2, 0), t2[r], l2[r]), equal_nan=True)


# ------------------------------------------------------------------ refusals (host side, before anything is enqueued)
P = 0x1000   # an aligned address that is never used: every call below is refused before anything is enqueued


def test_page_bytes(lib):
    assert thinfer.kv4_page_bytes(8, 128, 64) == 8 * 64 * 136 and thinfer.kv4_page_bytes(1, 64, 16) == 16 * 72
    for args, code in (((8, 96, 64), thinfer.EUNSUPPORTED), ((8, 128, 48), thinfer.EUNSUPPORTED), ((0, 128, 64), thinfer.EINVAL),
                       ((2000, 128, 64), thinfer.EUNSUPPORTED)):
        with pytest.raises(thinfer.ThinferError) as e:
            thinfer.kv4_page_bytes(*args)
        assert e.value.code == code and str(e.value)
    assert lib.thinfer_kv4_page_bytes(1, 64, 16, None) == thinfer.EINVAL


def test_rope_turns(lib):
    t = thinfer.rope_turns(10000.0, 64, device="cpu").numpy()
    assert np.allclose(t, 10000.0 ** (-2 * np.arange(32) / 64) / (2 * np.pi), rtol=1e-14)
    buf = (C.c_double * 4)()
    for args in ((0.0, 8, buf), (10000.0, 7, buf), (10000.0, 0, buf), (10000.0, 8, None), (float("nan"), 8, buf)):
        assert lib.thinfer_rope_turns(*args) == thinfer.EINVAL


def _call(fn, args, **change):
    return fn(*(change.get(n, v) for n, v in args.items()))


def _refusals(fn, args, cases):
    for change, code in cases:
        assert _call(fn, args, **change) == code, change
        assert thinfer.lib().thinfer_last_error(None)


def test_qk_norm_rope_refuses(lib):
    args = dict(q=P, qs=512, k=P, ks=256, qo=P, qos=512, ko=P, kos=256, qg=P, kg=P, turns=P, pos=P, tokens=2, hq=4, hkv=2, d=128,
                rot=128, halves=0, eps=1e-6, st=None)
    E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
    _refusals(lib.thinfer_op_qk_norm_rope, args, [
        *(({n: None}, E) for n in ("q", "k", "qo", "ko", "qg", "kg", "turns", "pos")),
        *(({n: 0}, E) for n in ("tokens", "hq", "hkv", "d")), ({"d": 96}, U), ({"rot": 136}, U), ({"rot": 24}, U), ({"rot": -16}, E),
        ({"halves": 2}, E), ({"eps": -1.0}, E), ({"eps": float("nan")}, E), ({"qs": 504}, E), ({"ks": 260}, E), ({"kos": 128}, E), ({"q": P + 8}, E),
        ({"ko": P + 2}, E), ({"turns": P + 4}, E), ({"pos": P + 2}, E)])
    # outputs over inputs that they do not replace, row by row: slices of one projection output do not overlap
    F, N = 1 << 24, 1 << 26
    args.update(q=F, qs=1024, k=F + 1024, ks=1024, qo=N, qos=512, ko=2 * N, kos=256, tokens=3)
    _refusals(lib.thinfer_op_qk_norm_rope, args, [
        ({"qo": F, "qos": 512}, E), ({"qo": F + 16, "qos": 1024}, E), ({"qo": F + 1024, "qos": 1024}, E), ({"ko": F, "kos": 1024}, E),
        ({"ko": F + 1040, "kos": 1024}, E), ({"ko": N + 512, "kos": 256}, E), ({"qo": F, "qos": 1024, "ko": F, "kos": 1024}, E),
        ({"qo": F + 1536, "qos": 1024}, E)])


def test_append_and_read_refuse(lib):
    E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
    common = [({"pool": None}, E), ({"pool": P + 8}, E), ({"table": None}, E), ({"table": P + 2}, E), ({"n_pages": 0}, E), ({"n_rows": 0}, E),
              ({"maxp": 0}, E), ({"maxp": 1 << 26}, U), ({"rows": None}, E), ({"pos": None}, E), ({"tokens": 0}, E), ({"tokens": -3}, E),
              ({"hkv": 0}, E), ({"d": 32}, U), ({"page": 8}, U), ({"page": 100}, U), ({"pos": P + 1}, E)]
    args = dict(pool=P, n_pages=4, table=P, n_rows=2, maxp=3, k=P, ks=256, v=P, vs=256, rows=P, pos=P, tokens=5, hkv=2, d=128, page=64, st=None)
    _refusals(lib.thinfer_op_kv4_append, args, common + [({"k": None}, E), ({"v": None}, E), ({"ks": 248}, E), ({"vs": 257}, E), ({"k": P + 2}, E)])
    args = dict(pool=P, n_pages=4, table=P, n_rows=2, maxp=3, ko=P, vo=P, ts=256, hs=128, rows=P, pos=P, tokens=5, hkv=2, d=128, page=64, st=None)
    _refusals(lib.thinfer_op_kv4_read, args, common + [({"ko": None}, E), ({"vo": P + 8}, E), ({"ts": 64}, E), ({"hs": 132}, E)])


def test_attention_refuses(lib):
    E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
    need = C.c_size_t(0)
    assert lib.thinfer_kv4_attention_workspace(2, 1, 8, 2, 128, C.byref(need)) == thinfer.OK and need.value > 0
    for bad in ((0, 1, 8, 2, 128), (2, 0, 8, 2, 128), (2, 1, 0, 2, 128), (2, 1, 8, 0, 128)):
        assert lib.thinfer_kv4_attention_workspace(*bad, C.byref(need)) == E
    assert lib.thinfer_kv4_attention_workspace(2, 1, 8, 2, 128, None) == E
    assert lib.thinfer_kv4_attention_workspace(2, 1, 8, 2, 128, C.byref(need)) == thinfer.OK
    args = dict(q=P, qs=1024, pool=P, n_pages=4, table=P, maxp=3, lens=P, out=P, batch=2, queries=1, hq=8, hkv=2, d=128, page=64, ws=P,
                wb=need.value, st=None)
    _refusals(lib.thinfer_op_kv4_attention, args, [
        *(({n: None}, E) for n in ("q", "pool", "table", "lens", "out", "ws")), *(({n: 0}, E) for n in ("batch", "queries", "hq", "hkv", "n_pages", "maxp")),
        ({"hq": 7}, U), ({"d": 80}, U), ({"page": 24}, U), ({"qs": 1016}, E), ({"qs": 1028}, E), ({"q": P + 4}, E), ({"out": P + 8}, E), ({"ws": P + 8}, E),
        ({"wb": need.value - 1}, thinfer.ECAPACITY), ({"maxp": 1 << 26}, U), ({"batch": 2049}, U), ({"queries": 70000}, U)])
    # an output or a workspace that overlaps an input, or each other
    q, table, lens, out, ws = ((1 << 24) * i for i in range(1, 6))
    args.update(q=q, table=table, lens=lens, out=out, ws=ws)
    _refusals(lib.thinfer_op_kv4_attention, args, [
        ({"out": q}, E), ({"out": q + 2048}, E), ({"out": q - 4080}, E), ({"out": table}, E), ({"lens": out + 16}, E), ({"ws": out}, E), ({"ws": q}, E),
        ({"ws": table}, E), ({"ws": lens}, E)])


def test_page_table_calls_refuse(lib):
    E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
    T, L, A, LO, R, S, TO = (0x10000 * i for i in range(1, 8))
    args = dict(t=T, l=L, a=A, lo=LO, r=R, rows=4, maxp=8, n_pages=32, page=16, st=None)
    _refusals(lib.thinfer_op_kv4_reserve, args, [
        *(({n: None}, E) for n in "tla"), ({"lo": None}, E), ({"r": None}, E), ({"rows": 0}, E), ({"maxp": 0}, E), ({"n_pages": -1}, E), ({"page": 17}, U),
        ({"rows": 4097}, U), ({"n_pages": (1 << 18) + 1}, U), ({"lo": L + 4}, E), ({"lo": A}, E), ({"r": L}, E), ({"r": LO + 8}, E), ({"l": L + 2}, E), ({"lo": T + 16}, E), ({"r": T + 8}, E)])
    need = C.c_size_t(0)
    assert lib.thinfer_kv4_pages_workspace(4, 32, C.byref(need)) == thinfer.OK and need.value >= 16 + 16 * 12
    assert lib.thinfer_kv4_pages_workspace(0, 32, C.byref(need)) == E and lib.thinfer_kv4_pages_workspace(4, 1 << 20, C.byref(need)) == U
    assert lib.thinfer_kv4_pages_workspace(4, 32, None) == E
    args = dict(pool=P, layers=2, n_pages=32, t=T, l=L, s=S, to=TO, lo=LO, r=R, rows=4, maxp=8, hkv=2, d=64, page=16, ws=P, wb=1 << 12, st=None)
    _refusals(lib.thinfer_op_kv4_fork, args, [
        *(({n: None}, E) for n in ("pool", "t", "l", "s", "to", "lo", "r", "ws")), ({"layers": 0}, E), ({"rows": 4097}, U), ({"to": T}, E), ({"to": T + 64}, E),
        ({"lo": L}, E), ({"lo": S}, E), ({"r": LO}, E), ({"r": TO + 8}, E), ({"r": R + 4}, E), ({"wb": 32}, thinfer.ECAPACITY), ({"d": 72}, U)])
    args = dict(pool=P, layers=2, n_pages=32, t=T, l=L, to=TO, live=R, rows=4, maxp=8, hkv=2, d=64, page=16, ws=P, wb=1 << 12, st=None)
    _refusals(lib.thinfer_op_kv4_compact, args, [
        *(({n: None}, E) for n in ("pool", "t", "l", "to", "live", "ws")), ({"layers": -1}, E), ({"to": T}, E), ({"live": L}, E), ({"live": TO}, E),
        ({"wb": 32}, thinfer.ECAPACITY), ({"n_pages": 1 << 19}, U)])


def test_the_binding_refuses_host_tensors_and_wrong_shapes(lib):
    import torch
    z = torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(4, 16 * 72, dtype=torch.uint8)
    kv = torch.zeros(2, 1, 64, dtype=torch.float16)
    for call in (lambda: thinfer.op_kv4_append(pool, z.view(1, 2), kv, kv, z, z, 16),
                 lambda: thinfer.op_kv4_read(pool, z.view(1, 2), z, z, 16, 64, torch.float16),
                 lambda: thinfer.op_kv4_attention(kv.view(2, 1, 1, 64), pool, z.view(2, 1), z, 16),
                 lambda: thinfer.op_kv4_reserve(z.view(2, 1), z, z, 4, 16),
                 lambda: thinfer.op_kv4_fork(pool[None], z.view(2, 1), z, z, 16, 64),
                 lambda: thinfer.op_kv4_compact(pool[None], z.view(2, 1), z, 16, 64),
                 lambda: thinfer.op_qk_norm_rope(kv, kv, kv[0, 0], kv[0, 0], 1e-6, torch.zeros(32, dtype=torch.float64), z)):
        with pytest.raises(thinfer.ThinferError) as e:
            call()
        assert e.value.code == thinfer.EINVAL and "CUDA" in str(e.value)
