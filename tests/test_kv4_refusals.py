"""Calls of the 4-bit paged cache and of the norm with rotation that write over what they read, or twice to one place, are
refused on the host, before anything is enqueued (no GPU needed)."""
import pytest

from paper_2605_25655_b200 import _build, thinfer

E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
# addresses that are never used: every call below is refused.  Far enough apart that nothing here reaches the next one
A = [(1 << 30) * (i + 1) for i in range(16)]


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return thinfer.lib()


def _refused(fn, args, cases, code=E):
    for change in cases:
        assert set(change) <= set(args)
        assert fn(*(change.get(n, v) for n, v in args.items())) == code, change
        assert thinfer.lib().thinfer_last_error(None)


def test_read_refuses_outputs_that_meet(lib):
    args = dict(pool=A[0], n_pages=4, table=A[1], n_rows=2, maxp=3, ko=A[2], vo=A[3], ts=256, hs=128, rows=A[4], pos=A[5], tokens=5, hkv=2, d=128,
                page=64, st=None)
    pool_end = A[0] + 4 * 2 * 64 * 136
    _refused(lib.thinfer_op_kv4_read, args, [
        {"vo": A[2]}, {"vo": A[2] + 256}, {"vo": A[2] - 512 * 4}, {"vo": A[2] + 16}, {"ts": 128}, {"ts": 192}, {"ts": 128, "hs": 512}, {"ts": 256, "hs": 512},
        {"ts": 256, "hs": 328}, {"ts": 384, "vo": A[2] + 2 * 136}, {"ts": 128, "hs": 640, "vo": A[2] + 2 * 5 * 128},
        {"ko": A[0]}, {"vo": pool_end - 16}, {"ko": A[0] - 16}, {"vo": A[1]}, {"table": A[2] + 64}, {"rows": A[2] + 1024}, {"pos": A[3]}])


def test_append_refuses_a_pool_over_its_inputs(lib):
    args = dict(pool=A[0], n_pages=4, table=A[1], n_rows=2, maxp=3, k=A[2], ks=256, v=A[3], vs=512, rows=A[4], pos=A[5], tokens=5, hkv=2, d=128,
                page=64, st=None)
    n = 4 * 2 * 64 * 136
    _refused(lib.thinfer_op_kv4_append, args, [
        {"k": A[0]}, {"v": A[0] + n - 16}, {"k": A[0] - (4 * 256 + 240) * 2}, {"v": A[0] - (4 * 512 + 240) * 2}, {"table": A[0]}, {"table": A[0] - 20},
        {"rows": A[0] + 64}, {"pos": A[0] - 16}])


def test_fork_and_compact_refuse_a_pool_or_workspace_over_another_tensor(lib):
    n = 2 * 32 * 2 * 16 * 72                            # bytes of the pool
    args = dict(pool=A[0], layers=2, n_pages=32, t=A[1], l=A[2], s=A[3], to=A[4], lo=A[5], r=A[6], rows=4, maxp=8, hkv=2, d=64, page=16, ws=A[7],
                wb=1 << 12, st=None)
    _refused(lib.thinfer_op_kv4_fork, args, [
        *({x: A[0] + n - 16} for x in ("t", "l", "s", "to", "lo", "r", "ws")), *({x: A[7] + 16} for x in ("t", "l", "s", "to", "lo", "r")),
        {"ws": A[0] - 16}, {"pool": A[1] - n + 16}, {"pool": A[6]}])
    args = dict(pool=A[0], layers=2, n_pages=32, t=A[1], l=A[2], to=A[4], live=A[6], rows=4, maxp=8, hkv=2, d=64, page=16, ws=A[7], wb=1 << 12, st=None)
    _refused(lib.thinfer_op_kv4_compact, args, [
        *({x: A[0] + n - 16} for x in ("t", "l", "to", "live", "ws")), *({x: A[7] + 16} for x in ("t", "l", "to", "live")), {"ws": A[0] - 16},
        {"pool": A[4] - n + 16}, {"pool": A[6]}])


def test_attention_refuses_outputs_over_the_pool(lib):
    args = dict(q=A[0], qs=1024, pool=A[1], n_pages=4, table=A[2], maxp=3, lens=A[3], out=A[4], batch=2, queries=1, hq=8, hkv=2, d=128, page=64, ws=A[5],
                wb=1 << 24, st=None)
    n = 4 * 2 * 64 * 136
    _refused(lib.thinfer_op_kv4_attention, args, [{"out": A[1]}, {"out": A[1] + n - 16}, {"out": A[1] - 16}, {"ws": A[1] + 16}, {"ws": A[1] - 64}])


def test_norm_refuses_outputs_over_gains_turns_and_positions(lib):
    args = dict(q=A[0], qs=1024, k=A[1], ks=256, qo=A[2], qos=1024, ko=A[3], kos=512, qg=A[4], kg=A[5], turns=A[6], pos=A[7], tokens=3, hq=4, hkv=2, d=128,
                rot=128, halves=0, eps=1e-6, st=None)
    q_row, k_row = 4 * 128 * 2, 2 * 128 * 2
    _refused(lib.thinfer_op_qk_norm_rope, args, [
        {"qg": A[2]}, {"kg": A[2] + 2048 + q_row - 16}, {"turns": A[2] + 2 * 2048 - 16}, {"pos": A[2] - 8}, {"pos": A[2] + 2 * 2048 + q_row - 4},
        {"qg": A[3] + 1024}, {"kg": A[3] - 240}, {"turns": A[3] + k_row - 8}, {"pos": A[3] + 2 * 1024 + k_row - 8}])


def test_strides_beyond_any_memory_are_refused(lib):
    big = 1 << 62
    args = dict(pool=A[0], n_pages=4, table=A[1], n_rows=2, maxp=3, ko=A[2], vo=A[3], ts=256, hs=128, rows=A[4], pos=A[5], tokens=5, hkv=2, d=128,
                page=64, st=None)
    _refused(lib.thinfer_op_kv4_read, args, [{"ts": big}, {"hs": big}, {"ts": 1 << 40, "tokens": (1 << 31) - 1}])
    args = dict(pool=A[0], n_pages=4, table=A[1], n_rows=2, maxp=3, k=A[2], ks=256, v=A[3], vs=512, rows=A[4], pos=A[5], tokens=5, hkv=2, d=128,
                page=64, st=None)
    _refused(lib.thinfer_op_kv4_append, args, [{"ks": big}, {"vs": big}, {"vs": 1 << 40, "tokens": (1 << 31) - 1}])
    args = dict(q=A[0], qs=1024, k=A[1], ks=256, qo=A[2], qos=1024, ko=A[3], kos=512, qg=A[4], kg=A[5], turns=A[6], pos=A[7], tokens=3, hq=4, hkv=2, d=128,
                rot=128, halves=0, eps=1e-6, st=None)
    _refused(lib.thinfer_op_qk_norm_rope, args, [{"qs": big}, {"ks": big}, {"qos": big}, {"kos": big}])
    args = dict(q=A[0], qs=1024, pool=A[1], n_pages=4, table=A[2], maxp=3, lens=A[3], out=A[4], batch=2, queries=1, hq=8, hkv=2, d=128, page=64, ws=A[5],
                wb=1 << 24, st=None)
    _refused(lib.thinfer_op_kv4_attention, args, [{"qs": big}])
