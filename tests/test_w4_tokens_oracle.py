"""Pins of the float64 definitions of the 4-bit weights and of the verification of drafts, and the refusals of their entry
points (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from oracle import tokens as tk
from oracle import w4
from paper_2605_25655_b200 import _build, thinfer

E, U = thinfer.EINVAL, thinfer.EUNSUPPORTED
# addresses that are never used: every call below is refused.  Far enough apart that nothing here reaches the next one
A = [(1 << 34) * (i + 1) for i in range(8)]


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return thinfer.lib()


# ------------------------------------------------------------------ the oracle
@pytest.mark.parametrize("n,k,group", [(16, 128, 128), (33, 136, 32), (7, 264, 64)])
def test_every_number_has_its_own_place(lib, n, k, group):
    tiles, blocks, per, (nc, ns, nz) = w4.sizes(n, k, group)
    every = {w4.code_at(r, c, n, k, group) for r in range(tiles * 16) for c in range(blocks * 128)}
    assert len(every) == 2 * nc and max(a for a, _ in every) == nc - 1
    params = [w4.param_at(r, j, n, k, group) for r in range(tiles * 16) for j in range(blocks * per)]
    assert len({p[0] for p in params}) == ns // 2 == max(p[0] for p in params) + 1
    assert len({p[1:] for p in params}) == 2 * nz and max(p[1] for p in params) == nz - 1
    size = C.c_size_t(0)
    assert lib.thinfer_w4_bytes(n, k, group, C.byref(size)) == thinfer.OK and size.value == nc + ns + nz == thinfer.w4_bytes(n, k, group)


@pytest.mark.parametrize("dt", [np.float16, "bf16"])
def test_quantised_weights_are_within_half_a_step(dt):
    rng = np.random.default_rng(1)
    eps = 2.0 ** -8 if dt == "bf16" else 2.0 ** -11
    w = w4.round_to(rng.standard_normal((40, 200)) * 0.02 + rng.standard_normal((40, 1)) * 0.01, dt)
    w[3], w[4, :64] = 0.0, 0.5
    codes, scales, zeros = w4.quantise(w, 64, dt)
    off = np.abs(w4.values(codes, scales, zeros, 64) - w)
    # half a step; a zero point moved by half a step and the rounding of the scale may cut as much again off the far end
    step = scales[:, np.arange(200) // 64]
    assert np.all(off <= step * (1.0 + 15 * eps)) and np.mean(off <= step * 0.5) > 0.99
    assert np.all(w4.values(codes, scales, zeros, 64)[w == 0] == 0)      # a zero stays a zero
    assert codes.min() == 0 and codes.max() == 15
    w[0, 0], w[1, 70] = np.nan, np.inf
    _, scales, _ = w4.quantise(w, 64, dt)
    assert np.isnan(scales[0, 0]) and np.isnan(scales[1, 1]) and not np.isnan(scales[0, 1])


def test_draws_follow_the_probabilities():
    p = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [tk.draw(p, u) for u in (0.0, 0.2499, 0.25, 0.74, 0.75, 0.9999)] == [1, 1, 3, 3, 4, 4]
    assert tk.draw(np.zeros(3), 0.5) == -1 and tk.draw(np.array([np.nan, -1.0, 2.0]), 0.9) == 2


def test_verification_keeps_the_targets_distribution():
    """Summed over the drafts and over a fine grid of random numbers, the first token has the target's probabilities."""
    p, q = np.array([0.5, 0.2, 0.3, 0.0]), np.array([0.1, 0.6, 0.2, 0.1])
    got, m = np.zeros(4), 400
    for d in range(4):
        for i in range(m):
            keep = (i + 0.5) / m * q[d] < p[d]
            if keep:
                got[d] += q[d] / m
            else:
                r = np.maximum(p - q, 0)
                got += q[d] / m * r / r.sum()
    assert np.allclose(got, p, atol=2 / m)
    tokens, accepted = tk.verify(np.stack([p, q])[None], q[None, None], [[1]], [[0.3, 0.0]])
    assert accepted == [1] and tokens == [[1, 0]]
    tokens, accepted = tk.verify(np.stack([p, q])[None], q[None, None], [[1]], [[0.4, 0.99]])
    assert accepted == [0] and tokens == [[2, -1]]
    assert tk.verify(np.stack([p, q])[None], None, [[3]], [[0.0, 0.6]])[0] == [[1, -1]]


def test_probabilities_of_the_ends():
    inf, nan = np.inf, np.nan
    got = tk.probs([[0, 0, -inf], [-inf] * 3, [nan, 0, 0], [inf, 0, inf], [1, 3, 3], [0, 1, 2]], [1, 1, 1, 1, 0, 2])
    assert np.allclose(got[0], [0.5, 0.5, 0]) and np.all(got[1] == 0) and np.isnan(got[2]).all() and np.isnan(got[3]).all()
    assert np.array_equal(got[4], [0, 1, 0]) and np.isclose(got[5, 2] / got[5, 1], np.exp(0.5))


# ------------------------------------------------------------------ refusals
def _refused(fn, args, cases):
    for change, code in cases:
        assert set(change) <= set(args)
        assert fn(*(change.get(n, v) for n, v in args.items())) == code, change
        assert thinfer.lib().thinfer_last_error(None)


SHAPES = [({"n": 0}, E), ({"n": -1}, E), ({"k": 0}, E), ({"k": 100}, U), ({"group": 16}, U), ({"group": 0}, E), ({"group": 256}, U), ({"group": 96}, U)]


def test_weights_calls_refuse(lib):
    size = C.c_size_t(0)
    assert lib.thinfer_w4_bytes(16, 128, 64, None) == E and lib.thinfer_w4_bytes(16, 12, 64, C.byref(size)) == U
    n = thinfer.w4_bytes(40, 264, 64)
    for fn, w, p in ((lib.thinfer_op_w4_quantize, "w", "packed"), (lib.thinfer_op_w4_read, "w", "packed")):
        args = dict(w=A[0], ws=272, packed=A[1], n=40, k=264, group=64, st=None)
        if fn is lib.thinfer_op_w4_read:
            args = dict(packed=A[1], w=A[0], ws=272, n=40, k=264, group=64, st=None)
        _refused(fn, args, SHAPES + [
            ({"w": None}, E), ({"packed": None}, E), ({"w": A[0] + 8}, E), ({"packed": A[1] + 8}, E), ({"ws": 256}, E), ({"ws": 268}, E), ({"ws": 1 << 62}, E),
            ({"ws": 1 << 48}, E), ({"packed": A[0]}, E), ({"packed": A[0] - n + 16}, E), ({"packed": A[0] + (39 * 272 + 256) * 2}, E), ({"w": A[1] + n - 16}, E)])


def test_linear_refuses(lib):
    n = thinfer.w4_bytes(40, 264, 64)
    args = dict(x=A[0], xs=272, packed=A[1], y=A[2], ys=40, rows=5, n=40, k=264, group=64, fp32=0, ws=None, wb=0, st=None)
    _refused(lib.thinfer_op_w4_linear, args, SHAPES + [
        *(({x: None}, E) for x in ("x", "packed", "y")), ({"rows": 0}, E), ({"rows": -2}, E), ({"rows": 65}, U), ({"fp32": 2}, E), ({"x": A[0] + 8}, E),
        ({"packed": A[1] + 4}, E), ({"y": A[2] + 1}, E), ({"y": A[2] + 2, "fp32": 1}, E), ({"xs": 256}, E), ({"xs": 268}, E), ({"ys": 39}, E), ({"xs": 1 << 60}, E),
        ({"ys": 1 << 60}, E), ({"y": A[0]}, E), ({"y": A[0] + 4 * 272 * 2 + 526}, E), ({"y": A[1] + n - 2}, E), ({"y": A[1] - 4 * 80 - 78}, E), ({"y": A[0] + 520, "ys": 272}, E)])


def test_linear_refuses_workspaces(lib):
    need = C.c_size_t(0)
    for bad, code in (((0, 40, 264, 64), E), ((65, 40, 264, 64), U), ((5, 0, 264, 64), E), ((5, 40, 264, 48), U)):
        assert lib.thinfer_w4_linear_workspace(*bad, C.byref(need)) == code
    assert lib.thinfer_w4_linear_workspace(5, 40, 264, 64, None) == E
    assert lib.thinfer_w4_linear_workspace(64, 40, 264, 64, C.byref(need)) == thinfer.OK and need.value == 0      # a small one needs none
    n_out, k = 2600, 8200
    assert lib.thinfer_w4_linear_workspace(64, n_out, k, 64, C.byref(need)) == thinfer.OK and need.value > 0
    n = thinfer.w4_bytes(n_out, k, 64)
    args = dict(x=A[0], xs=k, packed=A[1], y=A[2], ys=n_out, rows=64, n=n_out, k=k, group=64, fp32=0, ws=A[3], wb=need.value, st=None)
    _refused(lib.thinfer_op_w4_linear, args, [
        ({"ws": None}, E), ({"ws": A[3] + 8}, E), ({"wb": need.value - 1}, thinfer.ECAPACITY), ({"wb": 0}, thinfer.ECAPACITY), ({"ws": A[0]}, E), ({"ws": A[1] + n // 16 * 16 - 16}, E),
        ({"ws": A[2]}, E), ({"ws": A[1] - need.value // 16 * 16 + 16}, E), ({"y": A[3] + need.value - 2}, E), ({"x": A[3] + 16}, E)])


def test_probs_refuses(lib):
    args = dict(x=A[0], xs=1000, temp=A[1], p=A[2], ps=1000, rows=7, vocab=1000, st=None)
    _refused(lib.thinfer_op_token_probs, args, [
        ({"x": None}, E), ({"p": None}, E), ({"rows": 0}, E), ({"vocab": 0}, E), ({"vocab": -5}, E), ({"xs": 999}, E), ({"ps": 999}, E), ({"xs": 1 << 60}, E),
        ({"x": A[0] + 2}, E), ({"p": A[2] + 1}, E), ({"temp": A[1] + 2}, E), ({"p": A[0], "ps": 1001}, E), ({"p": A[0] + 4}, E), ({"p": A[0] - 6999 * 4}, E),
        ({"temp": A[2] + 64}, E), ({"temp": A[2] - 24}, E)])


def test_verify_refuses(lib):
    args = dict(p=A[0], pb=5000, pr=1000, q=A[1], qb=4000, qr=1000, d=A[2], u=A[3], c=A[4], t=A[5], a=A[6], batch=3, n=4, vocab=1000, st=None)
    _refused(lib.thinfer_op_verify_drafts, args, [
        *(({x: None}, E) for x in ("p", "d", "u", "t", "a")), ({"batch": 0}, E), ({"n": -1}, E), ({"n": 65536}, U), ({"vocab": 0}, E), ({"pb": -1}, E), ({"pr": -4}, E),
        ({"qb": -1}, E), ({"qr": 1 << 60}, E), ({"pb": 1 << 60}, E), *(({x: A[0] + 2}, E) for x in ("p", "q", "d", "u", "c", "t", "a")),
        *(({"t": A[i]}, E) for i in range(5)), *(({"a": A[i]}, E) for i in range(6)), ({"t": A[0] + 14999 * 4}, E), ({"a": A[1] - 8}, E), ({"a": A[5] + 56}, E)])


def test_the_binding_refuses_host_tensors(lib):
    import torch
    w, p, z = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(1, 2, 9), torch.zeros(1, 1, dtype=torch.int32)
    packed = torch.zeros(thinfer.w4_bytes(4, 64, 32), dtype=torch.uint8)
    for call in (lambda: thinfer.op_w4_quantize(w, 32), lambda: thinfer.op_w4_read(packed, 4, 64, 32, torch.float16), lambda: thinfer.op_w4_linear(w, packed, 4, 32),
                 lambda: thinfer.op_token_probs(p[0]), lambda: thinfer.op_verify_drafts(p, None, z, p[0, :, :1])):
        with pytest.raises(thinfer.ThinferError) as e:
            call()
        assert e.value.code == E and "CUDA" in str(e.value)
    with pytest.raises(thinfer.ThinferError) as e:
        thinfer.op_w4_read(packed, 4, 64, 32, torch.float32)
    assert e.value.code == U
