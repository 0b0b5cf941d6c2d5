"""Weights in 4 bits with group scales against their float64 definition (run with -m gpu on a B200).

Tolerances.  A stored result is rounded to the storage type once: EPS * |value| with EPS = 2^-11 (FP16) or 2^-8 (BF16), and
2^-25 at the bottom of FP16's subnormals.  What FP32 sums may add is written at each test.
"""
import numpy as np
import pytest

from oracle import w4

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


# ------------------------------------------------------------------ quantising and reading
def _weights(rng, n, k, t, kind):
    w = rng.standard_normal((n, k)) * 0.02
    if kind == "spread":                              # the whole range of the type, rows and groups of very different size
        low, high = (-24, 15) if t == "f16" else (-130, 126)
        w = rng.standard_normal((n, k)) * 2.0 ** rng.uniform(low, high, (n, k // 8)).repeat(8, 1)
        w = np.clip(w, -65504, 65504) if t == "f16" else np.clip(w, -3.3e38, 3.3e38)
    elif kind == "grid":                              # many quotients are the middle of two codes
        w = rng.integers(-15, 16, (n, k)) * 0.5 * 2.0 ** rng.integers(-8, 4, (n, 1))
    elif kind == "ends":
        w[0], w[-1, :8] = 0.0, [65504, -65504] * 4 if t == "f16" else [3.3e38, -3.3e38] * 4
        w[n // 2] = np.abs(w[n // 2])                 # a row without negative numbers, one without positive ones
        w[n // 3] = -np.abs(w[n // 3])
        w[2 % n, k - 1], w[5 % n, 0], w[5 % n, k - 1] = np.nan, np.inf, -np.inf
        w[7 % n, :16] = 2.0 ** -24 if t == "f16" else 2.0 ** -133
    return w4.round_to(w, DT[t])


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "spread", "grid", "ends"])
@pytest.mark.parametrize("n,k,group", [(1, 8, 32), (16, 128, 128), (17, 136, 64), (40, 1000, 32), (130, 392, 128), (33, 264, 32)])
def test_quantise_and_read(T, t, kind, n, k, group):
    torch, thinfer = T
    rng = np.random.default_rng(n * 7 + k + group)
    w = _weights(rng, n, k, t, kind)
    codes, scales, zeros = w4.quantise(w, group, DT[t])
    want = w4.pack(codes, scales, zeros, group, DT[t])
    wide = torch.full((n, k + 24), 9.0, dtype=_tt(torch, t), device="cuda")       # rows inside wider ones
    wide[:, 8:8 + k] = _dev(torch, w, t)
    packed = torch.full((want.size,), 255, dtype=torch.uint8, device="cuda")
    assert thinfer.op_w4_quantize(wide[:, 8:8 + k], group, packed=packed) is not None
    got = packed.cpu().numpy()
    assert np.array_equal(got, want), (np.nonzero(got != want)[0][:5], got[got != want][:5], want[got != want][:5])
    assert torch.equal(thinfer.op_w4_quantize(wide[:, 8:8 + k].contiguous(), group), packed)
    out = torch.full((n, k + 8), 9.0, dtype=_tt(torch, t), device="cuda")
    thinfer.op_w4_read(packed, n, k, group, _tt(torch, t), out=out[:, :k])
    with np.errstate(over="ignore"):
        back = w4.round_to(w4.values(codes, scales, zeros, group), DT[t])
    assert np.array_equal(_host(out[:, :k]), back, equal_nan=True) and torch.all(out[:, k:] == 9.0)
    assert torch.equal(thinfer.op_w4_read(packed, n, k, group, _tt(torch, t)).isnan(), out[:, :k].isnan())


# ------------------------------------------------------------------ products
def _random_packed(rng, n, k, group, t, whole):
    codes, zeros = rng.integers(0, 16, (n, k)), rng.integers(0, 16, (n, -(-k // group)))
    scales = 2.0 ** rng.integers(-3, 1, zeros.shape) if whole else w4.round_to(rng.uniform(0.004, 0.008, zeros.shape), DT[t])
    return w4.pack(codes, scales, zeros, group, DT[t]), w4.values(codes, scales, zeros, group)


SIZES = [(1, 16, 128, 128), (1, 4096, 256, 64), (2, 1, 8, 32), (3, 17, 40, 32), (5, 100, 1000, 64), (7, 1001, 136, 128), (8, 64, 4096, 128), (9, 33, 264, 32),
         (16, 500, 2048, 128), (17, 48, 520, 64), (24, 257, 1024, 32), (33, 130, 392, 128), (40, 31, 3000, 64), (64, 200, 1536, 128), (64, 15, 72, 32),
         (1, 40, 40960, 128), (16, 24, 30000, 32), (64, 20, 28672, 64), (4, 5000, 512, 128), (16, 9000, 136, 64), (64, 7000, 264, 32),
         # more than 10 (16) x 1024 tiles and blocks: tensor memory.  Few blocks and many rows, many blocks and few rows, one block
         (17, 1100, 20000, 64), (40, 5200, 4200, 128), (64, 2600, 8200, 128), (33, 2700, 13000, 32), (24, 41000, 640, 64), (64, 100000, 136, 128), (20, 170000, 120, 64),
         (32, 20000, 1784, 32), (64, 16, 1310728, 128)]


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("rows,n,k,group", SIZES)
def test_products_of_whole_numbers_are_exact(T, t, rows, n, k, group):
    """Tokens of small whole numbers and scales that are powers of two: every sum fits FP32, so nothing may be off at all."""
    torch, thinfer = T
    rng = np.random.default_rng(rows * 1000 + n + k)
    packed, w = _random_packed(rng, n, k, group, t, True)
    x = rng.integers(-3, 4, (rows, k)).astype(np.float64)
    wide = torch.full((rows, k + 8), float("nan"), dtype=_tt(torch, t), device="cuda")       # strided tokens
    wide[:, :k] = _dev(torch, x, t)
    packed = torch.from_numpy(packed).cuda()
    want = x @ w.T                                    # exact: multiples of 2^-3 below 2^21
    got = thinfer.op_w4_linear(wide[:, :k], packed, n, group, out_fp32=True)
    assert got.dtype == torch.float32 and np.array_equal(_host(got), want)
    out = torch.full((rows + 2, n + 3), 7.0, dtype=torch.float32, device="cuda")
    thinfer.op_w4_linear(wide[:, :k], packed, n, group, out=out[1:-1, 1:-2])
    assert np.array_equal(_host(out[1:-1, 1:-2]), want)
    assert torch.all(out[0] == 7) and torch.all(out[-1] == 7) and torch.all(out[:, 0] == 7) and torch.all(out[:, -2:] == 7)
    out = torch.full((rows + 2, n + 3), 7.0, dtype=_tt(torch, t), device="cuda")
    thinfer.op_w4_linear(_dev(torch, x, t), packed, n, group, out=out[1:-1, 1:-2])
    assert np.array_equal(_host(out[1:-1, 1:-2]), w4.round_to(want, DT[t]))
    assert torch.all(out[0] == 7) and torch.all(out[-1] == 7) and torch.all(out[:, 0] == 7) and torch.all(out[:, -2:] == 7)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [8, 9, 16, 17, 32, 33, 64])
def test_products_of_a_large_matrix_are_exact(T, t, rows):
    """The same for more than 80 x 1024 tiles and blocks, against the weights as they are read back (which has a test of its own)."""
    torch, thinfer = T
    n, k, group, tt = 20501, 8200, 128, _tt(torch, t)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    (nc, ns, nz) = w4.sizes(n, k, group)[3]
    packed = torch.randint(0, 256, (nc + ns + nz,), dtype=torch.uint8, device="cuda", generator=gen)
    packed[nc:nc + ns].view(tt).copy_(2.0 ** -torch.randint(0, 4, (ns // 2,), device="cuda", generator=gen).float())
    x = torch.randint(-2, 3, (rows, k), device="cuda", generator=gen).to(tt)
    w = thinfer.op_w4_read(packed, n, k, group, tt)
    want = torch.cat([x.double() @ part.double().T for part in w.split(4096)], 1)        # multiples of 2^-3 below 2^18
    got = thinfer.op_w4_linear(x, packed, n, group, out_fp32=True)
    assert torch.equal(got.double(), want)
    out = torch.full((rows + 1, n + 2), 7.0, dtype=tt, device="cuda")
    thinfer.op_w4_linear(x, packed, n, group, out=out[:-1, 1:-1])
    assert torch.equal(out[:-1, 1:-1], want.to(tt)) and torch.all(out[-1] == 7) and torch.all(out[:, 0] == 7) and torch.all(out[:, -1] == 7)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("rows,n,k,group", [(1, 700, 4096, 128), (4, 512, 8192, 64), (16, 300, 11008, 32), (33, 80, 5120, 128), (64, 160, 28672, 64), (64, 2600, 8192, 64),
                                            (24, 1100, 32768, 32)])
def test_products(T, t, rows, n, k, group):
    torch, thinfer = T
    rng = np.random.default_rng(rows + n + k)
    packed, w = _random_packed(rng, n, k, group, t, False)
    x = w4.round_to(rng.standard_normal((rows, k)), DT[t])
    want, size = w4.linear(x, w)
    # a sum of k terms in steps of 16 and of group by group: 2^-24 of the sums so far at each step, whose sizes wander like
    # the root of the number of terms, so that all of them together stay below 2^-22 of the root of the steps' number
    # times the result's typical size, size / sqrt(k); a matrix step that cuts instead of rounding doubles that
    tol = 2.0 ** -21 * np.sqrt(k / 16 + k / group) * size / np.sqrt(k)
    x, packed = _dev(torch, x, t), torch.from_numpy(packed).cuda()
    got = thinfer.op_w4_linear(x, packed, n, group, out_fp32=True)
    assert np.all(np.abs(_host(got) - want) <= tol)
    half = thinfer.op_w4_linear(x, packed, n, group)
    assert np.all(np.abs(_host(half) - want) <= tol + EPS[t] * np.abs(want) + 2.0 ** -25)
    for _ in range(3):                                # the same bits every time
        assert torch.equal(thinfer.op_w4_linear(x, packed, n, group, out_fp32=True), got)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("rows,n,k", [(1, 70, 600), (8, 70, 600), (13, 70, 600), (40, 70, 600), (20, 4000, 5200), (64, 4000, 5200)])
def test_what_is_not_finite_stays_in_its_row_and_column(T, t, rows, n, k):
    torch, thinfer = T
    rng = np.random.default_rng(rows)
    group = 64
    w = w4.round_to(rng.standard_normal((n, k)) * 0.02, DT[t])
    w[5, 70], w[37, 599] = np.nan, np.inf
    x = w4.round_to(rng.standard_normal((rows, k)), DT[t])
    x[rows // 2, 3] = np.inf
    x[0, 599] = np.nan
    got = _host(thinfer.op_w4_linear(_dev(torch, x, t), thinfer.op_w4_quantize(_dev(torch, w, t), group), n, group, out_fp32=True))
    fine = np.ones((rows, n), bool)
    fine[:, [5, 37]] = False
    fine[[0, rows // 2]] = False
    assert np.all(np.isfinite(got[fine])) and np.all(np.isnan(got[:, [5, 37]])) and np.all(np.isnan(got[0])) and not np.any(np.isfinite(got[rows // 2]))


def test_large_values(T):
    """FP16 tokens and weights at the top of the type: sums stay FP32, stored results beyond the type are infinity."""
    torch, thinfer = T
    x = torch.full((2, 256), 65504.0, dtype=torch.float16, device="cuda")
    w = torch.full((20, 256), 65504.0, dtype=torch.float16, device="cuda")
    w[3] = -w[3]
    packed = thinfer.op_w4_quantize(w, 128)
    got = thinfer.op_w4_linear(x, packed, 20, 128, out_fp32=True)
    scale = float(torch.tensor(65504 / 15, dtype=torch.float16))
    want = torch.full_like(got, 256 * 65504.0 * 15 * scale)
    want[:, 3] *= -1
    assert torch.all((got - want).abs() <= 2.0 ** -20 * want.abs()) and torch.equal(thinfer.op_w4_linear(x, packed, 20, 128), want.half())
    x = torch.full((2, 256), 2.0 ** 120, dtype=torch.bfloat16, device="cuda")      # 15 * 256 * 2^120 would not stay inside
    x[:, 32:] = 0
    w = torch.full((20, 256), 15 * 2.0 ** -100, dtype=torch.bfloat16, device="cuda")
    packed = thinfer.op_w4_quantize(w, 32)
    assert torch.all(thinfer.op_w4_linear(x, packed, 20, 32, out_fp32=True) == 32 * 15 * 2.0 ** 20)


def test_offsets_beyond_32_bits(T):
    """More than 2^31 bytes of codes, more than 2^32 weights."""
    torch, thinfer = T
    n, k, group, t = 65560, 65664, 128, torch.float16
    gen = torch.Generator(device="cuda").manual_seed(5)
    (nc, ns, nz) = w4.sizes(n, k, group)[3]
    assert nc > 2 ** 31 and thinfer.w4_bytes(n, k, group) == nc + ns + nz
    packed = torch.empty(nc + ns + nz, dtype=torch.uint8, device="cuda")
    for i in range(0, nc, 1 << 28):
        packed[i:min(nc, i + (1 << 28))] = torch.randint(0, 256, (min(nc, i + (1 << 28)) - i,), dtype=torch.uint8, device="cuda", generator=gen)
    packed[nc + ns:] = 0x88
    packed[nc:nc + ns].view(t).copy_(torch.full((ns // 2,), 2.0 ** -6, dtype=t, device="cuda"))
    w = thinfer.op_w4_read(packed, n, k, group, t)
    x = torch.randint(-1, 2, (3, k), device="cuda", generator=gen).to(t)
    got = thinfer.op_w4_linear(x, packed, n, group, out_fp32=True)
    for a, b in ((0, 100), (32700, 32800), (n - 100, n)):
        assert torch.equal(got[:, a:b].double(), x.double() @ w[a:b].double().T)
    # the last rows quantised with all the others and by themselves
    again = thinfer.op_w4_read(thinfer.op_w4_quantize(w, group), n, k, group, t)
    assert torch.equal(thinfer.op_w4_read(thinfer.op_w4_quantize(w[-24:], group), 24, k, group, t), again[-24:])
    # codes of the last whole tile and of the last, half filled one, byte by byte
    rows, cols = np.array([[n - 1], [n - 9], [n - 24]]), np.array([[0, 77, k - 1]])
    at, shift = w4.code_at(rows, cols, n, k, group)
    codes = (packed[torch.from_numpy(at).cuda()].long() >> torch.from_numpy(shift * np.ones_like(at)).cuda()) & 15
    assert torch.equal((codes - 8) * 2.0 ** -6, w[torch.from_numpy(rows).cuda(), torch.from_numpy(cols).cuda()].float())


def test_streams_and_graphs(T):
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(300, 520, generator=gen, device="cuda") * 0.02).half()
    x = torch.randn(6, 520, generator=gen, device="cuda").half()
    want = thinfer.op_w4_linear(x, thinfer.op_w4_quantize(w, 64), 300, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    packed = thinfer.op_w4_quantize(w, 64, stream=side)
    got = thinfer.op_w4_linear(x, packed, 300, 64, stream=side)
    back = thinfer.op_w4_read(packed, 300, 520, 64, torch.float16, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(back, thinfer.op_w4_read(packed, 300, 520, 64, torch.float16))
    # quantised, read back and multiplied in one graph, replayed on other numbers
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        packed = thinfer.op_w4_quantize(w, 64)
        y = thinfer.op_w4_linear(x, packed, 300, 64)
        z = thinfer.op_w4_linear(x[:1], packed, 300, 64, out_fp32=True)
    for _ in range(3):
        w.copy_((torch.randn(300, 520, generator=gen, device="cuda") * 0.02).half())
        x.copy_(torch.randn(6, 520, generator=gen, device="cuda").half())
        graph.replay()
        p = thinfer.op_w4_quantize(w, 64)
        assert torch.equal(y, thinfer.op_w4_linear(x, p, 300, 64)) and torch.equal(z, thinfer.op_w4_linear(x[:1], p, 300, 64, out_fp32=True))


def test_workspaces_graphs_and_streams_on_tensor_memory(T):
    """Two graphs that share a workspace, replayed in turn; calls on two streams at once with a workspace each; a workspace full of
    other numbers."""
    import ctypes as C
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, k, group = 2600, 8200, 128
    need = C.c_size_t(0)
    assert thinfer.lib().thinfer_w4_linear_workspace(40, n, k, group, C.byref(need)) == thinfer.OK and need.value > 0
    assert thinfer.lib().thinfer_w4_linear_workspace(16, n, k, group, C.byref(C.c_size_t(0))) == thinfer.OK
    packed = [thinfer.op_w4_quantize((torch.randn(n, k, generator=gen, device="cuda") * 0.02).half(), group) for _ in range(2)]
    x = [torch.randn(40, k, generator=gen, device="cuda").half() for _ in range(2)]
    want = [[thinfer.op_w4_linear(a, p, n, group, out_fp32=True) for a in x] for p in packed]
    workspace = torch.full((need.value,), 255, dtype=torch.uint8, device="cuda")
    graphs = []
    for p in packed:
        graph, held = torch.cuda.CUDAGraph(), x[0].clone()
        with torch.cuda.graph(graph):
            y = thinfer.op_w4_linear(held, p, n, group, out_fp32=True, workspace=workspace)
        graphs.append((graph, held, y))
    for turn in range(4):
        for i, (graph, held, y) in enumerate(graphs):
            held.copy_(x[turn % 2])
            graph.replay()
            assert torch.equal(y, want[i][turn % 2])
            workspace.fill_(turn * 37)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[thinfer.op_w4_linear(x[i], packed[i], n, group, out_fp32=True, stream=s) for _ in range(5)] for i, s in enumerate(streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i][i]) for i in range(2) for g in got[i])
    with pytest.raises(thinfer.ThinferError) as e:
        thinfer.op_w4_linear(x[0], packed[0], n, group, workspace=workspace[:-16])
    assert e.value.code == thinfer.ECAPACITY


def test_other_kernels_around_tensor_memory(T):
    """Products between the library's other kernels that use tensor memory, all chained in one stream."""
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, k = 2600, 8200
    w = (torch.randn(n, k, generator=gen, device="cuda") * 0.02).half()
    packed = thinfer.op_w4_quantize(w, 128)
    x = torch.randn(64, k, generator=gen, device="cuda").half()
    back = thinfer.op_w4_read(packed, n, k, 128, torch.float16)
    want, plain = thinfer.op_w4_linear(x, packed, n, 128), thinfer.op_linear(x, back)
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        got.append((thinfer.op_w4_linear(x, packed, n, 128), thinfer.op_linear(x, back)))
        got.append((thinfer.op_w4_linear(x, thinfer.op_w4_quantize(w, 128), n, 128), thinfer.op_linear(x, thinfer.op_w4_read(packed, n, k, 128, torch.float16))))
    assert all(torch.equal(a, want) and torch.equal(b, plain) for a, b in got)


def test_the_binding_refuses(T):
    torch, thinfer = T
    x, packed = torch.zeros(3, 64, dtype=torch.float16, device="cuda"), torch.zeros(thinfer.w4_bytes(20, 64, 32), dtype=torch.uint8, device="cuda")
    f32 = torch.zeros(3, 20, device="cuda")
    for call, code in (
            (lambda: thinfer.op_w4_linear(x, packed[:-1], 20, 32), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x, packed, 40, 32), thinfer.EINVAL),
            (lambda: thinfer.op_w4_linear(x, packed, 20, 48), thinfer.EUNSUPPORTED), (lambda: thinfer.op_w4_linear(x.float(), packed, 20, 32), thinfer.EUNSUPPORTED),
            (lambda: thinfer.op_w4_linear(x[:0], packed, 20, 32), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x.T, packed, 20, 32), thinfer.EINVAL),
            (lambda: thinfer.op_w4_linear(x, packed, 20, 32, out=f32[:2]), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x, packed, 20, 32, out=f32.double()), thinfer.EINVAL),
            (lambda: thinfer.op_w4_linear(x, packed, 20, 32, out=f32.bfloat16()), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x, packed, 20, 32, out=torch.zeros(20, 3, device="cuda").T), thinfer.EINVAL),
            (lambda: thinfer.op_w4_linear(torch.zeros(65, 64, dtype=torch.float16, device="cuda"), packed, 20, 32), thinfer.EUNSUPPORTED),
            (lambda: thinfer.op_w4_linear(x[:, 1:57], packed, 20, 32), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x, packed.cpu(), 20, 32), thinfer.EINVAL),
            (lambda: thinfer.op_w4_linear(x, None, 20, 32), thinfer.EINVAL), (lambda: thinfer.op_w4_linear(x, packed, "20", 32), thinfer.EINVAL),
            (lambda: thinfer.op_w4_quantize(x.float(), 32), thinfer.EUNSUPPORTED), (lambda: thinfer.op_w4_quantize(x, 33), thinfer.EUNSUPPORTED),
            (lambda: thinfer.op_w4_quantize(x[:, :60], 32), thinfer.EUNSUPPORTED), (lambda: thinfer.op_w4_quantize(x[0], 32), thinfer.EINVAL),
            (lambda: thinfer.op_w4_quantize(x, 32, packed=packed[:100]), thinfer.EINVAL), (lambda: thinfer.op_w4_read(packed, 20, 64, 32, torch.float16, out=x), thinfer.EINVAL),
            (lambda: thinfer.op_w4_read(packed, 20, 64, 32, torch.float16, out=torch.zeros(20, 64, device="cuda")), thinfer.EINVAL),
            (lambda: thinfer.op_w4_read(packed, 19, 128, 32, torch.float16), thinfer.OK)):
        if code == thinfer.OK:
            call()                                    # the same number of bytes
            continue
        with pytest.raises(thinfer.ThinferError) as e:
            call()
        assert e.value.code == code, e.value
