"""Weights in 4 bits and the choice of tokens at the ends: vocabularies that no cluster holds, a process whose first calls are
captured, several threads at once (run with -m gpu on a B200)."""
import threading

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


def _close(got, want, d_over_t, vocab):
    """As for shorter vocabularies: 2^-24 for the distance from the largest logit, for each addition of a thread among 512, and
    for twenty roundings more."""
    tol = 2.0 ** -24 * (np.abs(d_over_t) + 20 + vocab / 256) * want + 2.0 ** -126
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= tol[ok])


@pytest.mark.parametrize("vocab", [442361, 442362, 442363, 442366, 450001, 1000003])
def test_probabilities_of_very_long_vocabularies(T, vocab):
    torch, thinfer = T
    rng = np.random.default_rng(vocab)
    rows = 9
    x = (rng.standard_normal((rows, vocab)) * 3).astype(np.float32)
    x[1] = -INF
    x[2, vocab - 1] = NAN
    x[3, 2] = INF
    x[4, 5], x[4, vocab - 1] = x[4].max(), x[4].max()
    x[5], x[5, vocab // 2] = -3e38, 3e38
    x[6, ::3] = -INF
    x[7, 0] = NAN
    x[8, vocab - 2] = INF
    temp = np.array([0.7, 1, 1, 1, 0, 1, 1.5, -1, 0], np.float32)
    wide = torch.full((rows, vocab + 3), 99.0, device="cuda")
    wide[:, 1:-2] = torch.from_numpy(x).cuda()
    with np.errstate(over="ignore", invalid="ignore"):
        want = tk.probs(x, temp)
        far = x.astype(np.float64) - x.astype(np.float64).max(1, keepdims=True)
    far = np.where(np.isfinite(far), far, 0) / np.where(temp > 0, temp, 1)[:, None]
    far[5] = 0                                        # nothing but the largest is left
    temp = torch.from_numpy(temp).cuda()
    got = thinfer.op_token_probs(wide[:, 1:-2], temp)
    _close(got.double().cpu().numpy(), want, far, vocab)
    thinfer.op_token_probs(wide[:, 1:-2], temp, out=wide[:, 1:-2])
    assert torch.equal(wide[:, 1:-2].isnan(), got.isnan()) and torch.equal(wide[:, 1:-2].nan_to_num(7), got.nan_to_num(7))
    assert torch.all(wide[:, 0] == 99) and torch.all(wide[:, -2:] == 99)


@pytest.mark.parametrize("vocab", [131065, 262139, 1000003])
def test_verification_of_very_long_vocabularies(T, vocab):
    """What is drawn from lies at the first token, the last one, and around the middle of the walk over the vocabulary."""
    torch, thinfer = T
    places = sorted({0, 1, 4095, 4096, 16383, 16384, vocab // 2, vocab - 2, vocab - 1})
    batch, n = len(places), 2
    p = np.zeros((batch, n + 1, vocab), np.float32)
    for b, place in enumerate(places):
        p[b, :, place] = 1
    drafts = np.array([[place, (place + 1) % vocab] for place in places], np.int32)
    u = np.full((batch, n + 1), 0.5, np.float32)
    want, kept = tk.verify(p, None, drafts, u, None)
    tokens, accepted = thinfer.op_verify_drafts(torch.from_numpy(p).cuda(), None, torch.from_numpy(drafts).cuda(), torch.from_numpy(u).cuda())
    assert accepted.tolist() == list(kept) == [1] * batch
    assert tokens.tolist() == want and [t[1] for t in want] == places


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("rows,group", [(9, 32), (9, 64), (16, 64), (23, 32), (32, 64), (41, 64), (64, 32)])
def test_products_of_a_large_matrix_in_small_groups(T, t, rows, group):
    """Small whole numbers, more than 80 x 1024 tiles and blocks: nothing may be off, in any token row or behind the last one."""
    torch, thinfer = T
    n, k, tt = 20501, 8200, {"f16": torch.float16, "bf16": torch.bfloat16}[t]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randint(-7, 8, (n, k), device="cuda", generator=gen).to(tt)
    w[:, ::8], w[:, 1::8] = -7, 8                     # every group spans 15: codes are the numbers themselves
    packed = thinfer.op_w4_quantize(w, group)
    assert torch.equal(thinfer.op_w4_read(packed, n, k, group, tt), w)
    x = torch.randint(-2, 3, (rows, k), device="cuda", generator=gen).to(tt)
    want = torch.cat([x.double() @ part.double().T for part in w.split(4096)], 1)         # whole numbers below 2^18
    out = torch.full((rows + 1, n + 2), 7.0, dtype=torch.float32, device="cuda")
    thinfer.op_w4_linear(x, packed, n, group, out=out[:-1, 1:-1])
    assert torch.equal(out[:-1, 1:-1].double(), want) and torch.all(out[-1] == 7) and torch.all(out[:, 0] == 7) and torch.all(out[:, -1] == 7)


def test_first_calls_inside_a_capture():
    """A process that captures the very first call of each kind, and replays them on other numbers."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2605_25655_b200 import thinfer
torch.zeros(1, device="cuda")
gen = torch.Generator(device="cuda").manual_seed(0)
draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")
w, x, logits = (draw(2600, 8200) * 0.02).bfloat16(), draw(64, 8200).bfloat16(), draw(10, 9001)
drafts, u = torch.randint(0, 9001, (2, 4), generator=gen, device="cuda").int(), torch.rand(2, 5, generator=gen, device="cuda")
def step():
    packed = thinfer.op_w4_quantize(w, 128)
    p = thinfer.op_token_probs(logits)
    return [thinfer.op_w4_linear(x, packed, 2600, 128), thinfer.op_w4_linear(x[:3], packed, 2600, 128), thinfer.op_w4_linear(x[:16], packed, 2600, 128, out_fp32=True),
            thinfer.op_w4_read(packed, 2600, 8200, 128, torch.bfloat16), p, *thinfer.op_verify_drafts(p.view(2, 5, 9001), None, drafts, u)]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = step()
for _ in range(2):
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, step()))
    w.mul_(-1.25), x.mul_(0.5), logits.copy_(draw(10, 9001)), u.copy_(torch.rand(2, 5, generator=gen, device="cuda"))
print("equal")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert got.returncode == 0 and got.stdout.strip() == "equal", got.stderr


def test_threads_at_once(T):
    """Both storage types and all operators from four threads, each on a stream of its own."""
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(5)
    inputs = []
    for i in range(4):
        t = (torch.float16, torch.bfloat16)[i % 2]
        inputs.append(((torch.randn(1300 + 8 * i, 8200, generator=gen, device="cuda") * 0.02).to(t), torch.randn(64, 8200, generator=gen, device="cuda").to(t),
                       torch.randint(0, 4000, (8, 3), generator=gen, device="cuda").int(), torch.rand(8, 4, generator=gen, device="cuda")))

    def run(w, x, drafts, u, stream=None):
        n, k = w.shape
        packed = thinfer.op_w4_quantize(w, 64, stream=stream)
        y = thinfer.op_w4_linear(x, packed, n, 64, stream=stream)
        z = thinfer.op_w4_linear(x[:32], packed, n, 64, out_fp32=True, stream=stream)
        p = thinfer.op_token_probs(z, stream=stream).view(8, 4, n)
        return [y, z, p, *thinfer.op_verify_drafts(p, None, drafts, u, stream=stream)]
    want = [run(*i) for i in inputs]
    torch.cuda.synchronize()
    wrong = []

    def thread(i):
        try:
            torch.cuda.set_device(0)
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):           # what the calls allocate belongs to the stream
                for _ in range(20):
                    got = run(*inputs[i], stream=stream)
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        wrong.append(i)
        except BaseException as e:
            wrong.append(e)
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not wrong
