"""Weights in 4 bits and the choice of tokens: buffers that are written again between calls, numbers at the ends of their types, rows
and requests that differ in kind (run with -m gpu on a B200)."""
import numpy as np
import pytest

from oracle import tokens as tk
from oracle import w4
from paper_2605_25655_b200 import synth

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


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("between", ["nothing", "probabilities"])
def test_a_models_weights_read_back_in_front_of_a_step(T, mode, between):
    """4-bit weights read back into the tensors of a model, directly in front of each decode step or with another call between them:
    the same bits as with a pause behind the call."""
    torch, thinfer = T
    shape = synth.Shape(hidden=1024, n_q_heads=8, n_kv_heads=8, head_dim=128, ffn=2816, n_layers=1)
    layers = thinfer.to_device_layers([synth.layer_weights(shape, 0)])
    names = [n for n, w in layers[0].items() if w.dim() == 2]
    packed = [{n: thinfer.op_w4_quantize(layers[0][n] * by, 64) for n in names} for by in (1.0, -0.75)]
    x = torch.from_numpy(synth.hidden_states(shape, 0, (2, 24))).cuda()
    logits = torch.randn(64, 5000, device="cuda")

    def run(pause):
        ctx = thinfer.Context(shape, layers, max_batch=2, max_seq=32)
        ctx.set_launch_mode(mode)
        out = [ctx.prefill(x[:, :8].contiguous())]
        steps = [x[:, 8 + i].contiguous() for i in range(16)]
        for i, step in enumerate(steps):
            for n in reversed(names):
                w = layers[0][n]
                thinfer.op_w4_read(packed[i % 2][n], w.shape[0], w.shape[1], 64, torch.float16, out=w)
            if between == "probabilities":
                thinfer.op_token_probs(logits)
            if pause:
                torch.cuda.synchronize()
            out.append(ctx.decode_step(step))
            if pause:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert ctx.status() == 0
        ctx.close()
        return out
    for w, p in ((layers[0][n], packed[1][n]) for n in names):
        thinfer.op_w4_read(p, w.shape[0], w.shape[1], 64, torch.float16, out=w)
    want = run(True)
    assert torch.equal(layers[0][names[0]], thinfer.op_w4_read(packed[1][names[0]], *layers[0][names[0]].shape, 64, torch.float16))
    assert not torch.equal(want[-1], want[-2])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))


# ------------------------------------------------------------------ numbers at the ends of their types
def _whole(rng, rows, n, k, group, t, scale, token):
    """Packed weights with scales of 2^scale, tokens that are whole numbers times 2^token, and their products, which are exact in
    FP64: whole numbers below 2^19 times a power of two."""
    dt = {"float16": np.float16, "bfloat16": "bf16"}[t]
    codes, zeros = rng.integers(0, 16, (n, k)), rng.integers(0, 16, (n, -(-k // group)))
    of = np.arange(k) // group
    x = rng.integers(-3, 4, (rows, k)).astype(np.float64)
    want = (x @ (codes - zeros[:, of]).T.astype(np.float64)) * 2.0 ** (token + scale)
    return w4.pack(codes, np.full(zeros.shape, 2.0 ** scale), zeros, group, dt), x * 2.0 ** token, want


@pytest.mark.parametrize("t,scale,token", [("float16", -24, -24), ("float16", -14, -24), ("float16", 14, 13), ("bfloat16", -10, -133), ("bfloat16", 0, -126), ("bfloat16", -133, 0), ("bfloat16", -3, -117),
                                           ("bfloat16", 100, -130), ("bfloat16", 125, -133), ("bfloat16", 127, -60), ("bfloat16", -100, 120), ("bfloat16", -133, 126), ("bfloat16", 3, 100)])
@pytest.mark.parametrize("rows,n,k,group", [(1, 70, 600, 128), (8, 33, 392, 32), (16, 40, 1000, 64), (17, 2600, 8200, 128), (64, 2600, 8200, 128), (32, 2700, 8200, 32), (64, 2600, 8200, 64)])
def test_products_over_the_range_of_the_type(T, t, scale, token, rows, n, k, group):
    """Tokens and scales down to the smallest number of their type and up to the largest.  The results are whole numbers below 2^19
    times 2^-143 and more, multiples of FP32's smallest number 2^-149, and so are all sums on the way: nothing may be off."""
    torch, thinfer = T
    rng = np.random.default_rng(rows + k)
    packed, x, want = _whole(rng, rows, n, k, group, t, scale, token)
    x, packed = torch.from_numpy(x).to(getattr(torch, t)).cuda(), torch.from_numpy(packed).cuda()
    got = thinfer.op_w4_linear(x, packed, n, group, out_fp32=True)
    assert np.array_equal(got.double().cpu().numpy(), want)
    assert torch.equal(thinfer.op_w4_linear(x, packed, n, group), torch.from_numpy(want).cuda().to(getattr(torch, t)))


@pytest.mark.parametrize("rows,n,k,group", [(3, 70, 600, 128), (12, 33, 392, 32), (20, 2600, 8200, 128), (64, 2600, 8200, 32)])
def test_very_large_scales_beside_small_ones(T, rows, n, k, group):
    """BF16: weight rows with scales near the type's end and rows with small ones, in turn of 3 and 5.  Tokens of 2^-60 leave the
    former exact, and of the latter, which are multiples of 2^-160, each group's sum is rounded to a multiple of 2^-149 (sums of
    those are exact); tokens of 2^120 leave FP32 in the former rows only."""
    torch, thinfer = T
    rng = np.random.default_rng(rows)
    codes, zeros = rng.integers(0, 16, (n, k)), rng.integers(0, 16, (n, -(-k // group)))
    large = np.arange(n) % 8 < 3
    scale = np.where(large, 2.0 ** 127, 2.0 ** -100)[:, None]
    packed = torch.from_numpy(w4.pack(codes, np.broadcast_to(scale, zeros.shape), zeros, group, "bf16")).cuda()
    x = rng.integers(1, 4, (rows, k)).astype(np.float64)
    whole = x @ (codes - zeros[:, np.arange(k) // group]).T.astype(np.float64)        # below 2^19
    for token in (-60, 120):
        got = thinfer.op_w4_linear(torch.from_numpy(x * 2.0 ** token).bfloat16().cuda(), packed, n, group, out_fp32=True).double().cpu().numpy()
        want = whole * scale.T * 2.0 ** token
        fine = np.broadcast_to(~large, want.shape) if token > 0 else np.ones(want.shape, bool)
        tol = np.where(large | (token > 0), 0.0, -(-k // group) * 2.0 ** -150)
        assert np.all(np.abs(got - want)[fine] <= np.broadcast_to(tol, want.shape)[fine]) and not np.any(np.isfinite(got[~fine]) & (whole[~fine] != 0))


@pytest.mark.parametrize("vocab", [442367, 1000003, 3000001])
def test_sums_of_long_rows_do_not_drift(T, vocab):
    """Weights of one size, whose running sum in 32 bits would be rounded to the same side again and again.  Eight weights at a
    time are added up in FP32 (three roundings), the rest in FP64; a weight and the last product are off by 2^-24 for the
    distance d / T and for twenty roundings."""
    torch, thinfer = T
    weights = np.array([0.45, 0.3, 0.9, 0.7, 1 / 3])
    temp = np.array([1, 0.5, 2, 1, 1], np.float32)
    x = np.tile((np.log(weights) * temp).astype(np.float32)[:, None], (1, vocab))
    x[:, 17] = 0
    want = tk.probs(x, temp)
    got = thinfer.op_token_probs(torch.from_numpy(x).cuda(), torch.from_numpy(temp).cuda()).double().cpu().numpy()
    tol = 2.0 ** -24 * (np.abs(x) / temp[:, None] + 23) * want
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("vocab", [6, 3001, 150001, 450001])
def test_temperatures_over_their_range(T, vocab):
    """Logits and temperatures of any size: only the quotient d / T decides.  The distance d is rounded once; twenty roundings
    more, and the additions of a thread's weights, as for usual temperatures."""
    torch, thinfer = T
    top = np.float32(3.4e38)
    temp = np.array([3e38, 3e38, 1e38, 2e30, 1.5e30, 1e31, 2.0 ** 64, 2.0 ** 65, 1e25, INF, INF, 3e38, 1e-38, 2.0 ** -126, 2.0 ** -120], np.float32)
    size = np.array([3.4e38, 1e30, 3.4e38, 1e31, 1e30, 3.4e38, 1e20, 1e20, 1e25, 3.4e38, 1.0, 5.0, 2.0 ** -125, 2.0 ** -126, 2.0 ** -119])
    rng = np.random.default_rng(vocab)
    x = np.clip(rng.uniform(-1, 1, (len(temp), vocab)) * size[:, None], -top, top).astype(np.float32)
    x[:, 1], x[:, -1] = size, -size                   # the far ends
    x[:, 2] = -INF                                    # a masked token keeps its 0 at any temperature
    x[:2, 3] = -top
    with np.errstate(over="ignore"):
        want = tk.probs(x, temp)
    far = np.where(np.isneginf(x), 0, x.astype(np.float64).max(1, keepdims=True) - x) / np.maximum(temp, 2.0 ** -126).astype(np.float64)[:, None]
    want[12] = tk.probs(x[12:13], np.array([2.0 ** -126]))[0]      # smaller ones count as the smallest normal number
    got = thinfer.op_token_probs(torch.from_numpy(x).cuda(), torch.from_numpy(temp).cuda()).double().cpu().numpy()
    tol = 2.0 ** -24 * (far + 20 + min(vocab / 256, 90)) * want + 2.0 ** -126
    assert np.all(got[:, 2] == 0) and np.all(np.abs(got - want) <= tol), [(i, np.abs(got[i] - want[i]).max(), want[i].max()) for i in range(len(temp)) if np.any(np.abs(got[i] - want[i]) > tol[i])]


# ------------------------------------------------------------------ requests that differ, threads
@pytest.mark.parametrize("batch,n,vocab", [(1, 3, 33), (40, 4, 1000), (9, 2, 100003), (70, 7, 515), (3, 600, 40)])
def test_certain_drafts_of_ragged_counts(T, batch, n, vocab):
    """Drafts without probabilities, each request with a count of its own: padding, none, some, all, more than there are; most drafts
    stay, so that many requests keep all of their count and draw from the row behind it, of which nothing is taken off."""
    torch, thinfer = T
    rng = np.random.default_rng(batch + n + vocab)
    w = rng.random((batch, n + 1, vocab)) ** 8
    p = (w / w.sum(-1, keepdims=True)).astype(np.float32)
    drafts = rng.integers(0, vocab, (batch, n)).astype(np.int32)
    u = np.minimum(rng.random((batch, n + 1)), 1 - 2.0 ** -24).astype(np.float32)
    u[:, :n] = np.take_along_axis(p[:, :n], drafts[..., None], 2)[..., 0] * rng.choice([0.5, 2.0], (batch, n), p=[0.9, 0.1]).astype(np.float32)
    counts = (np.arange(batch) % (n + 4) - 1 if n < 20 else np.array([-1, 300, n + 2])).astype(np.int32)
    want, kept = tk.verify(p, None, drafts, u, counts)
    assert batch < 9 or any(0 < c < n and k == c for c, k in zip(counts, kept))
    tokens = torch.full((batch, n + 1), -77, dtype=torch.int32, device="cuda")
    accepted = torch.full((batch,), -77, dtype=torch.int32, device="cuda")
    cuda = [torch.from_numpy(a).cuda() for a in (p, drafts, u, counts)]
    thinfer.op_verify_drafts(cuda[0], None, cuda[1], cuda[2], cuda[3], tokens, accepted)
    for b in range(batch):
        assert (tokens[b].tolist(), int(accepted[b])) == (([-77] * (n + 1), -77) if want[b] is None else (want[b], kept[b])), b


def test_threads_finish_their_rounds(T):
    """Products on both kernels, probabilities and verification from four threads on streams of their own; every thread counts the
    rounds that it has compared, and none is left behind."""
    import threading
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(6)
    inputs = []
    for i in range(4):
        t = (torch.float16, torch.bfloat16)[i % 2]
        packed = thinfer.op_w4_quantize((torch.randn(2600 + 16 * i, 8200, generator=gen, device="cuda") * 0.02).to(t), 128)
        inputs.append((packed, 2600 + 16 * i, torch.randn(64, 8200, generator=gen, device="cuda").to(t), torch.randint(0, 2600, (16, 3), generator=gen, device="cuda").int(),
                       torch.rand(16, 4, generator=gen, device="cuda")))

    def run(packed, n, x, drafts, u):
        y = thinfer.op_w4_linear(x, packed, n, 128, out_fp32=True)
        p = thinfer.op_token_probs(y).view(16, 4, n)
        return [y, thinfer.op_w4_linear(x[:8], packed, n, 128), p, *thinfer.op_verify_drafts(p, None, drafts, u)]
    want = [run(*i) for i in inputs]
    torch.cuda.synchronize()
    rounds, equal = [0] * 4, [0] * 4

    def thread(i):
        torch.cuda.set_device(0)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = run(*inputs[i])
                stream.synchronize()
                rounds[i] += 1
                equal[i] += all(torch.equal(a, b) for a, b in zip(got, want[i]))
    threads = [threading.Thread(target=thread, args=(i,), daemon=True) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not any(t.is_alive() for t in threads) and rounds == equal == [20] * 4


@pytest.mark.parametrize("rows,vocab", [(40, 131069), (40, 131070), (40, 151936), (36, 221184), (40, 256000)])
def test_many_rows_of_long_vocabularies(T, rows, vocab):
    """Clusters of every size and slice, rows at every alignment.  At most 108 weights are added up by a thread, half of them
    in each of two sums, and twenty roundings more."""
    torch, thinfer = T
    rng = np.random.default_rng(vocab)
    x = (rng.standard_normal((rows, vocab)) * 4).astype(np.float32)
    temp = rng.uniform(0.5, 1.5, rows).astype(np.float32)
    temp[::7] = 0
    x[3, vocab - 1] = x[3].max() + 1
    wide = torch.full((rows, vocab + 1), 99.0, device="cuda")
    wide[:, 1:] = torch.from_numpy(x).cuda()
    want = tk.probs(x, temp)
    far = (x.max(1, keepdims=True).astype(np.float64) - x) / np.where(temp > 0, temp, 1)[:, None]
    got = thinfer.op_token_probs(wide[:, 1:], torch.from_numpy(temp).cuda())
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= 2.0 ** -24 * (far + 54 + 20) * want + 2.0 ** -126)
    thinfer.op_token_probs(wide[:, 1:], torch.from_numpy(temp).cuda(), out=wide[:, 1:])
    assert torch.equal(wide[:, 1:], got) and torch.all(wide[:, 0] == 99)


def test_the_longest_vocabulary(T):
    """2^31 - 1 tokens in a row that begins three numbers behind a 16-byte boundary, so that its last ones are numbers 2^31 and more
    of their walk: drawn, drafted, the largest logit, and its probability."""
    torch, thinfer = T
    vocab = 2 ** 31 - 1
    row = torch.zeros(vocab + 5, device="cuda")
    assert row.data_ptr() % 16 == 0
    p = row[3:3 + vocab].view(1, 1, vocab)
    empty = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    for places, u, token in (((vocab - 1,), 0.5, vocab - 1), ((vocab - 3, vocab - 2), 0.25, vocab - 3), ((5, vocab - 2), 0.75, vocab - 2), ((0, vocab - 1), 0.25, 0)):
        for place in places:
            p[0, 0, place] = 0.5
        tokens, accepted = thinfer.op_verify_drafts(p, None, empty, torch.full((1, 1), u, device="cuda"))
        assert tokens.tolist() == [[token]] and accepted.tolist() == [0]
        for place in places:
            p[0, 0, place] = 0
    draft = torch.tensor([[vocab - 1]], dtype=torch.int32, device="cuda")
    two = p.expand(1, 2, vocab)
    p[0, 0, vocab - 1], p[0, 0, vocab - 2] = 0.25, 0.75
    for u, want in ((0.2, [[vocab - 1, vocab - 2]]), (0.3, [[vocab - 2, -1]])):
        assert thinfer.op_verify_drafts(two, None, draft, torch.tensor([[u, 0.5]], device="cuda"))[0].tolist() == want
    logits = p[0]
    logits.zero_()
    logits[0, vocab - 1] = 20
    thinfer.op_token_probs(logits, torch.zeros(1, device="cuda"), out=logits)
    assert logits[0, vocab - 1] == 1 and logits[0, :vocab - 1].max() == 0
    logits[0, vocab - 1] = 20
    thinfer.op_token_probs(logits, out=logits)
    far = np.exp(-20.0)
    one = 1 / (1 + far * (vocab - 1))
    last, least, most = (float(v) for v in (logits[0, vocab - 1], logits[0, :vocab - 1].min(), logits[0, :vocab - 1].max()))
    tol = 2.0 ** -24 * (20 + 23)                      # the distance, twenty roundings, three more of the sums
    assert abs(last - one) <= tol * one and least == most and abs(most - far * one) <= tol * far * one
    assert torch.all(row[:3] == 0) and torch.all(row[3 + vocab:] == 0)
