"""Probabilities of logits, verification of drafted tokens, and a decode step of drafts with 4-bit weights and cache, against
their float64 definitions (run with -m gpu on a B200)."""
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


def _cuda(torch, x, dtype=np.float32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=dtype))).cuda()


# ------------------------------------------------------------------ probabilities
def _close(got, want, d_over_t, vocab):
    """The distance from the largest logit is rounded once (2^-24 of it), exp2 is good to two units, the product with its
    correction, the sum's inverse and the last product round once each; a sum in FP32 of vocab terms, at least 256 of
    them side by side, is off by 2^-24 for each that one thread adds and for the ten levels that join them.  Numbers below
    FP32's smallest normal one may be off by that."""
    tol = 2.0 ** -24 * (np.abs(d_over_t) + 10 + vocab / 256 + 10) * want + 2.0 ** -126
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= tol[ok])


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 32000), (3, 2), (5, 33), (2, 1000), (7, 4099), (300, 257), (2, 100003), (33, 8192), (4, 131072), (1, 200001), (1, 400000),
                                        (900, 5), (160, 20001)])
def test_probabilities(T, rows, vocab):
    torch, thinfer = T
    rng = np.random.default_rng(rows + vocab)
    x = (rng.standard_normal((rows, vocab)) * rng.choice([0.1, 4, 60], (rows, 1))).astype(np.float32)
    temp = rng.uniform(0.3, 2, rows).astype(np.float32)
    temp[2::5] = 0
    x[rng.random(x.shape) < 0.01] = -INF              # masked tokens
    if vocab > 40:
        x[0, 7], x[rows - 1, vocab - 1] = x[0].max(), x[rows - 1].max()      # ties
    wide = torch.full((rows, vocab + 3), 99.0, device="cuda")
    wide[:, 1:-2] = _cuda(torch, x)
    big = np.where(np.isneginf(x).all(1), 0, x.max(1)).astype(np.float64)[:, None]
    far = np.where(np.isneginf(x), 0, x - big)
    before = wide.clone()
    for t in (None, temp):
        want = tk.probs(x, t)
        by = np.where(temp > 0, temp, 1)[:, None] if t is not None else 1.0
        args = None if t is None else _cuda(torch, t)
        first = thinfer.op_token_probs(wide[:, 1:-2], args)
        _close(first.double().cpu().numpy(), want, far / by, vocab)
        assert torch.equal(wide, before)
        out = torch.full((rows, vocab + 2), 99.0, device="cuda")
        thinfer.op_token_probs(_cuda(torch, x), args, out=out[:, :vocab])
        _close(out[:, :vocab].double().cpu().numpy(), want, far / by, vocab)
        assert torch.all(out[:, vocab:] == 99)
    thinfer.op_token_probs(wide[:, 1:-2], _cuda(torch, temp), out=wide[:, 1:-2])          # in place
    assert torch.equal(wide[:, 1:-2], first) and torch.all(wide[:, :1] == 99) and torch.all(wide[:, -2:] == 99)


@pytest.mark.parametrize("vocab", [3, 50, 5000, 70001, 300000])
def test_ends_of_probabilities(T, vocab):
    torch, thinfer = T
    x = np.zeros((10, vocab), np.float32)
    x[0] = -INF
    x[1, 1:] = -INF                                   # one token left
    x[2, vocab - 1] = NAN
    x[3, 2] = INF
    x[4], x[4, vocab // 2] = -3e38, 3e38              # distances beyond FP32
    x[5] = 1e38
    x[6, -1] = 5
    x[7] = -INF
    x[8, 1] = INF
    x[9, 0] = NAN
    temp = np.array([1, 1, 1, 1, 1, 1e-30, 1e30, 0, -1, NAN], np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        want = tk.probs(x, np.where(np.isnan(temp), 0, temp))
        got = thinfer.op_token_probs(_cuda(torch, x), _cuda(torch, temp)).double().cpu().numpy()
    _close(got, want, np.zeros_like(want), vocab)
    assert np.all(got[0] == 0) and np.all(got[7] == 0) and got[8, 1] == 1 and got[8].sum() == 1 and np.isnan(got[[2, 3, 9]]).all()
    # temperatures at the ends: all of it on the largest, or equal shares
    x = np.tile(np.linspace(-1, 1, vocab, dtype=np.float32), (4, 1))
    got = thinfer.op_token_probs(_cuda(torch, x), _cuda(torch, [1e-38, 1e-45, 3e38, INF])).cpu().numpy()
    assert np.all(got[:2, -1] == 1) and np.all(got[:2, :-1] == 0) and np.allclose(got[2:], 1 / vocab, rtol=vocab * 2.0 ** -24)


# ------------------------------------------------------------------ verification
def _distributions(rng, shape, sharp=3.0):
    x = rng.standard_normal(shape) * sharp
    w = np.exp(x - x.max(-1, keepdims=True))
    return (w / w.sum(-1, keepdims=True)).astype(np.float32)


def _check(T, p, q, drafts, u, counts=None, dp=None, dq=None):
    torch, thinfer = T
    batch, n = p.shape[0], p.shape[1] - 1
    want, kept = tk.verify(p, q, drafts, u, counts)
    tokens = torch.full((batch, n + 1), -77, dtype=torch.int32, device="cuda")
    accepted = torch.full((batch,), -77, dtype=torch.int32, device="cuda")
    thinfer.op_verify_drafts(dp if dp is not None else _cuda(torch, p), None if q is None else (dq if dq is not None else _cuda(torch, q)),
                             _cuda(torch, drafts, np.int32).view(batch, n), _cuda(torch, u), None if counts is None else _cuda(torch, counts, np.int32), tokens, accepted)
    tokens, accepted = tokens.cpu().numpy(), accepted.cpu().numpy()
    for b in range(batch):
        if want[b] is None:                           # padding: left as it was
            assert np.all(tokens[b] == -77) and accepted[b] == -77
        else:
            assert accepted[b] == kept[b] and tokens[b].tolist() == want[b], (b, tokens[b], want[b])
    return tokens, accepted


@pytest.mark.parametrize("batch,n,vocab", [(1, 0, 1), (1, 1, 2), (3, 4, 33), (1, 4, 32000), (70, 3, 1000), (5, 8, 4097), (2, 2, 100003), (3, 1, 262145), (1, 0, 128000), (200, 2, 7),
                                           (1, 40, 515), (2, 600, 40), (160, 1, 9001)])
@pytest.mark.parametrize("how", ["drawn", "sure", "ragged"])
def test_verification(T, batch, n, vocab, how):
    rng = np.random.default_rng(batch * 100 + n + vocab)
    p = _distributions(rng, (batch, n + 1, vocab))
    near = np.log(p[:, :n].astype(np.float64) + 1e-30) + rng.standard_normal((batch, n, vocab)) * 0.3
    q = np.exp(near)
    q = (q / q.sum(-1, keepdims=True)).astype(np.float32)
    cum = np.cumsum(q.astype(np.float64), -1)
    drafts = np.minimum((cum <= rng.random((batch, n, 1)) * cum[..., -1:]).sum(-1), vocab - 1) if n else np.zeros((batch, 0))
    u = rng.random((batch, n + 1)).astype(np.float32)
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    if how == "sure":
        u[:, :n] *= 0.2
        _check(T, p, None, drafts, u)
        return
    counts = rng.integers(-1, n + 3, batch) if how == "ragged" else None
    _, accepted = _check(T, p, q, drafts, u, counts)
    if how == "drawn" and batch * n >= 100 and vocab > 100:
        assert 0 < accepted.sum() < batch * n


def test_uniforms_at_the_ends(T):
    rng = np.random.default_rng(0)
    p, q = _distributions(rng, (6, 3, 2000)), _distributions(rng, (6, 2, 2000))
    drafts = rng.integers(0, 2000, (6, 2))
    u = np.zeros((6, 3), np.float32)
    u[1:3, 2] = 1 - 2.0 ** -24
    u[2:4, :2] = 1 - 2.0 ** -24
    u[4, :2] = 2.0 ** -30
    p[5, :, :10] = 0                                  # u = 0 draws the first token that has a probability
    _check(T, p, q, drafts, u)
    _check(T, p, None, drafts, u)


def test_ends_of_verification(T):
    rng = np.random.default_rng(1)
    vocab, n = 5000, 2
    p, q = _distributions(rng, (12, n + 1, vocab)), _distributions(rng, (12, n, vocab))
    drafts = rng.integers(0, vocab, (12, n))
    u = np.full((12, n + 1), 0.5, np.float32)
    drafts[0, 0], drafts[1, 0], drafts[2, 1] = -1, vocab, 2 ** 31 - 1        # no tokens
    q[3] = p[3, :n]                                   # equal: every draft stays
    q[4, 0, drafts[4, 0]] = 0                         # a draft that could not have been drawn
    p[5, 0], q[5, 0], p[5, 0, 3] = 0, 0, 0.25         # a target with a single token, drafted elsewhere
    p[6, 0] = 0                                       # nothing to draw from
    p[7, 0] = q[7, 0] * np.float32(0.5)               # less than the draft everywhere: drawn from the target
    p[7, 0, drafts[7, 0]] = 0
    p[8, 0, ::2], p[8, 0, 1] = NAN, -1
    p[9, 0], q[9, 0] = 0, 0
    p[9, 0, -1], drafts[9, 0] = 1e-40, 4              # a single token of a denormal probability, the last one
    p[10] = 2.0 ** -140                               # rows that add up to a denormal number
    p[11, 0] *= 1e-20                                 # not normalised
    for uu in (0.0, 0.5, 1 - 2.0 ** -24):
        u[:, n] = uu
        _check(T, p, q, drafts, u)
        _check(T, p, None, drafts, u)


def test_strided_probabilities(T):
    torch, thinfer = T
    rng = np.random.default_rng(2)
    batch, n, vocab = 4, 3, 1001
    p, q = _distributions(rng, (batch, n + 1, vocab)), _distributions(rng, (batch, n, vocab))
    drafts, u = rng.integers(0, vocab, (batch, n)), rng.random((batch, n + 1)).astype(np.float32) * 0.9
    wide = torch.full((n + 1, batch, vocab + 7), NAN, device="cuda")
    wide[..., 3:-4] = _cuda(torch, p).transpose(0, 1)
    wq = torch.full((batch, n + 2, vocab + 2), NAN, device="cuda")
    wq[:, 1:-1, 2:] = _cuda(torch, q)
    _check(T, p, q, drafts, u, dp=wide[..., 3:-4].transpose(0, 1), dq=wq[:, 1:-1, 2:])
    # one distribution for all requests and drafts
    one = _cuda(torch, p[0, 0])
    _check(T, np.broadcast_to(p[0, 0], p.shape), np.broadcast_to(q[0, 0], q.shape), drafts, u, dp=one.expand(batch, n + 1, vocab), dq=_cuda(torch, q[0, 0]).expand(batch, n, vocab))


def test_a_long_vocabulary_beyond_32_bits(T):
    """Rows further apart than 2^31 elements."""
    torch, thinfer = T
    rng = np.random.default_rng(3)
    vocab, far = 2000, (1 << 31) + 5
    p, u = _distributions(rng, (2, 1, vocab)), rng.random((2, 1)).astype(np.float32)
    big = torch.empty(far + vocab, device="cuda")
    dp = big.as_strided((2, 1, vocab), (far, vocab, 1))
    dp.copy_(_cuda(torch, p))
    _check(T, p, None, np.zeros((2, 0)), u, dp=dp)
    x = rng.standard_normal((2, vocab)).astype(np.float32)
    dx = big.as_strided((2, vocab), (far, 1))
    dx.copy_(_cuda(torch, x))
    out = thinfer.op_token_probs(dx)
    _close(out.double().cpu().numpy(), tk.probs(x), x - x.max(1, keepdims=True), vocab)
    thinfer.op_token_probs(dx, out=dx)
    assert torch.equal(dx, out)


def test_bindings_refuse(T):
    torch, thinfer = T
    p, z, u = torch.zeros(2, 3, 9, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, device="cuda")
    for call in (
            lambda: thinfer.op_token_probs(p[0].half()), lambda: thinfer.op_token_probs(p), lambda: thinfer.op_token_probs(p[0].T), lambda: thinfer.op_token_probs(p[0, :0]),
            lambda: thinfer.op_token_probs(p[0], u[0, :2]), lambda: thinfer.op_token_probs(p[0], u[0].double()), lambda: thinfer.op_token_probs(p[0], out=p[0].double()),
            lambda: thinfer.op_token_probs(p[0, :2], out=p[0, 1:]), lambda: thinfer.op_token_probs(p[0], out=p[0, :2]), lambda: thinfer.op_token_probs(p[0], 1.0),
            lambda: thinfer.op_verify_drafts(p.double(), None, z, u), lambda: thinfer.op_verify_drafts(p, p, z, u), lambda: thinfer.op_verify_drafts(p[:, :, ::2], None, z, u),
            lambda: thinfer.op_verify_drafts(p, None, z.long(), u), lambda: thinfer.op_verify_drafts(p, None, z[:, :1], u), lambda: thinfer.op_verify_drafts(p, None, z, u[:, :2]),
            lambda: thinfer.op_verify_drafts(p, None, z, u, counts=z[0, :1]), lambda: thinfer.op_verify_drafts(p, None, z, u, tokens=z), lambda: thinfer.op_verify_drafts(p[:0], None, z[:0], u[:0]),
            lambda: thinfer.op_verify_drafts(p, p[:, :2].cpu(), z, u), lambda: thinfer.op_verify_drafts(p, None, z, u, accepted=z[0].long())):
        with pytest.raises(thinfer.ThinferError) as e:
            call()
        assert e.value.code == thinfer.EINVAL, e.value


# ------------------------------------------------------------------ all together
def test_a_captured_step_of_drafts(T):
    """Decode steps of three requests with four drafts each: 4-bit projections, keys and values appended to the 4-bit cache,
    attention of the five query tokens, the vocabulary projection, probabilities, verification, and the cache cut back to
    what stays.  Captured once and replayed, against the same calls one by one."""
    torch, thinfer = T
    gen = torch.Generator(device="cuda").manual_seed(3)
    batch, n, hidden, hq, hkv, d, vocab, page, group = 3, 4, 256, 4, 2, 64, 1003, 16, 64
    rows = batch * (n + 1)

    def weights(out, k):
        return thinfer.op_w4_quantize((torch.randn(out, k, generator=gen, device="cuda") * k ** -0.5).half(), group)
    qkv_out = (hq + 2 * hkv) * d
    wqkv, wo, head = weights(qkv_out, hidden), weights(hidden, hq * d), weights(vocab, hidden)
    steps = 6
    inputs = [((torch.randn(rows, hidden, generator=gen, device="cuda")).half(), torch.randint(0, vocab, (batch, n), generator=gen, device="cuda").int(),
               torch.rand(batch, n + 1, generator=gen, device="cuda"), torch.softmax(torch.randn(batch, n, vocab, generator=gen, device="cuda"), -1)) for _ in range(steps)]
    temp = torch.full((rows,), 1.3, device="cuda")
    row_of = torch.arange(batch, device="cuda", dtype=torch.int32).repeat_interleave(n + 1)
    behind = torch.arange(n + 1, device="cuda", dtype=torch.int32).repeat(batch)
    add = torch.full((batch,), n + 1, dtype=torch.int32, device="cuda")

    def fresh():
        pool = torch.zeros(20, thinfer.kv4_page_bytes(hkv, d, page), dtype=torch.uint8, device="cuda")
        return pool, torch.full((batch, 6), -1, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")

    def step(state, x, drafts, u, q):
        pool, table, lens = state
        first = lens[row_of.long()]
        thinfer.op_kv4_reserve(table, lens, add, pool.shape[0], page, lens_out=lens)
        qkv = thinfer.op_w4_linear(x, wqkv, qkv_out, group)
        heads = qkv.view(rows, hq + 2 * hkv, d)
        thinfer.op_kv4_append(pool, table, heads[:, hq:hq + hkv], heads[:, hq + hkv:], row_of, first + behind, page)
        o = thinfer.op_kv4_attention(heads[:, :hq].view(batch, n + 1, hq, d), pool, table, lens, page)
        h = x + thinfer.op_w4_linear(o.view(rows, hq * d), wo, hidden, group)
        p = thinfer.op_token_probs(thinfer.op_w4_linear(h, head, vocab, group, out_fp32=True), temp).view(batch, n + 1, vocab)
        tokens, accepted = thinfer.op_verify_drafts(p, q, drafts, u)
        lens.sub_(n - accepted)
        return tokens, accepted, p

    state, want = fresh(), []
    for x in inputs:
        tokens, accepted, p = step(state, *x)
        check, kept = tk.verify(p.cpu().numpy(), x[3].cpu().numpy(), x[1].tolist(), x[2].cpu().numpy())
        assert tokens.tolist() == check and accepted.tolist() == kept
        want.append((tokens.clone(), accepted.clone(), p.clone(), state[2].clone()))
    assert sum(int(w[1].sum()) for w in want) > 0 and state[2].max() <= 6 * page
    live, held = fresh(), [t.clone() for t in inputs[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(live, *held)
    for t, v in zip(live, fresh()):
        t.copy_(v)
    for x, w in zip(inputs, want):
        for a, b in zip(held, x):
            a.copy_(b)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((*out, live[2]), w))
    # only what the lengths still cover has to be the same; drafts that went are written over
    for a, b in ((live[1], state[1]),):
        for r in range(batch):
            used = -(-int(state[2][r]) // page)
            assert torch.equal(a[r, :used], b[r, :used])
