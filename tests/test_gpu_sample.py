"""Tokens drawn from logits, against the definition in float64 over sorted rows.

A draw, and a cut by weight, is held to the definition's own places: what it chose
has to be right for the number given, or for one closer to it than the weights'
rounding (2^-44 of the largest weight each, and some 2^-50 of float64's sums), of
which there is at most one neighbour."""

import math

import numpy as np
import pytest
import torch

from rows_helpers import dev

pytestmark = pytest.mark.gpu

INF = float("inf")


class Row:
    """The definition for one row: x float64 logits (of fp32 or bf16), settings as fp32 numbers."""

    def __init__(self, x, T=1.0, k=0, p=1.0, m=0.0):
        self.x = x
        self.order = np.lexsort((np.arange(len(x)), -x))
        self.order = self.order[x[self.order] > -INF]
        if T == 0:
            self.order = self.order[:1]
            T = 1.0
        y = (x[self.order] - x[self.order[0]]) / T
        self.y, w = y, np.exp(y)
        n = len(w) if not 0 < k < len(w) else k
        self.eps = len(x) * 2.0 ** -43
        self.cum = np.cumsum(w)
        self.w = w
        least = most = n
        if p < 1:
            ahead = self.cum[:n] - w[:n]
            least, most = (max(1, int((ahead < p * self.cum[n - 1] + e).sum())) for e in (-self.eps, self.eps))
        likely = [int((w >= m * (1 + e)).sum()) for e in (1e-12, -1e-12)]
        self.kept = range(max(1, min(least, likely[0])), max(1, min(most, likely[1])) + 1)

    def check(self, u, token, logprob, kept):
        assert kept in self.kept, (kept, self.kept)
        W = self.cum[kept - 1]
        place = int(np.flatnonzero(self.order == token)[0])
        assert place < kept
        assert self.cum[place] - self.w[place] <= u * W + self.eps and u * W < self.cum[place] + self.eps, (u, place)
        # a rounding to fp32, and what the weights' roundings move the sum by
        want = self.y[place] - math.log(W)
        assert abs(logprob - want) <= 2.0 ** -23 * abs(want) + 2 * self.eps / W + 1e-12


def call(lib, logits, T=None, k=None, p=None, m=None, u=None, vocab=None, stride=None, rows=None, stream=None, out=None):
    rows = logits.shape[0] if rows is None else rows
    vocab = logits.shape[1] if vocab is None else vocab
    f = lambda v: None if v is None else dev(np.broadcast_to(np.asarray(v, np.float32), rows), torch.float32)  # noqa: E731
    kk = None if k is None else dev(np.broadcast_to(np.asarray(k), rows))
    tok = torch.full((rows + 1,), -9, dtype=torch.int32, device="cuda")
    kept, lp = torch.full_like(tok, -9), torch.full((rows + 1,), 9.0, device="cuda")
    ws = torch.full((lib.sidp_sample_tokens_bytes(rows, vocab),), 255, dtype=torch.uint8, device="cuda")
    dtype = lib.SIDP_LOGITS_F32 if logits.dtype == torch.float32 else lib.SIDP_LOGITS_BF16
    args = f(T), kk, f(p), f(m), f(u)
    lib.sidp_sample_tokens(logits, dtype, rows, vocab, logits.shape[1] if stride is None else stride, *args, tok, lp, kept, ws, ws.numel(),
                           stream)
    torch.cuda.synchronize()
    assert tok[rows] == -9 and kept[rows] == -9 and lp[rows] == 9.0
    return tok[:rows].cpu().numpy(), lp[:rows].cpu().numpy(), kept[:rows].cpu().numpy()


def f32(v):
    return np.asarray(v, np.float32).astype(np.float64)


def check_rows(lib, logits, T, k, p, m, u):
    got = call(lib, logits.cuda(), T, k, p, m, u)
    x = logits.double().numpy()
    T, p, m, u = (f32(v) for v in (T, p, m, u))
    for r in range(len(x)):
        Row(x[r], T[r], int(k[r]), p[r], m[r]).check(u[r], *(g[r] for g in got))
    return got


def settings(rng, rows, vocab):
    T = np.where(rng.random(rows) < 0.1, 0, rng.uniform(0.1, 2.5, rows))
    k = np.where(rng.random(rows) < 0.5, 0, np.exp(rng.uniform(0, math.log(2 * vocab + 1), rows)).astype(int))
    p = np.where(rng.random(rows) < 0.4, 1.0, rng.uniform(0, 1, rows))
    m = np.where(rng.random(rows) < 0.6, 0.0, rng.uniform(0, 1, rows) ** 3)
    return T, k, p, m, rng.random(rows, np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (40, 7), (60, 63), (30, 1000), (24, 4097), (300, 1025), (16, 32001), (9, 128256),
                                        (2, 200003), (1, 1 << 20)])
def test_draws_match_the_definition(lib, dtype, rows, vocab):
    rng = np.random.default_rng(rows * 7 + vocab)
    for trial, std in enumerate((1.0, 4.0)):
        x = torch.tensor(std * rng.standard_normal((rows, vocab)), dtype=torch.float32).to(dtype)
        if trial and vocab > 8:
            x[:, rng.integers(0, vocab, 3)] += 20.0
        check_rows(lib, x, *settings(rng, rows, vocab))


@pytest.mark.parametrize("rows", [1024, 1025, 2600])
def test_more_rows_than_go_at_once(lib, rows):
    """The last rows, fewer, are cut into more segments than those before them."""
    rng = np.random.default_rng(rows)
    x = torch.tensor(rng.standard_normal((rows, 9001)), dtype=torch.float32).to(torch.bfloat16)
    check_rows(lib, x, *settings(rng, rows, 9001))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab,levels", [(500, 1), (5000, 3), (100000, 1), (100000, 2), (100000, 40)])
def test_equal_logits_go_by_index(lib, dtype, vocab, levels):
    """More tokens in a bin than are put in order at once, by value and by index."""
    rng = np.random.default_rng(levels)
    rows = 12
    x = torch.tensor(rng.integers(0, levels, (rows, vocab)) / 64.0, dtype=dtype)
    check_rows(lib, x, *settings(rng, rows, vocab))
    # temperature alone, and a top-k and a top-p that end among equals
    check_rows(lib, x, np.ones(rows), np.zeros(rows, int), np.ones(rows), np.zeros(rows), rng.random(rows))
    check_rows(lib, x, np.ones(rows), rng.integers(1, vocab, rows), np.ones(rows), np.zeros(rows), rng.random(rows))
    check_rows(lib, x, np.ones(rows), np.zeros(rows, int), rng.random(rows), np.zeros(rows), rng.random(rows))


def test_alike_logits_in_one_bin(lib):
    """Distinct logits a few units of the last place apart, around zero too, where whole numbers of keys are far apart."""
    rng = np.random.default_rng(5)
    x = np.float32(1.0) + rng.integers(0, 5000, (4, 20000)).astype(np.float32) * np.float32(2.0 ** -23)
    y = (rng.standard_normal((4, 20000)) * 2.0 ** rng.integers(-140, -10, (4, 20000))).astype(np.float32)
    for z in (x, y):
        for p, k in ((1.0, 0), (0.3, 0), (0.9, 7777), (1.0, 5001)):
            check_rows(lib, torch.tensor(z), np.ones(4), np.full(4, k), np.full(4, p), np.zeros(4), rng.random(4))


@pytest.mark.parametrize("vocab", [1, 3, 64, 1000, 4096, 70000, 1 << 20])
def test_closed_forms_of_equal_logits(lib, vocab):
    """n equal weights: the token is floor(u n), top-p keeps ceil(p n). u and p are fractions that fp32 and the sums hold exactly."""
    u = np.array([0, 2.0 ** -24, 0.25, 0.5, 0.75, 1 - 2.0 ** -24])
    x = torch.full((len(u), vocab), -3.25, device="cuda")
    tok, lp, kept = call(lib, x, u=u)
    assert np.array_equal(tok, np.floor(u * vocab)) and np.all(kept == vocab)
    np.testing.assert_allclose(lp, -math.log(vocab), rtol=2.0 ** -23, atol=1e-12)
    for p in (0.0, 0.25, 0.5, 0.75):
        n = max(1, math.ceil(p * vocab))
        tok, lp, kept = call(lib, x, T=0.7, p=p, u=u)
        assert np.all(kept == n) and np.array_equal(tok, np.floor(u * n))
    for k in (1, max(1, vocab // 3), vocab, vocab + 5):
        n = min(k, vocab)
        tok, lp, kept = call(lib, x, k=k, u=u)
        assert np.all(kept == n) and np.array_equal(tok, np.floor(u * n))


def test_the_shares_are_the_weights(lib):
    """8192 evenly spaced numbers over one row's logits: each token is drawn as often as its probability says, to one."""
    N, V = 8192, 50
    x = torch.randn(V, generator=torch.Generator().manual_seed(1)) * 2
    u = (np.arange(N) + 0.5) / N
    tok, lp, kept = call(lib, x.expand(N, V).contiguous().cuda(), T=0.8, u=u)
    p = torch.softmax(x.double() / np.float32(0.8).astype(np.float64), 0).numpy()
    assert np.all(np.abs(np.bincount(tok, minlength=V) - N * p) <= 1)
    assert np.all(np.diff(x.numpy()[tok]) <= 0) and np.all(kept == V)


def test_settings_at_their_ends(lib):
    rng = np.random.default_rng(2)
    x = torch.tensor(rng.standard_normal((6, 3000)), dtype=torch.float32)
    best = x.argmax(1).numpy()
    for kw in (dict(T=0), dict(k=1), dict(p=0), dict(m=1), dict(T=1e-30), dict(T=1e-45), dict(T=0, k=50, p=0.5, m=0.3)):
        tok, lp, kept = call(lib, x.cuda(), u=0.999, **kw)
        assert np.array_equal(tok, best), kw
        assert np.all(lp == 0), kw
        assert np.all(kept == (3000 if kw in (dict(T=1e-30), dict(T=1e-45)) else 1)), kw
    # a very hot row is even
    tok, lp, kept = call(lib, x.cuda(), T=3e38, u=0.5)
    order = np.lexsort((np.arange(3000), -x[0].numpy()))
    assert tok[0] == order[1500] and np.all(kept == 3000)
    np.testing.assert_allclose(lp, -math.log(3000), rtol=1e-6)
    for k in (-5, 0, 3000, 1 << 30, -(1 << 31)):  # off
        assert np.all(call(lib, x.cuda(), k=k, u=0.1)[2] == 3000)
    for p in (1.0, 1.5, INF):
        assert np.all(call(lib, x.cuda(), p=p, u=0.1)[2] == 3000)
    # without settings: temperature 1
    got, want = call(lib, x.cuda(), u=0.3), call(lib, x.cuda(), 1.0, 0, 1.0, 0.0, u=0.3)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_masked_rows(lib, dtype):
    rng = np.random.default_rng(3)
    x = torch.tensor(rng.standard_normal((9, 5000)), dtype=torch.float32).to(dtype)
    low = torch.finfo(dtype).min
    x[0, :] = -INF
    x[0, 4321] = -7.0  # one token left
    x[1, :] = -INF  # none
    x[2, 17] = INF
    x[3, 17] = float("nan")
    x[4, :] = low
    x[4, 99] = 1.0  # masked by the lowest value: counted, and never drawn
    x[5, :] = low  # all of them: even
    x[6, 100:] = -INF
    x[7, torch.arange(5000) % 3 > 0] = -INF
    u = np.full(9, 0.75, np.float32)
    tok, lp, kept = call(lib, x.cuda(), u=u)
    assert tok[0] == 4321 and lp[0] == 0 and kept[0] == 1
    for r in (1, 2, 3):
        assert tok[r] == -1 and np.isnan(lp[r]) and kept[r] == 0
    assert tok[4] == 99 and lp[4] == 0 and kept[4] == 5000
    assert tok[5] == 3750 and kept[5] == 5000
    assert kept[6] == 100 and kept[7] == 1667
    xs = x.double().numpy()
    for r in (6, 7, 8):
        Row(xs[r]).check(0.75, tok[r], lp[r], kept[r])
    greedy = call(lib, x.cuda(), T=0, u=u)[0]
    assert list(greedy[:6]) == [4321, -1, -1, -1, 99, 0]
    assert np.array_equal(call(lib, x.cuda(), k=3, u=u)[2], [1, 0, 0, 0, 3, 3, 3, 3, 3])


def test_settings_that_are_none(lib):
    x = torch.randn(5, 100, device="cuda")
    nan = float("nan")
    for kw in (dict(T=-1), dict(T=nan), dict(T=INF), dict(p=-0.1), dict(p=nan), dict(m=-0.1), dict(m=1.1), dict(m=nan), dict(u=1.0),
               dict(u=-0.1), dict(u=nan)):
        kw = {**dict(u=0.5), **kw}
        key = next(k for k in kw if k != "u" or len(kw) == 1)
        v = np.full(5, {"T": 1.0, "p": 0.9, "m": 0.1, "u": 0.5}[key], np.float32)
        v[2] = kw[key]  # one row's: the others are drawn
        tok, lp, kept = call(lib, x, **{**kw, key: v})
        assert tok[2] == -1 and np.isnan(lp[2]) and kept[2] == 0
        rest = [0, 1, 3, 4]
        assert np.all(tok[rest] >= 0) and np.all(np.isfinite(lp[rest])) and np.all(kept[rest] > 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_and_addresses(lib, dtype):
    """Rows at every place within 16 bytes, what lies between them NaN."""
    rng = np.random.default_rng(4)
    for pad in range(1, 9):
        V = 997
        buf = torch.full((6 * (V + pad) + 16,), float("nan"), dtype=dtype)
        x = torch.tensor(rng.standard_normal((6, V)), dtype=torch.float32).to(dtype)
        view = buf[pad:pad + 6 * (V + pad)].view(6, V + pad)
        view[:, :V] = x
        T, k, p, m, u = settings(rng, 6, V)
        big = buf.cuda()
        got = call(lib, big[pad:pad + 6 * (V + pad)].view(6, V + pad), T, k, p, m, u, vocab=V, stride=V + pad)
        want = call(lib, x.cuda(), T, k, p, m, u)
        assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_a_row_is_drawn_alike_alone_and_among_others(lib):
    """Bit for bit, whatever the number of rows, which decides how a row is shared out."""
    rng = np.random.default_rng(6)
    V = 50000
    x = torch.tensor(3 * rng.standard_normal((700, V)), dtype=torch.float32).to(torch.bfloat16).cuda()
    T, k, p, m, u = settings(rng, 700, V)
    want = call(lib, x, T, k, p, m, u)
    for rows in (1, 2, 3, 17, 64, 130, 300):
        got = call(lib, x[:rows], T[:rows], k[:rows], p[:rows], m[:rows], u[:rows])
        assert all(np.array_equal(a, b[:rows]) for a, b in zip(got, want)), rows


def test_rows_past_2_to_the_31_elements(lib):
    V, stride = 1000, 1 << 20
    rows = 2200  # 2.3e9 elements apart
    x = torch.zeros(rows, stride, dtype=torch.bfloat16, device="cuda")
    x[-1, :V] = torch.randn(V, device="cuda")
    x[-1, V:] = INF
    tok, lp, kept = call(lib, x, u=0.37, vocab=V, stride=stride)
    alone = call(lib, x[-1:, :V].contiguous(), u=0.37)
    assert tok[-1] == alone[0][0] and lp[-1] == alone[1][0] and kept[-1] == V and np.all(tok[:-1] == 370)


@pytest.mark.parametrize("rows", [3, 300])
def test_captured_and_replayed(lib, rows):
    V = 3001
    x = torch.zeros(rows, V, device="cuda")
    par = [torch.ones(rows, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.ones(rows, device="cuda"),
           torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")]
    tok, kept, lp = (torch.zeros(rows, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32))
    ws = torch.empty(lib.sidp_sample_tokens_bytes(rows, V), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        lib.sidp_sample_tokens(x, 1, rows, V, V, *par, tok, lp, kept, ws, ws.numel(), torch.cuda.current_stream())
    rng = np.random.default_rng(1)
    for _ in range(5):
        new = settings(rng, rows, V)
        x.copy_(torch.randn(rows, V, device="cuda") * 2)
        for a, b in zip(par, new):
            a.copy_(torch.tensor(b))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        want = call(lib, x, *new)
        for a, b in zip((tok, lp, kept), want):
            assert np.array_equal(a.cpu().numpy(), b)


def test_two_streams(lib):
    rng = np.random.default_rng(9)
    xs = [torch.tensor(rng.standard_normal((r, 40000)), dtype=torch.float32).cuda() for r in (5, 280)]
    sets = [settings(rng, len(x), 40000) for x in xs]
    want = [call(lib, x, *s) for x, s in zip(xs, sets)]
    streams = [torch.cuda.Stream() for _ in xs]
    held, outs = [], []
    for _ in range(3):
        for x, s, st in zip(xs, sets, streams):
            n = len(x)
            par = [torch.tensor(np.asarray(v, np.int32 if i == 1 else np.float32)).cuda() for i, v in enumerate(s)]
            o = [torch.zeros(n, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32)]
            ws = torch.empty(lib.sidp_sample_tokens_bytes(n, 40000), dtype=torch.uint8, device="cuda")
            held.append((par, o, ws, st, x))
            outs.append(o)
    torch.cuda.synchronize()
    for par, o, ws, st, x in held:
        lib.sidp_sample_tokens(x, 1, len(x), 40000, 40000, *par, o[0], o[1], o[2], ws, ws.numel(), st)
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        for a, b in zip(o, want[i % 2]):
            assert np.array_equal(a.cpu().numpy(), b)
