"""Log probabilities, ranks, entropy and top alternatives against 64-bit
definitions: sizes around the slices, misaligned rows, ties, masks, rows without
a distribution."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SLICE = 8192


def plain(x, targets, top):
    """x float64 [rows, vocab] (numpy); ties to the lowest token."""
    rows, vocab = x.shape
    lp = np.full(rows, np.nan)
    rank = np.full(rows, -1)
    ent = np.full(rows, np.nan)
    ids = np.full((rows, top), -1)
    lps = np.full((rows, top), np.nan)
    for r in range(rows):
        v = x[r]
        if np.isnan(v).any() or v.max() == np.inf or v.max() == -np.inf:
            continue
        m = v.max()
        with np.errstate(divide="ignore"):
            logp = v - m - np.log(np.exp(v - m).sum())
        p = np.exp(logp)
        ent[r] = -(p[p > 0] * logp[p > 0]).sum()
        order = np.lexsort((np.arange(vocab), -v))[:top]
        ids[r], lps[r] = order, logp[order]
        t = -1 if targets is None else targets[r]
        if 0 <= t < vocab:
            lp[r], rank[r] = logp[t], (v > v[t]).sum()
    return lp, rank, ent, ids, lps


def call(lib, logits, vocab, stride, targets, top, rows=None, offset=0, f32=None, stream=None, graph=None):
    """logits: a flat tensor; row r starts at offset + r * stride."""
    f32 = logits.dtype == torch.float32 if f32 is None else f32
    o = dict(lp=torch.full((rows + 1,), 9.0, device="cuda"), rank=torch.full((rows + 1,), 9, dtype=torch.int32, device="cuda"),
             ent=torch.full((rows + 1,), 9.0, device="cuda"),
             ids=torch.full((rows + 1, top), 9, dtype=torch.int32, device="cuda"),
             lps=torch.full((rows + 1, top), 9.0, device="cuda"))
    ws = torch.empty(lib.sidp_token_logprobs_bytes(rows, vocab, top), dtype=torch.uint8, device="cuda")
    lib.sidp_token_logprobs(logits.data_ptr() + offset * logits.element_size(), lib.SIDP_LOGITS_F32 if f32 else lib.SIDP_LOGITS_BF16,
                            rows, vocab, stride, targets, top, o["lp"], o["rank"], o["ent"], o["ids"], o["lps"], ws,
                            ws.numel(), stream)
    torch.cuda.synchronize()
    for k, v in o.items():
        assert (v[rows:] == 9).all(), k  # nothing behind the last row
    return {k: v[:rows].cpu().numpy() for k, v in o.items()}


def check(o, x, targets, top):
    lp, rank, ent, ids, lps = plain(x, targets, top)
    assert np.array_equal(o["rank"], rank)
    assert np.array_equal(o["ids"], ids)
    # fp32: exponents up to 256 in base 2 rounded once, 2^-24 of their size where the term counts (below 2^5), the sums' few
    # roundings, and the result's own three: 2^-18 absolute at these logits, 2^-21 relative
    for got, want in ((o["lp"], lp), (o["ent"], ent), (o["lps"], lps)):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got == -np.inf, want == -np.inf)
        fine = np.isfinite(want)
        assert np.all(np.abs(got[fine] - want[fine]) <= 2.0 ** -18 + 2.0 ** -21 * np.abs(want[fine]))


def data(rows, n, seed, dtype, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows * n + 64, generator=g) * scale).to(dtype)


def as_rows(flat, rows, vocab, stride, offset=0):
    return np.stack([flat[offset + r * stride:offset + r * stride + vocab].double().numpy() for r in range(rows)])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 1000, SLICE - 1, SLICE, SLICE + 1, 32000, 50001, 151936])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_logprobs_match_the_definition(lib, dtype, vocab, top):
    top = min(top, vocab)
    rows, stride = 3, vocab + 5
    flat = data(rows, stride, vocab + top, dtype)
    x = as_rows(flat, rows, vocab, stride)
    targets = [int(np.argmax(x[0])), vocab - 1, int(np.argmin(x[2]))]
    check(call(lib, flat.cuda(), vocab, stride, torch.tensor(targets, dtype=torch.int32, device="cuda"), top, rows=rows), x,
          targets, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", range(8))
def test_logprobs_of_misaligned_rows(lib, dtype, offset):
    vocab, stride, rows = 2 * SLICE - 3, 2 * SLICE + 1, 4  # each row at another offset again
    flat = data(rows, stride, offset, dtype)
    x = as_rows(flat, rows, vocab, stride, offset)
    targets = [0, vocab - 1, SLICE - offset, 5]
    check(call(lib, flat.cuda(), vocab, stride, torch.tensor(targets, dtype=torch.int32, device="cuda"), 6, rows=rows, offset=offset),
          x, targets, 6)


@pytest.mark.parametrize("vocab", [40, SLICE + 10, 40000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_ties_go_to_the_lowest_token(lib, vocab, dtype):
    """Few distinct values, all equal ones, zeros of both signs, the largest only at the end."""
    g = torch.Generator().manual_seed(vocab)
    rows = [torch.randint(0, 4, (vocab,), generator=g).float(), torch.full((vocab,), 2.5), torch.zeros(vocab),
            torch.arange(vocab).float().div(64).floor(), torch.zeros(vocab)]
    rows[2][::2] = -0.0
    rows[4][-3:] = 1.0
    x = torch.stack(rows).to(dtype)
    targets = [vocab - 1, 3, 1, 0, vocab - 2]
    o = call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 20, rows=5)
    check(o, x.double().numpy(), targets, 20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_under_masks(lib, dtype):
    """Masked by -inf: all but one, all but fewer than asked for, one whole slice, a block of allowed tokens; and masked by the
    type's lowest value."""
    vocab, rows, top = 3 * SLICE + 100, 6, 12
    x = data(rows, vocab, 1, dtype)[:rows * vocab].view(rows, vocab).clone()
    x[0] = -np.inf
    x[0, 20000] = -5.0
    x[1, torch.arange(vocab) % 3000 != 7] = -np.inf
    x[2, :SLICE] = -np.inf
    x[3, :2000] = -np.inf
    x[3, 5000:] = -np.inf
    x[4, torch.arange(vocab) % 2 == 0] = torch.finfo(dtype).min
    targets = [20000, 8, 3, 100, 0, 9]  # masked ones among them
    check(call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), top, rows=rows),
          x.double().numpy(), targets, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [300, SLICE + 500])
def test_logprobs_of_rows_without_a_distribution(lib, dtype, vocab):
    x = data(6, vocab, 2, dtype)[:6 * vocab].view(6, vocab).clone()
    x[0, vocab - 5] = np.nan
    x[1, 17] = np.inf
    x[2] = -np.inf
    x[3, 4], x[3, 200] = np.nan, np.inf
    x[4] = np.nan
    targets = [5, 6, 7, 200, 9, 10]
    check(call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 4, rows=6),
          x.double().numpy(), targets, 4)


def test_logprobs_of_sure_and_of_large_logits(lib):
    """A probability within 1e-7 of one, and logits near +-1e4, where only differences matter."""
    vocab = 20000
    x = data(4, vocab, 3, torch.float32)[:4 * vocab].view(4, vocab).clone()
    x[0, 77] = 40.0
    x[1] += 10000.0
    x[2] -= 10000.0
    x[3] *= 30
    targets = [77, 5, 6, int(x[3].argmax())]
    o = call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 3, rows=4)
    lp, rank, ent, ids, lps = plain(x.double().numpy(), targets, 3)
    assert np.array_equal(o["rank"], rank) and np.array_equal(o["ids"], ids)
    # the differences x - m are rounded to 2^-24 of themselves and log2 e is off by 2^-25.6 of them; where they are past 2^7 the
    # term is 0 and the given token's logprob rounds relative to itself
    for got, want in ((o["lp"], lp), (o["ent"], ent), (o["lps"], lps)):
        assert np.all(np.abs(got - want) <= 2.0 ** -17 + 2.0 ** -20 * np.abs(want))


def test_logprobs_entropy_beside_a_likely_token(lib):
    """A token of a fifth to four fifths of the probability among many unlikely ones, at every place of a lane's share: its weight
    may not swamp the others' in the entropy's sum."""
    vocab, rows = 128001, 24
    x = data(rows, vocab, 8, torch.float32, scale=2.0)[:rows * vocab].view(rows, vocab).clone()
    targets = [(r * 5333 + 17) % vocab for r in range(rows)]
    for r, t in enumerate(targets):
        x[r, t] = 13.0 + r / 8
    o = call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 2, rows=rows)
    lp, rank, ent, ids, lps = plain(x.double().numpy(), targets, 2)
    assert np.array_equal(o["rank"], rank) and np.array_equal(o["ids"], ids)
    # a lane adds 502 terms, each rounded to 2^-24 of a sum of at most 1 + 10: sqrt(502) * 11 * 2^-24 = 2^-15.9 if they all went to
    # one lane's sums; 256 lanes share them
    for got, want in ((o["lp"], lp), (o["ent"], ent), (o["lps"], lps)):
        assert np.max(np.abs(got - want)) <= 2.0 ** -16


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_rows_at_the_lowest_value(lib, dtype):
    """Every token at the type's lowest value is an even choice; next to it, the largest value takes all."""
    vocab = SLICE + 40
    x = torch.full((2, vocab), torch.finfo(dtype).min, dtype=dtype)
    x[1, 9000 % vocab] = 5.0
    targets = [4, 9000 % vocab]
    check(call(lib, x.flatten().cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 1, rows=2),
          x.double().numpy(), targets, 1)


def test_logprobs_targets_outside_and_missing_outputs(lib):
    vocab, rows = 1000, 5
    flat = data(rows, vocab, 4, torch.float32)
    x = as_rows(flat, rows, vocab, vocab)
    targets = [-1, vocab, 2147483647, -2147483648, 3]
    check(call(lib, flat.cuda(), vocab, vocab, torch.tensor(targets, dtype=torch.int32, device="cuda"), 2, rows=rows), x, targets, 2)
    check(call(lib, flat.cuda(), vocab, vocab, None, 2, rows=rows), x, None, 2)
    ws = torch.empty(lib.sidp_token_logprobs_bytes(rows, vocab, 0), dtype=torch.uint8, device="cuda")
    ent = torch.zeros(rows, device="cuda")
    lib.sidp_token_logprobs(flat.cuda(), 1, rows, vocab, vocab, None, 0, None, None, ent, None, None, ws, ws.numel())
    torch.cuda.synchronize()
    assert np.allclose(ent.cpu().numpy(), plain(x, None, 0)[2], atol=2.0 ** -18)


def test_logprobs_rows_past_32_bits(lib):
    """The last rows of logits that lie past 2^32 bytes."""
    vocab, stride, rows = 1000, 1 << 20, 2060
    flat = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    tail = torch.randn(vocab, generator=g, device="cuda").to(torch.bfloat16)
    flat[(rows - 1) * stride:(rows - 1) * stride + vocab] = tail
    o = call(lib, flat, vocab, stride, torch.full((rows,), 3, dtype=torch.int32, device="cuda"), 3, rows=rows)
    x = np.zeros((2, vocab))
    x[1] = tail.double().cpu().numpy()
    check({k: v[-2:] for k, v in o.items()}, x, [3, 3], 3)


@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 64001), (torch.float32, 32003)])
def test_logprobs_of_large_calls_are_those_of_small_ones(lib, dtype, vocab):
    """More logits than the caches hold, in one call and in two: the same bits, and some of the rows by their definition."""
    rows, top = 1200, 7
    g = torch.Generator(device="cuda").manual_seed(12)
    flat = (torch.randn(rows * vocab, generator=g, device="cuda") * 3).to(dtype)
    flat[5 * vocab:6 * vocab:2] = -torch.inf
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    whole = call(lib, flat, vocab, vocab, targets, top, rows=rows)
    for a in (0, rows // 2):
        part = call(lib, flat, vocab, vocab, targets[a:a + rows // 2], top, rows=rows // 2, offset=a * vocab)
        assert all(np.array_equal(part[k], whole[k][a:a + rows // 2], equal_nan=True) for k in whole)
    for r in (0, 5, rows - 1):
        x = flat[r * vocab:(r + 1) * vocab].double().cpu().numpy()[None]
        check({k: v[r:r + 1] for k, v in whole.items()}, x, [int(targets[r])], top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,stride", [(171, 8193, 8193), (300, 20011, 20024), (511, 9000, 9001)])
@pytest.mark.parametrize("top", [0, 1, 32])
def test_logprobs_of_hundreds_of_rows(lib, dtype, rows, vocab, stride, top):
    """Rows that nearly fill the chip, among them masked, equal, rising and odd ones."""
    flat = data(rows, stride, rows + top, dtype)
    for r, what in enumerate((-torch.inf, 0.0, torch.finfo(dtype).min)):
        flat[r * stride:r * stride + vocab] = what
    flat[2 * stride + 77] = 1.0
    flat[3 * stride:3 * stride + vocab] = torch.linspace(-20, 20, vocab).to(dtype)
    flat[4 * stride:4 * stride + vocab - 3] = -torch.inf
    flat[5 * stride + vocab - 1], flat[6 * stride + 5] = torch.nan, torch.inf
    targets = [(r * 37) % (vocab + 2) for r in range(rows)]
    o = call(lib, flat.cuda(), vocab, stride, torch.tensor(targets, dtype=torch.int32, device="cuda"), top, rows=rows)
    check(o, as_rows(flat, rows, vocab, stride), targets, top)


def test_logprobs_largest_vocabulary(lib):
    vocab = 1 << 20
    flat = data(1, vocab, 6, torch.bfloat16)
    x = as_rows(flat, 1, vocab, vocab)
    check(call(lib, flat.cuda(), vocab, vocab, torch.tensor([vocab - 1], dtype=torch.int32, device="cuda"), 32, rows=1), x,
          [vocab - 1], 32)


def test_logprobs_give_the_same_bits_again_and_captured(lib):
    vocab, rows, top = 30000, 9, 20
    flat = data(rows, vocab, 7, torch.bfloat16).cuda()
    targets = torch.arange(rows, dtype=torch.int32, device="cuda")
    first = call(lib, flat, vocab, vocab, targets, top, rows=rows)
    second = call(lib, flat, vocab, vocab, targets, top, rows=rows)
    assert all(np.array_equal(first[k], second[k]) for k in first)
    out = dict(lp=torch.zeros(rows, device="cuda"), rank=torch.zeros(rows, dtype=torch.int32, device="cuda"),
               ent=torch.zeros(rows, device="cuda"), ids=torch.zeros(rows, top, dtype=torch.int32, device="cuda"),
               lps=torch.zeros(rows, top, device="cuda"))
    ws = torch.empty(lib.sidp_token_logprobs_bytes(rows, vocab, top), dtype=torch.uint8, device="cuda")
    x = flat.clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.sidp_token_logprobs(x, 0, rows, vocab, vocab, targets, top, out["lp"], out["rank"], out["ent"], out["ids"], out["lps"],
                                ws, ws.numel(), torch.cuda.current_stream())
    for i in range(4):
        x.copy_(flat if i % 2 == 0 else flat.flip(0))
        ws.fill_(255)  # nothing in the workspace outlives a call
        g.replay()
        torch.cuda.synchronize()
        want = call(lib, x, vocab, vocab, targets, top, rows=rows)
        assert all(np.array_equal(out[k].cpu().numpy(), want[k]) for k in out)
