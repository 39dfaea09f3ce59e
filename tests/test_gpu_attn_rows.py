"""Causal attention of several new tokens a sequence over the paged cache, against
softmax(q K^T / sqrt(D)) V in float64. Whatever a call may not see is NaN: blocks of
nobody, and the places behind a sequence's last token."""

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from rows_helpers import BS, Handle, cfg_of, dev

pytestmark = pytest.mark.gpu


class Case:
    """Sequences of (cached, new) tokens in scattered blocks; keys and values are random, the rest of the cache NaN."""

    def __init__(self, lib, heads, lens, seed=0, regions=2, region=1, extra_blocks=3, nblk=None, q_std=1.5, max_seq=None, fill=float("nan"),
                 place=None):
        hq, hkv, D = heads
        self.lib, self.lens, self.region, self.in_use = lib, lens, region, []
        self.hq, self.hkv, self.D = hq, hkv, D
        need = [-(-(c + n) // BS) for c, n in lens]
        self.nblk = nblk or sum(need) + extra_blocks
        self.width = min(max(max(need), 1) + 1, 1 << 16)
        self.h = Handle(lib, cfg_of(hq, hkv, D), max_seq or max(64, max(c + n for c, n in lens)), self.nblk, regions, fill=fill)
        rng = np.random.default_rng(seed)
        blocks = (rng.permutation(self.nblk) if place is None else np.asarray(place)).tolist()
        self.tables = np.full((len(lens), self.width), -1)
        g = torch.Generator().manual_seed(seed)
        self.rows = sum(n for _, n in lens)
        self.kv = []
        for b, (c, n) in enumerate(lens):
            self.tables[b, :need[b]] = [blocks.pop() for _ in range(need[b])]
            k, v = (torch.randn(c + n, hkv, D, generator=g).to(torch.bfloat16) for _ in range(2))
            self.kv.append([k, v])
            self.put(b)
        self.q = (q_std * torch.randn(self.rows, hq, D, generator=g)).to(torch.bfloat16)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in lens])])

    def put(self, b):
        """Sequence b's keys and values into its blocks."""
        k, v = self.kv[b]
        t = torch.arange(len(k))
        blk = torch.as_tensor(self.tables[b])[t // BS].cuda()
        off = (t % BS).cuda()
        self.h.k[self.region][blk, :, :, off, :] = k.cuda().reshape(len(k), self.hkv, self.D // 8, 8)
        self.h.v[self.region][blk, :, :, off] = v.cuda()

    def run(self, max_rows=None, starts=None, ctx=None, tables=None, out=None, stream=None, sync=True):
        max_rows = self.rows if max_rows is None else max_rows
        q = torch.zeros(max(max_rows, self.rows) + 1, self.hq, self.D, dtype=torch.bfloat16, device="cuda")
        q[:self.rows] = self.q.cuda()
        out = torch.full((max(max_rows, self.rows) + 1, self.hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        ws = torch.full((max(1, self.lib.sidp_attention_rows_bytes(self.h.h, len(self.lens), max_rows)),), 255, dtype=torch.uint8,
                        device="cuda")
        starts = dev(self.starts if starts is None else starts)
        ctx = dev([c for c, _ in self.lens] if ctx is None else ctx)
        tables = dev(self.tables if tables is None else tables)
        torch.cuda.synchronize()
        self.lib.sidp_attention_rows(self.h.h, q, self.region, starts, ctx, tables, self.width, len(self.lens), max_rows, out, ws,
                                     ws.numel(), stream)
        # a call on a stream that torch does not know of reads these until it is waited for
        self.in_use.append((q, ws, starts, ctx, tables, out))
        if sync:
            self.h.sync()
            self.in_use.clear()
        return out

    def want(self):
        """(output, sum of p |v|) per row in float64."""
        out = np.zeros((self.rows, self.hq, self.D))
        mag = np.zeros_like(out)
        G, q = self.hq // self.hkv, f64(self.q)
        for b, (c, n) in enumerate(self.lens):
            if n == 0:
                continue
            k, v = f64(self.kv[b][0]), f64(self.kv[b][1])
            for h in range(self.hq):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = q[self.starts[b]:self.starts[b] + n, h] @ k[:, h // G].T / np.sqrt(self.D)
                    s = np.where(np.arange(c + n)[None] <= c + np.arange(n)[:, None], s, -np.inf)
                    p = np.exp(s - s.max(1, keepdims=True))
                    p /= p.sum(1, keepdims=True)
                    for i in range(n):  # only what the row sees: 0 * NaN is no part of the definition
                        vi = v[:c + i + 1, h // G]
                        out[self.starts[b] + i, h] = p[i, :c + i + 1] @ vi
                        mag[self.starts[b] + i, h] = p[i, :c + i + 1] @ np.abs(vi)
        return out, mag


def close(got, want, mag, what=""):
    """bf16 has 8 bits, so rounding to it is off by at most half of 2^-7, 2^-8 relative: of each probability (and 2^-12 of the
    sum for the fp32 exponents and sums), and once more of the result."""
    got = f64(got)
    assert np.all(np.isfinite(got)), what
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want) * 1.01
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.max(np.abs(got - want) / tol):.3g} of the tolerance"


HEADS = [(4, 2, 64), (8, 1, 64), (16, 1, 128), (5, 1, 128), (3, 3, 128), (64, 8, 128)]
LENS = {
    "one token each": [(0, 1), (5, 1), (15, 1), (16, 1), (63, 1), (64, 1), (200, 1)],
    "a few each": [(0, 2), (15, 3), (60, 8), (100, 5), (1000, 4)],
    "ragged": [(0, 5), (16, 16), (17, 100), (300, 33), (50, 0), (0, 129), (64, 64), (0, 0), (1, 63)],
    "one prompt": [(0, 333)],
    "one long chunk": [(777, 260)],
}


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", list(LENS), ids=str)
def test_attention_rows_match_the_definition(lib, heads, lens):
    c = Case(lib, heads, LENS[lens], seed=len(lens))
    out = c.run()
    close(out[:c.rows], *c.want(), what=lens)
    assert torch.all(out[c.rows:] == 7.0)
    c.h.close()


@pytest.mark.parametrize("heads,lens", [((8, 1, 128), [(6000, 4)]), ((8, 2, 64), [(3000, 1), (4095, 40), (10, 2), (64, 1)]),
                                        ((16, 1, 128), [(511, 1), (512, 1), (513, 1), (1024, 3), (0, 1), (1535, 1)]),
                                        ((4, 4, 64), [(2500, 700)])], ids=str)
def test_attention_rows_over_long_caches(lib, heads, lens):
    """Few rows and many keys: sequences are cut into runs and joined."""
    c = Case(lib, heads, lens, seed=5)
    close(c.run()[:c.rows], *c.want())
    c.h.close()


@pytest.mark.parametrize("lens", [[((1 << 20) - 3, 3)], [((1 << 20) - 1, 1)] + [(3, 1)] * 600], ids=["cut", "whole"])
def test_attention_rows_over_the_longest_cache(lib, lens):
    c = Case(lib, (1, 1, 64), lens, seed=6, regions=1, region=0)
    close(c.run()[:c.rows], *c.want())
    c.h.close()


@pytest.mark.parametrize("batch", [300, 1100, 4096])
def test_attention_rows_of_many_sequences(lib, batch):
    rng = np.random.default_rng(batch)
    lens = [(int(c), int(n)) for c, n in zip(rng.integers(0, 40, batch), rng.integers(0, 4, batch))]
    c = Case(lib, (4, 2, 64), lens, seed=2)
    close(c.run()[:c.rows], *c.want())
    c.h.close()


@pytest.mark.parametrize("max_rows", [1, 17, 400])
def test_attention_rows_behind_the_last_one_stay(lib, max_rows):
    """max_rows is a bound, the rows in use are row_starts' own."""
    lens = [(30, 5), (0, 12)] if max_rows > 1 else [(30, 1), (4, 0)]
    c = Case(lib, (8, 2, 64), lens)
    out = c.run(max_rows=max_rows)
    close(out[:c.rows], *c.want())
    assert torch.all(out[c.rows:] == 7.0)
    c.h.close()


def test_attention_rows_without_rows(lib):
    c = Case(lib, (4, 2, 64), [(10, 0), (0, 0)])
    out = c.run(max_rows=64)
    assert torch.all(out == 7.0)
    assert lib.sidp_attention_rows_bytes(c.h.h, 2, 0) == 0
    lib.sidp_attention_rows(c.h.h, out, 1, dev([0, 0, 0]), dev([10, 0]), dev(c.tables), c.width, 2, 0, out, None, 0)
    c.h.sync()
    c.h.close()


@pytest.mark.parametrize("heads", [(8, 1, 128), (4, 2, 64), (2, 2, 64)], ids=str)
@pytest.mark.parametrize("lens", [[(70, 90)], [(3, 4)], [(4000, 5)]], ids=str)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite_stay_out_of_rows_that_do_not_see_them(lib, heads, lens, value):
    """A later row's value (and key) in the same chunk: the rows before it are untouched, it and those behind it show it."""
    c = Case(lib, heads, lens)
    ctx, n = lens[0]
    clean, clean_mag = c.want()
    at = ctx + n // 2
    k, v = c.kv[0]
    v[at, :, 3], v[at, :, 40] = value, value
    v[ctx + n - 1, 0, 17] = -value
    c.put(0)
    out = c.run()[:c.rows]
    want, _ = c.want()
    touched = ~np.isfinite(want)
    assert touched.any() and not touched[:n // 2].any()
    got = f64(out)
    assert np.array_equal(np.isnan(got[touched]), np.isnan(want[touched]))
    inf = touched & ~np.isnan(want)
    assert np.array_equal(got[inf], want[inf])
    # the tolerance's magnitudes from the clean run: only the touched dims changed
    tol = (2.0 ** -8 + 2.0 ** -12) * clean_mag + 2.0 ** -8 * np.abs(clean) * 1.01
    assert np.all(np.abs(got - clean)[~touched] <= tol[~touched])
    # a key that is not a number reaches the rows that see it, whole
    k[at] = float("nan")
    v[at], v[ctx + n - 1, 0, 17] = 1.0, 1.0
    c.put(0)
    got = f64(c.run()[:c.rows])
    assert np.isnan(got[n // 2:]).all() and np.isfinite(got[:n // 2]).all()
    c.h.close()


def test_attention_rows_with_a_sharp_softmax(lib):
    """Scores of hundreds that rise and fall along the keys: the running reference moves up, and terms vanish."""
    c = Case(lib, (8, 2, 64), [(500, 70), (0, 90)], q_std=60.0)
    close(c.run()[:c.rows], *c.want())
    c.h.close()


@pytest.mark.parametrize("bad", [-1, "past"])
def test_attention_rows_bad_blocks_are_latched_and_stay_in_their_sequence(lib, bad):
    c = Case(lib, (8, 2, 64), [(100, 20), (90, 30), (0, 10)])
    tables = c.tables.copy()
    tables[1, 2] = c.nblk if bad == "past" else -1
    out = c.run(tables=tables, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    want, mag = c.want()
    for lo, hi in ((0, 20), (50, 60)):
        close(out[lo:hi], want[lo:hi], mag[lo:hi])
    c.h.close()


@pytest.mark.parametrize("what", ["ctx negative", "past the table", "past max_seq_len", "starts fall", "starts past max_rows"])
def test_attention_rows_bad_lengths_leave_the_others(lib, what):
    lens = [(100, 20), (90, 30), (0, 10)]
    c = Case(lib, (8, 2, 64), lens, max_seq=200)
    ctx, starts, max_rows = [100, 90, 0], list(c.starts), None
    if what == "ctx negative":
        ctx[1] = -5
    elif what == "past the table":
        ctx[1] = c.width * BS - 29
    elif what == "past max_seq_len":
        ctx[1] = 171
        c.tables = np.concatenate([c.tables, np.full((3, 8), -1)], 1)
        c.width += 8
    elif what == "starts fall":
        starts[1:] = [50, 20, 60]  # the second sequence ends before it starts; the third has rows 20..59
        ctx = [70, 0, 0]
    else:
        max_rows = 55
    out = c.run(ctx=ctx, starts=starts, max_rows=max_rows, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    want, mag = c.want()
    if what == "starts fall":
        return c.h.close()  # in bounds and latched is all that is asked
    close(out[:20], want[:20], mag[:20])
    if what == "starts past max_rows":
        close(out[20:50], want[20:50], mag[20:50])
        assert torch.all(out[50:] == 7.0)
    else:
        assert torch.all(out[20:50] == 7.0)
        close(out[50:60], want[50:60], mag[50:60])
    c.h.close()


def test_attention_rows_in_caches_past_32_bits(lib):
    """Blocks whose bytes and whose elements lie past 2^32."""
    nblk = (1 << 33) // (2 * 64 * BS * 2) // 2 + 4000  # K of 2 heads of 64: 4 KB a block, past 4 GB
    place = list(range(nblk - 20, nblk)) + [0, 1]
    c = Case(lib, (4, 2, 64), [(100, 30), (0, 20)], nblk=nblk, regions=1, region=0, place=place, fill=0.0)
    close(c.run()[:c.rows], *c.want())
    c.h.close()


def test_one_new_token_agrees_with_the_decode_attention(lib):
    lens = [(0, 1), (100, 1), (777, 1), (31, 1)]
    c = Case(lib, (64, 8, 128), lens, max_seq=1024)
    rows = c.run()[:4]
    lib.sidp_destroy(c.h.h)
    c.h.h = lib.sidp_create(lib.make_config(c.h.cfg, 4, 1024))
    lib.sidp_kv_attach(c.h.h, c.h.k, c.h.v, c.nblk, 2)
    out = torch.zeros(4, 64, 128, dtype=torch.bfloat16, device="cuda")
    lib.sidp_attention(c.h.h, c.q.cuda(), 1, dev([n for n, _ in lens]), dev(c.tables), c.width, 4, out)
    c.h.sync()
    want, mag = c.want()
    close(rows, want, mag)
    close(out, want, mag)
    c.h.close()


def test_attention_rows_on_two_streams_and_again(lib):
    """Calls that overlap, each with a workspace of its own, give the bits of calls alone."""
    a = Case(lib, (8, 2, 128), [(700, 50), (3, 90)], seed=1)
    b = Case(lib, (8, 2, 128), [(2500, 4)], seed=2)
    alone = [x.run().clone() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        outs = [x.run(stream=s, sync=False) for x, s in zip((a, b), streams)]
        torch.cuda.synchronize()
        for x, y in zip(outs, alone):
            assert torch.equal(x, y)
    a.h.close()
    b.h.close()


def test_attention_rows_captured_and_replayed(lib):
    """Lengths, tables and queries change between replays, up to the captured bounds; eager calls in between."""
    c = Case(lib, (8, 2, 64), [(300, 40), (20, 3), (0, 21)], seed=3)
    q = torch.zeros(c.rows, 8, 64, dtype=torch.bfloat16, device="cuda")
    starts, ctx, bt = dev(c.starts), dev([n for n, _ in c.lens]), dev(c.tables)
    out = torch.zeros_like(q)
    ws = torch.empty(lib.sidp_attention_rows_bytes(c.h.h, 3, c.rows), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        lib.sidp_attention_rows(c.h.h, q, 1, starts, ctx, bt, c.width, 3, c.rows, out, ws, ws.numel(), torch.cuda.current_stream())
    for new in ([40, 3, 21], [1, 1, 1], [0, 3, 9], [40, 3, 21]):
        st = np.concatenate([[0], np.cumsum(new)])
        starts.copy_(dev(st))
        q.copy_(torch.randn(q.shape, device="cuda"))
        out.fill_(7.0)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        c.q = q.cpu()
        assert torch.equal(out[:st[-1]], c.run(starts=st)[:st[-1]]) and torch.all(out[st[-1]:] == 7.0)
    c.h.close()


def test_attention_rows_refusals(lib):
    c = Case(lib, (4, 2, 64), [(10, 3)])
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    i = dev([0] * 8)
    need = lib.sidp_attention_rows_bytes(c.h.h, 1, 3)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    T, I, W = t.data_ptr(), i.data_ptr(), ws.data_ptr()

    def rc(h=c.h.h, q=T, region=0, starts=I, ctx=I, bt=I, width=2, batch=1, rows=3, out=T, w=W, n=need):
        return lib.raw_call("sidp_attention_rows", h, q, region, starts, ctx, bt, width, batch, rows, out, w, n, None)
    E = lib.SIDP_EINVAL
    assert rc(batch=0) == E and rc(batch=4097) == E and rc(rows=-1) == E and rc(rows=(1 << 20) + 1) == E
    assert rc(width=0) == E and rc(width=65537) == E and rc(region=2) == E and rc(region=-1) == E
    assert rc(q=None) == E and rc(starts=None) == E and rc(ctx=None) == E and rc(bt=None) == E and rc(out=None) == E
    assert rc(w=None) == E and rc(n=need - 1) == E and rc(w=W + 8) == E and rc(q=T + 2) == E and rc(out=T + 8) == E
    assert lib.raw_call("sidp_attention_rows", None, T, 0, I, I, I, 2, 1, 3, T, W, need, None) == E
    c.h.sync()
    assert lib.sidp_attention_rows_bytes(c.h.h, 4096, 1 << 20) > 0
    c.h.close()
    with Handle(lib, cfg_of(4, 2, 64), 64) as h:
        assert rc(h=h.h) == lib.SIDP_ESTATE  # no cache attached
