"""Attention of sequences of which groups share their first blocks, over both
caches, against softmax(q K^T / sqrt(D)) V of each sequence in float64."""

import numpy as np
import pytest
import torch

from gpu_helpers import kernels_of
from parts_helpers import Parts, close
from rows_helpers import BS, Handle, cfg_of, dev

pytestmark = pytest.mark.gpu

CACHES = ["bf16", "e4m3", "int8"]
CASES = {
    # (groups, lens): groups of (sequences, shared tokens), then (cached, new) of every sequence
    "one group": ([(6, 256)], [(256 + 13 * i, 1) for i in range(6)]),
    "nothing behind it": ([(5, 320)], [(320, 1)] * 5),
    "drafts of unlike length": ([(7, 192)], [(192 + 5 * i, i % 4) for i in range(7)]),
    "many rows": ([(40, 480)], [(480 + 3 * i, 1 + i % 3) for i in range(40)]),
    "two groups and others": ([(4, 160), (3, 640)], [(200, 1), (160, 2), (161, 1), (190, 1), (640, 1), (700, 3), (650, 1),
                                                     (20, 4), (0, 1), (333, 1)]),
    "odd lengths": ([(4, 16 * 13), (9, 16 * 7)], [(16 * 13 + i, 1) for i in range(4)] + [(16 * 7 + 50 * i, 1) for i in range(9)]),
    "ends in a block": ([(3, 200)], [(200, 0), (200, 0), (200, 1)]),
    "a group of one, a group of none": ([(1, 300), (0, 64), (3, 300 - 300 % 16)], [(300, 1)] + [(290, 1), (300, 2), (400, 1)]),
    "long and short rows": ([(5, 512)], [(512, 1), (520, 100), (512, 1), (530, 1), (600, 33)]),
    "short prefixes": ([(8, 32), (8, 96), (8, 112)], [(40 + i, 1) for i in range(8)] + [(96 + i, 2) for i in range(8)] +
                       [(112 + i, 1) for i in range(8)]),
}
HEADS = [(4, 2, 64), (16, 1, 128), (5, 1, 128), (2, 2, 128), (64, 8, 128)]


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("case", list(CASES), ids=str)
def test_shared_attention_matches_the_definition(lib, cache, heads, case):
    groups, lens = CASES[case]
    c = Parts(lib, cache, heads, lens, groups, seed=len(case))
    out = c.run()
    close(out[:c.rows], *c.want(), what=case)
    assert torch.all(out[c.rows:] == 7.0)
    c.close()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads,groups,lens", [
    ((8, 1, 128), [(3, 6000 - 6000 % 16)], [(6000, 4), (6100, 1), (7000, 1)]),
    ((8, 2, 64), [(20, 4096), (2, 2048)], [(4096 + 50 * i, 1) for i in range(20)] + [(3000, 1), (2048, 1)]),
    ((64, 8, 128), [(50, 1024)], [(1024 + 20 * i, 1) for i in range(50)]),
    ((16, 16, 64), [(130, 1600)], [(1600 + i, 1) for i in range(130)]),
    ((8, 8, 128), [(200, 800), (100, 800)], [(800 + i % 50, 1) for i in range(300)])], ids=str)
def test_long_prefixes_and_many_sequences(lib, cache, heads, groups, lens):
    """Shared tiles cut into runs, with as many items as fit the chip and with more."""
    c = Parts(lib, cache, heads, lens, groups, seed=4, regions=1, region=0)
    close(c.run()[:c.rows], *c.want())
    c.close()


@pytest.mark.parametrize("cache", CACHES)
def test_more_tiles_than_the_chip_holds(lib, cache):
    """Prompts beside many single tokens, some of them in groups."""
    rng = np.random.default_rng(3)
    groups = [(30, 256), (50, 512), (1, 64), (200, 128)]
    lens = []
    for n, s in groups:
        lens += [(s + int(rng.integers(0, 40)), int(rng.integers(0, 3))) for _ in range(n)]
    lens += [(int(rng.integers(0, 300)), int(rng.integers(1, 200))) for _ in range(40)]
    c = Parts(lib, cache, (8, 8, 64), lens, groups, seed=8, regions=1, region=0)
    out = c.run()
    close(out[:c.rows], *c.want())
    assert torch.all(out[c.rows:] == 7.0)
    c.close()


@pytest.mark.parametrize("groups,prefix", [(2048, 128), (4096, 16)])
def test_the_most_sequences_and_groups(lib, groups, prefix):
    """4096 sequences in pairs that share, and each a group of its own."""
    rng = np.random.default_rng(groups)
    lens = [(prefix + int(c), int(n)) for c, n in zip(rng.integers(0, 20, 4096), rng.integers(0, 2, 4096))]
    c = Parts(lib, "bf16", (4, 2, 64), lens, [(4096 // groups, prefix)] * groups, seed=1, regions=1, region=0)
    out = c.run()
    close(out[:c.rows], *c.want())
    assert torch.all(out[c.rows:] == 7.0)
    c.close()


@pytest.mark.parametrize("cache", CACHES)
def test_the_prefix_is_read_from_one_table(lib, cache):
    """Every other sequence's table is without the prefix's whole chunks: they are the group's, read once."""
    groups, lens = [(6, 256)], [(256 + 40 * i, 1) for i in range(6)]
    c = Parts(lib, cache, (16, 2, 64), lens, groups, seed=2)
    close(c.run()[:c.rows], *c.want())
    tables = c.tables.copy()
    tables[1:, :256 // BS] = -1
    close(c.run(tables=tables)[:c.rows], *c.want())  # no block is latched either
    c.close()


@pytest.mark.parametrize("cache", CACHES)
def test_without_groups_it_is_the_attention_of_rows(lib, cache):
    lens = [(100, 20), (90, 1), (0, 30), (2000, 1)]
    c = Parts(lib, cache, (8, 2, 128), lens, seed=2)
    out = c.run()
    close(out[:c.rows], *c.want())
    if cache != "bf16":
        assert torch.equal(out, c.run(shared=False))
    # group lengths of nothing: the same bits
    assert torch.equal(out, c.run(gstarts=[0, 2, 4], lens=[0, 0]))
    c.close()


def test_values_that_are_not_finite_reach_the_rows_that_see_them(lib):
    """In the prefix all rows of the group; behind it only the sequence's later ones."""
    groups, lens = [(4, 256)], [(256 + 10 * i, 2) for i in range(4)] + [(100, 1)]
    c = Parts(lib, "bf16", (8, 2, 64), lens, groups, seed=2)
    clean, mag = c.want()
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(clean) * 1.01
    c.kv[2][1][256 + 20 + 1, 0, 5] = float("inf")  # the last token of the third sequence
    c.put(2)
    got = c.run()[:c.rows].double().cpu().numpy()
    hit = np.zeros(got.shape, bool)
    hit[5, :4, 5] = True
    assert np.all(np.isposinf(got[hit])) and np.all(np.abs(got - clean)[~hit] <= tol[~hit])
    c.kv[2][1][256 + 20 + 1, 0, 5] = 1.0
    c.put(2)
    c.kv[0][1][77, 1, 9] = float("nan")
    c.put(0)
    got = c.run()[:c.rows].double().cpu().numpy()
    assert np.isnan(got[:8, 4:, 9]).all() and np.isfinite(got[8]).all() and np.isfinite(got[:, :4]).all()
    c.close()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("what,gstarts,shared", [
    ("order", [0, 5, 3], [256, 256]), ("range", [0, 3, 9], [256, 256]), ("negative start", [-1, 3, 7], [256, 256]),
    ("negative length", [0, 3, 7], [256, -16]), ("longer than a sequence", [0, 3, 7], [256, 272])])
def test_bad_groups_are_latched_and_rows_stay_right(lib, cache, what, gstarts, shared):
    groups, lens = [(3, 256), (4, 256)], [(256 + 40 * i, 1) for i in range(3)] + [(256 + 8 * i, 2) for i in range(4)]
    c = Parts(lib, cache, (8, 2, 64), lens, groups, seed=6)
    out = c.run(gstarts=gstarts, lens=shared, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    close(out[:c.rows], *c.want(), what=what)
    c.h.sync()
    c.close()


@pytest.mark.parametrize("cache", ["bf16", "int8"])
@pytest.mark.parametrize("what", ["ctx negative", "past the table", "starts past max_rows", "starts fall"])
def test_sequences_that_are_left_out(lib, cache, what):
    groups, lens = [(4, 256)], [(256 + 40 * i, 2) for i in range(4)] + [(100, 10)]
    c = Parts(lib, cache, (8, 2, 64), lens, groups, seed=6)
    ctx, starts, max_rows = [n for n, _ in lens], list(c.starts), None
    if what == "ctx negative":
        ctx[1] = -5
    elif what == "past the table":
        ctx[1] = c.width * BS
    elif what == "starts fall":
        starts[2] = 1
    else:
        max_rows = 9
    out = c.run(ctx=ctx, starts=starts, max_rows=max_rows, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    want, mag = c.want()
    if what == "starts fall":
        return c.close()
    if what == "starts past max_rows":
        close(out[:8], want[:8], mag[:8])
        assert torch.all(out[8:] == 7.0)
    else:
        assert torch.all(out[2:4] == 7.0)
        keep = [0, 1] + list(range(4, 18))
        close(out[keep], want[keep], mag[keep])
    c.close()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_shared_attention_captured_and_replayed(lib, cache):
    """Lengths, groups, tables and queries change between replays; eager calls in between, with a workspace of their own."""
    groups, lens = [(5, 256), (4, 160)], [(256 + 9 * i, 2) for i in range(5)] + [(160 + 9 * i, 1) for i in range(4)]
    c = Parts(lib, cache, (8, 2, 64), lens, groups, seed=3)
    q = torch.zeros(c.rows, 8, 64, dtype=torch.bfloat16, device="cuda")
    starts, ctx, bt, gs, sl = dev(c.starts), dev([n for n, _ in lens]), dev(c.tables), dev(c.gstarts), dev(c.shared)
    out = torch.zeros_like(q)
    ws = torch.empty(c.bytes(c.rows), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        lib.sidp_attention_shared(c.h.h, c.code(), q, 1, gs, sl, 2, starts, ctx, bt, c.width, 9, c.rows, out, ws, ws.numel(),
                                  torch.cuda.current_stream())
    for new, shared in (([2] * 5 + [1] * 4, [256, 160]), ([1] * 9, [128, 0]), ([0, 2, 1, 0, 0, 1, 1, 1, 0], [256, 160]),
                        ([2] * 5 + [1] * 4, [0, 160])):
        st = np.concatenate([[0], np.cumsum(new)])
        starts.copy_(dev(st))
        sl.copy_(dev(shared))
        q.copy_(torch.randn(q.shape, device="cuda"))
        out.fill_(7.0)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        want = c.run(starts=st, lens=shared, q=q.cpu())
        assert torch.equal(out[:st[-1]], want[:st[-1]]) and torch.all(out[st[-1]:] == 7.0)
        lib.sidp_sync(c.h.h)
    c.close()


def test_calls_side_by_side(lib):
    """Both streams busy with calls on one handle, each with a workspace of its own: the bits of calls alone."""
    a = Parts(lib, "bf16", (8, 2, 128), [(700 + i, 1) for i in range(9)], [(9, 640)], seed=1)
    alone = a.run().clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(4):
        outs += [a.run(stream=s, sync=False) for s in streams]
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, alone)
    a.close()


def test_three_launches(lib):
    c = Parts(lib, "bf16", (8, 2, 64), [(300, 1)] * 3, [(3, 288)], seed=1)
    c.run()
    q, out = (torch.zeros(3, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(c.bytes(3), dtype=torch.uint8, device="cuda")
    args = [dev(x) for x in (c.gstarts, c.shared, c.starts, [300] * 3, c.tables)]
    names = kernels_of(lambda: lib.sidp_attention_shared(c.h.h, 0, q, 1, args[0], args[1], 1, args[2], args[3], args[4], c.width, 3, 3, out,
                                                         ws, ws.numel()))
    assert len(names) == 3 and "plan" in names[0] and "join" in names[2], names
    c.close()


def test_refusals(lib):
    c = Parts(lib, "bf16", (4, 2, 64), [(10, 3)])
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    i = dev([0] * 8)
    need = lib.sidp_attention_shared_bytes(c.h.h, 0, 1, 3)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    T, I, W = t.data_ptr(), i.data_ptr(), ws.data_ptr()

    def rc(h=c.h.h, cache=0, q=T, region=0, gs=I, sl=I, groups=1, starts=I, ctx=I, bt=I, width=2, batch=1, rows=3, out=T, w=W, n=need):
        return lib.raw_call("sidp_attention_shared", h, cache, q, region, gs, sl, groups, starts, ctx, bt, width, batch, rows, out, w, n, None)
    E = lib.SIDP_EINVAL
    assert rc(cache=2) == E and rc(cache=-1) == E and rc(groups=-1) == E and rc(groups=2) == E and rc(gs=None) == E and rc(sl=None) == E
    assert rc(rows=0, w=None, n=0) == 0 and rc(gs=None, sl=None, groups=0, rows=0) == 0
    assert rc(batch=0) == E and rc(batch=4097) == E and rc(rows=-1) == E and rc(rows=(1 << 20) + 1) == E
    assert rc(width=0) == E and rc(width=65537) == E and rc(region=2) == E and rc(region=-1) == E
    assert rc(q=None) == E and rc(starts=None) == E and rc(ctx=None) == E and rc(bt=None) == E and rc(out=None) == E
    assert rc(w=None) == E and rc(n=need - 1) == E and rc(w=W + 8) == E and rc(q=T + 2) == E and rc(out=T + 8) == E
    assert rc(h=None) == E and rc(cache=1) == lib.SIDP_ESTATE  # no 8-bit cache attached
    f = lib.sidp_attention_shared_bytes
    assert f(c.h.h, 2, 1, 3) == 0 and f(None, 0, 1, 3) == 0 and f(c.h.h, 0, 0, 3) == 0 and f(c.h.h, 0, 1, 0) == 0
    assert f(c.h.h, 0, 4096, 1 << 20) > 0
    c.h.sync()
    c.close()
    with Handle(lib, cfg_of(1024, 1024, 64), 64) as h:  # 12288 tiles and half as many of groups, 1024 heads: past 2^32 threads
        assert f(h.h, 0, 4096, 1 << 20) == 0 and f(h.h, 0, 4096, 1 << 19) > 0
