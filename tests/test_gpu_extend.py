"""Block tables, row starts, positions and slots made on the GPU from request
lengths, against a plain loop over the sequences."""

import numpy as np
import pytest
import torch

from rows_helpers import Handle, cfg_of, dev

pytestmark = pytest.mark.gpu


def plain(ctx, new, free, taken, tables, nblk, max_rows):
    """(tables, row_starts, positions, slots, taken) by a loop; sequences are served until the first that does not fit."""
    tables, starts, positions, slots = [list(r) for r in tables], [0], [], []
    ended, width, blocks, rows = False, len(tables[0]), 0, 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        ok = c >= 0 and n >= 0 and c + n <= 16 * width
        if ok and n > 0 and not ended:
            have, need = -(-c // 16), -(-(c + n) // 16)
            ended = blocks + need - have > len(free) - taken or rows + n > max_rows
            if not ended:
                for j in range(have, need):
                    tables[b][j] = free[taken + blocks + j - have] if 0 <= free[taken + blocks + j - have] < nblk else -1
                blocks += need - have
                rows += n
                for p in range(c, c + n):
                    blk = tables[b][p // 16]
                    positions.append(p)
                    slots.append(blk * 16 + p % 16 if 0 <= blk < nblk else -1)
        starts.append(len(positions))
    return tables, starts, positions, slots, taken + blocks


def requests(ctx, width, nblk, seed, spare=7):
    """Tables holding the cached tokens' blocks, and the other blocks as the free list."""
    rng = np.random.default_rng(seed)
    perm = rng.permutation(nblk).tolist()
    tables = []
    for c in ctx:
        n = -(-max(0, c) // 16)
        tables.append([perm.pop() for _ in range(min(n, width))] + [-1] * (width - min(n, width)))
    return tables, perm


def call(lib, h, ctx, new, free, taken, tables, max_rows, in_place=False, stream=None):
    t = dict(ctx=dev(ctx), new=dev(new), free=dev(free if free else [0]), taken=dev([taken]), tables=dev(tables),
             starts=torch.full((len(ctx) + 2,), -99, dtype=torch.int32, device="cuda"),
             pos=torch.full((max_rows + 3,), -99, dtype=torch.int32, device="cuda"),
             slots=torch.full((max_rows + 3,), -99, dtype=torch.int32, device="cuda"))
    t["out"] = t["taken"] if in_place else torch.full((2,), -99, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    lib.sidp_kv_extend(h, t["ctx"], t["new"], len(ctx), t["free"], len(free), t["taken"], t["out"], t["tables"],
                       len(tables[0]), max_rows, t["starts"], t["pos"], t["slots"], stream)
    torch.cuda.synchronize()
    return t


def check(t, want, batch):
    tables, starts, positions, slots, taken = want
    n = len(positions)
    assert t["starts"].tolist() == starts + [-99]
    assert t["pos"].tolist()[:n] == positions and t["slots"].tolist()[:n] == slots
    assert set(t["pos"].tolist()[n:]) <= {-99} and set(t["slots"].tolist()[n:]) <= {-99}  # rows behind the last
    assert t["tables"].tolist() == tables
    assert t["out"].tolist()[0] == taken


@pytest.fixture(scope="module")
def handle(lib):
    with Handle(lib, cfg_of(2, 1, 64), 64) as h:
        yield h


@pytest.mark.parametrize("batch,ctx_hi,new_hi", [(1, 0, 1), (1, 100, 1), (1, 0, 3000), (3, 40, 33), (64, 300, 1), (255, 50, 40),
                                                (256, 1000, 2), (257, 64, 70), (1000, 40, 20), (4096, 64, 9)])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_matches_the_loop(lib, handle, batch, ctx_hi, new_hi, in_place):
    rng = np.random.default_rng(batch + new_hi)
    ctx = rng.integers(0, ctx_hi + 1, batch).tolist()
    new = rng.integers(0, new_hi + 1, batch).tolist()
    if batch == 1:
        new = [new_hi]
    width = -(-(ctx_hi + new_hi) // 16) + 1
    nblk = sum(-(-(c + n) // 16) for c, n in zip(ctx, new)) + 11
    tables, free = requests(ctx, width, nblk, batch)
    rows = sum(new)
    for max_rows in (rows, rows + 300):
        t = call(lib, handle.h, ctx, new, free, 2, tables, max_rows, in_place)
        handle.sync()
        check(t, plain(ctx, new, free, 2, tables, nblk, max_rows), batch)


def test_extend_at_block_borders(lib, handle):
    ctx = [0, 0, 0, 15, 15, 16, 16, 17, 31, 32, 5, 0]
    new = [0, 16, 17, 1, 2, 1, 16, 15, 1, 0, 0, 1]
    tables, free = requests(ctx, 4, 60, 1)
    t = call(lib, handle.h, ctx, new, free, 0, tables, sum(new))
    handle.sync()
    check(t, plain(ctx, new, free, 0, tables, 60, sum(new)), len(ctx))


@pytest.mark.parametrize("short", [0, 1, 2, 5, 17])
def test_extend_out_of_blocks_serves_those_before(lib, handle, short):
    ctx, new = [30, 0, 16, 10, 64, 3, 0, 31], [40, 33, 0, 100, 64, 5, 1, 1]  # 3, 3, 0, 6, 4, 0, 1, 0 blocks
    tables, free = requests(ctx, 12, 80, 4)
    free = free[:2 + 17 - short]
    t = call(lib, handle.h, ctx, new, free, 2, tables, 400)
    if short:
        with pytest.raises(lib.SidpError) as e:
            handle.sync()
        assert e.value.code == lib.SIDP_ENOBLOCKS
    handle.sync()
    check(t, plain(ctx, new, free, 2, tables, 80, 400), len(ctx))


@pytest.mark.parametrize("max_rows", [0, 1, 39, 40, 41, 100])
def test_extend_out_of_rows_serves_those_before(lib, handle, max_rows):
    ctx, new = [30, 0, 16], [40, 0, 60]
    tables, free = requests(ctx, 12, 80, 5)
    t = call(lib, handle.h, ctx, new, free, 0, tables, max_rows)
    if max_rows < 100:
        with pytest.raises(lib.SidpError) as e:
            handle.sync()
        assert e.value.code == lib.SIDP_EINVAL
    handle.sync()
    check(t, plain(ctx, new, free, 0, tables, 80, max_rows), len(ctx))


@pytest.mark.parametrize("in_place", [False, True])
def test_extend_lengths_that_sum_past_32_bits(lib, handle, in_place):
    """The most sequences of the most tokens, 2^32 in all, behind one that fits."""
    batch, width = lib.SIDP_EXTEND_MAX_BATCH, 65536
    i32 = dict(dtype=torch.int32, device="cuda")
    ctx, new = torch.zeros(batch, **i32), torch.full((batch,), 16 * width, **i32)
    new[0] = 21
    tables = torch.full((batch, width), -1, **i32)
    starts, pos, slots = torch.full((batch + 2,), -99, **i32), torch.full((100,), -99, **i32), torch.full((100,), -99, **i32)
    taken = dev([1])
    out = taken if in_place else dev([-99])
    lib.sidp_kv_extend(handle.h, ctx, new, batch, dev([3, 5, 7, 9]), 4, taken, out, tables, width, 100, starts, pos, slots)
    with pytest.raises(lib.SidpError) as e:
        handle.sync()
    assert e.value.code == lib.SIDP_EINVAL
    assert starts.tolist() == [0] + [21] * batch + [-99]
    assert pos.tolist() == list(range(21)) + [-99] * 79
    assert slots.tolist() == list(range(80, 96)) + list(range(112, 117)) + [-99] * 79
    assert out.tolist() == [3] and tables[0, :3].tolist() == [5, 7, -1]
    assert int((tables != -1).sum()) == 2


def test_extend_bad_lengths_leave_the_others_served(lib, handle):
    ctx, new = [5, -1, 20, 190, 7, 2147483647, 0], [3, 4, -2, 3, 20, 2147483647, 9]  # 193 tokens: past 12 blocks
    tables, free = requests([5, 0, 20, 190, 7, 0, 0], 12, 80, 6)
    t = call(lib, handle.h, ctx, new, free, 0, tables, 100)
    with pytest.raises(lib.SidpError) as e:
        handle.sync()
    assert e.value.code == lib.SIDP_EINVAL
    check(t, plain(ctx, new, free, 0, tables, 80, 100), len(ctx))


@pytest.mark.parametrize("taken", [-1, 100])
def test_extend_cursor_outside_the_list_hands_out_nothing(lib, handle, taken):
    ctx, new = [8, 16], [8, 1]  # the first needs no block
    tables, free = requests(ctx, 4, 40, 7)
    t = call(lib, handle.h, ctx, new, free, taken, tables, 20)
    with pytest.raises(lib.SidpError):
        handle.sync()
    assert t["starts"].tolist() == [0, 8, 8, -99] and t["tables"].tolist() == tables
    assert t["out"].tolist()[0] == taken


def test_extend_blocks_outside_the_cache_give_no_slot(lib):
    with Handle(lib, cfg_of(2, 1, 64), 64, nblk=20) as handle:
        ctx, new = [20, 5], [40, 3]
        tables, _ = requests(ctx, 5, 20, 8)
        tables[1][0] = 20  # past the cache
        free = [3, -4, 20, 7]
        t = call(lib, handle.h, ctx, new, free, 0, tables, 50)
        with pytest.raises(lib.SidpError) as e:
            handle.sync()
        assert e.value.code == lib.SIDP_EINVAL
        check(t, plain(ctx, new, free, 0, tables, 20, 50), 2)


def test_extend_captured_and_replayed_walks_the_free_list(lib, handle):
    """The cursor in place: every replay hands out the next blocks, eager work in between."""
    ctx0, new = [0, 0, 0], [16, 32, 5]
    tables, free = requests(ctx0, 10, 60, 9)
    s = torch.cuda.Stream()
    ctx, nw, fr, tk, bt = dev(ctx0), dev(new), dev(free), dev([0]), dev(tables)
    starts, pos, slots = dev([0] * 4), dev([0] * 64), dev([0] * 64)

    def go(stream):
        lib.sidp_kv_extend(handle.h, ctx, nw, 3, fr, len(free), tk, tk, bt, 10, 64, starts, pos, slots, stream)

    with torch.cuda.stream(s):
        go(s)
    torch.cuda.synchronize()
    tk.zero_()
    bt.copy_(dev(tables))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        go(torch.cuda.current_stream())
    want_tables, taken, c = tables, 0, list(ctx0)
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        want = plain(c, new, free, taken, want_tables, 60, 64)
        want_tables, taken = want[0], want[4]
        assert bt.tolist() == want_tables and tk.tolist() == [taken]
        assert slots.tolist()[:53] == want[3] and starts.tolist() == want[1]
        c = [a + b for a, b in zip(c, new)]
        ctx += nw
        handle.sync()


def test_extend_refusals(lib, handle):
    t = {k: dev([0] * 8) for k in ("ctx", "new", "free", "taken", "out", "bt", "starts", "pos", "slots")}
    p = {k: v.data_ptr() for k, v in t.items()}

    def rc(batch=1, num_free=1, width=1, max_rows=1, **null):
        a = {k: None if k in null else v for k, v in p.items()}
        return lib.raw_call("sidp_kv_extend", handle.h, a["ctx"], a["new"], batch, a["free"], num_free, a["taken"], a["out"],
                            a["bt"], width, max_rows, a["starts"], a["pos"], a["slots"], None)
    E = lib.SIDP_EINVAL
    assert rc(batch=0) == E and rc(batch=4097) == E and rc(num_free=-1) == E
    assert rc(width=0) == E and rc(width=65537) == E and rc(max_rows=-1) == E and rc(max_rows=(1 << 20) + 1) == E
    for k in p:
        assert rc(**{k: True}) == E, k
    assert rc(num_free=0, free=True) == lib.SIDP_OK  # no list, no blocks needed
    assert rc(max_rows=0, pos=True, slots=True) == lib.SIDP_OK
    handle.sync()
