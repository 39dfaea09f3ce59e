"""Causal attention of several new tokens a sequence over the 8-bit cache, against
softmax(q K^T / sqrt(D)) V in float64 over what the codes stand for."""

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from kv8_helpers import Handle8
from parts_helpers import Parts, close
from rows_helpers import BS, Handle, cfg_of, dev

pytestmark = pytest.mark.gpu

KINDS = ["e4m3", "int8"]
HEADS = [(4, 2, 64), (8, 1, 64), (16, 1, 128), (5, 1, 128), (3, 3, 128), (64, 8, 128)]
LENS = {
    "one token each": [(0, 1), (5, 1), (15, 1), (16, 1), (31, 1), (32, 1), (63, 1), (64, 1), (200, 1)],
    "a few each": [(0, 2), (15, 3), (60, 8), (100, 5), (1000, 4)],
    "ragged": [(0, 5), (16, 16), (17, 100), (300, 33), (50, 0), (0, 129), (64, 64), (0, 0), (1, 63)],
    "one prompt": [(0, 333)],
    "one long chunk": [(777, 260)],
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", list(LENS), ids=str)
def test_attention_rows8_match_the_definition(lib, kind, heads, lens):
    c = Parts(lib, kind, heads, LENS[lens], seed=len(lens))
    out = c.run(shared=False)
    close(out[:c.rows], *c.want(), what=lens)
    assert torch.all(out[c.rows:] == 7.0)
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,lens", [((8, 1, 128), [(6000, 4)]), ((8, 2, 64), [(3000, 1), (4095, 40), (10, 2), (64, 1)]),
                                        ((16, 1, 128), [(511, 1), (512, 1), (513, 1), (1024, 3), (0, 1), (1535, 1)]),
                                        ((8, 8, 128), [(2000 + 77 * i, 1) for i in range(9)]),
                                        ((4, 4, 64), [(2500, 700)]), ((2, 1, 128), [(40000, 2)])], ids=str)
def test_attention_rows8_over_long_caches(lib, kind, heads, lens):
    """Few rows and many keys: sequences are cut into runs and joined, block ids are fetched in groups."""
    c = Parts(lib, kind, heads, lens, seed=5)
    close(c.run(shared=False)[:c.rows], *c.want())
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("chunks", list(range(1, 12)) + [31, 32, 33, 34, 35, 36, 63, 64, 65, 66, 67, 68])
def test_every_number_of_chunks(lib, kind, chunks):
    """Whole and ragged last chunks, through each end of the loop over chunks and of the fetches in front of it."""
    for edge in (0, 1, 15, 16, 17, 31):
        n = 32 * chunks - edge
        for new in (1, 5):
            if n < new:
                continue
            c = Parts(lib, kind, (4, 2, 64) if edge % 2 else (8, 1, 128), [(n - new, new)], seed=chunks)
            close(c.run(shared=False)[:c.rows], *c.want(), what=f"{n} keys, {new} rows")
            c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch", [300, 1100, 4096])
def test_attention_rows8_of_many_sequences(lib, kind, batch):
    rng = np.random.default_rng(batch)
    lens = [(int(c), int(n)) for c, n in zip(rng.integers(0, 90, batch), rng.integers(0, 3, batch))]
    c = Parts(lib, kind, (4, 2, 64), lens, seed=batch, regions=1, region=0)
    out = c.run(shared=False)
    close(out[:c.rows], *c.want())
    assert torch.all(out[c.rows:] == 7.0)
    c.close()


@pytest.mark.parametrize("kind", KINDS)
def test_attention_rows8_with_a_sharp_softmax_and_uneven_scales(lib, kind):
    """Scores of hundreds that rise and fall along the keys; tokens of very different sizes, and zeros."""
    c = Parts(lib, kind, (8, 2, 64), [(500, 70), (0, 90)], q_std=60.0)
    close(c.run(shared=False)[:c.rows], *c.want())
    rng = np.random.default_rng(0)
    for b, (k, v) in enumerate(c.kv):
        k *= torch.tensor(2.0 ** rng.integers(-30, 1, (len(k), 2, 1))).to(torch.bfloat16)
        v *= torch.tensor(2.0 ** rng.integers(-30, 20, (len(k), 2, 1))).to(torch.bfloat16)
        k[::7], v[::5] = 0, 0
        c.put(b)
    close(c.run(shared=False)[:c.rows], *c.want())
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", [(8, 1, 128), (4, 2, 64)], ids=str)
@pytest.mark.parametrize("lens", [[(70, 90)], [(3, 4)], [(4000, 5)]], ids=str)
@pytest.mark.parametrize("which", [0, 1])
def test_a_token_without_a_scale_stays_out_of_rows_that_do_not_see_it(lib, kind, heads, lens, which):
    c = Parts(lib, kind, heads, lens)
    ctx, n = lens[0]
    want, mag = c.want()
    at = ctx + n // 2
    c.kv[0][which][at, 0, 3] = float("inf") if which else float("nan")
    c.put(0)
    got = f64(c.run(shared=False)[:c.rows])
    G = heads[0] // heads[1]
    assert np.isnan(got[n // 2:, :G]).all()
    clean = np.ones(got.shape, bool)
    clean[n // 2:, :G] = False
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want) * 1.01
    assert np.all(np.abs(got - want)[clean] <= tol[clean])
    c.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bad", [-1, "past"])
def test_attention_rows8_bad_blocks_are_latched_and_stay_in_their_sequence(lib, kind, bad):
    c = Parts(lib, kind, (8, 2, 64), [(100, 20), (90, 30), (0, 10)])
    tables = c.tables.copy()
    tables[1, 2] = c.nblk if bad == "past" else -1
    out = c.run(shared=False, tables=tables, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    want, mag = c.want()
    for lo, hi in ((0, 20), (50, 60)):
        close(out[lo:hi], want[lo:hi], mag[lo:hi])
    c.close()


@pytest.mark.parametrize("what", ["ctx negative", "past the table", "past max_seq_len", "starts fall", "starts past max_rows"])
def test_attention_rows8_bad_lengths_leave_the_others(lib, what):
    lens = [(100, 20), (90, 30), (0, 10)]
    c = Parts(lib, "e4m3", (8, 2, 64), lens, max_seq=200)
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
        starts[1:] = [50, 20, 60]
        ctx = [70, 0, 0]
    else:
        max_rows = 55
    out = c.run(shared=False, ctx=ctx, starts=starts, max_rows=max_rows, sync=False)
    with pytest.raises(lib.SidpError) as e:
        c.h.sync()
    assert e.value.code == lib.SIDP_EINVAL
    want, mag = c.want()
    if what == "starts fall":
        return c.close()  # in bounds and latched is all that is asked
    close(out[:20], want[:20], mag[:20])
    if what == "starts past max_rows":
        close(out[20:50], want[20:50], mag[20:50])
        assert torch.all(out[50:] == 7.0)
    else:
        assert torch.all(out[20:50] == 7.0)
        close(out[50:60], want[50:60], mag[50:60])
    c.close()


def test_attention_rows8_in_caches_past_32_bits(lib):
    nblk = (1 << 32) // (2 * 64 * BS) + 4000
    place = list(range(nblk - 20, nblk)) + [0, 1]
    c = Parts(lib, "int8", (4, 2, 64), [(100, 30), (0, 20)], nblk=nblk, regions=1, region=0, place=place)
    close(c.run(shared=False)[:c.rows], *c.want())
    c.close()


def test_attention_rows8_on_two_streams_and_again(lib):
    a = Parts(lib, "e4m3", (8, 2, 128), [(700, 50), (3, 90)], seed=1)
    b = Parts(lib, "e4m3", (8, 2, 128), [(2500, 4)], seed=2)
    alone = [x.run(shared=False).clone() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        outs = [x.run(shared=False, stream=s, sync=False) for x, s in zip((a, b), streams)]
        torch.cuda.synchronize()
        for x, y in zip(outs, alone):
            assert torch.equal(x, y)
    a.close()
    b.close()


def test_attention_rows8_without_rows_and_refusals(lib):
    c = Parts(lib, "int8", (4, 2, 64), [(10, 3)])
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    i = dev([0] * 8)
    need = lib.sidp_attention_rows8_bytes(c.h.h, 1, 3)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    T, I, W = t.data_ptr(), i.data_ptr(), ws.data_ptr()

    def rc(h=c.h.h, q=T, region=0, starts=I, ctx=I, bt=I, width=2, batch=1, rows=3, out=T, w=W, n=need):
        return lib.raw_call("sidp_attention_rows8", h, q, region, starts, ctx, bt, width, batch, rows, out, w, n, None)
    E = lib.SIDP_EINVAL
    assert rc(rows=0, w=None, n=0) == 0
    assert rc(batch=0) == E and rc(batch=4097) == E and rc(rows=-1) == E and rc(rows=(1 << 20) + 1) == E
    assert rc(width=0) == E and rc(width=65537) == E and rc(region=2) == E and rc(region=-1) == E
    assert rc(q=None) == E and rc(starts=None) == E and rc(ctx=None) == E and rc(bt=None) == E and rc(out=None) == E
    assert rc(w=None) == E and rc(n=need - 1) == E and rc(w=W + 8) == E and rc(q=T + 2) == E and rc(out=T + 8) == E
    assert lib.raw_call("sidp_attention_rows8", None, T, 0, I, I, I, 2, 1, 3, T, W, need, None) == E
    c.h.sync()
    assert lib.sidp_attention_rows8_bytes(c.h.h, 4096, 1 << 20) > 0
    assert lib.sidp_attention_rows8_bytes(None, 1, 1) == 0 and lib.sidp_attention_rows8_bytes(c.h.h, 0, 1) == 0
    c.close()
    with Handle(lib, cfg_of(4, 2, 64), 64, 4) as h:
        assert rc(h=h.h) == lib.SIDP_ESTATE  # a bf16 cache only
    with Handle8(lib, cfg_of(1, 1, 64), 64, 4, "e4m3") as h:
        assert lib.raw_call("sidp_attention_rows", h.h, T, 0, I, I, I, 2, 1, 3, T, W, need, None) == lib.SIDP_ESTATE
