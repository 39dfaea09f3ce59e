"""Infinite values in sidp_attention_shared over the bf16 cache: each row that sees one
has it in that dim, sign and all, as from sidp_attention_rows, whatever the size of the
tile that reads it."""

import numpy as np
import pytest

from gpu_helpers import f64
from parts_helpers import Parts

pytestmark = pytest.mark.gpu

INF = float("inf")
HEADS = [(4, 2, 64), (8, 1, 128), (16, 1, 128), (3, 3, 64), (64, 8, 128)]


def best_key(c, b, lo, hi):
    """The key of sequence b, of lo .. hi - 1, with the highest score of its first row's first head: weight 1 beside its reference."""
    score = c.held[b][0][lo:hi, 0] @ f64(c.q)[c.starts[b], 0]
    return lo + int(np.argmax(score))


def check(c, rows, clean, mag, infinite):
    """infinite: [(rows, first head, heads, dim, value)]; the rest is what it was without."""
    got = f64(rows)
    touched = np.zeros(got.shape, bool)
    for who, h0, hn, d, value in infinite:
        assert np.all(got[who, h0:h0 + hn, d] == value), (value, got[who, h0:h0 + hn, d])
        touched[who, h0:h0 + hn, d] = True
    # the bounds of parts_helpers.close
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(clean) * 1.01 + 2.0 ** -107
    assert np.all(np.abs(got - clean)[~touched] <= tol[~touched])


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("ctx", [0, 1, 5, 31, 32, 200, 3000])
def test_a_row_of_its_own(lib, heads, ctx, value):
    """No group: each sequence one row, with one key up to runs that are joined; infinite are the highest scored key and the row's own."""
    c = Parts(lib, "bf16", heads, [(ctx, 1), (ctx + 40, 1)], seed=ctx)
    clean, mag = c.want()
    G = heads[0] // heads[1]
    top = best_key(c, 0, 0, ctx + 1)
    v = c.kv[0][1]
    v[top, 0, 3] = value
    v[ctx, :, 9] = -value
    c.put(0)
    check(c, c.run()[:2], clean, mag, [([0], 0, G, 3, value), ([0], 0, heads[0], 9, -value)])
    c.close()


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("heads,batch", [((64, 8, 128), 512), ((4, 2, 64), 1100)], ids=str)
def test_many_short_sequences(lib, heads, batch, value):
    """More tiles than the chip holds at once: short ones go by a wave each, longer ones by a workgroup."""
    lens = [(int(n), 1) for n in np.random.default_rng(batch).integers(0, 70, batch)]
    lens[1] = (2000, 1)
    c = Parts(lib, "bf16", heads, lens, seed=3, regions=1, region=0)
    clean, mag = c.want()
    G = heads[0] // heads[1]
    hits = []
    for b in (0, 1, batch // 2, batch - 1):
        v = c.kv[b][1]
        v[best_key(c, b, 0, lens[b][0] + 1), 0, 3] = value
        v[lens[b][0], :, 9] = -value
        c.put(b)
        hits += [([b], 0, G, 3, value), ([b], 0, heads[0], 9, -value)]
    check(c, c.run()[:batch], clean, mag, hits)
    c.close()


@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("members,rows", [(2, 1), (4, 1), (16, 1), (40, 1), (7, 2)])
@pytest.mark.parametrize("prefix", [128, 1600])
def test_in_a_shared_prefix_and_behind_it(lib, heads, members, rows, prefix, value):
    """Group tiles of 2 to 320 pairs (those of at most 16 and others), in one run and in several; a key by its own sequence as well."""
    lens = [(prefix + 9 * i, rows) for i in range(members)] + [(50, 1)]
    c = Parts(lib, "bf16", heads, lens, [(members, prefix)], seed=members)
    clean, mag = c.want()
    G, hq = heads[0] // heads[1], heads[0]
    group = list(range(members * rows))
    v = c.kv[0][1]
    v[best_key(c, 0, 0, prefix), 0, 3] = value
    v[prefix - 1, :, 7] = -value
    for b in range(1, members):
        c.kv[b][1][:prefix] = v[:prefix]
    last = members - 1
    c.kv[last][1][prefix + 9 * last, :, 9] = value  # its first row's own: every row of the sequence sees it
    c.put(0)
    c.put(last)
    mine = list(range(last * rows, members * rows))
    check(c, c.run()[:c.rows], clean, mag, [(group, 0, G, 3, value), (group, 0, hq, 7, -value), (mine, 0, hq, 9, value)])
    c.close()
