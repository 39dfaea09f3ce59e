"""Attention of a few rows over the longest caches and in the largest ones, with keys
planted so that every stretch of the cache decides a dim of its own: a run of keys
that is lost or read twice, or an offset that wraps, cannot hide among a million others."""

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from rows_helpers import BS, Handle, cfg_of, dev
from test_gpu_attn_rows import Case

LONGEST = 1 << 20
D = 64
CHUNK = 32


def planted(tokens, seed):
    """(keys, values, places) of one head: 64 stretches with four heavy keys each, their first, their last and two between; a heavy
    key's value is 1 in its stretch's dim alone. The other keys are light."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    k = 0.5 * torch.randn(tokens, 1, D, generator=g)
    v = 0.25 * torch.randn(tokens, 1, D, generator=g)
    k[:, :, 0] = 0
    edges = [tokens * i // D // CHUNK * CHUNK for i in range(D)] + [tokens - 7]  # all before the last rows' own keys
    places = np.stack([[a, b - 1, *rng.choice(np.arange(a + 1, b - 1), 2, replace=False)] for a, b in zip(edges, edges[1:])])
    for i in range(D):
        k[places[i]], v[places[i]] = 0, 0
        k[places[i], 0, 0] = 8
        v[places[i], 0, i] = 1
    return k.to(torch.bfloat16), v.to(torch.bfloat16), places.ravel()


def queries(rows, seed):
    """Scores of 16, 15, .. at the heavy keys, below 2 at the others."""
    q = 0.25 * torch.randn(rows, 1, D, generator=torch.Generator().manual_seed(seed))
    q[:, 0, 0] = 16 - torch.arange(rows)
    return q.to(torch.bfloat16)


def weights(q, k, cached):
    """[rows, tokens] in float64, of a sequence of `cached` tokens before its rows."""
    s = f64(q)[:, 0] @ f64(k)[:, 0].T / np.sqrt(D)
    s[np.arange(len(k))[None] > cached + np.arange(len(q))[:, None]] = -np.inf
    return np.exp(s - s.max(1, keepdims=True))


def answer(w, v):
    """(output, sum of p |v|)."""
    p, x = w / w.sum(1, keepdims=True), f64(v)[:, 0]
    return p @ x, p @ np.abs(x)


def tolerance(want, mag, light=0.0):
    """Weights of 16 bits (2^-15), fp32 exponents and sums (2^-12), the result's rounding. `light`: the light keys' share of the
    weights. A chunk of them may be below half a step of the fp32 sum that it joins, so all of them may be missing there."""
    return (2.0 ** -15 + 2.0 ** -12 + light) * mag + 2.0 ** -8 * np.abs(want) * 1.01


def test_a_lost_stretch_would_show():
    """The oracle with keys left out is far outside the tolerance: each planted key alone, each 32nd of the cache, a chunk at every
    border of these; and a stretch read in another's place."""
    n = 1 << 16  # a sixteenth of the longest: the planted keys outweigh the light ones even more there than here
    k, v, places = planted(n, 1)
    q = queries(3, 1)
    w = weights(q, k, n - 3)
    want, mag = answer(w, v)
    # light keys weigh little, also sixteen times as many of them
    light = 16 * (1 - w[:, places].sum(1, keepdims=True) / w.sum(1, keepdims=True))
    assert light.max() < 2.0 ** -6
    tol = tolerance(want, mag, light)

    x = f64(v)[:, 0]
    whole, total = w @ x, w.sum(1, keepdims=True)

    def shows(gone, instead=slice(0, 0)):
        """Without the keys of a stretch, or with another's in their place."""
        top = whole - w[:, gone] @ x[gone] + w[:, instead] @ x[instead]
        out = top / (total - w[:, gone].sum(1, keepdims=True) + w[:, instead].sum(1, keepdims=True))
        return (np.abs(out - want) > 8 * tol).any(1).all()
    for place in places:
        assert shows(slice(place, place + 1)), place
    for i in range(32):
        a, b = n * i // 32, n * (i + 1) // 32
        assert shows(slice(a, b)), i
        assert shows(slice(a, a + CHUNK)) and shows(slice(b - CHUNK, b)), i
        other = (a + n // 2) % n
        assert shows(slice(a, b), slice(other, other + b - a)), i


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[(LONGEST - 3, 3)], [(LONGEST - 1, 1)] + [(3, 1)] * 600, [(LONGEST - 130, 130)],
                                  [(LONGEST - 40, 2), (LONGEST // 2 + 777, 5)]], ids=["cut", "whole", "two tiles", "two long"])
def test_every_stretch_of_the_longest_cache_counts(lib, lens):
    c = Case(lib, (1, 1, D), lens, seed=6, regions=1, region=0)
    want, tol = np.zeros((c.rows, D)), np.full((c.rows, D), np.inf)
    for b, (ctx, n) in enumerate(lens):
        at = slice(c.starts[b], c.starts[b] + n)
        if ctx < 1000:
            continue  # there to fill the chip
        k, v, places = planted(ctx + n, 7 + b)
        c.kv[b] = [k, v]
        c.put(b)
        c.q[at] = queries(n, 8 + b) if n < 8 else queries(1, 8).repeat(n, 1, 1)
        for r in [0, n // 2, n - 1]:
            row = c.starts[b] + r
            w = weights(c.q[row:row + 1], k[:ctx + r + 1], ctx + r)
            x, mag = answer(w, v[:ctx + r + 1])
            seen = places[places <= ctx + r]
            light = 1 - w[:, seen].sum() / w.sum()
            want[row] = x[0]
            # more rows than a tile: weights of 8 bits
            tol[row] = tolerance(x, mag, light)[0] + (2.0 ** -8 * mag[0] if n > 128 else 0)
    got = f64(c.run()[:c.rows])[:, 0]
    off = np.abs(got - want) / tol
    assert np.isfinite(got).all() and off.max() <= 1, (off.max(), np.unravel_index(off.argmax(), off.shape))
    c.h.close()


@pytest.mark.gpu
def test_appends_and_attention_past_2_to_the_32_elements(lib):
    """K and V of 2^32 elements and more, 8.6 GB each: rows appended to the last blocks, and attended there; where an offset of 32
    bits would land nothing is written, and what stands there is NaN."""
    heads, nblk = (4, 2, D), (1 << 32) // (2 * D * BS) + 4000
    assert nblk * 2 * D * BS > 1 << 32
    lens = [(100, 30), (0, 20)]
    place = list(range(nblk - 20, nblk))
    c = Case(lib, heads, lens, nblk=nblk, regions=1, region=0, place=place)
    # the keys and values of the rows come by the call itself (positions turned as its own tables turn them)
    qkv = torch.randn(50, 8 * D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    pos = np.concatenate([np.arange(ctx, ctx + n) for ctx, n in lens])
    seq = np.repeat(np.arange(2), [n for _, n in lens])
    slots = c.tables[seq, pos // BS] * BS + pos % BS
    assert slots.min() * 2 * D > 1 << 32
    q = torch.zeros(50, 4, D, dtype=torch.bfloat16, device="cuda")
    lib.sidp_rope_append_rows(c.h.h, qkv.cuda(), 8 * D, 50, None, dev(pos), dev(slots), None, None, 0, q)
    c.h.sync()
    blk, off = torch.as_tensor(slots // BS).cuda(), torch.as_tensor(slots % BS).cuda()
    k = c.h.k[0][blk, :, :, off, :].reshape(50, 2, D).cpu()
    v = c.h.v[0][blk, :, :, off].cpu()
    assert torch.equal(v, qkv[:, 6 * D:].view(50, 2, D))
    # the same rows in a small cache: the same keys
    with Handle(lib, cfg_of(*heads), 200, 8) as small:
        near = np.arange(50)
        lib.sidp_rope_append_rows(small.h, qkv.cuda(), 8 * D, 50, None, dev(pos), dev(near), None, None, 0, torch.zeros_like(q))
        small.sync()
        assert torch.equal(small.keys()[:50].cpu(), k)
    wrapped = torch.as_tensor((slots * 2 * D - (1 << 32)) // (2 * D * BS)).cuda()
    assert int(wrapped.min()) >= 0 and torch.isnan(c.h.k[0][wrapped]).all() and torch.isnan(c.h.v[0][wrapped]).all()
    for b, (ctx, n) in enumerate(lens):
        at = slice(c.starts[b], c.starts[b] + n)
        c.kv[b][0][ctx:], c.kv[b][1][ctx:] = k[at], v[at]
    c.q = q.cpu()
    got, (want, mag) = f64(c.run()[:50]), c.want()
    assert np.isfinite(got).all() and np.all(np.abs(got - want) <= tolerance(want, mag))
    c.h.close()
