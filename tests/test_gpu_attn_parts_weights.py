"""How exactly the softmax weights reach their values in sidp_attention_rows8 and
sidp_attention_shared: sixteen bits where the header says so, on every path that such a
row can take (its own keys by a workgroup or by a wave, its group's by a small tile or a
large one), and eight bits in the other calls."""

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from parts_helpers import Parts

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (8, 1, 128), (16, 1, 128), (3, 3, 64), (64, 8, 128)]
CACHES = ["bf16", "e4m3", "int8"]
# Scores of two sizes, whose weights beside the other are 1 + 0.47 * 2^-8 and 1 - 0.47 * 2^-8: bf16 has neither, the nearest is 1 (its
# steps are 2^-7 above 1 and 2^-8 below), whichever of the two is the reference.
RISE = 0.47 * 2.0 ** -8


def close(got, want, mag, bits, what=""):
    """A weight's significand has `bits` bits: cut to 8 and the rest, below 2^-7, rounded to 8 bits (2^-8): 2^-15 relative (and 2^-23
    of it that an infinite value is kept by, below every other rounding); or rounded to 8 bits once: 2^-8. The exponents, scales and
    sums are fp32 (2^-12 holds scores of hundreds). Then the result's rounding."""
    assert np.all(np.isfinite(got)), what
    tol = ({16: 2.0 ** -15, 8: 2.0 ** -8}[bits] + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want) * 1.01
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-30))
    assert worst <= 1, f"{what}: worst {worst:.3g} of the tolerance"


def plant(c):
    """Every other key scores RISE more, with a value of -1 beside 1: what is left is the difference that eight bits lose. The rows'
    own keys weigh nothing. All numbers but the -60s are ones that the codes hold exactly."""
    D = c.D
    for b, (k, v) in enumerate(c.kv):
        ctx = c.lens[b][0]
        odd = torch.arange(len(k)) % 2 == 1
        k[:] = 0
        k[odd, :, 0] = 1.0
        k[ctx:, :, 0] = 0
        k[ctx:, :, 1] = -60.0
        v[:] = 1
        v[odd] = -1
        c.put(b)
    c.q[:] = 0
    c.q[:, :, 0] = np.log1p(RISE) * D ** 0.5
    c.q[:, :, 1] = D ** 0.5


def check(c, out, rows, bits):
    want, mag = c.want()
    got = np.abs(want[rows])
    # a shift of RISE / 2 between halves of weights that sum to 1 is what bf16 weights, all 1, would lose: three times the bound of 16
    assert np.all(got > 0.9 * RISE / 2) and np.all(got < 1.1 * RISE / 2) and RISE / 2 > 3 * (2.0 ** -15 + 2.0 ** -12)
    close(f64(out)[rows], want[rows], mag[rows], bits)


def fitting(c, pairs):
    """Rows of sequences with at most this many (row, head) pairs."""
    G = c.hq // c.hkv
    return np.concatenate([np.arange(c.starts[b], c.starts[b] + n) for b, (_, n) in enumerate(c.lens) if 0 < n * G <= pairs])


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("ctx", [64, 640, 3200])
def test_weights_of_few_rows(lib, cache, heads, ctx):
    """By a workgroup's waves: a row, as many as make 16 pairs, and (bf16) a whole tile; the longest are cut into runs and joined."""
    G = heads[0] // heads[1]
    lens = [(ctx, 1), (ctx, max(1, 16 // G))] + ([(ctx, 128 // G)] if cache == "bf16" else [])
    c = Parts(lib, cache, heads, lens, seed=1)
    plant(c)
    everyone = fitting(c, 16 if cache != "bf16" else 128)
    assert len(everyone) == c.rows
    check(c, c.run(shared=True), everyone, 16)
    if cache != "bf16":
        check(c, c.run(shared=False), everyone, 16)
    c.close()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads,batch", [((64, 8, 128), 512), ((4, 2, 64), 1100)], ids=str)
def test_weights_of_many_short_sequences(lib, cache, heads, batch):
    """More tiles than the chip holds: sequences of average length are a wave's each, the longest a workgroup's."""
    G = heads[0] // heads[1]
    lens = [(64, 1 + (i % 3 == 0) * (16 // G - 1) * (cache != "bf16")) for i in range(batch)]
    lens[7] = (4000, 1)
    c = Parts(lib, cache, heads, lens, seed=2, regions=1, region=0)
    plant(c)
    check(c, c.run(shared=True), fitting(c, 16), 16)
    if cache != "bf16":
        check(c, c.run(shared=False), fitting(c, 16), 16)
    c.close()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("size", ["small", "sixteen", "a tile", "more"])
@pytest.mark.parametrize("prefix", [128, 1600])
def test_weights_of_shared_tokens(lib, cache, heads, size, prefix):
    """Groups of 2 rows, of 16 pairs, of a whole tile and of more, with little behind their prefix."""
    G = heads[0] // heads[1]
    members = max(2, {"small": 2, "sixteen": 16 // G, "a tile": 128 // G, "more": 128 // G + 3}[size])
    c = Parts(lib, cache, heads, [(prefix + 2 * (i % 3), 1) for i in range(members)], [(members, prefix)], seed=3)
    plant(c)
    most = 128 if cache == "bf16" else 16
    check(c, c.run(), np.arange(members), 16 if members * G <= most else 8)
    c.close()


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_weights_of_more_rows_are_rounded_once(lib, cache, heads):
    """Past 16 pairs over the 8-bit cache, up to a tile and past it."""
    G = heads[0] // heads[1]
    c = Parts(lib, cache, heads, [(640, 16 // G + 1), (640, 64 // G + 1), (640, 128 // G + 1)], seed=4)
    plant(c)
    check(c, c.run(shared=False), np.arange(c.rows), 8)
    c.close()


@pytest.mark.parametrize("cache", CACHES)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_random_rows_with_weights_of_sixteen_bits(lib, cache, heads):
    G = heads[0] // heads[1]
    lens = [(300, 1), (17, max(1, 16 // G)), (3000, 1), (0, 1)] + [(400 + i, 1) for i in range(max(2, 16 // G))]
    c = Parts(lib, cache, heads, lens[4:] + lens[:4], [(len(lens) - 4, 384)], seed=5)
    want, mag = c.want()
    out = f64(c.run())
    grouped = (len(lens) - 4) * G
    first = 0 if grouped <= (128 if cache == "bf16" else 16) else len(lens) - 4
    close(out[first:c.rows], want[first:], mag[first:], 16)
    c.close()
