"""How exactly the softmax weights of several new tokens a sequence reach their
values: sixteen bits in sequences whose rows fit a tile (as in the attention of a
decode step), eight in longer ones, and infinite values in both."""

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from rows_helpers import dev
from test_gpu_attn_rows import Case

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (8, 1, 128), (16, 1, 128), (3, 3, 64)]


def close(got, want, mag, bits, what=""):
    """A weight's significand has `bits` bits: cut to 8 and the rest, below 2^-7, rounded to 8 bits (2^-8): 2^-15 relative; or
    rounded to 8 bits once: 2^-8. The exponents and sums are fp32 (2^-12 holds scores of hundreds). Then the result's rounding."""
    got = f64(got)
    assert np.all(np.isfinite(got)), what
    tol = ({16: 2.0 ** -15, 8: 2.0 ** -8}[bits] + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want) * 1.01
    worst = np.max(np.abs(got - want) / np.maximum(tol, 1e-30))
    assert worst <= 1, f"{what}: worst {worst:.3g} of the tolerance"


def tile_rows(heads):
    return 128 // (heads[0] // heads[1])


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("ctx", [0, 7, 300, 5000])
def test_rows_of_one_tile_have_weights_of_sixteen_bits(lib, heads, ctx):
    """Random keys and values: one row, two, a full tile; the last cut into runs by its length."""
    c = Case(lib, heads, [(ctx, 1), (ctx + 9, 2), (ctx // 2, tile_rows(heads))], seed=ctx)
    close(c.run()[:c.rows], *c.want(), bits=16)
    c.h.close()


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("rows", ["one", "a tile", "more"])
@pytest.mark.parametrize("signs", ["unlike", "alike"])
def test_weights_that_all_round_the_same_way(lib, heads, rows, signs):
    """Half of the keys have weight 1 and half one that rounds down to it from nearly halfway: values of unlike signs leave the
    difference alone, which eight bits lose, and with values alike the sum of weights and their products part."""
    n = {"one": 1, "a tile": tile_rows(heads), "more": 2 * tile_rows(heads) + 3}[rows]
    ctx = 640
    c = Case(lib, heads, [(ctx, n)], seed=1)
    D = heads[2]
    score = np.log(1 + 0.97 * 2.0 ** -8)
    k, v = c.kv[0]
    odd = (torch.arange(ctx + n) % 2 == 1) & (torch.arange(ctx + n) >= 32)  # the reference is a score of the first 32 keys
    k[:] = 0
    k[odd, :, 0] = score * D ** 0.5
    k[ctx:, :, 0] = -60.0 * D ** 0.5  # the rows' own keys weigh nothing
    v[:] = 1
    if signs == "unlike":
        v[odd] = -1
    c.q[:] = 0
    c.q[:, :, 0] = 1
    c.put(0)
    want, mag = c.want()
    # what 8 bits make of it: every weight of the odd keys is 1
    w = np.where(odd[:ctx].numpy(), np.exp(f64(k[:ctx, 0, 0]) / D ** 0.5), 1.0)
    lost = np.sum((1 - w) * f64(v[:ctx, 0, 0])) / w.sum()
    assert abs(lost) > (6 if signs == "unlike" else 0) * 2.0 ** -12
    close(c.run()[:c.rows], want, mag, bits=8 if rows == "more" else 16, what=f"off by {lost:.3g} in eight bits")
    c.h.close()


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", [[(200, 1)], [(200, 8)], [(200, 300)], [(3000, 3)], [(70, 90), (40, 1)]], ids=str)
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_infinite_values_that_every_row_sees(lib, heads, lens, value):
    """In chunks that all rows see whole: the dim is infinite, its sign kept, the others are what they were."""
    c = Case(lib, heads, lens, seed=3)
    clean, mag = c.want()
    v = c.kv[0][1]
    v[5, :, 3], v[20, :, 3], v[33, 0, 7] = value, value, -value
    c.put(0)
    got = f64(c.run()[:c.rows])
    G = heads[0] // heads[1]
    first = slice(0, lens[0][1])
    assert np.all(got[first, :, 3] == value) and np.all(got[first, :G, 7] == -value)
    touched = np.zeros(got.shape, bool)
    touched[first, :, 3] = True
    touched[first, :G, 7] = True
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(clean) * 1.01
    assert np.all(np.abs(got - clean)[~touched] <= tol[~touched])
    c.h.close()


def test_a_drafted_token_is_checked_with_the_weights_of_its_decode_step(lib):
    """Four tokens at once, and each by itself through the attention of the decode step: nearly always the same bits."""
    lens = [(300, 4), (1500, 4), (17, 4)]
    c = Case(lib, (64, 8, 128), lens, seed=4, max_seq=2048)
    rows = c.run()[:c.rows]
    want, mag = c.want()
    h = lib.sidp_create(lib.make_config(c.h.cfg, c.rows, 2048))
    lib.sidp_kv_attach(h, c.h.k, c.h.v, c.nblk, 2)
    pos = dev([n + i for n, m in lens for i in range(m)])
    out = torch.zeros(c.rows, 64, 128, dtype=torch.bfloat16, device="cuda")
    lib.sidp_attention(h, c.q.cuda(), 1, pos, dev(c.tables.repeat(4, 0)), c.width, c.rows, out)
    lib.sidp_sync(h)
    close(rows, want, mag, bits=16)
    close(out, want, mag, bits=16)
    # before their rounding the two differ by at most 2^-15 of the magnitudes (P's second part) and the order of fp32 sums, so a result
    # is rounded otherwise where it lies that near to the middle of a step of 2^-8: one in 128 values as large as the magnitudes, a
    # few in a hundred of those at a quarter of them. Weights of 8 bits would change about every third.
    same = (rows == out).double().mean().item()
    lib.sidp_destroy(h)
    c.h.close()
    assert same > 0.95, same
