"""The 8-bit cache: rows appended to it and read back, against the definition of
its codes in float64. Places that no row writes hold a byte of their own, which
has to stay."""

import ctypes

import numpy as np
import pytest
import torch

from gpu_helpers import f64
from kv8_helpers import Handle8, codes_of, half_step, scale_of, values_of
from rows_helpers import BS, Handle, cfg_of, dev, turn

pytestmark = pytest.mark.gpu
FILL = 0x35


def rows_of(hq, hkv, D, rows, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn(rows, (hq + 2 * hkv) * D, generator=g)).to(torch.bfloat16)


def slots_of(kind, rows, nblk, seed=0):
    if kind == "scattered":
        return np.random.default_rng(seed).permutation(nblk * BS)[:rows]
    if kind == "run":  # of consecutive tokens, from the middle of a block
        return 5 + np.arange(rows)
    if kind == "blocks":  # a sequence's tokens in blocks out of order, from the middle of one
        place = np.random.default_rng(seed).permutation(nblk)
        p = 11 + np.arange(rows)
        return place[p // BS] * BS + p % BS
    raise KeyError(kind)


def append(lib, h, qkv, slots, pos, region=0, g_q=None, g_k=None, rows=None, count=None, stride=None, stream=None):
    hq, D = h.cfg["num_q_heads"], h.cfg["head_dim"]
    rows = len(qkv) if rows is None else rows
    q = torch.full((len(qkv) + 1, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.sidp_rope_append_rows8(h.h, qkv, qkv.shape[1] if stride is None else stride, rows, count, dev(pos), dev(slots), g_q, g_k, region,
                               q, stream)
    return q


def check_cache(h, region, slots, k, v, fill=FILL, exact_k=False):
    """Cached rows against keys and values in float64; everything else is as it was. Values are bf16, so that their codes are the
    definition's bit for bit; keys come from fp32: 4 roundings of the larger pair member (2^-22 of the head's largest)."""
    kc, ks, vc, vs = h.key_codes(region), h.key_scales(region), h.value_codes(region), h.value_scales(region)
    np.testing.assert_array_equal(vs[slots], scale_of(v, h.kind))
    np.testing.assert_array_equal(vc[slots], codes_of(v, vs[slots], h.kind))
    want = scale_of(k, h.kind)
    if exact_k:
        np.testing.assert_array_equal(ks[slots], want)
        # as numbers: -0 cos + 0 sin is 0
        np.testing.assert_array_equal(values_of(kc[slots], h.kind), values_of(codes_of(k, want, h.kind), h.kind))
    else:
        most = np.max(np.abs(k), -1)
        if h.kind == "e4m3":
            near = np.abs(most / want / 448 - 1) < 1e-6  # either power of two
            near |= np.abs(most / want / 224 - 1) < 1e-6
            assert np.all((ks[slots] == want) | near)
        else:
            np.testing.assert_allclose(ks[slots], want, rtol=2.0 ** -20)
        got = values_of(kc[slots], h.kind) * ks[slots][..., None]
        tol = half_step(k, ks[slots], h.kind) * (1 + 2.0 ** -18) + 2.0 ** -21 * most[..., None]
        assert np.all(np.abs(got - k) <= tol), np.max(np.abs(got - k) / tol)
    rest = np.ones(h.nblk8 * BS, bool)
    rest[slots] = False
    assert np.all(kc[rest] == fill) and np.all(vc[rest] == fill)
    assert np.all(np.isnan(ks[rest])) and np.all(np.isnan(vs[rest]))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (5, 1, 128), (64, 8, 128), (3, 3, 128)], ids=str)
@pytest.mark.parametrize("rows,where", [(1, "run"), (7, "scattered"), (45, "run"), (100, "blocks"), (2100, "blocks")])
def test_append_matches_the_definition(lib, kind, heads, rows, where):
    hq, hkv, D = heads
    if rows > 1000 and hq > 8:
        pytest.skip("the long tile is covered by the smaller heads")
    nblk = rows // BS + 6
    cfg = cfg_of(hq, hkv, D)
    with Handle8(lib, cfg, 5000, nblk, kind, regions=2, fill=FILL) as h, Handle(lib, cfg, 5000, nblk) as plain:
        qkv = rows_of(hq, hkv, D, rows, rows)
        pos = (np.arange(rows) * 7 + 3) % 5000
        slots = slots_of(where, rows, nblk, 1)
        q = append(lib, h, qkv.cuda(), slots, pos, region=1)
        h.sync()
        x = f64(qkv).reshape(rows, hq + 2 * hkv, D)
        freqs = 1e4 ** (-2.0 * np.arange(D // 2) / D)
        check_cache(h, 1, slots, turn(x[:, hq:hq + hkv], pos, freqs, 1.0, False), x[:, hq + hkv:])
        assert torch.all(h.k8[0] == FILL) and torch.all(h.v8[0] == FILL)
        # queries are the bf16 append's
        want = torch.zeros_like(q)
        lib.sidp_rope_append_rows(plain.h, qkv.cuda(), qkv.shape[1], rows, None, dev(pos), dev(slots), None, None, 0, want)
        plain.sync()
        assert torch.equal(q[:rows], want[:rows]) and torch.all(q[rows:] == 7.0)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("layout,rot,D", [("interleaved", 32, 64), ("half", 48, 128), ("interleaved", 128, 128)])
def test_append_with_norms_layouts_and_strides(lib, kind, layout, rot, D):
    hq, hkv, rows, nblk = 8, 2, 37, 12
    cfg = cfg_of(hq, hkv, D, qk_norm=1)
    with Handle8(lib, cfg, 300, nblk, kind, fill=FILL) as h:
        lib.sidp_set_rope(h.h, lib.make_rope(layout=layout, rotary_dim=rot, theta=5e5))
        qkv = rows_of(hq, hkv, D, rows, 3)
        wide = torch.full((rows, qkv.shape[1] + 24), float("nan"), dtype=torch.bfloat16)
        wide[:, :qkv.shape[1]] = qkv
        g = (1 + 0.1 * torch.randn(2, D, generator=torch.Generator().manual_seed(5))).to(torch.bfloat16)
        pos, slots = np.arange(rows) * 8, slots_of("blocks", rows, nblk, 2)
        gc = g.cuda()
        append(lib, h, wide.cuda(), slots, pos, g_q=gc[0], g_k=gc[1])
        h.sync()
        x = f64(qkv).reshape(rows, hq + 2 * hkv, D)
        k = x[:, hq:hq + hkv]
        k = k / np.sqrt(np.mean(k * k, -1, keepdims=True) + 1e-6) * f64(g[1])
        freqs = 5e5 ** (-2.0 * np.arange(rot // 2) / rot)
        check_cache(h, 0, slots, turn(k, pos, freqs, 1.0, layout == "interleaved"), x[:, hq + hkv:])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_append_of_all_magnitudes(lib, kind):
    """Position 0 turns nothing: keys are bf16 as they are, and their codes the definition's bit for bit. Heads of one size and of
    many, powers of two, zeros, the smallest and the largest numbers; NaN and infinities make a head NaN."""
    D, hkv, nblk = 64, 4, 40
    rng = np.random.default_rng(7)
    rows = 600
    x = rng.standard_normal((rows, 2 * hkv, D)) * 2.0 ** rng.integers(-20, 20, (rows, 2 * hkv, 1))
    x[:200] *= 2.0 ** rng.integers(-14, 3, (200, 2 * hkv, D))
    x[200:220] = 0
    x[220:260] = 2.0 ** rng.integers(-30, 30, (40, 2 * hkv, D))
    x[260:280] *= 1e-38 / np.abs(x[260:280]).max(-1, keepdims=True)
    x[280:300] *= 3e38 / np.abs(x[280:300]).max(-1, keepdims=True)
    x[300:320] = 448 * 2.0 ** rng.integers(-5, 5, (20, 2 * hkv, 1))
    x[320:340] = 1e-44 * rng.integers(0, 9, (20, 2 * hkv, D))
    x[340:350, :, 3] = np.inf
    x[350:360, ::2, 5] = -np.inf
    x[360:370, 1::2, 63] = np.nan
    qkv = torch.tensor(np.concatenate([np.ones((rows, hkv, D)), x], 1).reshape(rows, -1), dtype=torch.float64).to(torch.bfloat16)
    with Handle8(lib, cfg_of(hkv, hkv, D), 64, nblk, kind, fill=FILL) as h:
        slots = slots_of("scattered", rows, nblk, 4)
        append(lib, h, qkv.cuda(), slots, np.zeros(rows, int))
        h.sync()
        y = f64(qkv).reshape(rows, 3 * hkv, D)
        check_cache(h, 0, slots, y[:, hkv:2 * hkv], y[:, 2 * hkv:], exact_k=True)
        # and read back: NaN where there is no scale, else code * scale in fp32, once rounded
        k, v = (torch.full((rows, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lib.sidp_kv8_read(h.h, 0, rows, None, dev(slots), k, v)
        h.sync()
        for got, codes, scales in ((k, h.key_codes(), h.key_scales()), (v, h.value_codes(), h.value_scales())):
            want = torch.tensor(values_of(codes[slots], kind).astype(np.float32) * scales[slots][..., None].astype(np.float32)).to(torch.bfloat16)
            np.testing.assert_array_equal(f64(got), f64(want))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_are_left_out(lib, kind, D):
    hq, hkv, rows, nblk = 4, 2, 50, 8
    with Handle8(lib, cfg_of(hq, hkv, D), 100, nblk, kind, fill=FILL) as h:
        qkv = rows_of(hq, hkv, D, rows, 9).cuda()
        slots, pos = slots_of("run", rows, nblk), np.arange(rows)
        slots[[3, 20]] = -1  # cached nowhere, their queries still come
        q = append(lib, h, qkv, slots, pos, count=dev([41]))
        h.sync()
        assert torch.all(q[41:] == 7.0) and not torch.any(torch.all(q[:41] == 7.0, -1))
        live = np.array([s for s in slots[:41] if s >= 0])
        touched = ~np.all(h.key_codes() == FILL, (1, 2))
        assert sorted(np.flatnonzero(touched)) == sorted(live)
        np.testing.assert_array_equal(np.flatnonzero(~np.isnan(h.value_scales()[:, 0])), np.sort(live))
        # read back: rows behind the count, and of negative slots, as they were
        k, v = (torch.full((rows, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lib.sidp_kv8_read(h.h, 0, rows, dev([41]), dev(slots), k, v)
        h.sync()
        for got in (k, v):
            assert torch.all(got[41:] == 7.0) and torch.all(got[[3, 20]] == 7.0)
        only = torch.full_like(k, 7.0)
        lib.sidp_kv8_read(h.h, 0, rows, None, dev(slots), None, only)
        h.sync()
        assert torch.equal(only[:41], v[:41])
        # a position or a slot outside latches, and its row alone is left out
        for bad_pos, bad_slot in ((100, 7), (-1, 7), (5, nblk * BS), (5, 1 << 30)):
            before = h.key_codes(), h.value_codes()
            append(lib, h, qkv[:1], [bad_slot], [bad_pos])
            with pytest.raises(lib.SidpError):
                h.sync()
            np.testing.assert_array_equal(before[0], h.key_codes())
            np.testing.assert_array_equal(before[1], h.value_codes())
        before = k.clone()
        lib.sidp_kv8_read(h.h, 0, 2, None, dev([nblk * BS, 7]), k, None)
        with pytest.raises(lib.SidpError):
            h.sync()
        assert torch.equal(k[0], before[0])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_rows_past_2_to_the_31(lib, kind):
    """The last blocks of a cache of more than 2^32 bytes a side."""
    D, hkv = 128, 8
    nblk = (1 << 32) // (hkv * D * BS) + 40
    with Handle8(lib, cfg_of(8, hkv, D), 64, nblk, kind, fill=FILL) as h:
        rows = 40
        qkv = rows_of(8, hkv, D, rows, 2)
        slots = np.arange(nblk * BS - rows, nblk * BS)
        append(lib, h, qkv.cuda(), slots, np.zeros(rows, int))
        k, v = (torch.zeros(rows, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lib.sidp_kv8_read(h.h, 0, rows, None, dev(slots), k, v)
        h.sync()
        x = f64(qkv).reshape(rows, -1, D)
        for got, want in ((k, x[:, 8:16]), (v, x[:, 16:])):
            s = scale_of(want, kind)
            tol = half_step(want, s, kind) * (1 + 2.0 ** -20) + 2.0 ** -8 * np.abs(want) * 1.1
            assert np.all(np.abs(f64(got) - want) <= tol)
        assert torch.all(h.v8[0, :nblk - 4] == FILL)


def test_captured_appends_and_reads(lib):
    """Append and read captured into a graph, replayed with other rows, slots and counts."""
    hq, hkv, D, rows, nblk = 8, 2, 64, 33, 9
    with Handle8(lib, cfg_of(hq, hkv, D), 100, nblk, "e4m3", fill=FILL) as h, Handle8(lib, cfg_of(hq, hkv, D), 100, nblk, "e4m3", fill=FILL) as e:
        qkv, pos, slots = rows_of(hq, hkv, D, rows, 1).cuda(), dev(np.arange(rows)), dev(slots_of("run", rows, nblk))
        count = dev([rows])
        out = [torch.zeros(rows, n, D, dtype=torch.bfloat16, device="cuda") for n in (hq, hkv, hkv)]

        def both(h, q, k, v, stream):
            lib.sidp_rope_append_rows8(h.h, qkv, qkv.shape[1], rows, count, pos, slots, None, None, 0, q, stream)
            lib.sidp_kv8_read(h.h, 0, rows, count, slots, k, v, stream)
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        with torch.cuda.graph(g, stream=s):
            both(h, *out, torch.cuda.current_stream())
        for i in range(4):
            qkv.copy_(rows_of(hq, hkv, D, rows, 10 + i))
            slots.copy_(dev(slots_of("scattered", rows, nblk, i)))
            count.fill_(rows - i)
            want = [torch.zeros_like(o) for o in out]
            for o in out:
                o.zero_()
            g.replay()
            both(e, *want, torch.cuda.current_stream())
            h.sync()
            e.sync()
            for a, b in zip(out, want):
                assert torch.equal(a, b)
            assert torch.equal(h.k8, e.k8) and torch.equal(h.v8, e.v8)
            assert torch.equal(h.scales.nan_to_num(9.0), e.scales.nan_to_num(9.0))


def test_refusals(lib):
    E, S = lib.SIDP_EINVAL, lib.SIDP_ESTATE
    cfg = cfg_of(4, 2, 64)
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    with Handle(lib, cfg, 64) as h:
        attach = lambda *a: lib.raw_call("sidp_kv8_attach", h.h, *[ctypes.c_void_p(x) if isinstance(x, int) and x > 1000 else x for x in a])  # noqa: E731
        ap = lambda **k: lib.raw_call("sidp_rope_append_rows8", h.h, *{**dict(qkv=ctypes.c_void_p(p), stride=ctypes.c_int64(512), rows=2,  # noqa: E731
            count=None, pos=ctypes.c_void_p(p), slots=ctypes.c_void_p(p), gq=None, gk=None, region=0, q=ctypes.c_void_p(p), st=None), **k}.values())
        rd = lambda **k: lib.raw_call("sidp_kv8_read", h.h, *{**dict(region=0, rows=2, count=None, slots=ctypes.c_void_p(p),  # noqa: E731
            k=ctypes.c_void_p(p), v=ctypes.c_void_p(p), st=None), **k}.values())
        assert ap() == S and rd() == S  # nothing attached
        for bad in ((0, p, p, p, 2, 1), (3, p, p, p, 2, 1), (1, None, p, p, 2, 1), (1, p, None, p, 2, 1), (1, p, p, None, 2, 1),
                    (1, p + 8, p, p, 2, 1), (1, p, p + 4, p, 2, 1), (1, p, p, p + 8, 2, 1), (1, p, p, p, 0, 1), (1, p, p, p, 2, 0)):
            assert attach(*bad) == E, bad
        assert ap() == S
        assert attach(2, p, p + 8192, p + 16384, 2, 2) == 0
        for bad in (dict(qkv=None), dict(stride=ctypes.c_int64(511)), dict(stride=ctypes.c_int64(516)), dict(rows=-1), dict(rows=(1 << 20) + 1),
                    dict(pos=None), dict(slots=None), dict(q=None), dict(region=2), dict(region=-1), dict(qkv=ctypes.c_void_p(p + 8)),
                    dict(q=ctypes.c_void_p(p + 2))):
            assert ap(**bad) == E, bad
        for bad in (dict(region=2), dict(region=-1), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(slots=None), dict(k=None, v=None),
                    dict(k=ctypes.c_void_p(p + 8)), dict(v=ctypes.c_void_p(p + 2))):
            assert rd(**bad) == E, bad
        assert ap(rows=0) == 0 and rd(rows=0) == 0
        # the bf16 calls still want a bf16 cache
        assert lib.raw_call("sidp_rope_append_rows", h.h, ctypes.c_void_p(p), ctypes.c_int64(512), 2, None, ctypes.c_void_p(p),
                            ctypes.c_void_p(p), None, None, 0, ctypes.c_void_p(p), None) == S
        h.sync()
        # after a HIP error the handle takes no more calls
        lib.sidp_debug_inject_hip_error(h.h, 719)
        assert rd() == lib.SIDP_EHIP and rd() == S and ap() == S and attach(1, p, p, p, 1, 1) == S
