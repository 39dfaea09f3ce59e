"""Rotary positions of every layout, part and scaling, in the append of many rows
and in the decode step, against complex multiplication in 64 bits."""

import numpy as np
import pytest
import torch

import oracle
import synth
from gpu_helpers import Stack, assert_bf16_within_ulp, bits, f64
from rows_helpers import BS, Handle, cfg_of, dev, turn

pytestmark = pytest.mark.gpu

SCALES = {
    "none": dict(theta=1e4),
    "linear": dict(theta=1e4, scaling="linear", factor=4.0),
    "llama3": dict(theta=5e5, scaling="llama3", factor=8.0, original_len=8192),
    "yarn": dict(theta=1e6, scaling="yarn", factor=4.0, original_len=32768),
}


def inputs(cfg, rows, nblk, max_seq, seed, stride=None, holes=False):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    heads, D = cfg["num_q_heads"] + 2 * cfg["num_kv_heads"], cfg["head_dim"]
    stride = stride or heads * D
    qkv = torch.randn(rows, stride, generator=g).to(torch.bfloat16)
    pos = rng.integers(0, max_seq, rows)
    pos[0] = max_seq - 1
    slots = rng.permutation(nblk * BS)[:rows]
    if holes:
        slots[rng.random(rows) < 0.3] = -1
    gq = (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16)
    gk = (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16)
    return qkv, pos, slots, gq, gk


def want_rows(cfg, qkv, pos, gq, gk, freqs, scale, interleaved):
    hq, hkv, D = cfg["num_q_heads"], cfg["num_kv_heads"], cfg["head_dim"]
    x = f64(qkv)[:, :(hq + 2 * hkv) * D].reshape(len(qkv), -1, D)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if cfg["qk_norm"]:
        q = oracle.rms_norm(q, f64(gq), cfg["qk_norm_eps"])
        k = oracle.rms_norm(k, f64(gk), cfg["qk_norm_eps"])
    return turn(q, pos, freqs, scale, interleaved), turn(k, pos, freqs, scale, interleaved), v


def tol(x, scale):
    """fp32 evaluation: the table's rounding and three roundings of a turned pair, each 2^-24 of the pair's size, the QK-norm's
    sum of at most 128 squares (2^-21 relative at worst): 2^-19 of the largest value covers both components."""
    return 2.0 ** -19 * np.max(np.abs(x)) * scale


@pytest.mark.parametrize("heads", [(4, 2, 64, 0), (8, 8, 64, 1), (8, 1, 128, 0), (5, 1, 128, 1), (64, 8, 128, 1)])
@pytest.mark.parametrize("layout,part,scaling", [("half", 1.0, "none"), ("half", 1.0, "llama3"), ("half", 0.25, "linear"),
                                                ("half", 0.75, "yarn"), ("interleaved", 1.0, "yarn"),
                                                ("interleaved", 0.25, "llama3"), ("interleaved", 0.5, "none")])
@pytest.mark.parametrize("rows", [1, 37])
def test_rope_rows_match_the_definition(lib, heads, layout, part, scaling, rows):
    cfg = cfg_of(*heads)
    D, nblk, max_seq = cfg["head_dim"], 6, 5000
    rot = int(D * part)
    with Handle(lib, cfg, max_seq, nblk, regions=2, fill=3.0) as h:
        rope = lib.make_rope(layout=layout, rotary_dim=rot, **SCALES[scaling])
        lib.sidp_set_rope(h.h, rope)
        freqs, scale = lib.sidp_rope_frequencies(rope, D)
        width = (heads[0] + 2 * heads[1]) * D
        qkv, pos, slots, gq, gk = inputs(cfg, rows, nblk, max_seq, rows, stride=width + 24, holes=rows > 1)
        q_out = torch.full((rows + 1, heads[0], D), 5.0, dtype=torch.bfloat16, device="cuda")
        before_k, before_v = h.k.clone(), h.v.clone()
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), width + 24, rows, None, dev(pos), dev(slots), gq.cuda(), gk.cuda(), 1, q_out)
        h.sync()
        q, k, v = want_rows(cfg, qkv, pos, gq, gk, freqs, scale, layout == "interleaved")
        assert_bf16_within_ulp(bits(q_out[:rows]), q, what="q", abs_tol=tol(q, scale))
        kept = slots >= 0
        assert_bf16_within_ulp(bits(h.keys(1)[torch.as_tensor(slots[kept])]), k[kept], what="k", abs_tol=tol(k, scale))
        assert np.array_equal(f64(h.values(1)[torch.as_tensor(slots[kept])]), v[kept])
        # nothing else is written: other slots, the other region, the row behind the last
        assert torch.all(q_out[rows] == 5.0)
        untouched = torch.ones(nblk * BS, dtype=torch.bool)
        untouched[torch.as_tensor(slots[kept])] = False
        assert torch.all(h.keys(1)[untouched.cuda()] == 3.0) and torch.all(h.values(1)[untouched.cuda()] == 3.0)
        assert torch.equal(h.k[0], before_k[0]) and torch.equal(h.v[0], before_v[0])


@pytest.mark.parametrize("rows", [63, 64, 65, 257, 2100])
@pytest.mark.parametrize("start", [0, 5, 8, 15])
def test_rope_rows_of_whole_prompts(lib, rows, start):
    """Consecutive positions in consecutive slots of scattered blocks, as prompts bring them, from any offset in a block."""
    cfg = cfg_of(8, 4, 128)
    nblk = (rows + start) // BS + 3
    with Handle(lib, cfg, 4096, nblk, fill=3.0) as h:
        rng = np.random.default_rng(rows)
        table = rng.permutation(nblk)
        pos = np.arange(start, start + rows)
        slots = table[pos // BS] * BS + pos % BS
        qkv, _, _, gq, gk = inputs(cfg, rows, nblk, 4096, rows)
        q_out = torch.zeros(rows, 8, 128, dtype=torch.bfloat16, device="cuda")
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), 16 * 128, rows, None, dev(pos), dev(slots), None, None, 0, q_out)
        h.sync()
        freqs = 1e4 ** (-np.arange(64) / 64)
        q, k, v = want_rows(cfg, qkv, pos, gq, gk, freqs, 1.0, False)
        assert_bf16_within_ulp(bits(q_out), q, what="q", abs_tol=tol(q, 1))
        at = torch.as_tensor(slots)
        assert_bf16_within_ulp(bits(h.keys()[at]), k, what="k", abs_tol=tol(k, 1))
        assert np.array_equal(f64(h.values()[at]), v)
        untouched = torch.ones(nblk * BS, dtype=torch.bool)
        untouched[at] = False
        assert torch.all(h.keys()[untouched.cuda()] == 3.0) and torch.all(h.values()[untouched.cuda()] == 3.0)


@pytest.mark.parametrize("heads", [(4, 2, 64, 1), (5, 1, 128, 0)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_rows_of_long_calls_are_those_of_short_ones(lib, heads, layout):
    """Many rows at random places in one call and in calls of a hundred: the same bits."""
    cfg, rows, nblk = cfg_of(*heads), 2200, 150
    with Handle(lib, cfg, 5000, nblk, fill=3.0) as h:
        lib.sidp_set_rope(h.h, lib.make_rope(layout=layout, rotary_dim=heads[2] // 2, theta=1e4))
        qkv, pos, slots, gq, gk = inputs(cfg, rows, nblk, 5000, 11, holes=True)
        qkv, pos, slots, gq, gk = qkv.cuda(), dev(pos), dev(slots), gq.cuda(), gk.cuda()
        out = torch.zeros(2, rows, heads[0], heads[2], dtype=torch.bfloat16, device="cuda")
        lib.sidp_rope_append_rows(h.h, qkv, qkv.shape[1], rows, None, pos, slots, gq, gk, 0, out[0])
        h.sync()
        k, v = h.k.clone(), h.v.clone()
        h.k.fill_(3.0)
        h.v.fill_(3.0)
        for a in range(0, rows, 100):
            b = a + 100
            lib.sidp_rope_append_rows(h.h, qkv[a:b], qkv.shape[1], 100, None, pos[a:b], slots[a:b], gq, gk, 0, out[1, a:b])
        h.sync()
        assert torch.equal(out[0], out[1]) and torch.equal(h.k, k) and torch.equal(h.v, v)


@pytest.mark.parametrize("count", [-3, 0, 1, 70, 200, 1000])
def test_rope_rows_in_use_are_read_on_the_device(lib, count):
    cfg, rows = cfg_of(4, 2, 64), 200
    with Handle(lib, cfg, 512, 20, fill=3.0) as h:
        qkv, pos, slots, _, _ = inputs(cfg, rows, 20, 512, 3)
        out = [torch.full((rows, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), 512, rows, None, dev(pos), dev(slots), None, None, 0, out[0])
        h.sync()
        k, v = h.keys().clone(), h.values().clone()
        h.k.fill_(3.0)
        h.v.fill_(3.0)
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), 512, rows, dev([count]), dev(pos), dev(slots), None, None, 0, out[1])
        h.sync()
        n = min(rows, max(0, count))
        assert torch.equal(out[1][:n], out[0][:n]) and torch.all(out[1][n:] == 5.0)
        used, rest = torch.as_tensor(slots[:n]), torch.as_tensor(slots[n:])
        assert torch.equal(h.keys()[used], k[used]) and torch.equal(h.values()[used], v[used])
        assert torch.all(h.keys()[rest] == 3.0) and torch.all(h.values()[rest] == 3.0)


def test_rope_rows_with_bad_places_leave_the_others(lib):
    cfg, rows = cfg_of(4, 2, 64), 80
    with Handle(lib, cfg, 512, 20, fill=3.0) as h:
        qkv, pos, slots, _, _ = inputs(cfg, rows, 20, 512, 3)
        good = torch.zeros(rows, 4, 64, dtype=torch.bfloat16, device="cuda")
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), 512, rows, None, dev(pos), dev(slots), None, None, 0, good)
        h.sync()
        k, v = h.keys().clone(), h.values().clone()
        h.k.fill_(3.0)
        h.v.fill_(3.0)
        bad_pos, bad_slots = pos.copy(), slots.copy()
        bad_pos[[3, 50]] = [-1, 512]
        bad_slots[[4, 51, 79]] = [320, 2147483647, -7]
        out = torch.full((rows, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), 512, rows, None, dev(bad_pos), dev(bad_slots), None, None, 0, out)
        with pytest.raises(lib.SidpError) as e:
            h.sync()
        assert e.value.code == lib.SIDP_EINVAL
        h.sync()
        left_out = torch.tensor([3, 50], device="cuda")
        assert torch.all(out[left_out] == 5.0)
        written = torch.ones(rows, dtype=torch.bool, device="cuda")
        written[left_out] = False
        assert torch.equal(out[written], good[written])  # a row without a place still gets its query
        cached = [r for r in range(rows) if r not in (3, 4, 50, 51, 79)]
        at, rest = torch.as_tensor(slots[cached]), torch.as_tensor(slots[[3, 4, 50, 51, 79]])
        assert torch.equal(h.keys()[at], k[at]) and torch.equal(h.values()[at], v[at])
        assert torch.all(h.keys()[rest] == 3.0) and torch.all(h.values()[rest] == 3.0)


@pytest.mark.parametrize("heads", [(4, 2, 64, 0), (64, 8, 128, 1)])
@pytest.mark.parametrize("layout,part,scaling", [("half", 1.0, "none"), ("half", 1.0, "yarn"), ("half", 0.5, "none"),
                                                ("interleaved", 1.0, "llama3")])
def test_single_token_append_gives_the_same_bits(lib, heads, layout, part, scaling):
    cfg, rows, nblk = cfg_of(*heads), 30, 40
    D = cfg["head_dim"]
    with Handle(lib, cfg, 512, nblk, regions=2) as h:
        lib.sidp_destroy(h.h)
        h.h = lib.sidp_create(lib.make_config(cfg, rows, 512))
        lib.sidp_kv_attach(h.h, h.k, h.v, nblk, 2)
        lib.sidp_set_rope(h.h, lib.make_rope(layout=layout, rotary_dim=int(D * part), **SCALES[scaling]))
        qkv, pos, _, gq, gk = inputs(cfg, rows, nblk, 512, 5)
        pos = pos % 16
        table = np.random.default_rng(1).permutation(nblk)[:rows]
        args = (dev(pos), dev(table[:, None]), 1, rows)
        out = [torch.zeros(rows, heads[0], D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        lib.sidp_rope_append(h.h, qkv.cuda(), *args, gq.cuda(), gk.cuda(), 0, out[0])
        lib.sidp_rope_append_rows(h.h, qkv.cuda(), qkv.shape[1], rows, None, dev(pos), dev(table * BS + pos), gq.cuda(), gk.cuda(),
                                  1, out[1])
        h.sync()
        assert torch.equal(out[0], out[1]) and torch.equal(h.k[0], h.k[1]) and torch.equal(h.v[0], h.v[1])


@pytest.mark.parametrize("layout,part,scaling", [("half", 0.5, "linear"), ("interleaved", 1.0, "llama3"), ("half", 1.0, "yarn")])
def test_decode_steps_use_the_rope_and_lose_it_again(lib, layout, part, scaling):
    """The key that a step's first layer caches, and streamed steps against resident ones, bit for bit."""
    cfg = synth.get_config("tiny_layer", num_layers=2)
    st = Stack(cfg, gains="random", regions=2)
    try:
        def step(flags):
            st.reset()
            st.dec.step(st.hidden, st.positions, st.bt, flags, copy=torch.cuda.Stream())
            st.dec.sync()
            return st.hidden.clone(), st.dec.k_cache.clone()

        first = step(lib.SIDP_RESIDENT)
        rope = lib.make_rope(layout=layout, rotary_dim=int(64 * part), **SCALES[scaling])
        st.dec.set_rope(rope)
        resident, streamed = step(lib.SIDP_RESIDENT), step(lib.SIDP_STREAMED)
        assert torch.equal(resident[0], streamed[0]) and torch.equal(resident[1], streamed[1])
        assert not torch.equal(resident[1], first[1])
        w = st.layer_weights(0)
        x = oracle.round_to_bf16(oracle.rms_norm(st.x0.double().cpu().numpy(), oracle.bf16_bits_to_f64(w["g_attn"]), cfg["rms_eps"]))
        k = oracle.round_to_bf16(x @ oracle.bf16_bits_to_f64(w["w_k"]).T).reshape(st.batch, 2, 64)
        freqs, scale = lib.sidp_rope_frequencies(rope, 64)
        want = turn(k, st.ctx, freqs, scale, layout == "interleaved")
        tables = np.asarray(st.tables)
        nat = st.dec.k_natural(0)  # [block][head][token][d]
        got = np.stack([f64(nat[int(tables[b, c // 16]), :, c % 16]) for b, c in enumerate(st.ctx)])
        # the projection's sum may round to the other bf16 neighbour, two halves of a pair at once
        assert np.max(np.abs(got - want)) <= 2.0 ** -6 * scale * np.max(np.abs(k))
        st.dec.set_rope(None)
        again = step(lib.SIDP_RESIDENT)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    finally:
        st.close()


def test_rope_rows_captured_and_replayed(lib):
    cfg, rows = cfg_of(8, 2, 128), 90
    with Handle(lib, cfg, 512, 20) as h:
        qkv, pos, slots, _, _ = inputs(cfg, rows, 20, 512, 3)
        x, p, sl, n = qkv.cuda(), dev(pos), dev(slots), dev([rows])
        out, ref = (torch.zeros(rows, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            lib.sidp_rope_append_rows(h.h, x, x.shape[1], rows, n, p, sl, None, None, 0, out, torch.cuda.current_stream())
        for i in range(3):
            x.copy_(torch.randn(x.shape, device="cuda"))
            p.copy_((p + 1) % 512)
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            k = h.k.clone()
            lib.sidp_rope_append_rows(h.h, x, x.shape[1], rows, n, p, sl, None, None, 0, ref)
            h.sync()
            assert torch.equal(out, ref) and torch.equal(h.k, k)


def test_rope_rows_refusals(lib):
    cfg = cfg_of(4, 2, 64, qk_norm=1)
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    i = dev([0] * 8)
    with Handle(lib, cfg, 64, 4) as h:
        def rc(handle=h.h, x=t.data_ptr(), stride=512, rows=1, pos=i.data_ptr(), slots=i.data_ptr(), gq=t.data_ptr(),
               gk=t.data_ptr(), region=0, out=t.data_ptr()):
            return lib.raw_call("sidp_rope_append_rows", handle, x, stride, rows, None, pos, slots, gq, gk, region, out, None)
        E = lib.SIDP_EINVAL
        assert rc(rows=-1) == E and rc(rows=(1 << 20) + 1) == E and rc(stride=511) == E and rc(stride=516) == E
        assert rc(x=None) == E and rc(pos=None) == E and rc(slots=None) == E and rc(out=None) == E
        assert rc(gq=None) == E and rc(gk=None) == E and rc(gq=t.data_ptr() + 2) == E
        assert rc(x=t.data_ptr() + 8) == E and rc(out=t.data_ptr() + 4) == E
        assert rc(region=1) == E and rc(region=-1) == E
        assert rc(rows=0, x=None, pos=None, slots=None, out=None) == lib.SIDP_OK
        with pytest.raises(lib.SidpError):
            lib.sidp_set_rope(h.h, lib.make_rope(rotary_dim=128))
        h.sync()
    with Handle(lib, cfg, 64) as h:
        assert rc(handle=h.h) == lib.SIDP_ESTATE  # no cache attached
