"""Performance cases of the operators of one serving iteration that come after the
calls of perf/operators.py: a KV cache of 8 bits, attention that computes a
prefix shared by several sequences once, and tokens drawn from logits, with the
plain torch form of each.

  cache8   QK-norm, rotary positions and the append of many rows to a cache of
           8-bit codes with a scale for each token and KV head, and those rows
           read back as bf16 (sidp_rope_append_rows8, sidp_kv8_read)
  attn8    causal attention of each sequence's new rows over the 8-bit cache
           (sidp_attention_rows8)
  shared   the same, over either cache, for groups of sequences whose first
           blocks are the same ones (sidp_attention_shared)
  sample   a token of each row of logits, drawn by temperature, top-k, top-p and
           min-p from a given random number (sidp_sample_tokens)

A case holds numbers only; inputs come from the seed alone. Lengths of a case
are evenly spread over its range and dealt out by the seed, so that its work
does not depend on the seed.
"""

import math

import torch

own = False

BS = 16  # tokens per KV block

# query heads, KV heads, head dim, QK-norm (the shapes of synth/configs.py, and few-head ones)
HEADS = {
    "70b": (64, 8, 128, 0),
    "qwen3": (64, 8, 128, 1),
    "tiny": (4, 2, 64, 0),
    "mha": (16, 16, 64, 0),
}


def listed():
    return [
        # A draft model's few rows into an int8 cache: nothing but latency.
        dict(name="cache8_tiny_8", kind="cache8", heads="tiny", type="int8", layout="interleaved", rot=32, batch=8, clo=16,
             chi=64, nlo=1, nhi=1),
        # A decode iteration's keys and values, QK-norm: a token each of the headline batch.
        dict(name="cache8_qwen3_256", kind="cache8", heads="qwen3", type="e4m3", layout="half", rot=128, batch=256,
             clo=1024, chi=8000, nlo=1, nhi=1),
        # Prompt chunks of a prefill iteration, ragged.
        dict(name="cache8_70b_prompts", kind="cache8", heads="70b", type="e4m3", layout="half", rot=128, batch=8, clo=0,
             chi=2000, nlo=300, nhi=1748),
        # A decode iteration: a token each over long caches, bound by the cache's bytes.
        dict(name="attn8_decode_64", kind="attn8", heads="70b", type="e4m3", batch=64, clo=1024, chi=8190, nlo=1, nhi=1),
        # Drafted tokens checked against an int8 cache.
        dict(name="attn8_verify_16", kind="attn8", heads="70b", type="int8", batch=16, clo=512, chi=4091, nlo=1, nhi=7),
        # Ragged prompt chunks over what is cached of them: bound by the matrix units.
        dict(name="attn8_chunks_8", kind="attn8", heads="70b", type="e4m3", batch=8, clo=0, chi=4096, nlo=1, nhi=1021),
        # Eight answers of one prompt, the first tokens: the smallest call.
        dict(name="shared_8", kind="shared", heads="70b", type="bf16", groups=1, batch=8, plo=2048, phi=2048, clo=0, chi=60,
             nlo=1, nhi=1),
        # Several prompts with several drafted answers each, in the 8-bit cache, odd lengths.
        dict(name="shared_groups8", kind="shared", heads="70b", type="e4m3", groups=6, batch=72, plo=500, phi=3500, clo=1,
             chi=777, nlo=1, nhi=3),
        # The headline batch under one long instruction.
        dict(name="shared_256", kind="shared", heads="70b", type="bf16", groups=1, batch=256, plo=8192, phi=8192, clo=0,
             chi=1000, nlo=1, nhi=1),
        # The next token of a single sequence.
        dict(name="sample_1", kind="sample", rows=1, vocab=128256, pad=0, f32=False, k=0.99, p=0.99, m=0.0, cold=0.0,
             masked=0.0),
        # A decode iteration's tokens from fp32 logits: every user's own settings, some greedy, some under a grammar's mask.
        dict(name="sample_256", kind="sample", rows=256, vocab=151936, pad=128, f32=True, k=0.5, p=0.5, m=0.25, cold=0.1,
             masked=0.2),
        # Many samples at a temperature and nothing else, an odd vocabulary.
        dict(name="sample_512_plain", kind="sample", rows=512, vocab=32001, pad=0, f32=False, k=0.0, p=0.0, m=0.0, cold=0.0,
             masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cache8", "attn8", "attn8", "shared", "shared", "sample", "sample"])
    if kind == "cache8":
        heads = rng.choice(["70b", "qwen3", "tiny", "mha"])
        D = HEADS[heads][2]
        batch = _log_int(rng, 1, 256)
        nhi = min(_log_int(rng, 1, 4096), 8192 // batch)
        clo = rng.choice([0, _log_int(rng, 1, 20000)])
        return dict(kind=kind, heads=heads, type=rng.choice(["e4m3", "int8"]), layout=rng.choice(["half", "interleaved"]),
                    rot=rng.choice([16 * rng.randint(1, D // 16), D]), batch=batch, clo=clo, chi=clo + _log_int(rng, 1, 4000),
                    nlo=rng.randint(1, nhi), nhi=nhi)
    if kind == "attn8":
        heads = rng.choice(["70b", "70b", "tiny", "mha"])
        hq = HEADS[heads][0]
        batch = _log_int(rng, 1, 64)
        nhi = min(_log_int(rng, 1, 1024), 8192 // batch)
        # the whole rectangle of scores stays below the largest listed one
        most = min(64 * 8192 * 4096 // (batch * nhi * hq) - nhi, 32768, 400000 // batch)
        chi = _log_int(rng, 1, max(1, most))
        return dict(kind=kind, heads=heads, type=rng.choice(["e4m3", "int8"]), batch=batch, clo=rng.randint(0, chi), chi=chi,
                    nlo=rng.choice([nhi, rng.randint(batch < 2, nhi)]), nhi=nhi)
    if kind == "shared":
        heads = rng.choice(["70b", "70b", "tiny", "mha"])
        batch = _log_int(rng, 2, 256)
        phi = _log_int(rng, 16, 8192)
        chi = _log_int(rng, 1, max(1, min(4000, 256 * 9000 // batch - phi)))
        return dict(kind=kind, heads=heads, type=rng.choice(["bf16", "bf16", "e4m3", "int8"]), groups=_log_int(rng, 1, min(batch, 16)),
                    batch=batch, plo=rng.randint(1, phi), phi=phi, clo=rng.randint(0, chi), chi=chi, nlo=rng.randint(0, 1),
                    nhi=rng.randint(1, 4) if batch < 64 else 1)
    vocab = rng.choice([_log_int(rng, 1000, 160000), 128256, 151936])
    rows = _log_int(rng, 1, min(512, 256 * 151936 // vocab))
    return dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, rng.randint(1, 64)]), f32=rng.random() < 0.5,
                k=rng.choice([0.0, 0.5, 1.0]), p=rng.choice([0.0, 0.5, 1.0]), m=rng.choice([0.0, 0.5]),
                cold=rng.choice([0.0, 0.2]), masked=rng.choice([0.0, 0.5]))


# ---------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + salt * 7919 + 31) & ((1 << 62) - 1))
    return g


def _randn(shape, seed, salt, std=1.0):
    t = torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=torch.float32)
    return t.mul_(std).to(torch.bfloat16)


def _rand(shape, seed, salt):
    return torch.rand(shape, generator=_gen(seed, salt), device="cuda")


def _lens(lo, hi, n):
    """n lengths evenly spread over [lo, hi]."""
    return [lo + ((hi - lo) * i) // max(1, n - 1) for i in range(n)]


def _dealt(lo, hi, n, seed, salt):
    g = torch.Generator()
    g.manual_seed((seed * 1_000_003 + salt * 104729 + 3) & ((1 << 62) - 1))
    v = torch.tensor(_lens(lo, hi, n), dtype=torch.int32)
    return v[torch.randperm(n, generator=g)]


def _sizes(case):
    """Sequences of each group: as even as they can be, the first ones longer."""
    n, B = case.get("groups", 0), case["batch"]
    return [B // n + (i < B % n) for i in range(n)]


def _paged(case, seed):
    """Request lengths and block tables, the new tokens' blocks among them, blocks in random order. In a case with groups the first
    blocks of a group's sequences are the same."""
    B = case["batch"]
    tail, new = _dealt(case["clo"], case["chi"], B, seed, 1), _dealt(case["nlo"], case["nhi"], B, seed, 2)
    sizes = torch.tensor(_sizes(case), dtype=torch.int64)
    groups = sizes.numel()
    if groups:
        prefix = _dealt(case["plo"], case["phi"], groups, seed, 4).long()
        held = prefix // BS  # whole blocks are shared; the tail of the prefix is each sequence's own
        group = torch.repeat_interleave(torch.arange(groups), sizes)
        ctx = (tail.long() + prefix[group]).to(torch.int32)
    else:
        prefix, held = torch.zeros(0, dtype=torch.int64), torch.zeros(1, dtype=torch.int64)
        group = torch.zeros(B, dtype=torch.int64)
        ctx = tail
    alone = (ctx + new + BS - 1).long() // BS - held[group]
    width = int((alone + held[group]).max()) + 2
    total = int(alone.sum() + held.sum()) + 5
    perm = torch.randperm(total, generator=_gen(seed, 3), device="cuda").to(torch.int32)
    first_shared = torch.cumsum(held, 0) - held
    first_alone = torch.cumsum(alone, 0) - alone + held.sum()
    col = torch.arange(width)[None, :]
    in_prefix = col < held[group][:, None]
    at = torch.where(in_prefix, first_shared[group][:, None] + col, first_alone[:, None] + col - held[group][:, None])
    mine = col < (alone + held[group])[:, None]
    tables = torch.where(mine.cuda(), perm[at.clamp_(max=total - 1).cuda()], torch.full((), -1, dtype=torch.int32, device="cuda"))
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.cumsum(new, 0)
    gstarts = torch.zeros(groups + 1, dtype=torch.int32)
    gstarts[1:] = torch.cumsum(sizes, 0)
    return dict(B=B, rows=int(starts[-1]), nblk=total, width=width, ctx=ctx.cuda(), new=new.cuda(), starts=starts.cuda(),
                tables=tables.contiguous(), longest_new=int(new.max()), longest=int((ctx + new).max()), groups=groups,
                gstarts=gstarts.cuda(), shared=(held * BS).to(torch.int32).cuda() if groups else None)


def _row_places(p):
    """Position and cache slot of every new row."""
    seq = torch.repeat_interleave(torch.arange(p["B"], device="cuda"), p["new"].long(), output_size=p["rows"])
    pos = p["ctx"].long()[seq] + torch.arange(p["rows"], device="cuda") - p["starts"].long()[seq]
    return pos, p["tables"].long()[seq, pos // BS] * BS + pos % BS


def _quantised(x, kind):
    """Codes and scales of vectors along the last axis, fp32. e4m3: the least power of two that brings the largest magnitude to 448 =
    0.875 * 2^9 at most; int8: the largest magnitude over 127."""
    most = x.abs().amax(-1, keepdim=True)
    if kind == "e4m3":
        m, e = torch.frexp(most)
        scale = torch.ldexp(torch.ones_like(most), (e - 9 + (m > 0.875)).clamp(min=-126))
        return (x / scale).to(torch.float8_e4m3fn).view(torch.uint8), scale.squeeze(-1)
    scale = (most / 127.0).clamp(min=2.0 ** -126)
    return torch.round(x / scale).clamp(-127, 127).to(torch.int8).view(torch.uint8), scale.squeeze(-1)


def _values(codes, kind):
    return codes.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).float()


class _Handle:
    """A library handle, with the given caches attached; freed with its state."""

    def __init__(self, heads, max_seq_len, s, kind):
        import paper_2605_28095_amd as sidp
        hq, hkv, D, norm = HEADS[heads]
        cfg = dict(num_layers=1, hidden=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, ffn_dim=64, qkv_bias=0,
                   qk_norm=norm, rms_eps=1e-6, qk_norm_eps=1e-6, rope_theta=1e4, block_size=BS)
        self.sidp = sidp
        self.h = None
        self.h = sidp.sidp_create(sidp.make_config(cfg, 1, max_seq_len))
        if kind == "bf16":
            sidp.sidp_kv_attach(self.h, s["k"], s["v"], s["nblk"], 1)
        else:
            sidp.sidp_kv8_attach(self.h, sidp.SIDP_KV_E4M3 if kind == "e4m3" else sidp.SIDP_KV_INT8, s["k"], s["v"],
                                 s["scales"], s["nblk"], 1)

    def __del__(self):
        if self.h is not None:
            self.sidp.sidp_destroy(self.h)
            self.h = None


def _caches(nblk, hkv, D, kind, seed):
    """One region of a cache of normal keys and values in the library's layouts: bf16 K [block][head][d / 8][token][d % 8], V
    [block][head][d][token]; 8 bits the same with 16 dims a piece, and scales [block][head][K, V][token]."""
    k, v = _randn((nblk, hkv, BS, D), seed, 10), _randn((nblk, hkv, BS, D), seed, 11)
    if kind == "bf16":
        return dict(k=k.view(nblk, hkv, BS, D // 8, 8).transpose(2, 3).contiguous(), v=v.transpose(2, 3).contiguous())
    kc, ks = _quantised(k.float(), kind)
    vc, vs = _quantised(v.float(), kind)
    return dict(k=kc.view(nblk, hkv, BS, D // 16, 16).transpose(2, 3).contiguous(), v=vc.transpose(2, 3).contiguous(),
                scales=torch.stack([ks, vs], 2).contiguous())


def _prepare_cache8(case, seed):
    hq, hkv, D, norm = HEADS[case["heads"]]
    p = _paged(case, seed)
    pos, slot = _row_places(p)
    s = dict(case=case, rows=p["rows"], nblk=p["nblk"], positions=pos.to(torch.int32), slots=slot.to(torch.int32))
    s |= _caches(p["nblk"], hkv, D, case["type"], seed)
    s["qkv"] = _randn((p["rows"], (hq + 2 * hkv) * D), seed, 12)
    s["g_q"] = (1 + _randn((D,), seed, 13, 0.1).float()).to(torch.bfloat16) if norm else None
    s["g_k"] = (1 + _randn((D,), seed, 14, 0.1).float()).to(torch.bfloat16) if norm else None
    for name, heads in (("q_out", hq), ("k_out", hkv), ("v_out", hkv)):
        s[name] = torch.zeros((p["rows"], heads, D), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2605_28095_amd as sidp
        s["handle"] = _Handle(case["heads"], p["longest"], s, case["type"])
        sidp.sidp_set_rope(s["handle"].h, sidp.make_rope(layout=case["layout"], rotary_dim=case["rot"], theta=1e4))
    else:
        inv = 1e4 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        angle = torch.arange(p["longest"], dtype=torch.float64, device="cuda")[:, None] * inv[None, :]
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def _prepare_attn(case, seed):
    hq, hkv, D, _ = HEADS[case["heads"]]
    p = _paged(case, seed)
    s = dict(p, case=case, q=_randn((p["rows"], hq, D), seed, 15, 1.5))
    s |= _caches(p["nblk"], hkv, D, case["type"], seed)
    s["out"] = torch.zeros((p["rows"], hq, D), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2605_28095_amd as sidp
        h = s["handle"] = _Handle(case["heads"], max(64, p["longest"]), s, case["type"])
        most = max(1, p["rows"])
        if case["kind"] == "shared":
            s["cache"] = sidp.SIDP_CACHE_BF16 if case["type"] == "bf16" else sidp.SIDP_CACHE_8BIT
            size = sidp.sidp_attention_shared_bytes(h.h, s["cache"], p["B"], most)
        else:
            size = sidp.sidp_attention_rows8_bytes(h.h, p["B"], most)
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


def _prepare_sample(case, seed):
    R, V = case["rows"], case["vocab"]
    x = torch.randn((R, V + case["pad"]), generator=_gen(seed, 20), device="cuda")
    x *= 0.5 + 2.5 * _rand((R, 1), seed, 21)
    likely = torch.randint(0, V, (R, 8), generator=_gen(seed, 22), device="cuda")
    x.scatter_add_(1, likely, 14.0 * _rand((R, 1), seed, 23) * _rand((R, 8), seed, 24))  # a handful of tokens that the model has in mind
    if case["masked"]:
        under = _rand((R, 1), seed, 25) < case["masked"]
        out = _rand((R, V + case["pad"]), seed, 26) < 0.995
        out.scatter_(1, likely, False)
        x.masked_fill_(under & out, -math.inf)
    pick = lambda share, salt: _rand((R,), seed, salt) < share  # noqa: E731
    off = torch.zeros(R, device="cuda")
    s = dict(case=case, logits=x.to(torch.float32 if case["f32"] else torch.bfloat16))
    s["temperature"] = torch.where(pick(case["cold"], 27), off, 0.5 + _rand((R,), seed, 28))
    s["top_k"] = torch.where(pick(case["k"], 29), torch.randint(1, 200, (R,), generator=_gen(seed, 30), device="cuda"), 0).to(torch.int32)
    s["top_p"] = torch.where(pick(case["p"], 31), 0.5 + 0.49 * _rand((R,), seed, 32), off + 1)
    s["min_p"] = torch.where(pick(case["m"], 33), 0.2 * _rand((R,), seed, 34), off)
    s["uniform"] = _rand((R,), seed, 35)
    s["token"] = torch.zeros(R, dtype=torch.int32, device="cuda")
    s["kept"] = torch.zeros(R, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.zeros(R, device="cuda")
    if own:
        import paper_2605_28095_amd as sidp
        s["ws"] = torch.empty(sidp.sidp_sample_tokens_bytes(R, V), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return {"cache8": _prepare_cache8, "attn8": _prepare_attn, "shared": _prepare_attn, "sample": _prepare_sample}[case["kind"]](case, seed)


# ---------------------------------------------------------------- one pass

def _cache8(s):
    c = s["case"]
    hq, hkv, D, norm = HEADS[c["heads"]]
    R, rot, kind = s["rows"], c["rot"], c["type"]
    x = s["qkv"].float().view(R, hq + 2 * hkv, D)
    qk, v = x[:, :hq + hkv], x[:, hq + hkv:]
    if norm:
        gain = torch.cat([s["g_q"].float().expand(hq, D), s["g_k"].float().expand(hkv, D)])
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + 1e-6) * gain
    cos, sin = s["cos"][s["positions"].long()][:, None, :], s["sin"][s["positions"].long()][:, None, :]
    if c["layout"] == "half":
        a, b = qk[..., :rot // 2], qk[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin, qk[..., rot:]], -1)
    else:
        a, b = qk[..., 0:rot:2], qk[..., 1:rot:2]
        turned = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), qk[..., rot:]], -1)
    blk, off = s["slots"].long() // BS, s["slots"].long() % BS
    kc, ks = _quantised(turned[:, hq:], kind)
    vc, vs = _quantised(v, kind)
    s["k"][blk, :, :, off, :] = kc.view(R, hkv, D // 16, 16)
    s["v"][blk, :, :, off] = vc
    s["scales"][blk, :, 0, off] = ks
    s["scales"][blk, :, 1, off] = vs
    k_back = _values(s["k"][blk, :, :, off, :].reshape(R, hkv, D), kind) * s["scales"][blk, :, 0, off][..., None]
    v_back = _values(s["v"][blk, :, :, off], kind) * s["scales"][blk, :, 1, off][..., None]
    return dict(q=turned[:, :hq].to(torch.bfloat16), k=k_back.to(torch.bfloat16), v=v_back.to(torch.bfloat16))


def _cache8_own(s):
    import paper_2605_28095_amd as sidp
    h, stream = s["handle"].h, torch.cuda.current_stream()
    sidp.sidp_rope_append_rows8(h, s["qkv"], s["qkv"].shape[1], s["rows"], None, s["positions"], s["slots"], s["g_q"], s["g_k"],
                                0, s["q_out"], stream)
    sidp.sidp_kv8_read(h, 0, s["rows"], None, s["slots"], s["k_out"], s["v_out"], stream)
    return dict(q=s["q_out"], k=s["k_out"], v=s["v_out"])


def _attn(s):
    c = s["case"]
    hq, hkv, D, _ = HEADS[c["heads"]]
    B, n, G, kind = s["B"], max(1, s["longest_new"]), hq // hkv, c["type"]
    S = s["width"] * BS
    tables = s["tables"].long().clamp(min=0)
    # [B][head][d][token], [B][head][token][d]
    if kind == "bf16":
        k = s["k"][tables].permute(0, 2, 3, 5, 1, 4).reshape(B, hkv, D, S).float()
        v = s["v"][tables].permute(0, 2, 1, 4, 3).reshape(B, hkv, S, D).float()
    else:
        scales = s["scales"][tables].permute(3, 0, 2, 1, 4).reshape(2, B, hkv, S)
        k = _values(s["k"][tables].permute(0, 2, 3, 5, 1, 4).reshape(B, hkv, D, S), kind).mul_(scales[0][:, :, None, :])
        v = _values(s["v"][tables].permute(0, 2, 1, 4, 3).reshape(B, hkv, S, D), kind).mul_(scales[1][..., None])
    i = torch.arange(n, device="cuda")
    row = (s["starts"][:-1, None].long() + i).clamp(max=max(0, s["rows"] - 1))  # the rows of each sequence, padded to the longest
    q = s["q"][row].float().view(B, n, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, D)
    p = torch.matmul(q, k).mul_(1 / math.sqrt(D)).view(B, hkv, n, G, S)
    seen = torch.arange(S, device="cuda") <= (s["ctx"].long()[:, None] + i)[..., None]
    p.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    o = torch.matmul(p.view(B, hkv, n * G, S), v).view(B, hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, hq, D)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), s["new"].long(), output_size=s["rows"])
    at = torch.arange(s["rows"], device="cuda") - s["starts"].long()[seq]
    return o[seq, at].to(torch.bfloat16)


def _attn8_own(s):
    import paper_2605_28095_amd as sidp
    sidp.sidp_attention_rows8(s["handle"].h, s["q"], 0, s["starts"], s["ctx"], s["tables"], s["width"], s["B"], s["rows"],
                              s["out"], s["ws"], s["ws"].numel(), torch.cuda.current_stream())
    return s["out"]


def _shared_own(s):
    import paper_2605_28095_amd as sidp
    sidp.sidp_attention_shared(s["handle"].h, s["cache"], s["q"], 0, s["gstarts"], s["shared"], s["groups"], s["starts"],
                               s["ctx"], s["tables"], s["width"], s["B"], s["rows"], s["out"], s["ws"], s["ws"].numel(),
                               torch.cuda.current_stream())
    return s["out"]


def _sample(s):
    V = s["case"]["vocab"]
    x, order = torch.sort(s["logits"][:, :V].float(), dim=1, descending=True, stable=True)  # of equal ones the lowest first
    cold = s["temperature"] == 0
    heat = torch.where(cold, 1.0, s["temperature"]).double()
    y = (x.double() - x[:, :1].double()) / heat[:, None]
    w = y.exp()
    at = torch.arange(V, device="cuda")[None, :]
    k = torch.where(s["top_k"] > 0, s["top_k"], V).long().clamp(max=V)
    k = torch.where(cold, 1, k)
    cum = w.cumsum(1)
    total = cum.gather(1, k[:, None] - 1)
    keep = (at < k[:, None]) & (w >= s["min_p"].double()[:, None]) & (x > -math.inf)
    ahead = cum - w
    keep &= (ahead < s["top_p"].double()[:, None] * total) | (s["top_p"][:, None] >= 1) | (at == 0)
    kept = keep.sum(1)
    weight = cum.gather(1, kept[:, None] - 1)
    place = torch.minimum((cum <= s["uniform"].double()[:, None] * weight).sum(1), kept - 1)
    logprob = y.gather(1, place[:, None]) - weight.log()
    return dict(token=order.gather(1, place[:, None])[:, 0].to(torch.int32), logprob=logprob[:, 0].float(), kept=kept.to(torch.int32))


def _sample_own(s):
    import paper_2605_28095_amd as sidp
    c = s["case"]
    sidp.sidp_sample_tokens(s["logits"], sidp.SIDP_LOGITS_F32 if c["f32"] else sidp.SIDP_LOGITS_BF16, c["rows"], c["vocab"],
                            s["logits"].shape[1], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["token"],
                            s["logprob"], s["kept"], s["ws"], s["ws"].numel(), torch.cuda.current_stream())
    return dict(token=s["token"], logprob=s["logprob"], kept=s["kept"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"cache8": _cache8_own, "attn8": _attn8_own, "shared": _shared_own, "sample": _sample_own}[kind](state)
    return {"cache8": _cache8, "attn8": _attn, "shared": _attn, "sample": _sample}[kind](state)


# ---------------------------------------------------------------- work

def work(case):
    kind = case["kind"]
    if kind == "sample":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * V * (4 if case["f32"] else 2) + 32 * R, "flops": 4 * R * V}
    B = case["batch"]
    tail, new = _lens(case["clo"], case["chi"], B), _lens(case["nlo"], case["nhi"], B)
    rows = sum(new)
    hq, hkv, D, _ = HEADS[case["heads"]]
    if kind == "cache8":
        # bf16 rows in, queries out, codes and scales out and in, rows out
        return {"bytes": rows * (2 * (hq + 2 * hkv) * D + 2 * hq * D + 2 * hkv * (2 * D + 8) + 4 * hkv * D + 8),
                "flops": rows * (hq + 2 * hkv) * D * 6}
    token = hkv * (4 * D if case["type"] == "bf16" else 2 * D + 8)  # bytes of a cached token
    sizes = _sizes(case)
    prefix = _lens(case["plo"], case["phi"], len(sizes)) if sizes else []
    # the deal pairs lengths, rows and prefixes at random: each at its mean
    before = sum(tail) / B + (sum(prefix) / len(prefix) if prefix else 0)
    once = sum(tail) + rows + sum(prefix)
    return {"bytes": 4 * rows * hq * D + int(token * once), "flops": int(4 * hq * D * sum(n * (before + (n + 1) / 2) for n in new))}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_codes(x, kind):
    """The values that vectors along the last axis, in 64 bits, are held as."""
    most = x.abs().amax(-1, keepdim=True)
    if kind == "int8":
        step = most / 127
        return torch.where(most > 0, torch.round(x / step) * step, 0.0)
    scale = torch.exp2(torch.ceil(torch.log2(most / 448)))
    z = x / scale
    # three bits behind the leading one, down to an exponent of -6
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(most > 0, torch.round(z / step) * step * scale, 0.0)


def _exact_cache8(case, seed):
    hq, hkv, D, norm = HEADS[case["heads"]]
    s = _prepare_cache8(dict(case), seed)
    R, rot = s["rows"], case["rot"]
    x = s["qkv"].double().view(R, hq + 2 * hkv, D)
    if norm:
        for lo, hi, g in ((0, hq, s["g_q"]), (hq, hq + hkv, s["g_k"])):
            part = x[:, lo:hi]
            x[:, lo:hi] = part / torch.sqrt(part.square().mean(-1, keepdim=True) + 1e-6) * g.double()
    # each pair is a complex number turned by its angle
    turn = torch.tensor([math.exp(-2 * i / rot * math.log(1e4)) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * turn)
    qk = x[:, :hq + hkv, :rot]
    half = case["layout"] == "half"
    pair = qk.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if half else qk.unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None, :])
    x[:, :hq + hkv, :rot] = (z.transpose(-1, -2) if half else z).flatten(-2)
    return dict(q=x[:, :hq].contiguous(), k=_exact_codes(x[:, hq:hq + hkv], case["type"]), v=_exact_codes(x[:, hq + hkv:], case["type"]))


def _exact_attn(case, seed):
    hq, hkv, D, _ = HEADS[case["heads"]]
    G = hq // hkv
    s = _prepare_attn(dict(case), seed)
    out = torch.zeros((s["rows"], hq, D), dtype=torch.float64, device="cuda")
    starts, ctx, tables = s["starts"].tolist(), s["ctx"].tolist(), s["tables"].long()

    def held(codes, scale):  # token rows of codes as numbers
        if case["type"] == "bf16":
            return codes.double()
        return codes.view(torch.float8_e4m3fn if case["type"] == "e4m3" else torch.int8).double() * scale.reshape(-1, 1).double()

    for b in range(case["batch"]):
        n, keys = starts[b + 1] - starts[b], ctx[b] + starts[b + 1] - starts[b]
        if n == 0:
            continue
        blocks = tables[b, :(keys + BS - 1) // BS]
        sees = torch.arange(keys, device="cuda")[None, :] <= ctx[b] + torch.arange(n, device="cuda")[:, None]
        for g in range(hkv):
            sc = s["scales"][blocks, g] if "scales" in s else None
            kk = held(s["k"][blocks, g].permute(0, 2, 1, 3).reshape(-1, D), None if sc is None else sc[:, 0])[:keys]
            vv = held(s["v"][blocks, g].permute(0, 2, 1).reshape(-1, D), None if sc is None else sc[:, 1])[:keys]
            q = s["q"][starts[b]:starts[b + 1], g * G:(g + 1) * G].double().reshape(n * G, D)
            score = (q @ kk.T.contiguous() / math.sqrt(D)).view(n, G, keys)
            score = score.masked_fill(~sees[:, None, :], -math.inf)
            out[starts[b]:starts[b + 1], g * G:(g + 1) * G] = (torch.softmax(score, -1).view(n * G, keys) @ vv).view(n, G, D)
    return out


def _exact_sample(case, seed):
    s = _prepare_sample(dict(case), seed)
    R, V = case["rows"], case["vocab"]
    logprob = torch.zeros(R, dtype=torch.float64, device="cuda")
    heat, ks, ps, ms, us = (s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "uniform"))
    for r in range(R):
        if heat[r] == 0:
            continue  # one token, log 1
        x, _ = torch.sort(s["logits"][r, :V].double(), descending=True, stable=True)
        x = x[x > -math.inf] / heat[r]
        if 0 < ks[r] < x.numel():
            x = x[:ks[r]]
        p = torch.softmax(x, 0)
        n = x.numel()
        if ps[r] < 1:
            n = 1 + int((p.cumsum(0)[:-1] < ps[r]).sum())
        n = min(n, int((p >= ms[r] * p[0]).sum()))
        lp = torch.log_softmax(x[:n], 0)
        logprob[r] = lp[min(n - 1, int((lp.exp().cumsum(0) <= us[r]).sum()))]
    return dict(token=None, logprob=logprob, kept=None)


def exact(case, seed):
    return {"cache8": _exact_cache8, "attn8": _exact_attn, "shared": _exact_attn, "sample": _exact_sample}[case["kind"]](case, seed)
