"""Performance cases of the operators around the decode step that take several
tokens of a sequence at once (prompts, prompt chunks, drafted tokens) and that
read answers out of logits, with the plain torch form of each.

  extend   block tables, row starts, positions and cache slots of one iteration,
           from request lengths (sidp_kv_extend)
  rope     QK-norm, rotary positions (half or interleaved pairs, part of the
           head, scaled for long contexts) and the append of many rows to the
           paged cache (sidp_set_rope, sidp_rope_append_rows)
  attn     causal attention of each sequence's new rows over its paged cache
           (sidp_attention_rows)
  logp     log probabilities of given tokens, their ranks, the entropy and the
           most likely alternatives (sidp_token_logprobs)

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

# scaling of the rotary frequencies: kind, base, factor, original length (low 1 / high 4 and beta 1 / 32 throughout)
ROPES = {
    "plain": ("none", 1e4, 1.0, 0),
    "linear": ("linear", 1e4, 4.0, 4096),
    "banded": ("llama3", 5e5, 8.0, 8192),
    "yarn": ("yarn", 1e6, 4.0, 32768),
}


def listed():
    return [
        # One sequence's next token: the smallest call, nothing but latency.
        dict(name="extend_1", kind="extend", batch=1, clo=100, chi=100, nlo=1, nhi=1),
        # An iteration of the headline batch: a token a sequence, contexts up to 8K.
        dict(name="extend_256", kind="extend", batch=256, clo=1024, chi=8191, nlo=1, nhi=1),
        # Many ragged prompts taken in at once, some sequences idle or partly cached.
        dict(name="extend_prompts", kind="extend", batch=512, clo=0, chi=700, nlo=0, nhi=511),
        # A draft model's few rows: interleaved pairs over part of a 64-wide head.
        dict(name="rope_tiny_8", kind="rope", heads="tiny", layout="interleaved", rot=32, rope="plain", batch=8,
             clo=16, chi=64, nlo=1, nhi=1),
        # A decode iteration far into long contexts, QK-norm and scaled frequencies.
        dict(name="rope_qwen3_256", kind="rope", heads="qwen3", layout="half", rot=128, rope="yarn", batch=256,
             clo=2000, chi=32000, nlo=1, nhi=1),
        # Prompt chunks of a prefill iteration, ragged, frequencies scaled in bands.
        dict(name="rope_70b_prompts", kind="rope", heads="70b", layout="half", rot=128, rope="banded", batch=8,
             clo=0, chi=2000, nlo=300, nhi=1748),
        # Four drafted tokens a sequence checked against long caches: bound by the cache's bytes.
        dict(name="attn_verify_16", kind="attn", heads="70b", batch=16, clo=1024, chi=8187, nlo=4, nhi=4),
        # Ragged chunks over partly filled caches, as a chunked prefill mixes them with single tokens.
        dict(name="attn_chunks_8", kind="attn", heads="70b", batch=8, clo=0, chi=4096, nlo=1, nhi=1021),
        # A whole long prompt: bound by the matrix units.
        dict(name="attn_prompt_8k", kind="attn", heads="70b", batch=1, clo=0, chi=0, nlo=8192, nhi=8192),
        # The answer of a single sequence.
        dict(name="logp_1", kind="logp", rows=1, vocab=128256, pad=0, f32=False, top=5, none=0.0, masked=0.0),
        # A decode iteration's answers in fp32, some of them under a grammar's mask, rows padded to a stride.
        dict(name="logp_256", kind="logp", rows=256, vocab=151936, pad=128, f32=True, top=20, none=0.1, masked=0.25),
        # Prompt scoring: every token of several prompts, an odd vocabulary.
        dict(name="logp_prompt_2048", kind="logp", rows=2048, vocab=128001, pad=0, f32=False, top=1, none=0.0,
             masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["extend", "rope", "rope", "attn", "attn", "attn", "logp", "logp"])
    if kind == "extend":
        batch = _log_int(rng, 1, 1024)
        nhi = min(_log_int(rng, 1, 4096), 2 * 65536 // batch)
        clo = rng.choice([0, _log_int(rng, 1, 2000)])
        return dict(kind=kind, batch=batch, clo=clo, chi=clo + _log_int(rng, 1, 6000), nlo=rng.randint(batch < 2, nhi), nhi=nhi)
    if kind == "rope":
        heads = rng.choice(["70b", "qwen3", "tiny", "mha"])
        D = HEADS[heads][2]
        batch = _log_int(rng, 1, 256)
        nhi = min(_log_int(rng, 1, 4096), 8192 // batch)
        clo = rng.choice([0, _log_int(rng, 1, 20000)])
        return dict(kind=kind, heads=heads, layout=rng.choice(["half", "interleaved"]),
                    rot=rng.choice([16 * rng.randint(1, D // 16), D]), rope=rng.choice(sorted(ROPES)), batch=batch,
                    clo=clo, chi=clo + _log_int(rng, 1, 4000), nlo=rng.randint(1, nhi), nhi=nhi)
    if kind == "attn":
        heads = rng.choice(["70b", "70b", "tiny", "mha"])
        hq = HEADS[heads][0]
        batch = _log_int(rng, 1, 64)
        nhi = min(_log_int(rng, 1, 4096), 8192 // batch)
        # the whole rectangle of scores stays below the largest listed one
        most = min(64 * 8192 * 4096 // (batch * nhi * hq) - nhi, 32768, 400000 // batch)
        chi = _log_int(rng, 1, max(1, most))
        return dict(kind=kind, heads=heads, batch=batch, clo=rng.randint(0, chi), chi=chi,
                    nlo=rng.choice([nhi, rng.randint(batch < 2, nhi)]), nhi=nhi)
    vocab = rng.choice([_log_int(rng, 1000, 160000), 128256, 151936])
    rows = min(_log_int(rng, 1, 2048), 2048 * 64000 // vocab)
    return dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, rng.randint(1, 64)]), f32=rng.random() < 0.5,
                top=rng.choice([0, 1, 5, 20, rng.randint(1, 32)]), none=rng.choice([0.0, 0.3]),
                masked=rng.choice([0.0, 0.5]))


# ---------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + salt * 7919 + 29) & ((1 << 62) - 1))
    return g


def _randn(shape, seed, salt, std=1.0):
    t = torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=torch.float32)
    return t.mul_(std).to(torch.bfloat16)


def _lens(lo, hi, n):
    """n lengths evenly spread over [lo, hi]."""
    return [lo + ((hi - lo) * i) // max(1, n - 1) for i in range(n)]


def _dealt(lo, hi, n, seed, salt):
    g = torch.Generator()
    g.manual_seed((seed * 1_000_003 + salt * 104729 + 3) & ((1 << 62) - 1))
    v = torch.tensor(_lens(lo, hi, n), dtype=torch.int32)
    return v[torch.randperm(n, generator=g)]


def _paged(case, seed, complete):
    """Request lengths and block tables: blocks in random order; the tables hold
    the cached tokens' blocks and, with `complete`, the new ones' too."""
    B = case["batch"]
    ctx, new = _dealt(case["clo"], case["chi"], B, seed, 1), _dealt(case["nlo"], case["nhi"], B, seed, 2)
    have, need = (ctx + BS - 1) // BS, (ctx + new + BS - 1) // BS
    width = (case["chi"] + case["nhi"] + BS - 1) // BS + 2
    held = need if complete else have
    total = int((ctx + new).sum()) // BS + B + 5
    perm = torch.randperm(total, generator=_gen(seed, 3), device="cuda").to(torch.int32)
    start = torch.cumsum(held, 0) - held
    col = torch.arange(width)
    at = (start[:, None] + col[None, :]).clamp_(max=total - 1).cuda()
    tables = torch.where((col[None, :] < held[:, None]).cuda(), perm[at], torch.full((), -1, dtype=torch.int32, device="cuda"))
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.cumsum(new, 0)
    return dict(B=B, rows=int(starts[-1]), nblk=total, width=width, ctx=ctx.cuda(), new=new.cuda(),
                starts=starts.cuda(), tables=tables.contiguous(), free=perm[int(held.sum()):].contiguous(),
                longest_new=int(new.max()), longest=int((ctx + new).max()))


def _row_places(p):
    """Sequence, position and cache slot of every new row."""
    seq = torch.repeat_interleave(torch.arange(p["B"], device="cuda"), p["new"].long(), output_size=p["rows"])
    pos = p["ctx"].long()[seq] + torch.arange(p["rows"], device="cuda") - p["starts"].long()[seq]
    slot = p["tables"].long()[seq, pos // BS] * BS + pos % BS
    return seq, pos, slot


def _frequencies(kind, base, factor, original, rot):
    """Angle per position of each pair (64 bits) and the factor on cos and sin."""
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if kind == "linear":
        return inv / factor, 1.0
    if kind == "llama3":  # wavelengths past original / 1 are stretched, those under original / 4 kept, a ramp between
        turns = original * inv / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return keep * inv + (1 - keep) * inv / factor, 1.0
    if kind == "yarn":  # ramp over the pairs between those that turn 32 times and once in the original length
        at = lambda n: rot * math.log(original / (n * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=torch.float64) - lo) / (hi - lo if hi > lo else 0.001)).clamp(0, 1)
        return ramp * inv / factor + (1 - ramp) * inv, 0.1 * math.log(factor) + 1.0
    return inv, 1.0


class _Handle:
    """A library handle, with the given caches attached; freed with its state."""

    def __init__(self, heads, max_seq_len, k=None, v=None, nblk=0):
        import paper_2605_28095_amd as sidp
        hq, hkv, D, norm = HEADS[heads]
        cfg = dict(num_layers=1, hidden=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, ffn_dim=64, qkv_bias=0,
                   qk_norm=norm, rms_eps=1e-6, qk_norm_eps=1e-6, rope_theta=1e4, block_size=BS)
        self.sidp = sidp
        self.h = None
        self.h = sidp.sidp_create(sidp.make_config(cfg, 1, max_seq_len))
        if k is not None:
            sidp.sidp_kv_attach(self.h, k, v, nblk, 1)

    def __del__(self):
        if self.h is not None:
            self.sidp.sidp_destroy(self.h)
            self.h = None


def _caches(nblk, hkv, D, seed):
    """One region of the paged cache in the library's layouts, K [block][head][d / 8][token][d % 8], V [block][head][d][token]."""
    return _randn((nblk, hkv, D // 8, BS, 8), seed, 10), _randn((nblk, hkv, D, BS), seed, 11)


def _prepare_extend(case, seed):
    p = _paged(case, seed, False)
    s = dict(p, case=case, taken=torch.tensor([3], dtype=torch.int32, device="cuda"))
    s["free"] = torch.cat([torch.full((3,), -7, dtype=torch.int32, device="cuda"), p["free"]])  # three handed out before
    s["taken_out"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["starts"] = torch.zeros(p["B"] + 1, dtype=torch.int32, device="cuda")
    s["positions"] = torch.zeros(max(1, p["rows"]), dtype=torch.int32, device="cuda")
    s["slots"] = torch.zeros(max(1, p["rows"]), dtype=torch.int32, device="cuda")
    if own:
        s["handle"] = _Handle("tiny", 64)
    return s


def _prepare_rope(case, seed):
    hq, hkv, D, norm = HEADS[case["heads"]]
    p = _paged(case, seed, True)
    _, pos, slot = _row_places(p)
    k, v = _caches(p["nblk"], hkv, D, seed)
    s = dict(case=case, rows=p["rows"], nblk=p["nblk"], positions=pos.to(torch.int32), slots=slot.to(torch.int32), k=k, v=v)
    s["qkv"] = _randn((p["rows"], (hq + 2 * hkv) * D), seed, 12)
    s["g_q"] = (1 + _randn((D,), seed, 13, 0.1).float()).to(torch.bfloat16) if norm else None
    s["g_k"] = (1 + _randn((D,), seed, 14, 0.1).float()).to(torch.bfloat16) if norm else None
    s["q_out"] = torch.zeros((p["rows"], hq, D), dtype=torch.bfloat16, device="cuda")
    kind, base, factor, original = ROPES[case["rope"]]
    if own:
        import paper_2605_28095_amd as sidp
        s["handle"] = _Handle(case["heads"], p["longest"], k, v, p["nblk"])
        sidp.sidp_set_rope(s["handle"].h, sidp.make_rope(layout=case["layout"], rotary_dim=case["rot"], theta=base,
                                                         scaling=kind, factor=factor, original_len=original))
    else:
        inv, mul = _frequencies(kind, base, factor, original, case["rot"])
        angle = torch.arange(p["longest"], dtype=torch.float64, device="cuda")[:, None] * inv.cuda()[None, :]
        s["cos"], s["sin"] = (angle.cos() * mul).float(), (angle.sin() * mul).float()
    return s


def _prepare_attn(case, seed):
    hq, hkv, D, _ = HEADS[case["heads"]]
    p = _paged(case, seed, True)
    k, v = _caches(p["nblk"], hkv, D, seed)
    s = dict(p, case=case, k=k, v=v, q=_randn((p["rows"], hq, D), seed, 15, 1.5))
    s["out"] = torch.zeros((p["rows"], hq, D), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2605_28095_amd as sidp
        s["handle"] = _Handle(case["heads"], max(64, p["longest"]), k, v, p["nblk"])
        s["ws"] = torch.empty(sidp.sidp_attention_rows_bytes(s["handle"].h, p["B"], max(1, p["rows"])), dtype=torch.uint8,
                              device="cuda")
    return s


def _prepare_logp(case, seed):
    R, V = case["rows"], case["vocab"]
    dt = torch.float32 if case["f32"] else torch.bfloat16
    x = torch.randn((R, V + case["pad"]), generator=_gen(seed, 20), device="cuda")
    x *= 0.5 + 2.5 * torch.rand((R, 1), generator=_gen(seed, 21), device="cuda")
    targets = torch.randint(0, V, (R,), generator=_gen(seed, 22), device="cuda")
    sure = torch.rand((R, 1), generator=_gen(seed, 23), device="cuda")
    x.scatter_add_(1, targets[:, None], 14.0 * sure)  # from a guess to a token that the model is sure of
    if case["masked"]:
        under = torch.rand((R, 1), generator=_gen(seed, 24), device="cuda") < case["masked"]
        out = torch.rand((R, V + case["pad"]), generator=_gen(seed, 25), device="cuda") < 0.995
        out.scatter_(1, targets[:, None], False)
        x.masked_fill_(under & out, -math.inf)
    targets = targets.to(torch.int32)
    if case["none"]:
        targets[torch.rand(R, generator=_gen(seed, 26), device="cuda") < case["none"]] = -1
    s = dict(case=case, logits=x.to(dt), targets=targets)
    s["logprob"] = torch.zeros(R, device="cuda")
    s["entropy"] = torch.zeros(R, device="cuda")
    s["rank"] = torch.zeros(R, dtype=torch.int32, device="cuda")
    s["top_ids"] = torch.zeros((R, case["top"]), dtype=torch.int32, device="cuda")
    s["top_logprobs"] = torch.zeros((R, case["top"]), device="cuda")
    if own:
        import paper_2605_28095_amd as sidp
        s["ws"] = torch.empty(sidp.sidp_token_logprobs_bytes(R, V, case["top"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return {"extend": _prepare_extend, "rope": _prepare_rope, "attn": _prepare_attn, "logp": _prepare_logp}[case["kind"]](case, seed)


# ---------------------------------------------------------------- one pass

def _extend(s):
    ctx, new, B, rows = s["ctx"].long(), s["new"].long(), s["B"], s["rows"]
    have = (ctx + BS - 1) // BS
    add = (ctx + new + BS - 1) // BS - have
    first = torch.cumsum(add, 0) - add + s["taken"].long()
    starts = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
    starts[1:] = torch.cumsum(new, 0)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), new, output_size=rows)
    pos = ctx[seq] + torch.arange(rows, device="cuda") - starts[seq]
    blk = pos // BS
    ahead = blk - have[seq]
    ids = torch.where(ahead >= 0, s["free"][(first[seq] + ahead).clamp(0, s["free"].numel() - 1)], s["tables"][seq, blk])
    s["tables"][seq, blk] = ids
    return dict(tables=s["tables"], starts=starts.to(torch.int32), positions=pos.to(torch.int32),
                slots=(ids.long() * BS + pos % BS).to(torch.int32), taken=(s["taken"] + add.sum()).to(torch.int32))


def _extend_own(s):
    import paper_2605_28095_amd as sidp
    sidp.sidp_kv_extend(s["handle"].h, s["ctx"], s["new"], s["B"], s["free"], s["free"].numel(), s["taken"], s["taken_out"],
                        s["tables"], s["width"], s["rows"], s["starts"], s["positions"], s["slots"],
                        torch.cuda.current_stream())
    return dict(tables=s["tables"], starts=s["starts"], positions=s["positions"][:s["rows"]], slots=s["slots"][:s["rows"]],
                taken=s["taken_out"])


def _rope(s):
    c = s["case"]
    hq, hkv, D, norm = HEADS[c["heads"]]
    R, rot = s["rows"], c["rot"]
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
    turned = turned.to(torch.bfloat16)
    blk, off = s["slots"].long() // BS, s["slots"].long() % BS
    s["k"][blk, :, :, off, :] = turned[:, hq:].reshape(R, hkv, D // 8, 8)
    s["v"][blk, :, :, off] = v.to(torch.bfloat16)
    return dict(q=turned[:, :hq].contiguous(), k=s["k"], v=s["v"])


def _rope_own(s):
    import paper_2605_28095_amd as sidp
    sidp.sidp_rope_append_rows(s["handle"].h, s["qkv"], s["qkv"].shape[1], s["rows"], None, s["positions"], s["slots"],
                               s["g_q"], s["g_k"], 0, s["q_out"], torch.cuda.current_stream())
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _attn(s):
    c = s["case"]
    hq, hkv, D, _ = HEADS[c["heads"]]
    B, n, G = s["B"], max(1, s["longest_new"]), hq // hkv
    S = s["width"] * BS
    tables = s["tables"].long().clamp(min=0)
    k = s["k"][tables].permute(0, 2, 3, 5, 1, 4).reshape(B, hkv, D, S).float()  # [B][head][d][token]
    v = s["v"][tables].permute(0, 2, 1, 4, 3).reshape(B, hkv, S, D).float()
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


def _attn_own(s):
    import paper_2605_28095_amd as sidp
    sidp.sidp_attention_rows(s["handle"].h, s["q"], 0, s["starts"], s["ctx"], s["tables"], s["width"], s["B"],
                             s["rows"], s["out"], s["ws"], s["ws"].numel(), torch.cuda.current_stream())
    return s["out"]


def _logp(s):
    c = s["case"]
    V = c["vocab"]
    x = s["logits"][:, :V].float()
    given = s["targets"].long()
    some = given >= 0
    xt = x.gather(1, given.clamp(min=0)[:, None])
    m = x.amax(1, keepdim=True)
    e = (x - m).exp_()
    total = e.sum(1, keepdim=True)
    entropy = total.log() - torch.where(e > 0, e * (x - m), 0.0).sum(1, keepdim=True) / total
    rank = (x > xt).sum(1)
    if c["top"]:
        # the order of the values, then the lowest index, as one whole number
        bits = (x + 0.0).view(torch.int32)
        key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long() * (1 << 32) + (V - 1 - torch.arange(V, device="cuda"))
        top = V - 1 - (key.topk(c["top"], 1)[0] & 0xFFFFFFFF)
    else:
        top = torch.zeros((c["rows"], 0), dtype=torch.int64, device="cuda")
    nan = torch.full((), math.nan, device="cuda")
    return dict(logprob=torch.where(some, (xt - m - total.log())[:, 0], nan), entropy=entropy[:, 0],
                rank=torch.where(some, rank, -1).to(torch.int32), top_ids=top.to(torch.int32),
                top_logprobs=x.gather(1, top) - m - total.log())


def _logp_own(s):
    import paper_2605_28095_amd as sidp
    c = s["case"]
    sidp.sidp_token_logprobs(s["logits"], sidp.SIDP_LOGITS_F32 if c["f32"] else sidp.SIDP_LOGITS_BF16, c["rows"], c["vocab"],
                             s["logits"].shape[1], s["targets"], c["top"], s["logprob"], s["rank"], s["entropy"],
                             s["top_ids"], s["top_logprobs"], s["ws"], s["ws"].numel(), torch.cuda.current_stream())
    return dict(logprob=s["logprob"], entropy=s["entropy"], rank=s["rank"], top_ids=s["top_ids"],
                top_logprobs=s["top_logprobs"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"extend": _extend_own, "rope": _rope_own, "attn": _attn_own, "logp": _logp_own}[kind](state)
    return {"extend": _extend, "rope": _rope, "attn": _attn, "logp": _logp}[kind](state)


# ---------------------------------------------------------------- work

def work(case):
    kind = case["kind"]
    if kind == "logp":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * V * (4 if case["f32"] else 2) + R * (16 + 8 * case["top"]), "flops": 6 * R * V}
    B = case["batch"]
    ctx, new = _lens(case["clo"], case["chi"], B), _lens(case["nlo"], case["nhi"], B)
    rows = sum(new)
    if kind == "extend":
        # lengths, starts, positions and slots, a table entry read or written for each block touched
        return {"bytes": 12 * B + 8 * rows + 8 * (rows // BS + B) + 12, "flops": 0}
    hq, hkv, D, norm = HEADS[case["heads"]]
    if kind == "rope":
        return {"bytes": rows * (4 * (hq + 2 * hkv) * D + 8 + 4 * case["rot"]), "flops": rows * (hq + hkv) * D * 4}
    # the deal pairs contexts and chunks at random: each at its mean
    mean = sum(ctx) / B
    keys = sum(n * (mean + (n + 1) / 2) for n in new)
    return {"bytes": 4 * rows * hq * D + 4 * hkv * D * (sum(ctx) + rows) + 4 * sum(ctx) // BS, "flops": 4 * hq * D * keys}


# ---------------------------------------------------------------- the definition in 64 bits

def _turn_per_position(kind, base, factor, original, rot, i):
    """The angle by which pair i turns at each position."""
    w = math.exp(-2 * i / rot * math.log(base))
    if kind == "none":
        return w
    if kind == "linear":
        return w / factor
    if kind == "llama3":
        length = 2 * math.pi / w
        if length < original / 4.0:
            return w
        if length > original / 1.0:
            return w / factor
        t = (original / length - 1.0) / (4.0 - 1.0)
        return (1 - t) * w / factor + t * w
    ends = [rot / 2 * math.log(original / (2 * math.pi * n), base) for n in (32.0, 1.0)]
    lo, hi = max(0, math.floor(ends[0])), min(rot - 1, math.ceil(ends[1]))
    t = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001)))
    return w * (1 - t) + w / factor * t


def _exact_rope(case, seed):
    hq, hkv, D, norm = HEADS[case["heads"]]
    s = _prepare_rope(dict(case), seed)
    R, rot = s["rows"], case["rot"]
    kind, base, factor, original = ROPES[case["rope"]]
    inv = torch.tensor([_turn_per_position(kind, base, factor, original, rot, i) for i in range(rot // 2)], dtype=torch.float64)
    mul = 1.0 + 0.1 * math.log(factor) if kind == "yarn" else 1.0
    x = s["qkv"].double().view(R, hq + 2 * hkv, D)
    if norm:
        for lo, hi, g in ((0, hq, s["g_q"]), (hq, hq + hkv, s["g_k"])):
            part = x[:, lo:hi]
            x[:, lo:hi] = part / torch.sqrt(part.square().mean(-1, keepdim=True) + 1e-6) * g.double()
    # each pair is a complex number turned by its angle
    turn = torch.polar(torch.full((), mul, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * inv.cuda())
    qk = x[:, :hq + hkv, :rot]
    pair = qk.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" else qk.unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None, :])
    x[:, :hq + hkv, :rot] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
    k, v = s["k"].double(), s["v"].double()
    # the caches with tokens as rows
    kt = k.permute(0, 3, 1, 2, 4).reshape(-1, hkv, D)
    vt = v.permute(0, 3, 1, 2).reshape(-1, hkv, D)
    kt[s["slots"].long()] = x[:, hq:hq + hkv]
    vt[s["slots"].long()] = x[:, hq + hkv:]
    n = s["nblk"]
    return dict(q=x[:, :hq].contiguous(), k=kt.view(n, BS, hkv, D // 8, 8).permute(0, 2, 3, 1, 4).contiguous(),
                v=vt.view(n, BS, hkv, D).permute(0, 2, 3, 1).contiguous())


def _exact_attn(case, seed):
    hq, hkv, D, _ = HEADS[case["heads"]]
    G = hq // hkv
    s = _prepare_attn(dict(case), seed)
    out = torch.zeros((s["rows"], hq, D), dtype=torch.float64, device="cuda")
    starts, ctx, tables = s["starts"].tolist(), s["ctx"].tolist(), s["tables"].long()
    for b in range(case["batch"]):
        n, keys = starts[b + 1] - starts[b], ctx[b] + starts[b + 1] - starts[b]
        if n == 0:
            continue
        blocks = tables[b, :(keys + BS - 1) // BS]
        sees = torch.arange(keys, device="cuda")[None, :] <= ctx[b] + torch.arange(n, device="cuda")[:, None]
        for g in range(hkv):
            kk = s["k"][blocks, g].double().permute(0, 2, 1, 3).reshape(-1, D)[:keys]
            vv = s["v"][blocks, g].double().permute(0, 2, 1).reshape(-1, D)[:keys]
            q = s["q"][starts[b]:starts[b + 1], g * G:(g + 1) * G].double().reshape(n * G, D)
            score = (q @ kk.T.contiguous() / math.sqrt(D)).view(n, G, keys)
            score = score.masked_fill(~sees[:, None, :], -math.inf)
            out[starts[b]:starts[b + 1], g * G:(g + 1) * G] = (torch.softmax(score, -1).view(n * G, keys) @ vv).view(n, G, D)
    return out


def _exact_logp(case, seed):
    s = _prepare_logp(dict(case), seed)
    R, V = case["rows"], case["vocab"]
    logprob = torch.full((R,), math.nan, dtype=torch.float64, device="cuda")
    entropy = torch.zeros(R, dtype=torch.float64, device="cuda")
    tops = torch.zeros((R, case["top"]), dtype=torch.float64, device="cuda")
    for r0 in range(0, R, 256):
        lp = torch.log_softmax(s["logits"][r0:r0 + 256, :V].double(), 1)
        t = s["targets"][r0:r0 + 256].long()
        logprob[r0:r0 + 256] = torch.where(t >= 0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], math.nan)
        entropy[r0:r0 + 256] = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
        tops[r0:r0 + 256] = lp.topk(case["top"], 1)[0]
    return dict(logprob=logprob, entropy=entropy, rank=None, top_ids=None, top_logprobs=tops)


def exact(case, seed):
    if case["kind"] == "extend":
        return None  # whole numbers only
    return {"rope": _exact_rope, "attn": _exact_attn, "logp": _exact_logp}[case["kind"]](case, seed)
