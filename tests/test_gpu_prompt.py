"""The calls around a decode step as a serving program runs them together: two
iterations of ragged prompt chunks (tables and slots from request lengths, norm,
QKV projection, rotary append, attention, output projection, FFN), then the
framework's own decode step on the cache that they filled, then the output
projection and log probabilities. Checked against the oracle, one token at a time."""

import numpy as np
import pytest
import torch

import oracle
import synth
from gpu_helpers import bits, row_rel_err
from rows_helpers import dev

pytestmark = pytest.mark.gpu

# per-row inf-norm error of the residual stream after two layers: as the decode step's own parity tests
TOL = 5e-3
V = 1003


class Prompt:
    """Layers, caches and work buffers for up to `rows` new tokens an iteration."""

    def __init__(self, lib, cfg, batch, rows, nblk, width):
        self.lib, self.cfg, self.batch, self.rows, self.width = lib, cfg, batch, rows, width
        self.dec = lib.WaSDecoder(cfg, max(batch, rows), 256, nblk, cfg["num_layers"])
        self.w = []
        for l in range(cfg["num_layers"]):
            w = {k: v.cuda() for k, v in synth.layer_weights(cfg, l, seed=1, gains="random").items()}
            self.dec.load_layer(l, w)
            H, F = cfg["hidden"], cfg["ffn_dim"]

            def packed(m):
                p = torch.empty(lib.sidp_packed_bytes(*m.shape), dtype=torch.uint8, device="cuda")
                lib.sidp_pack_linear(m, m.shape[0], m.shape[1], p)
                return p
            gu = torch.empty(lib.sidp_packed_bytes(2 * (-(-F // 32) * 32), H), dtype=torch.uint8, device="cuda")
            lib.sidp_pack_gate_up(w["w_gate"], w["w_up"], F, H, gu)
            self.w.append(dict(w, qkv=packed(torch.cat([w["w_q"], w["w_k"], w["w_v"]])), o=packed(w["w_o"]), gu=gu, d=packed(w["w_down"])))
        self.head_w = (0.05 * torch.randn(V, cfg["hidden"], generator=torch.Generator().manual_seed(9))).to(torch.bfloat16)
        self.head = packed(self.head_w.cuda())
        self.gain = (1 + 0.1 * torch.randn(cfg["hidden"], generator=torch.Generator().manual_seed(8))).to(torch.bfloat16)
        torch.cuda.synchronize()
        self.tables = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
        self.free = dev(np.random.default_rng(4).permutation(nblk))
        self.taken = dev([0])
        self.starts, self.pos, self.slots = dev([0] * (batch + 1)), dev([0] * rows), dev([0] * rows)
        self.ws = torch.empty(lib.sidp_attention_rows_bytes(self.dec.h, batch, rows), dtype=torch.uint8, device="cuda")

    def extend(self, ctx, new):
        self.lib.sidp_kv_extend(self.dec.h, ctx, new, self.batch, self.free, self.free.numel(), self.taken, self.taken, self.tables,
                                self.width, self.rows, self.starts, self.pos, self.slots)

    def layers(self, x, ctx, n):
        """x fp32 [n, H] in place through every layer."""
        lib, c, h = self.lib, self.cfg, self.dec.h
        H, D, F = c["hidden"], c["head_dim"], c["ffn_dim"]
        hq, hkv = c["num_q_heads"], c["num_kv_heads"]
        N = (hq + 2 * hkv) * D
        y, qkv = torch.empty(n, H, dtype=torch.bfloat16, device="cuda"), torch.empty(n, N, dtype=torch.bfloat16, device="cuda")
        q, o = (torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        a = torch.empty(n, F, dtype=torch.bfloat16, device="cuda")
        for l, w in enumerate(self.w):
            lib.sidp_rmsnorm(x, w["g_attn"], c["rms_eps"], y, n, H)
            lib.sidp_linear(h, y, n, H, w["qkv"], N, lib.SIDP_EPI_BF16, None, None, qkv)
            lib.sidp_rope_append_rows(h, qkv, N, n, self.starts[self.batch:], self.pos, self.slots, w.get("g_q"), w.get("g_k"), l, q)
            lib.sidp_attention_rows(h, q, l, self.starts, ctx, self.tables, self.width, self.batch, n, o, self.ws, self.ws.numel())
            lib.sidp_linear(h, o, n, hq * D, w["o"], H, lib.SIDP_EPI_RESID, None, x, x)
            lib.sidp_rmsnorm(x, w["g_mlp"], c["rms_eps"], y, n, H)
            lib.sidp_linear(h, y, n, H, w["gu"], F, lib.SIDP_EPI_SWIGLU, None, None, a)
            lib.sidp_linear(h, a, n, F, w["d"], H, lib.SIDP_EPI_RESID, None, x, x)


@pytest.mark.parametrize("qk_norm", [0, 1])
def test_prompt_chunks_then_a_decode_step_then_answers(lib, qk_norm):
    cfg = synth.get_config("tiny_layer", num_layers=2, qk_norm=qk_norm, qkv_bias=0)
    H, L = cfg["hidden"], cfg["num_layers"]
    chunks = [[17, 0, 40, 1], [5, 23, 1, 16]]
    batch, rows, nblk, width = 4, 64, 20, 6
    p = Prompt(lib, cfg, batch, rows, nblk, width)
    total = [sum(c[b] for c in chunks) for b in range(batch)]
    g = torch.Generator().manual_seed(3)
    tokens = [torch.randn(t + 1, H, generator=g) for t in total]  # each sequence's inputs, one more for the decode step
    ctx = dev([0] * batch)
    done = [0] * batch
    got = [torch.zeros(t + 1, H) for t in total]
    for new in chunks:
        n = sum(new)
        x = torch.cat([tokens[b][done[b]:done[b] + new[b]] for b in range(batch)]).cuda()
        p.extend(ctx, dev(new))
        p.layers(x, ctx, n)
        p.dec.sync()
        assert p.starts.tolist() == np.concatenate([[0], np.cumsum(new)]).tolist()
        at = 0
        for b in range(batch):
            got[b][done[b]:done[b] + new[b]] = x[at:at + new[b]].cpu()
            at, done[b] = at + new[b], done[b] + new[b]
        ctx += dev(new)
    # the framework's decode step takes the next token of every sequence; its block comes from the same call
    p.extend(ctx, dev([1] * batch))
    hidden = torch.stack([t[-1] for t in tokens]).cuda()
    p.dec.step(hidden, ctx, p.tables, lib.SIDP_RESIDENT)
    p.dec.sync()
    assert p.pos.tolist()[:batch] == total
    for b in range(batch):
        got[b][-1] = hidden[b].cpu()

    w = [{k: bits(v) for k, v in p.w[l].items() if k.startswith(("w_", "g_", "b_"))} for l in range(L)]
    for b in range(batch):
        k = [np.zeros((6, cfg["num_kv_heads"], 16, cfg["head_dim"])) for _ in range(L)]
        v = [np.zeros_like(k[0]) for _ in range(L)]
        want = np.concatenate([oracle.decode_stack(tokens[b][t:t + 1].double().numpy(), w, cfg, k, v, np.array([t]), np.arange(6)[None])
                               for t in range(total[b] + 1)])
        err = row_rel_err(got[b].double().numpy(), want)
        assert err.max() <= TOL, (b, err)

    # answers: the last hidden state of every sequence through the final norm and the output projection
    y = torch.empty(batch, H, dtype=torch.bfloat16, device="cuda")
    logits = torch.empty(batch, V, dtype=torch.bfloat16, device="cuda")
    lib.sidp_rmsnorm(hidden, p.gain.cuda(), cfg["rms_eps"], y, batch, H)
    lib.sidp_linear(p.dec.h, y, batch, H, p.head, V, lib.SIDP_EPI_BF16, None, None, logits)
    targets = dev([0, 5, V - 1, 77])
    lp, rank, ent = torch.zeros(batch, device="cuda"), dev([0] * batch), torch.zeros(batch, device="cuda")
    ids, lps = torch.zeros(batch, 5, dtype=torch.int32, device="cuda"), torch.zeros(batch, 5, device="cuda")
    ws = torch.empty(lib.sidp_token_logprobs_bytes(batch, V, 5), dtype=torch.uint8, device="cuda")
    lib.sidp_token_logprobs(logits, lib.SIDP_LOGITS_BF16, batch, V, V, targets, 5, lp, rank, ent, ids, lps, ws, ws.numel())
    p.dec.sync()
    want = torch.log_softmax(logits.double().cpu(), 1)
    at = want.gather(1, targets.cpu().long()[:, None])
    assert torch.allclose(lp.cpu().double(), at[:, 0], atol=2.0 ** -18)
    assert torch.equal(rank.cpu().long(), (want > at).sum(1))
    assert torch.allclose(ent.cpu().double(), -(want.exp() * want).sum(1), atol=2.0 ** -18)
    assert torch.equal(logits.cpu().gather(1, ids.cpu().long()), logits.cpu().topk(5, 1)[0])
    full = oracle.rms_norm(hidden.double().cpu().numpy(), oracle.bf16_bits_to_f64(bits(p.gain)), cfg["rms_eps"])
    exact = full @ p.head_w.double().numpy().T
    # logits of size up to 4: two roundings to bf16 (the norm's output averaged over 256 terms, the logit itself)
    assert np.max(np.abs(logits.double().cpu().numpy() - exact)) <= 2.0 ** -5
    p.dec.close()
