"""Several answers to each of a few prompts, as a serving loop draws them: slots of new
tokens, their projection, positions and keys into the 8-bit cache, attention that
reads each prompt once, logits, a draw. Each step's parts against float64 from what
the step itself holds, and the loop captured into a graph against the same steps
launched one by one."""

import numpy as np
import pytest
import torch

from gpu_helpers import assert_bf16_within_ulp, bits, dot_abs_tol, f64
from kv8_helpers import Handle8, half_step, values_of
from parts_helpers import close
from rows_helpers import BS, cfg_of, dev, turn
from test_gpu_sample import Row

pytestmark = pytest.mark.gpu

HQ, HKV, D, H, V = 8, 2, 64, 128, 1003
GROUPS = [(6, 144), (3, 160)]  # (answers, prompt tokens), and one more request by itself
ALONE = 37
BATCH = 10
FIRST = {0: 144, 6: 160, 9: ALONE}  # the sequence that brings a prompt, and its length
WIDTH, NBLK, STEPS = 14, 64, 20


class Big(Handle8):
    """Handle8 with projections of up to 512 rows."""

    def __init__(self, lib, cfg, kind):
        super().__init__(lib, cfg, WIDTH * BS, NBLK, kind)
        self.close()
        self.h = lib.sidp_create(lib.make_config(cfg, 512, WIDTH * BS))
        lib.sidp_kv8_attach(self.h, {"e4m3": lib.SIDP_KV_E4M3, "int8": lib.SIDP_KV_INT8}[kind], self.k8, self.v8, self.scales, NBLK, 1)


class Loop:
    def __init__(self, lib, kind):
        self.lib = lib
        g = torch.Generator().manual_seed(11)
        self.h = Big(lib, cfg_of(HQ, HKV, D, hidden=H, ffn=2048), kind)  # the scratch of projections goes by the widest
        self.n_qkv = (HQ + 2 * HKV) * D
        self.emb = torch.randn(V, H, generator=g).to(torch.bfloat16).cuda()
        self.w_qkv = (0.1 * torch.randn(self.n_qkv, H, generator=g)).to(torch.bfloat16)
        self.w_head = (0.15 * torch.randn(V, HQ * D, generator=g)).to(torch.bfloat16)
        self.qkv_p, self.head_p = self.packed(self.w_qkv), self.packed(self.w_head)
        self.free = dev(np.random.default_rng(1).permutation(NBLK))
        self.taken, self.ctx = dev([0]), dev([0] * BATCH)
        self.tables = torch.full((BATCH, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.one = dev([1] * BATCH)
        self.gstarts, self.shared = dev([0, 6, 9]), dev([s for _, s in GROUPS])
        self.tokens = dev(np.random.default_rng(2).integers(0, V, BATCH))
        # settings of every kind side by side
        self.T = [1.0, 0.7, 1.3, 0.0, 1.0, 2.0, 1.0, 0.9, 1.0, 0.0]
        self.k = [0, 50, 0, 0, 5, 400, 0, 0, 1, 3]
        self.p = [1.0, 0.9, 0.95, 1.0, 1.0, 0.8, 1.0, 0.5, 1.0, 1.0]
        self.m = [0.0, 0.0, 0.02, 0.0, 0.0, 0.01, 0.0, 0.0, 0.0, 0.0]
        f = lambda v: dev(v, torch.float32)  # noqa: E731
        self.set = f(self.T), dev(self.k), f(self.p), f(self.m)
        self.us = np.random.default_rng(3).random((STEPS, BATCH), np.float32)
        self.u = f(self.us[0])
        self.lp, self.kept = torch.zeros(BATCH, device="cuda"), dev([0] * BATCH)
        self.ws_s = torch.empty(lib.sidp_sample_tokens_bytes(BATCH, V), dtype=torch.uint8, device="cuda")
        self.bufs(BATCH)

    def packed(self, m):
        p = torch.empty(self.lib.sidp_packed_bytes(*m.shape), dtype=torch.uint8, device="cuda")
        self.lib.sidp_pack_linear(m.cuda(), m.shape[0], m.shape[1], p)
        torch.cuda.synchronize()
        return p

    def bufs(self, rows):
        b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.qkv, self.q, self.o, self.logits = b(rows, H), b(rows, self.n_qkv), b(rows, HQ, D), b(rows, HQ, D), b(rows, V)
        self.starts, self.pos, self.slots = dev([0] * (BATCH + 1)), dev([0] * rows), dev([0] * rows)
        self.ws = torch.full((self.lib.sidp_attention_shared_bytes(self.h.h, self.lib.SIDP_CACHE_8BIT, BATCH, rows),), 255,
                             dtype=torch.uint8, device="cuda")

    def forward(self, new, rows, groups, stream=None):
        """The layer of `rows` new tokens whose inputs are in x."""
        lib, h = self.lib, self.h.h
        lib.sidp_kv_extend(h, self.ctx, new, BATCH, self.free, NBLK, self.taken, self.taken, self.tables, WIDTH, rows, self.starts,
                           self.pos, self.slots, stream)
        lib.sidp_linear(h, self.x, rows, H, self.qkv_p, self.n_qkv, lib.SIDP_EPI_BF16, None, None, self.qkv, stream)
        lib.sidp_rope_append_rows8(h, self.qkv, self.n_qkv, rows, self.starts[BATCH:], self.pos, self.slots, None, None, 0, self.q, stream)
        lib.sidp_attention_shared(h, lib.SIDP_CACHE_8BIT, self.q, 0, self.gstarts, self.shared, groups, self.starts, self.ctx, self.tables,
                                  WIDTH, BATCH, rows, self.o, self.ws, self.ws.numel(), stream)

    def prompts(self):
        new = [FIRST.get(b, 0) for b in range(BATCH)]
        rows = sum(new)
        self.bufs(rows)
        self.x.copy_(self.emb[torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(5)).cuda()])
        self.forward(dev(new), rows, 0)
        self.h.sync()
        for first, (n, s) in zip((0, 6), GROUPS):
            self.tables[first:first + n, :s // BS] = self.tables[first, :s // BS]
        self.ctx.copy_(dev([144] * 6 + [160] * 3 + [ALONE]))
        self.bufs(BATCH)

    def step(self, stream=None):
        torch.index_select(self.emb, 0, self.tokens, out=self.x)
        self.forward(self.one, BATCH, 2, stream)
        self.lib.sidp_linear(self.h.h, self.o, BATCH, HQ * D, self.head_p, V, self.lib.SIDP_EPI_BF16, None, None, self.logits, stream)
        self.lib.sidp_sample_tokens(self.logits, self.lib.SIDP_LOGITS_BF16, BATCH, V, V, *self.set, self.u, self.tokens, self.lp, self.kept,
                                    self.ws_s, self.ws_s.numel(), stream)
        self.ctx.add_(1)

    def state(self):
        return [t.clone() for t in (self.tokens, self.lp, self.kept, self.logits, self.o, self.tables, self.ctx, self.taken)]

    def check(self, n, kind):
        """The step just done, part by part."""
        ctx, tables = self.ctx.cpu().numpy() - 1, self.tables.cpu().numpy()
        assert self.pos.tolist() == ctx.tolist()
        qkv = f64(self.qkv).reshape(BATCH, HQ + 2 * HKV, D)
        w = 1e4 ** (-np.arange(D // 2) * 2.0 / D)
        kc, ks = values_of(self.h.key_codes(), kind), self.h.key_scales()
        vc, vs = values_of(self.h.value_codes(), kind), self.h.value_scales()
        want, mag = np.zeros((BATCH, HQ, D)), np.zeros((BATCH, HQ, D))
        q = f64(self.q)
        true_k = turn(qkv[:, HQ:HQ + HKV], ctx, w, 1.0, False)
        for b in range(BATCH):
            t = np.arange(ctx[b] + 1)
            at = tables[b][t // BS] * BS + t % BS
            assert at[-1] == self.slots[b]
            k, v = kc[at] * ks[at][..., None], vc[at] * vs[at][..., None]
            for got, true, scale in ((k[-1], true_k[b], ks[at[-1]]), (v[-1], qkv[b, HQ + HKV:], vs[at[-1]])):
                # the code's half step, and what fp32 turns and tables of fp32 cosines are off by
                assert np.all(np.abs(got - true) <= half_step(true, scale, kind) * (1 + 2.0 ** -10) + 2.0 ** -19 * np.abs(true).max())
            for g in range(HKV):
                i = slice(g * HQ // HKV, (g + 1) * HQ // HKV)
                s = q[b, i] @ k[:, g].T / np.sqrt(D)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                want[b, i], mag[b, i] = p @ v[:, g], p @ np.abs(v[:, g])
        close(self.o, want, mag, f"step {n}")
        o, head = f64(self.o).reshape(BATCH, -1), f64(self.w_head)
        assert_bf16_within_ulp(bits(self.logits), o @ head.T, what="logits", abs_tol=dot_abs_tol(o, head))
        x = f64(self.logits)
        f = lambda v: np.asarray(v, np.float32).astype(np.float64)  # noqa: E731
        T, p, m, u = f(self.T), f(self.p), f(self.m), f(self.us[n])
        for r in range(BATCH):
            Row(x[r], T[r], self.k[r], p[r], m[r]).check(u[r], int(self.tokens[r]), float(self.lp[r]), int(self.kept[r]))
        # beside the log probabilities of given tokens: those drawn from all at temperature 1 have the same, the greedy ones are the likeliest
        lib, lp = self.lib, torch.zeros(BATCH, device="cuda")
        rank, top, top_lp = dev([-9] * BATCH), dev([-9] * BATCH), torch.zeros(BATCH, device="cuda")
        ws = torch.empty(lib.sidp_token_logprobs_bytes(BATCH, V, 1), dtype=torch.uint8, device="cuda")
        lib.sidp_token_logprobs(self.logits, lib.SIDP_LOGITS_BF16, BATCH, V, V, self.tokens, 1, lp, rank, None, top, top_lp, ws, ws.numel())
        torch.cuda.synchronize()
        for r in range(BATCH):
            if self.T[r] == 0 or self.k[r] == 1:
                assert self.tokens[r] == top[r] and rank[r] == 0 and self.lp[r] == 0 and self.kept[r] == 1
            elif self.T[r] == 1 and not self.k[r] and self.p[r] == 1 and not self.m[r]:
                # fp32 sums of 1003 terms in any order: 1003 2^-24 < 2^-14 relative, which is what the logarithm moves by
                assert abs(lp[r] - self.lp[r]) <= 2.0 ** -14 + 2.0 ** -22 * abs(lp[r]) and self.kept[r] == V


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_answers_drawn_over_shared_prompts_in_the_8_bit_cache(lib, kind):
    loop = Loop(lib, kind)
    loop.prompts()
    start = [t.clone() for t in (loop.tokens, loop.ctx, loop.taken, loop.tables)]
    states = []
    for n in range(STEPS):
        loop.u.copy_(dev(loop.us[n], torch.float32))
        loop.step()
        loop.h.sync()
        states.append(loop.state())
        if n % 6 == 0 or n == STEPS - 1:
            loop.check(n, kind)
    assert int(loop.taken[0]) == 9 + 10 + 3 + 9 * 2 + 1  # prompts', and 20 tokens from 144, 160 and 37 on
    assert len(set(states[-1][0].tolist())) > 1

    for t, s in zip((loop.tokens, loop.ctx, loop.taken, loop.tables), start):
        t.copy_(s)
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        loop.step(torch.cuda.current_stream())
    for n in range(STEPS):
        loop.u.copy_(dev(loop.us[n], torch.float32))
        loop.ws.fill_(255)
        loop.ws_s.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for name, a, b in zip(("tokens", "logprobs", "kept", "logits", "attention", "tables", "ctx", "taken"), loop.state(), states[n]):
            assert torch.equal(a, b), (n, name)
    loop.h.sync()
    loop.h.close()
