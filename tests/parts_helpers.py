"""Requests over either cache, groups of them with the same leading blocks, and
softmax(q K^T / sqrt(D)) V of each in float64 over what the cache holds. Whatever a
call may not see is NaN: in the bf16 cache the numbers, in the 8-bit one codes and
scales."""

import numpy as np
import torch

from gpu_helpers import f64
from kv8_helpers import Handle8
from rows_helpers import BS, Handle, cfg_of, dev


class Parts:
    """groups: [(sequences, shared tokens)] from sequence 0 on; lens: (cached, new) of every sequence, the shared ones included."""

    def __init__(self, lib, cache, heads, lens, groups=(), seed=0, regions=2, region=1, q_std=1.5, max_seq=None, nblk=None, place=None,
                 std=1.0):
        hq, hkv, D = heads
        self.lib, self.cache, self.lens, self.region, self.in_use = lib, cache, lens, region, []
        self.hq, self.hkv, self.D = hq, hkv, D
        self.gstarts = np.concatenate([[0], np.cumsum([n for n, _ in groups])]).astype(int)
        self.shared = [s for _, s in groups]
        need = [-(-(c + n) // BS) for c, n in lens]
        self.width = max(max(need), 1) + 1
        total = sum(need) + 5
        self.nblk = nblk or total
        cfg = cfg_of(hq, hkv, D)
        most = max_seq or max(64, max(c + n for c, n in lens))
        if cache == "bf16":
            self.h = Handle(lib, cfg, most, self.nblk, regions, fill=float("nan"))
        else:
            self.h = Handle8(lib, cfg, most, self.nblk, cache, regions)
        blocks = (np.random.default_rng(seed).permutation(self.nblk) if place is None else np.asarray(place)).tolist()
        self.tables = np.full((len(lens), self.width), -1)
        g = torch.Generator().manual_seed(seed)
        self.kv = []
        for b, (c, n) in enumerate(lens):
            i = int(np.searchsorted(self.gstarts, b, side="right")) - 1
            same = self.shared[i] if i < len(groups) else 0
            first = self.gstarts[i] if i < len(groups) else b
            held = -(-same // BS) if b > first else 0  # blocks that are the first sequence's
            k, v = (std * torch.randn(c + n, hkv, D, generator=g).to(torch.bfloat16) for _ in range(2))
            if b > first:
                assert same % BS == 0 or n == 0 or same == c, "a shared block in part belongs to nobody else's tokens"
                m = min(same, c + n)
                k[:m], v[:m] = self.kv[first][0][:m], self.kv[first][1][:m]
                self.tables[b, :held] = self.tables[first, :held]
            self.tables[b, held:need[b]] = [blocks.pop() for _ in range(need[b] - held)]
            self.kv.append([k, v])
        self.held = [None] * len(lens)
        for b in range(len(lens)):
            self.put(b)
        self.rows = sum(n for _, n in lens)
        self.q = (q_std * torch.randn(self.rows, hq, D, generator=g)).to(torch.bfloat16)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in lens])])

    def put(self, b):
        """Sequence b's keys and values into its blocks."""
        k, v = self.kv[b]
        if len(k) == 0:
            self.held[b] = (np.zeros((0, self.hkv, self.D)),) * 2
            return
        t = np.arange(len(k))
        slots = self.tables[b][t // BS] * BS + t % BS
        if self.cache != "bf16":
            self.held[b] = self.h.put(self.region, slots, f64(k), f64(v))
            return
        blk, off = torch.as_tensor(slots // BS).cuda(), torch.as_tensor(slots % BS).cuda()
        self.h.k[self.region][blk, :, :, off, :] = k.cuda().reshape(len(k), self.hkv, self.D // 8, 8)
        self.h.v[self.region][blk, :, :, off] = v.cuda()
        self.held[b] = f64(k), f64(v)

    def bytes(self, max_rows, batch=None, shared=True):
        batch = len(self.lens) if batch is None else batch
        if shared:
            return self.lib.sidp_attention_shared_bytes(self.h.h, self.code(), batch, max_rows)
        return self.lib.sidp_attention_rows8_bytes(self.h.h, batch, max_rows)

    def code(self):
        return self.lib.SIDP_CACHE_BF16 if self.cache == "bf16" else self.lib.SIDP_CACHE_8BIT

    def run(self, shared=True, max_rows=None, starts=None, ctx=None, tables=None, gstarts=None, lens=None, stream=None, sync=True, q=None):
        """The call; `shared`: sidp_attention_shared with the groups, else sidp_attention_rows8."""
        max_rows = self.rows if max_rows is None else max_rows
        qq = torch.zeros(max(max_rows, self.rows) + 1, self.hq, self.D, dtype=torch.bfloat16, device="cuda")
        qq[:self.rows] = (self.q if q is None else q).cuda()
        out = torch.full_like(qq, 7.0)
        ws = torch.full((max(1, self.bytes(max_rows, shared=shared)),), 255, dtype=torch.uint8, device="cuda")
        starts = dev(self.starts if starts is None else starts)
        ctx = dev([c for c, _ in self.lens] if ctx is None else ctx)
        tables = dev(self.tables if tables is None else tables)
        gs = dev(self.gstarts if gstarts is None else gstarts)
        sl = dev(self.shared if lens is None else lens)
        torch.cuda.synchronize()
        rest = (starts, ctx, tables, self.width, len(self.lens), max_rows, out, ws, ws.numel(), stream)
        if shared:
            self.lib.sidp_attention_shared(self.h.h, self.code(), qq, self.region, gs, sl, len(sl), *rest)
        else:
            self.lib.sidp_attention_rows8(self.h.h, qq, self.region, *rest)
        # a call on a stream that torch does not know of reads these until it is waited for
        self.in_use.append((qq, ws, starts, ctx, tables, gs, sl, out))
        if sync:
            self.h.sync()
            self.in_use.clear()
        return out

    def want(self):
        """(output, sum of p |v|) per row in float64."""
        out = np.zeros((self.rows, self.hq, self.D))
        mag = np.zeros_like(out)
        G, q = self.hq // self.hkv, f64(self.q)
        for b, (c, n) in enumerate(self.lens):
            if n == 0:
                continue
            k, v = self.held[b]
            for g in range(self.hkv):
                at = slice(self.starts[b], self.starts[b] + n)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = np.einsum("nhd,td->nht", q[at, g * G:(g + 1) * G], k[:, g]) / np.sqrt(self.D)
                    seen = np.arange(c + n)[None] <= c + np.arange(n)[:, None]
                    s = np.where(seen[:, None], s, -np.inf)
                    p = np.exp(s - s.max(-1, keepdims=True))
                    p /= p.sum(-1, keepdims=True)
                if np.isfinite(v[:, g]).all():
                    out[at, g * G:(g + 1) * G] = p @ v[:, g]
                    mag[at, g * G:(g + 1) * G] = p @ np.abs(v[:, g])
                else:
                    for i in range(n):  # only what the row sees: 0 * NaN is no part of the definition
                        out[self.starts[b] + i, g * G:(g + 1) * G] = p[i, :, :c + i + 1] @ v[:c + i + 1, g]
        return out, mag

    def close(self):
        self.h.close()


def close(got, want, mag, what=""):
    """bf16 has 8 bits, so rounding to it is off by at most half of 2^-7, 2^-8 relative: of each probability (and 2^-12 of the
    sum for the fp32 exponents, scales and sums), and once more of the result. Numbers below 2^-126 need not be kept: a weight times
    its value's scale there, times a code of at most 448 < 2^9, is below 2^-117, and 2^10 keys of them below 2^-107; the sum of the
    weights that they are divided by is 1 or more, for the reference is a score of the row's own."""
    got = f64(got)
    assert np.all(np.isfinite(got)), what
    tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * np.abs(want) * 1.01 + 2.0 ** -107
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.max(np.abs(got - want) / tol):.3g} of the tolerance"
