"""sidp_attention_shared at its largest: a million rows over a million keys, whose tiles'
chunks sum to more than 2^32, groups under a long prefix among them."""

import numpy as np
import pytest
import torch

from rows_helpers import BS, Handle, cfg_of, dev
from test_parts_plan_host import longest_call

pytestmark = pytest.mark.gpu


def test_more_than_2_to_the_32_chunks(lib):
    """Every sequence reads the same 65536 blocks; rows of each kind against float64. Scores have a deviation of 6, so that a few of the
    keys that a row sees decide it."""
    _, _, _, seqs, groups = longest_call()
    B, width, hq, D = len(seqs), (1 << 20) // BS, 16, 64
    rows, ctx = np.array([n for n, _ in seqs]), np.array([c for _, c in seqs])
    starts = np.concatenate([[0], np.cumsum(rows)])
    total = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(1)
    with Handle(lib, cfg_of(hq, 1, D), 1 << 20, width, 1) as h:
        h.k.copy_(torch.randn(h.k.shape, generator=g, device="cuda") * 1.5)
        h.v.copy_(torch.randn(h.v.shape, generator=g, device="cuda"))
        table = torch.randperm(width, generator=g, device="cuda").to(torch.int32)
        tables = table.expand(B, width).contiguous()
        q = torch.randn(total, hq, D, generator=g, device="cuda", dtype=torch.bfloat16) * 4
        out = torch.full_like(q, 7.0)
        need = lib.sidp_attention_shared_bytes(h.h, lib.SIDP_CACHE_BF16, B, total)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        args = (dev([a for a, _, _ in groups] + [groups[-1][1]]), dev([32 * c for _, _, c in groups]), len(groups), dev(starts), dev(ctx))
        torch.cuda.synchronize()
        lib.sidp_attention_shared(h.h, lib.SIDP_CACHE_BF16, q, 0, *args, tables, width, B, total, out, ws, need)
        h.sync()
        k = h.k[0][table.long()].permute(0, 3, 1, 2, 4).reshape(width * BS, D).double()
        v = h.v[0][table.long()].permute(0, 3, 1, 2).reshape(width * BS, D).double()
        last = B - 1
        for b, i in [(0, 0), (7, 0), (8, 0), (40, 0), (71, 0), (72, 0), (72, 256), (100, 13), (B // 2, 128), (last, 0), (last, 256)]:
            row, seen = int(starts[b]) + i, int(ctx[b]) + i + 1
            p = torch.softmax(q[row].double() @ k[:seen].T.contiguous() / D ** 0.5, -1)
            want, mag = p @ v[:seen], p @ v[:seen].abs()
            # the bounds of parts_helpers.close
            tol = (2.0 ** -8 + 2.0 ** -12) * mag + 2.0 ** -8 * want.abs() * 1.01
            assert torch.all((out[row].double() - want).abs() <= tol), (b, i)
        assert torch.isfinite(out).all()
