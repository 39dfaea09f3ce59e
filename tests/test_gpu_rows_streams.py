"""The calls that take several tokens a sequence, and the answers, on two streams at
once: calls on one handle that really overlap, each with outputs and a workspace of
its own, give the bits of calls alone."""

import numpy as np
import pytest
import torch

from rows_helpers import BS, Handle, cfg_of, dev
from test_gpu_attn_rows import Case
from test_gpu_extend import plain, requests

pytestmark = pytest.mark.gpu

ROUNDS = 6


def at_once(calls):
    """calls: one function of (round, stream) a stream. Everything is prepared and the device idle; both streams first sleep, so that
    the calls of all rounds wait in both queues and then run side by side."""
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
    for r in range(ROUNDS):
        for call, s in zip(calls, streams):
            call(r, s)
    assert not any(s.query() for s in streams)  # nothing has been waited for while the calls were made
    torch.cuda.synchronize()


def alone(calls):
    for call in calls:
        for r in range(ROUNDS):
            call(r, None)
            torch.cuda.synchronize()


def test_attention_rows_side_by_side(lib):
    """One handle: whole tiles of many rows beside cut tiles of few."""
    parts = [[(700, 50), (3, 90), (1200, 300)], [(2500, 4), (5000, 3)]]
    c = Case(lib, (8, 2, 128), parts[0] + parts[1], seed=1)
    jobs, seq = [], 0
    for part in parts:
        rows, batch = sum(n for _, n in part), len(part)
        job = dict(rows=rows, batch=batch, starts=dev(np.concatenate([[0], np.cumsum([n for _, n in part])])),
                   ctx=dev([n for n, _ in part]), tables=dev(c.tables[seq:seq + batch]),
                   q=[(1.5 * torch.randn(rows, 8, 128, device="cuda")).to(torch.bfloat16) for _ in range(ROUNDS)])
        job["ws"] = torch.full((lib.sidp_attention_rows_bytes(c.h.h, batch, rows),), 255, dtype=torch.uint8, device="cuda")
        jobs.append(job)
        seq += batch

    def results():
        for j in jobs:
            j["out"] = [torch.full_like(q, 7.0) for q in j["q"]]
        return [j["out"] for j in jobs]

    def call_of(j):
        return lambda r, s: lib.sidp_attention_rows(c.h.h, j["q"][r], c.region, j["starts"], j["ctx"], j["tables"], c.width, j["batch"],
                                                    j["rows"], j["out"][r], j["ws"], j["ws"].numel(), s)
    calls = [call_of(j) for j in jobs]
    want = results()
    alone(calls)
    assert not any(torch.all(o == 7.0) for outs in want for o in outs)
    got = results()
    at_once(calls)
    c.h.sync()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    c.h.close()


def test_row_appends_side_by_side(lib):
    """One handle, a region each: a long call beside a short one."""
    cfg, sizes, nblk = cfg_of(8, 2, 128, qk_norm=1), (2200, 70), 140
    with Handle(lib, cfg, 4096, nblk, regions=2, fill=3.0) as h:
        W = 12 * 128
        gains = [(1 + 0.1 * torch.randn(128, device="cuda")).to(torch.bfloat16) for _ in range(2)]
        jobs = []
        for region, rows in enumerate(sizes):
            rng = np.random.default_rng(region)
            jobs.append(dict(rows=rows, region=region, pos=dev(rng.integers(0, 4096, rows)), slots=dev(rng.permutation(nblk * BS)[:rows]),
                             qkv=[torch.randn(rows, W, device="cuda").to(torch.bfloat16) for _ in range(ROUNDS)]))

        def results():
            h.k.fill_(3.0)
            h.v.fill_(3.0)
            for j in jobs:
                j["out"] = [torch.full((j["rows"], 8, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(ROUNDS)]
            return [j["out"] for j in jobs]

        def call_of(j):
            return lambda r, s: lib.sidp_rope_append_rows(h.h, j["qkv"][r], W, j["rows"], None, j["pos"], j["slots"], *gains, j["region"],
                                                          j["out"][r], s)
        calls = [call_of(j) for j in jobs]
        want = results()
        alone(calls)
        k, v = h.k.clone(), h.v.clone()
        assert not torch.all(k == 3.0)
        got = results()
        at_once(calls)
        h.sync()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert torch.equal(h.k, k) and torch.equal(h.v, v)  # the last round's rows of each stream


def test_block_tables_side_by_side(lib):
    """One handle, free lists of their own: a cursor in place, walking, beside one that is not."""
    with Handle(lib, cfg_of(2, 1, 64), 64) as h:
        jobs = []
        for seed, (batch, width) in enumerate([(300, 12), (5, 200)]):
            rng = np.random.default_rng(seed)
            ctx, new = rng.integers(0, 20, batch).tolist(), rng.integers(0, 9 if batch > 10 else 400, batch).tolist()
            nblk = ROUNDS * (sum(-(-n // 16) + 1 for n in new) + batch * 2)
            tables, free = requests(ctx, width, nblk, seed)
            rows = sum(new)
            j = dict(ctx=ctx, new=new, nblk=nblk, tables=tables, free=free, rows=rows, batch=batch, width=width, in_place=seed == 0,
                     d_ctx=dev(ctx), d_new=dev(new), d_free=dev(free), cursor=dev([0]))
            j["t"] = [dict(tables=dev(tables), starts=dev([-99] * (batch + 1)), pos=dev([-99] * rows), slots=dev([-99] * rows),
                           out=dev([-99])) for _ in range(ROUNDS)]
            jobs.append(j)

        def call_of(j):
            def call(r, s):
                t = j["t"][r]
                out = j["cursor"] if j["in_place"] else t["out"]
                lib.sidp_kv_extend(h.h, j["d_ctx"], j["d_new"], j["batch"], j["d_free"], len(j["free"]), j["cursor"], out, t["tables"],
                                   j["width"], j["rows"], t["starts"], t["pos"], t["slots"], s)
            return call
        at_once([call_of(j) for j in jobs])
        h.sync()
        for j in jobs:
            taken = 0
            for t in j["t"]:
                tables, starts, positions, slots, after = plain(j["ctx"], j["new"], j["free"], taken, j["tables"], j["nblk"], j["rows"])
                assert t["tables"].tolist() == tables and t["starts"].tolist() == starts
                assert t["pos"].tolist() == positions and t["slots"].tolist() == slots
                if j["in_place"]:
                    taken = after
                else:
                    assert t["out"].tolist() == [after]
            assert j["cursor"].tolist() == [taken]


def test_log_probabilities_side_by_side(lib):
    """Rows in segments that are joined beside rows of one launch."""
    V = 60001
    jobs = []
    for rows, top in ((3, 20), (200, 5)):
        jobs.append(dict(rows=rows, top=top, targets=dev(np.random.default_rng(rows).integers(0, V, rows)),
                         x=[(3 * torch.randn(rows, V, device="cuda")).to(torch.bfloat16) for _ in range(ROUNDS)],
                         ws=torch.full((lib.sidp_token_logprobs_bytes(rows, V, top),), 255, dtype=torch.uint8, device="cuda")))

    def results():
        for j in jobs:
            n, top = j["rows"], j["top"]
            j["out"] = [(torch.zeros(n, device="cuda"), dev([9] * n), torch.zeros(n, device="cuda"),
                         torch.zeros(n, top, dtype=torch.int32, device="cuda"), torch.zeros(n, top, device="cuda")) for _ in range(ROUNDS)]
        return [j["out"] for j in jobs]

    def call_of(j):
        return lambda r, s: lib.sidp_token_logprobs(j["x"][r], lib.SIDP_LOGITS_BF16, j["rows"], V, V, j["targets"], j["top"], *j["out"][r],
                                                    j["ws"], j["ws"].numel(), s)
    calls = [call_of(j) for j in jobs]
    want = results()
    alone(calls)
    got = results()
    at_once(calls)
    for j, a, b in zip(jobs, want, got):
        for r, (x, y) in enumerate(zip(a, b)):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
            full = torch.log_softmax(j["x"][r].double(), 1).gather(1, j["targets"].long()[:, None])[:, 0]
            assert torch.allclose(x[0].double(), full, atol=2.0 ** -18)
