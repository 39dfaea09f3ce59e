"""The plan of attention over the 8-bit cache and over shared prefixes, on the CPU: with
the header that the kernel takes its arithmetic from, every list of items fits the
places that the workspace keeps for it, up to the most rows and the longest caches."""

import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2605_28095_amd", "csrc", "parts_plan.h")
SUM = "typedef uint64_t ChunkSum;"

# Reads calls: "batch groups max_rows tm slots", then "rows ctx" of each sequence and "first end shared_chunks" of each group. Prints
# entries, cuts and rows of records, each with the places there are, and the workgroup's longest run.
PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "parts_plan.h"
using namespace sidp;
struct Tile { int rows, chunks; bool group, rec; };
int main() {
  int B, G, max_rows, tm, slots;
  while (scanf("%d %d %d %d %d", &B, &G, &max_rows, &tm, &slots) == 5) {
    std::vector<int> rows(B), ctx(B), of(B, -1);
    for (int b = 0; b < B; b++) if (scanf("%d %d", &rows[b], &ctx[b]) != 2) return 1;
    std::vector<Tile> tiles;
    std::vector<int> shared(G);
    for (int i = 0; i < G; i++) {
      int first, end, chunks, all = 0, own = 0;
      if (scanf("%d %d %d", &first, &end, &chunks) != 3) return 1;
      for (int b = first; b < end; b++) all += rows[b], own += (rows[b] + tm - 1) / tm;
      if (!group_shares(chunks, all, own, tm)) continue;
      shared[i] = chunks;
      for (int b = first; b < end; b++) of[b] = i;
      for (int r = 0; r < all; r += tm) tiles.push_back({std::min(tm, all - r), chunks, true, true});
    }
    const int gtiles = (int)tiles.size();
    for (int b = 0; b < B; b++)
      for (int r = 0; r < rows[b]; r += tm) {
        const int end = std::min(rows[b], r + tm), from = of[b] >= 0 ? shared[of[b]] : 0;
        tiles.push_back({end - r, (ctx[b] + end + 31) / 32 - from, false, of[b] >= 0});
      }
    const PartsCaps caps = parts_caps(B, max_rows, tm, slots, G > 0);
    const int threads = 64 * std::max(2, std::min(16, (std::max(B, caps.tiles + (G > 0 ? caps.tiles / 2 : 0)) + 63) / 64));
    ChunkSum total = 0;
    int longest = 1;
    for (const Tile& x : tiles) total += x.chunks, longest = std::max(longest, x.chunks);
    const bool few = (int)tiles.size() < slots && (int)tiles.size() <= threads;
    int run = longest;
    if (few) {
      const int least = least_run(total, slots, longest);
      if (tiles_are_cut(longest, least)) {
        const int safe = safe_run(total, slots, (int)tiles.size(), least);
        int j = 0;
        for (; j < kTries - 1; j++) {
          long n = 0;
          for (const Tile& x : tiles) n += (x.chunks + try_run(j, least, safe) - 1) / try_run(j, least, safe);
          if (n <= slots) break;
        }
        run = std::min(run, try_run(j, least, safe));
      }
    } else if (gtiles > 0 && slots > 0) {
      run = group_run(total, slots, longest);
    }
    long entries = 0, cuts = 0, recs = 0;
    int most = 0;
    for (const Tile& x : tiles) {
      const int parts = few || x.group ? (x.chunks + run - 1) / run : 1;
      entries += parts;
      if (parts > 1 || x.rec) recs += (long)parts * x.rows, cuts += !x.group;
      most = std::max(most, (x.chunks + parts - 1) / parts);
    }
    const int wave = wave_item(total, 4, slots, longest);
    if (wave < kWaveLeast) return 2;
    printf("%ld %d %ld %d %ld %d %d\n", entries, caps.entries, cuts, caps.cuts, recs, caps.recs, most);
  }
  return 0;
}
"""


def build(where, header):
    (where / "parts_plan.h").write_text(header)
    (where / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", str(where), str(where / "plan.cpp"), "-o", str(where / "plan")], check=True, timeout=120)
    return str(where / "plan")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    with open(HEADER) as f:
        return build(tmp_path_factory.mktemp("plan"), f.read())


def lists(program, calls):
    text = []
    for max_rows, tm, slots, seqs, groups in calls:
        text.append(f"{len(seqs)} {len(groups)} {max_rows} {tm} {slots}")
        text += ["%d %d" % s for s in seqs] + ["%d %d %d" % g for g in groups]
    r = subprocess.run([program], input="\n".join(text), capture_output=True, text=True, check=True, timeout=120)
    out = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert len(out) == len(calls)
    return out


def fits(found):
    return all(found[i] <= found[i + 1] for i in (0, 2, 4))


def chunks_of(rows, ctx, tm):
    end = np.minimum(np.arange(0, rows, tm) + tm, rows)
    return int(((ctx + end + 31) // 32).sum())


def longest_call():
    """16 query heads of one KV head, tiles of 8 rows: 72 sequences of a row in groups of eight under 32000 chunks, and 4024 of 257 rows,
    whose 132792 tiles' chunks sum to just more than 2^32."""
    tm, n, rows, prefix = 8, 4024, 257, 32000
    rest = 9 * prefix + 72  # the groups' tiles, and what is left of their sequences
    ctx = next(c for c in range(32 * 32000, (1 << 20) - rows, 8) if n * chunks_of(rows, c + 8, tm) + rest >= 1 << 32)
    short, each = (1 << 32) - rest - n * chunks_of(rows, ctx, tm), chunks_of(rows, ctx + 8, tm) - chunks_of(rows, ctx, tm)
    longer = -(-short // each)  # so many of them have 8 keys more
    assert 0 < longer <= n and each < 32
    groups = [(8 * i, 8 * i + 8, prefix) for i in range(9)]
    return 72 + rows * n, tm, 512, [(1, 32 * prefix)] * 72 + [(rows, ctx + 8)] * longer + [(rows, ctx)] * (n - longer), groups


def test_the_longest_lists_fit(plan):
    """A million rows over the longest caches; groups' runs are of an even share of it all."""
    call = longest_call()
    assert call[0] <= 1 << 20 and len(call[3]) <= 4096
    (found,) = lists(plan, [call])
    assert fits(found), found
    assert found[0] == 9 + 4024 * 33 + 72  # an even share of all is longer than any tile: nothing is cut
    full = [(1 << 20, 8, 512, [(256, (1 << 20) - 256)] * 4096, []), (1 << 20, 8, 1, [(256, (1 << 20) - 256)] * 4096, []),
            (1 << 20, 128, 0, [(256, (1 << 20) - 256)] * 4096, [(0, 4096, 32760)]),
            (4096, 128, 64, [(1, (1 << 20) - 1)] * 4096, [(0, 4096, 32767)]), (4096, 8, 1, [(1, (1 << 20) - 1)] * 4096, [(0, 4096, 32767)])]
    for found in lists(plan, full):
        assert fits(found), found


def test_a_sum_of_32_bits_is_seen(tmp_path):
    """The same list with a sum that wraps: groups' tiles in runs far too short, past the places for their records."""
    with open(HEADER) as f:
        header = f.read()
    assert header.count(SUM) == 1
    program = build(tmp_path, header.replace(SUM, "typedef uint32_t ChunkSum;"))
    (found,) = lists(program, [longest_call()])
    assert not fits(found)


def test_lists_of_all_kinds_fit(plan):
    rng = np.random.default_rng(7)
    calls = []
    for _ in range(400):
        B = int(np.exp(rng.uniform(0, np.log(4096))))
        tm = 128 // int(rng.integers(1, 17))
        slots = int(rng.choice([0, 1, 2, 7, 32, 64, 128, 256, 512]))
        most_rows = max(1, min(int(np.exp(rng.uniform(0, np.log(400)))), (1 << 20) // B))
        rows = rng.integers(0, most_rows + 1, B) if rng.random() < 0.7 else rng.integers(0, 2, B)
        if rows.sum() == 0:
            rows[0] = 1
        ctx = np.exp(rng.uniform(0, np.log(rng.choice([50, 2000, 1 << 20])), B)).astype(int) - 1
        ctx = np.minimum(ctx, (1 << 20) - rows)
        groups = []
        if rng.random() < 0.8:
            cuts = np.unique(np.concatenate([[0], rng.integers(0, B + 1, int(rng.integers(1, 40)))]))
            for a, b in zip(cuts[:-1], cuts[1:]):
                c = int(ctx[a:b].max()) if rng.random() < 0.5 else int(ctx[a:b].min())
                ctx[a:b] = np.maximum(ctx[a:b], c)
                rows[a:b] = np.minimum(rows[a:b], (1 << 20) - ctx[a:b])
                groups.append((int(a), int(b), c // 32))
        total = max(1, int(rows.sum()))
        calls.append((total if rng.random() < 0.5 else min(1 << 20, 2 * total), tm, slots, list(zip(rows.tolist(), ctx.tolist())), groups))
    cut = 0
    for call, found in zip(calls, lists(plan, calls)):
        assert fits(found), (call[:3], found)
        cut += found[4] > 0
    assert cut > 100  # lists with records among them
