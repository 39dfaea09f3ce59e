"""What sidp_sync says of a batch that did not fit: the reason of the first sequence
that ended it, whatever the ones behind it would have met."""

import numpy as np
import pytest

from rows_helpers import Handle, cfg_of
from test_gpu_extend import call, check, plain, requests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def handle(lib):
    with Handle(lib, cfg_of(2, 1, 64), 64) as h:
        yield h


# lengths (none cached), blocks in the free list, max_rows, what ended the batch
CASES = {
    "blocks, then more rows than fit": ([16, 40, 40, 40], 1, 100, "ENOBLOCKS"),
    "blocks, then one that alone has too many rows": ([5, 33, 90], 2, 50, "ENOBLOCKS"),
    "blocks at the first": ([40, 200], 2, 100, "ENOBLOCKS"),
    "blocks, then idle ones, then rows": ([16, 20, 0, 0, 200], 1, 64, "ENOBLOCKS"),
    "blocks, then one longer than its table": ([16, 20, 0, 0, 300], 1, 64, "EINVAL"),  # 300 > 16 * 13
    "rows, then more blocks than there are": ([16, 60, 40, 200], 6, 60, "EINVAL"),
    "rows and blocks at the same sequence": ([16, 90, 1], 2, 60, "EINVAL"),
    "blocks alone": ([16, 40, 16], 2, 100, "ENOBLOCKS"),
    "rows alone": ([16, 40, 16], 20, 50, "EINVAL"),
}


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("ahead", [0, 62, 63, 255, 300, 1000])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_reports_the_first_reason(lib, handle, case, ahead, in_place):
    """`ahead` sequences of one row in a block that they have already: the sequences of the case lie in other lanes, waves and
    threads' shares."""
    new, blocks, max_rows, reason = CASES[case]
    ctx, new = [1] * ahead + [0] * len(new), [1] * ahead + new
    width, nblk = 13, ahead + 40
    tables, free = requests(ctx, width, nblk, ahead)
    free, max_rows = free[:3 + blocks], max_rows + ahead
    t = call(lib, handle.h, ctx, new, free, 3, tables, max_rows, in_place)
    with pytest.raises(lib.SidpError) as e:
        handle.sync()
    assert e.value.code == getattr(lib, "SIDP_" + reason)
    handle.sync()  # said once
    check(t, plain(ctx, new, free, 3, tables, nblk, max_rows), len(ctx))


def test_extend_reports_lengths_that_are_no_lengths_beside_missing_blocks(lib, handle):
    """A sequence that the table cannot hold is an input error wherever it stands, before or behind the one without blocks."""
    for at in (0, 3):
        ctx, new = [0, 0, 0], [16, 40, 1]
        ctx.insert(at, -1)
        new.insert(at, 2)
        tables, free = requests([max(0, c) for c in ctx], 4, 30, 1)
        t = call(lib, handle.h, ctx, new, free[:2], 0, tables, 100)
        with pytest.raises(lib.SidpError) as e:
            handle.sync()
        assert e.value.code == lib.SIDP_EINVAL
        check(t, plain(ctx, new, free[:2], 0, tables, 30, 100), len(ctx))
        assert np.diff(t["starts"].tolist()[:5]).tolist().count(16) == 1
