"""The largest calls of sidp_kv8_read: as many rows as the header says, and refused past them."""

import pytest
import torch

from kv8_helpers import Handle8
from gpu_helpers import f64
from rows_helpers import BS, cfg_of, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hkv,rows", [(64, 1 << 20), (128, 1 << 20), (256, 1 << 19), (1024, 1 << 17)])
def test_the_most_rows_that_are_read_at_once(lib, hkv, rows):
    """Few of them in use, first and last of the call's tiles beside them empty."""
    D, nblk, used = 64, 4, 40
    g = torch.Generator().manual_seed(hkv)
    x = torch.randn(used, hkv, D, generator=g).to(torch.bfloat16)
    with Handle8(lib, cfg_of(hkv, hkv, D), 64, nblk, "int8") as h:
        slots = torch.randperm(nblk * BS, generator=g)[:used].numpy()
        held = h.put(0, slots, f64(x), -f64(x))
        at = torch.full((rows,), -1, dtype=torch.int32)
        at[:used] = torch.as_tensor(slots)
        k, v = (torch.full((used + 1, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lib.sidp_kv8_read(h.h, 0, rows, None, at.cuda(), k, v)  # negative slots: their rows are nobody's
        h.sync()
        for got, want in zip((k, v), held):
            assert torch.equal(got[:used].cpu(), torch.tensor(want).to(torch.bfloat16))
            assert torch.all(got[used:] == 7.0)
        count = dev([used])
        lib.sidp_kv8_read(h.h, 0, rows, count, at.cuda(), v, None)
        h.sync()
        assert torch.equal(v[:used], k[:used])
        more = lib.raw_call("sidp_kv8_read", h.h, 0, rows + 1, count.data_ptr(), at.data_ptr(), k.data_ptr(), None, None)
        assert more == lib.SIDP_EINVAL
