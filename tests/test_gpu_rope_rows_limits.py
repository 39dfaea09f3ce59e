"""The most rows of a row append: sizes that one launch cannot cover are refused."""

import pytest
import torch

from rows_helpers import Handle, cfg_of

pytestmark = pytest.mark.gpu

FAKE = 1 << 20  # an aligned address that a refused call never reads


@pytest.mark.parametrize("hkv,most", [(8, 1 << 20), (1024, None)])
def test_rows_times_heads_past_a_launch_are_refused(lib, hkv, most):
    # 2 workgroups a KV head and 64 rows, one a row, 256 threads each, fewer than 2^32 threads in all
    first_too_many = 1
    while 2 * -(-first_too_many // 64) * hkv + first_too_many < 1 << 24:
        first_too_many += 64
    with Handle(lib, cfg_of(hkv, hkv, 64), 64, 1) as h:
        def rc(rows):
            return lib.raw_call("sidp_rope_append_rows", h.h, FAKE, 3 * hkv * 64, rows, None, FAKE, FAKE, None, None, 0, FAKE, None)
        assert rc(lib.SIDP_MAX_ROWS + 1) == lib.SIDP_EINVAL
        if most is None:
            assert first_too_many < lib.SIDP_MAX_ROWS
            assert rc(first_too_many) == lib.SIDP_EINVAL and rc(lib.SIDP_MAX_ROWS) == lib.SIDP_EINVAL
        else:
            assert first_too_many > most
        # the handle is as it was: a small call runs
        qkv = torch.ones(1, 3 * hkv * 64, dtype=torch.bfloat16, device="cuda")
        q = torch.zeros(1, hkv, 64, dtype=torch.bfloat16, device="cuda")
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        lib.sidp_rope_append_rows(h.h, qkv, qkv.shape[1], 1, None, zero, zero, None, None, 0, q)
        h.sync()
        assert torch.all(q == 1) and torch.all(h.keys()[0] == 1) and torch.all(h.values()[0] == 1)
