"""Host side of the 8-bit cache: sizes, refusals that are decided before any GPU
work, and the tests' own coder against torch's."""

import numpy as np
import pytest
import torch

import paper_2605_28095_amd as sidp
from kv8_helpers import E4M3, codes_of, half_step, scale_of, to_e4m3, values_of
from rows_helpers import cfg_of

E = sidp.SIDP_EINVAL
FAKE = 1 << 20


def test_the_coder_of_the_tests_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 20001), E4M3[:127], (E4M3[:126] + E4M3[1:127]) / 2, [2.0 ** -10, 2.0 ** -11, 0.0, -0.0]])
    want = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(to_e4m3(x.astype(np.float32).astype(np.float64)), want)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_codes_are_within_half_a_step(kind):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((500, 64)) * 2.0 ** rng.integers(-30, 30, (500, 1))
    x[:100] *= 2.0 ** rng.integers(-8, 8, (100, 64))
    s = scale_of(x, kind)
    if kind == "e4m3":
        assert np.all(np.max(np.abs(x), 1) <= 448 * s) and np.all(np.max(np.abs(x), 1) > 224 * s)
        assert np.all(np.frexp(s)[0] == 0.5)
    got = values_of(codes_of(x, s, kind), kind) * s[:, None]
    assert np.all(np.abs(got - x) <= half_step(x, s, kind) * (1 + 2.0 ** -22))  # int8: the scale itself is fp32


def test_scales_of_nothing_and_of_no_number():
    for kind in ("e4m3", "int8"):
        assert scale_of(np.zeros((1, 4)), kind)[0] == 2.0 ** -126
        assert np.isnan(scale_of(np.array([[1.0, np.inf]]), kind)[0]) and np.isnan(scale_of(np.array([[1.0, np.nan]]), kind)[0])


def test_sizes():
    cfg = sidp.make_config(cfg_of(8, 2, 64), 1, 64)
    assert sidp.sidp_kv8_region_bytes(cfg, 10) == 10 * 2 * 16 * 64 == sidp.sidp_kv_region_bytes(cfg, 10) // 2
    assert sidp.sidp_kv8_scale_bytes(cfg, 10) == 10 * 2 * 2 * 16 * 4
    assert sidp.sidp_kv8_region_bytes(cfg, 0) == 0 and sidp.sidp_kv8_scale_bytes(cfg, -1) == 0
    assert sidp.sidp_kv8_region_bytes(cfg, 1 << 30) == (1 << 30) * 2 * 16 * 64
    cfg.head_dim = 80
    assert sidp.sidp_kv8_region_bytes(cfg, 10) == 0 and sidp.sidp_kv8_scale_bytes(cfg, 10) == 0


def test_calls_refuse_a_missing_handle():
    assert sidp.raw_call("sidp_kv8_attach", None, 1, FAKE, FAKE, FAKE, 1, 1) == E
    assert sidp.raw_call("sidp_rope_append_rows8", None, FAKE, 512, 1, None, FAKE, FAKE, None, None, 0, FAKE, None) == E
    assert sidp.raw_call("sidp_kv8_read", None, 0, 1, None, FAKE, FAKE, FAKE, None) == E
