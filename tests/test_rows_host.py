"""Host side of the calls around the decode step that take several tokens a
sequence or read logits: rotary frequencies against their formulas and against
transformers' own, and every refusal that is decided before any GPU work."""

import ctypes
import math

import numpy as np
import pytest

import paper_2605_28095_amd as sidp

E = sidp.SIDP_EINVAL
FAKE = 1 << 20  # an aligned address that a refused call never reads


def _want(rot, theta, scaling, factor, original, low=1.0, high=4.0, slow=1.0, fast=32.0):
    """Pair by pair, from wavelengths instead of turns."""
    out = []
    edge = lambda n: rot / 2 * math.log(original / (2 * math.pi * n), theta)  # noqa: E731
    for i in range(rot // 2):
        w = math.exp(-2 * i / rot * math.log(theta))
        length = 2 * math.pi / w
        if scaling == "linear":
            w /= factor
        elif scaling == "llama3":
            if length > original / low:
                w /= factor
            elif length >= original / high:
                t = (original / length - low) / (high - low)
                w = (1 - t) * w / factor + t * w
        elif scaling == "yarn":
            a, b = max(0, math.floor(edge(fast))), min(rot - 1, math.ceil(edge(slow)))
            t = min(1, max(0, (i - a) / (b - a if b > a else 0.001)))
            w = w * (1 - t) + w / factor * t
        out.append(w)
    return np.array(out)


@pytest.mark.parametrize("rot,head_dim", [(16, 64), (64, 64), (48, 128), (128, 128)])
@pytest.mark.parametrize("scaling,theta,factor,original", [
    ("none", 1e4, 1.0, 0), ("linear", 1e4, 8.0, 0), ("llama3", 5e5, 8.0, 8192), ("llama3", 5e5, 32.0, 8192),
    ("yarn", 1e6, 4.0, 32768), ("yarn", 1e4, 16.0, 2048)])
def test_frequencies_follow_their_formulas(rot, head_dim, scaling, theta, factor, original):
    got, scale = sidp.sidp_rope_frequencies(
        sidp.make_rope(rotary_dim=rot, theta=theta, scaling=scaling, factor=factor, original_len=original), head_dim)
    want = _want(rot, theta, scaling, factor, original)
    # a few roundings of 2^-53 in log, exp and the blend, the logarithms' arguments up to 14
    np.testing.assert_allclose(got, want, rtol=1e-13, atol=0)
    assert scale == pytest.approx(0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0, rel=1e-15)


@pytest.mark.parametrize("scaling,theta,factor,original", [("llama3", 5e5, 8.0, 8192), ("yarn", 1e6, 4.0, 32768)])
def test_frequencies_agree_with_transformers(scaling, theta, factor, original):
    from transformers import LlamaConfig
    from transformers.modeling_rope_utils import ROPE_INIT_FUNCTIONS
    rope = dict(rope_type=scaling, factor=factor, original_max_position_embeddings=original)
    if scaling == "llama3":
        rope.update(low_freq_factor=1.0, high_freq_factor=4.0)
    cfg = LlamaConfig(hidden_size=1024, num_attention_heads=8, head_dim=128, max_position_embeddings=original, rope_theta=theta,
                      rope_scaling=rope)
    if hasattr(cfg, "rope_parameters") and cfg.rope_parameters is not None:
        cfg.rope_parameters["rope_theta"] = theta
    want, scale = ROPE_INIT_FUNCTIONS[scaling](cfg, "cpu")
    got, mul = sidp.sidp_rope_frequencies(
        sidp.make_rope(rotary_dim=128, theta=theta, scaling=scaling, factor=factor, original_len=original), 128)
    # theirs are computed in float32: the power's exponent alone is off by 2^-24 ln(theta) < 14 * 2^-24
    np.testing.assert_allclose(got, want.double().numpy(), rtol=32 * 2.0 ** -24, atol=0)
    assert mul == pytest.approx(scale, rel=1e-6)


@pytest.mark.parametrize("change", [
    dict(layout=2), dict(rotary_dim=0), dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=144), dict(theta=1.0),
    dict(theta=float("nan")), dict(theta=float("inf")), dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.0),
    dict(scaling=1, factor=float("inf")), dict(scaling=2, original_len=0), dict(scaling=2, high_freq=1.0),
    dict(scaling=2, low_freq=0.0), dict(scaling=3, original_len=0), dict(scaling=3, beta_fast=1.0),
    dict(scaling=3, beta_slow=-1.0), dict(scaling=3, attn_factor=-0.5), dict(scaling=3, factor=0.5),
    dict(scaling=3, attn_factor=float("nan"))])
def test_rope_refusals(change):
    rope = sidp.make_rope(theta=1e4, factor=4.0, original_len=4096)
    for k, v in change.items():
        setattr(rope, k, v)
    out, scale = (ctypes.c_double * 64)(), ctypes.c_double()
    assert sidp.raw_call("sidp_rope_frequencies", ctypes.byref(rope), 128, out, ctypes.byref(scale)) == E


def test_rope_refuses_head_dims_and_missing_arguments():
    rope = sidp.make_rope(rotary_dim=96)
    out, scale = (ctypes.c_double * 64)(), ctypes.c_double()
    call = lambda *a: sidp.raw_call("sidp_rope_frequencies", *a)  # noqa: E731
    assert call(ctypes.byref(rope), 64, out, ctypes.byref(scale)) == E  # more turned dims than the head has
    assert call(ctypes.byref(rope), 96, out, ctypes.byref(scale)) == E
    assert call(None, 128, out, ctypes.byref(scale)) == E
    assert call(ctypes.byref(rope), 128, None, ctypes.byref(scale)) == E
    assert call(ctypes.byref(rope), 128, out, None) == E
    assert sidp.raw_call("sidp_set_rope", None, ctypes.byref(rope)) == E
    with pytest.raises(KeyError):
        sidp.make_rope(layout="diagonal")


def test_calls_refuse_a_missing_handle():
    assert sidp.raw_call("sidp_kv_extend", None, FAKE, FAKE, 1, FAKE, 1, FAKE, FAKE, FAKE, 1, 1, FAKE, FAKE, FAKE, None) == E
    assert sidp.raw_call("sidp_rope_append_rows", None, FAKE, 512, 1, None, FAKE, FAKE, None, None, 0, FAKE, None) == E


def test_logprob_workspace_sizes():
    f = sidp.sidp_token_logprobs_bytes
    assert f(1, 1, 0) > 0 and f(1, 1, 1) > 0
    assert f(1, 1, 2) == 0  # more alternatives than tokens
    assert f(1, 1000, 33) == 0 and f(1, 1000, -1) == 0
    assert f(0, 1000, 1) == 0 and f(-1, 1000, 1) == 0 and f((1 << 20) + 1, 1000, 1) == 0
    assert f(1, 0, 0) == 0 and f(1, (1 << 20) + 1, 0) == 0
    # a row in segments keeps sums and its best of each; rows that fill the chip are not cut and keep nothing
    assert f(1, 1 << 20, 32) >= 2 * (16 + 32 * 8) and 0 < f(1 << 20, 1 << 20, 32) <= f(1, 1 << 20, 32)
    assert f(7, 50000, 5) >= 7 * 7 * (16 + 40)


def test_logprob_refusals():
    big = 1 << 30

    def call(logits=FAKE, dtype=1, rows=2, vocab=1000, stride=1000, targets=FAKE, top=3, ids=FAKE, lps=FAKE, ws=FAKE, n=big):
        return sidp.raw_call("sidp_token_logprobs", logits, dtype, rows, vocab, stride, targets, top, FAKE, FAKE, FAKE, ids,
                             lps, ws, n, None)
    assert call(rows=-1) == E and call(rows=(1 << 20) + 1) == E
    assert call(rows=0) == sidp.SIDP_OK  # nothing to do, nothing launched
    assert call(vocab=0) == E and call(vocab=(1 << 20) + 1, stride=1 << 21) == E
    assert call(stride=999) == E
    assert call(dtype=2) == E and call(dtype=-1) == E
    assert call(top=-1) == E and call(top=33) == E and call(vocab=2, top=3) == E
    assert call(logits=None) == E and call(logits=FAKE + 2) == E and call(logits=FAKE + 1, dtype=0) == E
    assert call(ids=None) == E and call(lps=None) == E
    assert call(ws=None) == E and call(ws=FAKE + 8) == E
    assert call(n=sidp.sidp_token_logprobs_bytes(2, 1000, 3) - 256) == E
