"""Refusals of sidp_sample_tokens that are decided before any GPU work."""

import importlib.util
import os
import subprocess

import pytest

import paper_2605_28095_amd as sidp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

E = sidp.SIDP_EINVAL
FAKE = 1 << 20  # an aligned address that a refused call never reads


def test_workspace_sizes():
    f = sidp.sidp_sample_tokens_bytes
    assert f(1, 1) > 0 and f(1 << 16, 1 << 20) > 0
    assert f(0, 10) == 0 and f(-1, 10) == 0 and f((1 << 16) + 1, 10) == 0 and f(1, 0) == 0 and f(1, (1 << 20) + 1) == 0


def test_refusals():
    def call(logits=FAKE, dtype=1, rows=2, vocab=1000, stride=1000, u=FAKE, tokens=FAKE, ws=FAKE, n=1 << 30):
        return sidp.raw_call("sidp_sample_tokens", logits, dtype, rows, vocab, stride, None, None, None, None, u, tokens, None, None, ws, n,
                             None)
    assert call(rows=0) == sidp.SIDP_OK  # nothing to do, nothing launched
    assert call(rows=-1) == E and call(rows=(1 << 16) + 1) == E
    assert call(vocab=0) == E and call(vocab=(1 << 20) + 1, stride=1 << 21) == E and call(stride=999) == E
    assert call(dtype=2) == E and call(dtype=-1) == E
    assert call(logits=None) == E and call(logits=FAKE + 2) == E and call(logits=FAKE + 1, dtype=0) == E
    assert call(u=None) == E and call(tokens=None) == E
    assert call(ws=None) == E and call(ws=FAKE + 8) == E and call(n=sidp.sidp_sample_tokens_bytes(2, 1000) - 1) == E


def test_lds_is_addressed_as_lds(tmp_path):
    """A flat access decides by its address register alone, before its offset is added, whether it goes to LDS: the compiler may put
    the register in front of the first byte of LDS, which faults. The kernels' LDS accesses say what they are, and none is flat."""
    spec = importlib.util.spec_from_file_location("sidp_build_flags", os.path.join(ROOT, "paper_2605_28095_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "sample.s")
    subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "k_sample.hip"), "-o", out], check=True,
                   capture_output=True, timeout=300)
    with open(out) as f:
        lines = [line.split(";")[0].strip() for line in f]
    assert any(line.startswith("ds_") for line in lines)
    assert [line for line in lines if line.startswith(("flat_", "s_swappc"))] == []
