"""Waits of the attention of several new tokens a sequence, in the code that is
built: a wave that reaches a barrier has no LDS operation of its own under way, so
what lies behind the barrier (tiles that other waves load over the ones it read,
values that they change by atomics) cannot meet it."""

import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("sidp_build_flags", os.path.join(ROOT, "paper_2605_28095_amd", "build.py"))
build = importlib.util.module_from_spec(spec)
spec.loader.exec_module(build)

WAIT = re.compile(r"\bs_waitcnt\b.*\blgkmcnt\(0\)")


def barriers(lines):
    """(line number, whether it is waited for LDS right before it) of every barrier: back from it, the wait comes before any LDS
    operation and before the block's start."""
    for i, line in enumerate(lines):
        if not re.search(r"^\s*s_barrier\b", line):
            continue
        waited = False
        for back in reversed(lines[:i]):
            code = back.split(";")[0].strip()
            if WAIT.search(code):
                waited = True
                break
            if code.startswith("ds_") or code.endswith(":") or code.startswith(("s_branch", "s_cbranch")):
                break
        yield i, waited


def test_the_reader_sees_a_missing_wait():
    good = ["x:", "  ds_read_b128 v[0:3], v4", "  s_waitcnt vmcnt(8) lgkmcnt(0)", "  s_add_u32 s0, s0, s1", "  s_barrier"]
    assert list(barriers(good)) == [(4, True)]
    assert list(barriers([good[0], good[2], good[1], good[4]])) == [(3, False)]  # a read behind the wait
    assert list(barriers([good[1], "  s_waitcnt vmcnt(8)", good[4]])) == [(2, False)]
    assert list(barriers([good[1], good[2], ".LBB0_1:", good[4]])) == [(3, False)]  # another way in
    assert list(barriers([good[1], "  s_waitcnt lgkmcnt(1)", good[4]])) == [(2, False)]


def test_no_lds_operation_is_under_way_at_a_barrier(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "rows.s")
    subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "k_attn_rows.hip"), "-o", out],
                   check=True, capture_output=True, timeout=300)
    with open(out) as f:
        text = f.read()
    kernels = re.findall(r"^(_Z\w*11k_attn_rowsILi\d+E\w*):(.*?)^\.Lfunc_end", text, re.M | re.S)
    assert len(kernels) == 2  # heads of 64 and of 128
    for name, body in kernels:
        lines = body.splitlines()
        found = list(barriers(lines))
        assert len(found) >= 8, name
        missing = [i for i, waited in found if not waited]
        assert not missing, f"{name}: {len(missing)} of {len(found)} barriers without a wait, first at line {missing[0]}"
