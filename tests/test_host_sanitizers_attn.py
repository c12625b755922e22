"""The attention plan's host code under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only): its validation,
work lists and argument checks (tests/test_attn_plan.py) against the host-sanitized library in a child process."""
import os
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, _gcc_runtime


def test_attention_plan_clean_under_asan_and_ubsan():
    asan, ubsan = _gcc_runtime("libasan.so"), _gcc_runtime("libubsan.so")
    if not (asan and ubsan):
        pytest.skip("gcc's sanitizer runtimes are not installed")
    from paper_2607_28848_amd import build as pkg_build
    lib = pkg_build.build_host_asan()
    env = dict(os.environ)
    pre = env.get("LD_PRELOAD")
    env.update({
        "LD_PRELOAD": asan + ":" + ubsan + ((":" + pre) if pre else ""),
        "ASAN_OPTIONS": "detect_leaks=0:verify_asan_link_order=0:abort_on_error=1",
        "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1",
        "DSV_LIBRARY": lib,
        "PYTHONPATH": ROOT + ((":" + env["PYTHONPATH"]) if env.get("PYTHONPATH") else ""),
    })
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_attn_plan.py"],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    log = res.stdout + res.stderr
    assert res.returncode == 0, log[-6000:]
    for marker in ("runtime error:", "AddressSanitizer"):
        assert marker not in log, log[-6000:]
    assert " passed" in log
