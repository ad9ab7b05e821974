"""The attention entries' host code (sizes, strides, spans, parts, workspaces) under
AddressSanitizer and UndefinedBehaviorSanitizer, in the build and manner of
test_sanitized_cpu.py."""
import os
import shutil
import sys

import pytest

from test_sanitized_cpu import ROOT, _exported, _load, _run_pytest


@pytest.mark.skipif(shutil.which("nm") is None, reason="binutils nm not available")
def test_attention_entries_under_sanitizers():
    sys.path.insert(0, os.path.join(ROOT, "paper_2308_15152_amd"))
    build_sanitized = _load("paper_2308_15152_amd/build_sanitized.py", "sgemm_emu_build_sanitized")
    lib = build_sanitized.build()
    assert "__asan_" in _exported(lib) and "__ubsan_" in _exported(lib), "not instrumented"
    _run_pytest({"SGEMM_EMU_LIB": lib, "LD_PRELOAD": build_sanitized.asan_runtime()},
                ["tests/test_attention_cpu.py"], [])
