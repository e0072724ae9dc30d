"""The timing records of launches (csrc/prof.h) are made inside C entry points: neither function may throw."""
import os
import subprocess

import pytest

from paper_2609_34318_amd import build_lib

SOURCE = """
#include "prof.h"
static_assert(noexcept(hydra::prof_begin("", hipStream_t{})), "prof_begin");
static_assert(noexcept(hydra::prof_end(0, hipStream_t{})), "prof_end");
"""


@pytest.mark.skipif(not os.path.exists(build_lib.HIPCC), reason="hipcc not available")
def test_records_do_not_throw(tmp_path):
    src = tmp_path / "records.cpp"
    src.write_text(SOURCE)
    r = subprocess.run([build_lib.HIPCC, "-x", "hip", "-std=c++17", f"--offload-arch={build_lib.ARCH}", "-fsyntax-only",
                        f"-I{build_lib.CSRC}", str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
