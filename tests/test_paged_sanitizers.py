"""Host side of the paged cache under sanitizers, and its launches of very many rows, on the CPU (tests/san/).  No kernel runs."""
import os
import shutil

import pytest

from tests.test_sanitizers import HIPCC, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_host_side_of_the_paged_calls_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    exe = str(tmp_path / "paged_abi_san")
    csrc = os.path.join(ROOT, "paper_2410_07590_amd", "csrc")
    # each -fsanitize= sits directly behind -Xarch_host: only the host pass is instrumented
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
          "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wl,--unresolved-symbols=ignore-all",
          "-o", exe, os.path.join(SAN, "paged_abi_san.cpp"), os.path.join(csrc, "tr_api.hip"), os.path.join(csrc, "tr_paged_api.hip")])
    assert "paged abi sanitizer run ok: 4000 mixes" in _run([exe, "4000"])


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_launches_of_very_many_rows_are_legal(tmp_path):
    from paper_2410_07590_amd import binding as B
    B.lib()
    exe = str(tmp_path / "paged_launches")
    _run(["g++", "-O1", "-std=c++17", "-Wall", "-rdynamic", "-o", exe, os.path.join(SAN, "paged_launches.cpp"), "-ldl"])
    assert "paged launches ok" in _run([exe, B.lib_path()])
