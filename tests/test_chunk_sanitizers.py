"""The host side of the calls for chunks (csrc/akvq_chunk_api.hip) under AddressSanitizer and UndefinedBehaviorSanitizer, host pass only, with
the launchers replaced by stubs that check bounds, tiles and grids (tests/sanitize/chunk_driver.cpp): sizes at the ends of the
int range, page sizes, heads, strides and splits, in all pairs."""
import os
import shutil

import pytest

from test_sanitizers import ROOT, SAN, _run


def test_chunk_calls_under_address_and_ub_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "chunk_san")
    host_san = [x for flag in SAN for x in ("-Xarch_host", flag)]
    out = _run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", *host_san, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                os.path.join(ROOT, "paper_2501_15021_amd", "csrc", "akvq_chunk_api.hip"),
                "-x", "hip", os.path.join(ROOT, "tests", "sanitize", "chunk_driver.cpp"), "-o", exe], exe)
    assert int(out.split()[1]) >= 1000
