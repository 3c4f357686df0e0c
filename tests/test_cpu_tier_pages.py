"""The host side of the paged cache (eta_page_api.cpp: argument checks, plans, workspace carve-up)
built with g++ under the address and undefined-behaviour sanitizers against stub launchers; no GPU."""
import os
import shutil

import pytest

from test_cpu_tier import CSRC, INC, ROCM_INC, TIER, _build_and_run

pytestmark = pytest.mark.skipif(
    shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM_INC, "hip", "hip_runtime_api.h")),
    reason="g++ or the HIP headers not available")


def test_page_api_sanitized(tmp_path):
    _build_and_run(tmp_path, "page_harness",
                   [os.path.join(CSRC, f) for f in ("eta_api.cpp", "eta_page_api.cpp")] + [os.path.join(TIER, "page_harness.cpp")],
                   ["-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INC, "-I" + INC, "-I" + CSRC])
