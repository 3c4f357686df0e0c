"""The host side of the operators around the gated prefill (eta_train_api.cpp: argument
checks, work plans, workspace carve-up) built with g++ under the address and
undefined-behaviour sanitizers against stub launchers; no GPU."""
import os
import shutil

import pytest

from test_cpu_tier import CSRC, INC, ROCM_INC, TIER, _build_and_run

pytestmark = pytest.mark.skipif(
    shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM_INC, "hip", "hip_runtime_api.h")),
    reason="g++ or the HIP headers not available")


def test_train_api_sanitized(tmp_path):
    _build_and_run(tmp_path, "train_harness",
                   [os.path.join(CSRC, "eta_train_api.cpp"), os.path.join(TIER, "train_harness.cpp")],
                   ["-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INC, "-I" + INC, "-I" + CSRC])
