"""The row operators' plans (row_plans.hpp, as the library compiles it) and the
workspaces derived from them, on the CPU under AddressSanitizer and
UndefinedBehaviorSanitizer."""
import os
import shutil

import pytest

from test_host_sanitizers import CSRC, NATIVE, ROCM, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")),
                                reason="g++ or the HIP headers are not available")


@pytest.mark.timeout(600)
def test_plans(tmp_path):
    exe = str(tmp_path / "row_plan_checks")
    _build(exe, [os.path.join(NATIVE, "row_plan_checks.cpp"), os.path.join(CSRC, "row_ops.cpp")],
           ["-fsanitize=address,undefined", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-Wno-unknown-pragmas"],
           libs=["-L", os.path.join(ROCM, "lib"), "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}"])
    rc, out, err = _run(exe, {"ASAN_OPTIONS": "detect_leaks=0", "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert rc == 0 and "row plan checks ok" in out, (out + err)[-4000:]
    assert "runtime error" not in err and "AddressSanitizer" not in err, err[-4000:]
