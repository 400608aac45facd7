"""The vocabulary's operators' host code (vocab_ops.cpp) and plans under
AddressSanitizer and UndefinedBehaviorSanitizer on the CPU, with the launchers stubbed
out: seeded random sizes, the overlap rules against brute force."""
import os
import shutil

import pytest

from test_host_sanitizers import CSRC, NATIVE, ROCM, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")),
                                reason="g++ or the HIP headers are not available")


@pytest.mark.timeout(600)
def test_vocabulary_operators_host_code(tmp_path):
    exe = str(tmp_path / "vocab_checks")
    _build(exe, [os.path.join(NATIVE, "vocab_checks.cpp"), os.path.join(CSRC, "vocab_ops.cpp")],
           ["-fsanitize=address,undefined", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-Wno-unknown-pragmas"],
           libs=["-L", os.path.join(ROCM, "lib"), "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}"])
    rc, out, err = _run(exe, {"ASAN_OPTIONS": "detect_leaks=0", "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert rc == 0 and "vocabulary checks ok" in out, (out + err)[-4000:]
    assert "runtime error" not in err and "AddressSanitizer" not in err, err[-4000:]
