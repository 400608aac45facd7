"""What the vocabulary's operators launch (vocab_plans.hpp), under AddressSanitizer and
UndefinedBehaviorSanitizer on the CPU: the choices as a call makes them, with both types of
gradients, and the zeros of few tokens byte by byte."""
import os
import shutil

import pytest

from test_host_sanitizers import NATIVE, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not available")


@pytest.mark.timeout(600)
def test_launches(tmp_path):
    exe = str(tmp_path / "vocab_launches")
    _build(exe, [os.path.join(NATIVE, "vocab_launches.cpp")], ["-fsanitize=address,undefined"])
    rc, out, err = _run(exe, {"ASAN_OPTIONS": "detect_leaks=0", "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert rc == 0 and "vocabulary launches ok" in out, (out + err)[-4000:]
    assert "runtime error" not in err and "AddressSanitizer" not in err, err[-4000:]
