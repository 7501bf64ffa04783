"""The host code of routing, combining, products of codes and the AdamW step under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): the tests of their checks of arguments, sizes and memory run against a library
whose host code is instrumented."""
import os
import subprocess

import pytest

from tests.test_sanitizers import HIPCC, ROOT, _clang_asan_runtime, _run

TESTS = ["test_route.py", "test_combine.py", "test_int8.py", "test_adamw.py"]


@pytest.mark.skipif(not os.path.exists(HIPCC) or _clang_asan_runtime() is None, reason="hipcc and clang's ASan runtime")
def test_routing_host_code_under_asan_ubsan(tmp_path):
    lib = str(tmp_path / "libpnn_asan.so")
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-O1", "-Xarch_device", "-O0", "-std=c++17", "-fPIC", "-shared",
                           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
                           "-Xarch_host", "-fno-omit-frame-pointer",
                           "-o", lib, os.path.join(ROOT, "paper_2304_09590_amd", "csrc", "pnn.hip")],
                          stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    first, *rest = [os.path.join(ROOT, "tests", t) for t in TESTS]
    setup = ("import os, torch\nfrom paper_2304_09590_amd import pnn\n"
             f"pnn.LIB_PATH = {lib!r}\n"
             f"os.environ['PYTEST_ADDOPTS'] = \"-m 'not gpu' \" + {' '.join(rest)!r}")
    _run(tmp_path, setup, first, lib, _clang_asan_runtime())
