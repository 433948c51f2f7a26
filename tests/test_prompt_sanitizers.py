"""Host code of the rotary, prompt and shared-prefix operators under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU: builds their sources with the sanitizers applied to the host
compilation and runs tests/host_prompt_driver.cpp, which reaches no kernel launch."""

import os
import subprocess

import pytest

from paper_2608_00531_amd import build as pbuild
from test_host_sanitizers import HERE, SANITIZE, _run


@pytest.mark.skipif(not os.path.exists(pbuild.hipcc()), reason="hipcc not available")
def test_host_code_under_asan_and_ubsan(tmp_path):
    rocm = os.path.dirname(os.path.dirname(pbuild.hipcc()))
    clangxx = os.path.join(rocm, "llvm", "bin", "clang++")
    if not os.path.exists(clangxx):
        pytest.skip("ROCm clang++ not available")
    flags = [f for f in pbuild.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    objs = []
    for src in ("api.cpp", "tree_attn.hip", "rope.hip", "prompt_attn.hip"):
        objs.append(str(tmp_path / (src + ".o")))
        _run([pbuild.hipcc()] + flags + SANITIZE + ["-c", "-I", pbuild.INCLUDE, "-I", pbuild.CSRC,
                                                    os.path.join(pbuild.CSRC, src), "-o", objs[-1]], str(tmp_path))
    host_san = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    exe = str(tmp_path / "driver")
    _run([clangxx, "-O1", "-g", "-std=c++17"] + host_san +
         ["-I", pbuild.INCLUDE, os.path.join(HERE, "host_prompt_driver.cpp")] + objs +
         ["-L", os.path.join(rocm, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(rocm, "lib"), "-o", exe], str(tmp_path))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = res.stdout + res.stderr
    assert res.returncode == 0 and "0 failure(s)" in res.stdout, out
    assert "runtime error" not in out and "AddressSanitizer" not in out, out
