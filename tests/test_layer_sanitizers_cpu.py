"""Host sanitizer runs of the gated-delta layer: the oracle's delta rule and the
C-ABI layer's host code, built with AddressSanitizer and
UndefinedBehaviorSanitizer into standalone executables (tests/sanitize/), as
test_sanitizers_cpu.py does for the rest of the library."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers_cpu import CSRC, HERE, HIPCC, INCLUDE, ROOT, SAN_HOST, _clean_env, _run


def _passes(exe):
    res = subprocess.run([exe], capture_output=True, text=True, env=_clean_env(), timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "all checks passed" in res.stdout
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_oracle_delta_under_sanitizers(tmp_path):
    exe = str(tmp_path / "oracle_asan")
    _run(["gcc", "-O1", "-g", "-std=c11", "-fno-omit-frame-pointer", "-pthread", "-fsanitize=address,undefined",
          "-fno-sanitize-recover=all", os.path.join(ROOT, "oracle", "precog_oracle.c"),
          os.path.join(HERE, "layer_oracle_driver.c"), "-o", exe, "-lm"], str(tmp_path))
    _passes(exe)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_layer_abi_under_sanitizers(tmp_path):
    common = ["-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-I", INCLUDE,
              "-I", CSRC] + SAN_HOST
    objs = []
    for src in (os.path.join(CSRC, "precog_abi.cpp"), os.path.join(CSRC, "layer_abi.cpp"),
                os.path.join(HERE, "launch_stubs.cpp"), os.path.join(HERE, "layer_stubs.cpp"),
                os.path.join(HERE, "layer_abi_driver.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([HIPCC] + common + ["-c", src, "-o", obj], str(tmp_path))
        objs.append(obj)
    exe = str(tmp_path / "layer_asan")
    _run([HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"] +
         objs + ["-o", exe], str(tmp_path))
    _passes(exe)
