"""The host layer of rotary positions and of pages in 8 bits (argument checks, planning, workspace sizes) under the address and
undefined-behaviour sanitizers, driven through ordinary and extreme arguments (tests/sanitize/e4m3_driver.cpp).  CPU only."""
import os
import subprocess

import pytest

import test_sanitizers as S


def test_e4m3_host_layer_under_sanitizers(tmp_path):
    from paper_2606_00535_amd import build as B
    if not os.path.isdir(B.BUILD_DIR) or not all(
            os.path.exists(os.path.join(B.BUILD_DIR, os.path.basename(s) + ".o")) for s in B.sources()):
        B.build()
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc is not installed")
    host = [x for flag in S.SAN for x in ("-Xarch_host", flag)]     # host code only: the device code is built as usual
    api, driver = str(tmp_path / "api_san.o"), str(tmp_path / "e4m3_driver.o")
    subprocess.run([B.HIPCC] + [f for f in B.CFLAGS if f != "-O3"] + ["-O1", "-g"] + host +
                   ["-c", os.path.join(B.CSRC, "dreams_api.hip"), "-o", api], check=True, capture_output=True)
    subprocess.run([B.HIPCC, "-O1", "-g", "-std=c++17"] + host +
                   ["-I" + B.INCLUDE, "-I/opt/rocm/include", "-D__HIP_PLATFORM_AMD__", "-c",
                    os.path.join(S.HERE, "e4m3_driver.cpp"), "-o", driver], check=True, capture_output=True)
    objs = [os.path.join(B.BUILD_DIR, os.path.basename(s) + ".o") for s in B.sources()
            if os.path.basename(s) != "dreams_api.hip"]
    exe = str(tmp_path / "e4m3_driver")
    subprocess.run([B.HIPCC, "--offload-arch=" + B.ARCH] + host + ["-o", exe, driver, api] + objs,
                   check=True, capture_output=True)
    assert "e4m3 driver: ok" in S._run(exe, tmp_path)
