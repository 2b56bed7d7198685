"""The workspace checks of the paged attention, in a CPU build with sanitizers and stub launchers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_attention_workspaces_under_sanitizers(tmp_path):
    san, csrc = os.path.join(ROOT, "tests", "abi_sanitize"), os.path.join(ROOT, "paper_2605_28760_amd", "csrc")
    exe = str(tmp_path / "decode_workspace_check")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-static-libasan", "-static-libubsan", "-D__HIP_PLATFORM_AMD__",
           "-I/opt/rocm/include", "-I" + csrc, os.path.join(csrc, "zo_abi.cpp"), os.path.join(csrc, "zo_decode_abi.cpp"),
           os.path.join(san, "launch_stubs.cpp"), os.path.join(san, "decode_stubs.cpp"),
           os.path.join(san, "decode_workspace_check.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert " 0 failed" in run.stdout, run.stdout
