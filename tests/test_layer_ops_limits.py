"""Which sizes the operators around an attention take, against recorded launches: nothing is run and nothing allocated."""
import os
import subprocess

from test_host_launch_model import CSRC, ROOT, STUB


def test_sizes_that_are_taken_and_refused(tmp_path):
    exe = str(tmp_path / "layer_limits")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-fno-sanitize-recover=undefined",
           "-I", STUB, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *(os.path.join(CSRC, f) for f in ("layer_api.cpp", "pattern_compiler.cpp")),
           os.path.join(STUB, "layer_limits.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
