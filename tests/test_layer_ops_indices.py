"""The index arithmetic that the kernels around an attention share with the host (csrc/layer_index.h), under UBSan, at the ends of the
sizes that the calls take: what a work-group, a wave or a thread takes covers everything once and nothing else."""
import os
import subprocess

import pytest

from test_host_launch_model import CSRC, ROOT, STUB


@pytest.fixture(scope="module")
def indices(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("layer_indices") / "layer_indices")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-fno-sanitize-recover=undefined",
           "-I", STUB, "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(STUB, "layer_indices.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return exe


@pytest.mark.parametrize("part", ["rows", "rope", "quantise", "joins"])
def test_everything_once(indices, part):
    res = subprocess.run([indices, part], capture_output=True, text=True, timeout=600, env=dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1"))
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
