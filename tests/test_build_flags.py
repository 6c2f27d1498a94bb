"""How the sources are compiled."""
import os

from paper_2506_03065_amd import build as b


def flags(monkeypatch, source):
    monkeypatch.setattr(b, "hipcc_path", lambda: "hipcc")
    return b.compile_command(source, "out.o")


def test_what_is_said_of_nan_is_not_left_to_the_compiler(monkeypatch):
    """The operators around the attention define what happens with infinities and NaN."""
    for s in ("norm_kernels.hip", "rope_kernels.hip", "blockscale_kernels.hip", "layer_api.cpp"):
        assert s in b.SOURCES
        assert not {"-fno-honor-nans", "-ffinite-math-only", "-ffast-math", "-Ofast"} & set(flags(monkeypatch, s))


def test_every_source_is_compiled_for_the_chip_without_packed_fp32(monkeypatch):
    for s in b.SOURCES:
        cmd = flags(monkeypatch, s)
        assert "--offload-arch=gfx950" in cmd and "-packed-fp32-ops" in cmd and os.path.join(b.CSRC, s) in cmd
        assert cmd[cmd.index("-packed-fp32-ops") - 3:cmd.index("-packed-fp32-ops")] == ["-Xclang", "-target-feature", "-Xclang"]
