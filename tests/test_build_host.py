"""CPU-only checks of what the build rebuilds and of what it needs for what."""
import os

import pytest

from paper_2511_15927_amd import build


def test_an_object_is_as_old_as_all_that_its_source_includes():
    """Headers that a source reaches through others count: an object of an older one would be linked with objects of the newer one."""
    def names(src):
        return {os.path.basename(p) for p in build.includes_of(os.path.join(build.CSRC, src))}
    for src in ("embed.hip", "norm.hip", "scores.hip", "clip.hip"):
        assert names(src) == {src, "model_ops.h", "kernels.h", "launch.h", "bimamba.h"}
    assert names("bwd_inst.hip") == {"bwd_inst.hip", "kernels.h", "launch.h", "bwd_kernels.h"}
    assert "ssd_wide.h" in names("ssd_wide_inst.hip") and "ssd_kernels.h" in names("ssd_wide_inst.hip")
    assert names("torch_calls.cpp") == {"torch_calls.cpp", "bimamba.h"}
    # every header is reached by some source
    every = set().union(*(names(f) for f in os.listdir(build.CSRC) if not f.endswith(".h")))
    assert {f for f in os.listdir(build.CSRC) if f.endswith(".h")} <= every


def test_the_library_is_linked_without_what_the_extension_module_needs(monkeypatch, tmp_path):
    """A machine without g++ or the headers of Python and torch gets the C library, and an error that names what is missing."""
    ran = []
    monkeypatch.setattr(build, "_run", lambda cmd: ran.append(cmd) or "")
    monkeypatch.setattr(build, "OBJ", str(tmp_path))

    def missing(force):
        raise RuntimeError("no torch headers")
    monkeypatch.setattr(build, "compile_calls", missing)
    with pytest.raises(RuntimeError, match="no torch headers"):
        build.build(force=True)
    assert all(cmd[0] == "hipcc" for cmd in ran)
    assert sum("-shared" in cmd and build.LIB in cmd for cmd in ran) == 1 and "-shared" in ran[-1]
