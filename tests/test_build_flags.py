"""The flags each source of the library is compiled with: those of all files everywhere, the accumulators' form where it belongs."""
import os

import pytest

from paper_2605_11354_amd import build


@pytest.mark.parametrize("src", build.SOURCES)
def test_flags(src, monkeypatch):
    def check():
        flags, form = build.flags_of(src), "-amdgpu-mfma-vgpr-form=1"
        assert flags[:len(build.FLAGS)] == build.FLAGS and "-packed-fp32-ops" in flags
        assert (form in flags) == (src not in build.AGPR_FORM)
        if form in flags:
            assert flags[flags.index(form) - 1] == "-mllvm"
    check()
    monkeypatch.setattr(build, "FLAGS", build.FLAGS + ["-DANOTHER"])                         # a flag appended reaches every file
    check()


def test_sources_are_there():
    assert set(build.AGPR_FORM) <= set(build.SOURCES) and all(os.path.exists(os.path.join(build.CSRC, s)) for s in build.SOURCES)
