"""The build's steps (commands recorded, nothing compiled)."""
import os

import pytest

from paper_2601_21896_amd import build


@pytest.fixture
def steps(monkeypatch, tmp_path):
    done = []
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libpafu.so"))
    monkeypatch.setattr(build, "CALL", str(tmp_path / "_paged_call.so"))
    monkeypatch.setattr(build, "hipcc", lambda: "hipcc")

    def run(cmd):
        target = os.path.basename(cmd[cmd.index("-o") + 1])
        if target == "_paged_call.so":
            raise RuntimeError("no headers")
        done.append(target)
        return ""
    monkeypatch.setattr(build, "_run", run)
    return done


def test_a_module_that_does_not_compile_leaves_the_library(steps, tmp_path):
    (tmp_path / "_paged_call.so").write_text("of an older source")
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert steps[-1] == "libpafu.so" and len(steps) == len(build.SOURCES) + 1
    assert not (tmp_path / "_paged_call.so").exists()     # not one that belongs to another library


def test_a_study_build_makes_no_module(steps, tmp_path):
    build.build(out="study.so")
    assert steps[-1] == "study.so" and len(steps) == len(build.SOURCES) + 1
