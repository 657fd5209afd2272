"""The build script: what it compiles again and what it takes over (a stand-in for nvcc, no compiler runs)."""
import os
import stat

import pytest

from paper_2609_13285_b200 import build as gbuild

NVCC = """#!/bin/sh
echo "$@" >> "$NVCC_SAYS"
while [ $# -gt 0 ]; do
  if [ "$1" = -o ]; then echo "part" > "$2"; fi
  shift
done
exit ${NVCC_RC:-0}
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A tree of its own with empty sources; tree() = the command lines since the last call."""
    csrc = tmp_path / "package" / "csrc"
    csrc.mkdir(parents=True)
    (tmp_path / "include").mkdir()
    for source, headers in gbuild.SOURCES.items():
        for f in [source] + headers:
            (csrc / f).write_text("")
            os.utime(csrc / f, (1, 1))
    nvcc, says = tmp_path / "nvcc", tmp_path / "says"
    nvcc.write_text(NVCC)
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IEXEC)
    monkeypatch.setattr(gbuild, "CSRC", str(csrc))
    monkeypatch.setattr(gbuild, "LIB", str(tmp_path / "package" / "libgva.so"))
    for name in ("GVA_LIBRARY", "GVA_EXTRA_NVCC_FLAGS", "NVCC_RC"):
        monkeypatch.delenv(name, raising=False)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.setenv("NVCC_SAYS", str(says))

    def said():
        lines = says.read_text().splitlines() if says.exists() else []
        says.unlink(missing_ok=True)
        return lines
    return said


def compiled(lines):
    return sorted(s for s in gbuild.SOURCES for line in lines if " -c" in " " + line and s + " " in line)


def test_nothing_is_done_twice(tree):
    gbuild.build()
    assert compiled(tree()) == sorted(gbuild.SOURCES)
    gbuild.build()
    assert tree() == []
    os.unlink(gbuild.LIB)
    gbuild.build()
    lines = tree()
    assert compiled(lines) == [] and len(lines) == 1 and "-shared" in lines[0]
    gbuild.build(force=True)
    assert compiled(tree()) == sorted(gbuild.SOURCES)


def test_a_newer_source_is_compiled_again(tree):
    gbuild.build()
    tree()
    source = sorted(gbuild.SOURCES)[0]
    os.utime(os.path.join(gbuild.CSRC, source), (2 ** 32, 2 ** 32))
    gbuild.build()
    assert compiled(tree()) == [source]


def test_other_flags_are_not_answered_with_old_objects(tree, monkeypatch):
    gbuild.build()
    tree()
    os.unlink(gbuild.LIB)
    monkeypatch.setenv("GVA_EXTRA_NVCC_FLAGS", "-DGVA_SOMETHING=1")
    gbuild.build()
    lines = tree()
    assert compiled(lines) == sorted(gbuild.SOURCES)
    assert all("-DGVA_SOMETHING=1" in line for line in lines if "-shared" not in line)


def test_verbose_prints_what_every_source_gives(tree):
    gbuild.build()
    tree()
    os.unlink(gbuild.LIB)
    gbuild.build(verbose=True)
    assert compiled(tree()) == sorted(gbuild.SOURCES)


def test_what_a_failed_compiler_left_is_not_linked(tree, monkeypatch):
    monkeypatch.setenv("NVCC_RC", "1")
    with pytest.raises(RuntimeError):
        gbuild.build()
    tree()
    monkeypatch.delenv("NVCC_RC")
    gbuild.build()
    assert compiled(tree()) == sorted(gbuild.SOURCES)
