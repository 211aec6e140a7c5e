"""The library's build script with a stand-in for the compiler: what an interrupted build leaves is not taken as built."""
import os
import stat

import pytest

COMPILER = """#!/bin/sh
# writes half of its output, then the rest; a file "die_<word>" beside this script ends it in between for outputs with that word
here=$(dirname "$0"); out=""; last=""
for a in "$@"; do [ "$last" = "-o" ] && out="$a"; last="$a"; done
printf half > "$out"
for f in "$here"/die_*; do
  [ -e "$f" ] || continue
  case "$out" in *"${f##*/die_}"*) kill -9 $$ ;; esac
done
printf ' whole' >> "$out"
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    from paper_2207_02849_b200 import build
    csrc = tmp_path / "pkg" / "csrc"
    csrc.mkdir(parents=True)
    (tmp_path / "include").mkdir()
    (tmp_path / "include" / "betty.h").write_text("")
    for n in ("one.cu", "two.cu"):
        (csrc / n).write_text("")
    cc = tmp_path / "nvcc"
    cc.write_text(COMPILER)
    cc.chmod(cc.stat().st_mode | stat.S_IXUSR)
    for k, v in dict(PKG_DIR=str(tmp_path / "pkg"), ROOT=str(tmp_path), CSRC=str(csrc), LIB_PATH=str(tmp_path / "pkg" / "lib.so"),
                     SOURCES=["one.cu", "two.cu"], FAMILY_SOURCES=[], _nvcc=lambda: str(cc)).items():
        monkeypatch.setattr(build, k, v)
    return build, tmp_path


def _read(path):
    with open(path) as f:
        return f.read()


@pytest.mark.parametrize("word", ["two.o", "lib.so"])
def test_an_interrupted_output_is_made_again(tree, word):
    build, root = tree
    (root / ("die_" + word)).write_text("")
    with pytest.raises(RuntimeError):
        build.build()
    os.remove(root / ("die_" + word))
    assert _read(build.build()) == "half whole"
    made = sorted(os.listdir(os.path.join(build.PKG_DIR, "_build")))
    assert made == ["one.o", "two.o"]
    for n in made:
        assert _read(os.path.join(build.PKG_DIR, "_build", n)) == "half whole"


def test_only_what_is_older_than_its_sources_is_compiled(tree):
    build, root = tree
    build.build()
    objs = [os.path.join(build.PKG_DIR, "_build", n) for n in ("one.o", "two.o")]
    for f in objs + [build.LIB_PATH]:
        os.utime(f, (2e9, 2e9))
    os.utime(os.path.join(build.CSRC, "two.cu"), (2.1e9, 2.1e9))
    build.build()
    assert os.path.getmtime(objs[0]) == 2e9 and os.path.getmtime(objs[1]) != 2e9
