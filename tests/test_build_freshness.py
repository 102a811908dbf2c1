"""Which objects a build compiles again: those whose sources, flags or compiler changed, and those whose compilation did not end.  A script stands in for
the compiler, so nothing is compiled."""
import os
import stat

import pytest

from paper_2510_01565_b200 import build

COMPILER = """#!/bin/sh
if [ "$1" = --version ]; then echo release {version}; exit 0; fi
for last; do true; done
case " $* " in *" -c "*) ;; *) while [ $# -gt 0 ]; do [ "$1" = -o ] && echo linked > "$2"; shift; done; exit 0;; esac
while [ $# -gt 0 ]; do
  [ "$1" = -MF ] && dep="$2"
  [ "$1" = -c ] && src="$2"
  shift
done
echo "$src" >> {log}
echo "$last : $src" > "$dep"
echo object > "$last"
exit {code}
"""


@pytest.fixture
def project(tmp_path, monkeypatch):
    """Two sources; compile(version, code) builds and names what was compiled."""
    sources = [tmp_path / "one.cu", tmp_path / "two.cu"]
    for s in sources:
        s.write_text("source")
        os.utime(s, (1e9, 1e9))
    log, compiler = tmp_path / "log", tmp_path / "nvcc"
    monkeypatch.setenv("NVCC", str(compiler))
    for name, value in (("SOURCES", [str(s) for s in sources]), ("OBJECTS", str(tmp_path / "obj")), ("LIB", str(tmp_path / "lib.so")),
                        ("build_marshal", lambda: None), ("_newest_source_mtime", lambda: float("inf"))):
        monkeypatch.setattr(build, name, value)

    def compile(version=1, code=0, **kw):
        log.write_text("")
        compiler.write_text(COMPILER.format(version=version, log=log, code=code))
        compiler.chmod(compiler.stat().st_mode | stat.S_IEXEC)
        try:
            build.build_library(**kw)
        finally:
            done = sorted(os.path.basename(line) for line in log.read_text().split())
        return done
    compile.sources = sources
    return compile


def test_only_what_changed_is_compiled_again(project):
    assert project() == ["one.cu", "two.cu"]
    assert project() == []
    project.sources[1].write_text("changed")
    assert project() == ["two.cu"]
    assert project() == []
    assert project(verbose=True) == []
    assert project(force=True) == ["one.cu", "two.cu"]


def test_other_flags_compile_everything_again(project, monkeypatch):
    project()
    monkeypatch.setattr(build, "NVCC_FLAGS", build.NVCC_FLAGS + ["-DX=1"])
    assert project() == ["one.cu", "two.cu"]
    assert project() == []


def test_another_compiler_compiles_everything_again(project):
    project()
    assert project(version=2) == ["one.cu", "two.cu"]
    assert project(version=2) == []


def test_an_object_that_a_failed_compilation_left_is_not_used(project):
    project()
    project.sources[0].write_text("broken")
    with pytest.raises(RuntimeError):
        project(code=1)                                  # (this compiler leaves an object behind)
    assert project() == ["one.cu"]


def test_a_source_that_changes_while_it_is_compiled_is_compiled_again(project, monkeypatch):
    project()
    project.sources[0].write_text("changed")
    popen = build.subprocess.Popen

    def slow(cmd, **kw):
        job = popen(cmd, **kw)
        if "-c" not in cmd:
            return job
        job.wait()
        now = os.path.getmtime(cmd[-1])
        os.utime(project.sources[0], (now + 5, now + 5))               # saved again before the object was written
        os.utime(cmd[-1], (now + 10, now + 10))
        return job
    monkeypatch.setattr(build.subprocess, "Popen", slow)
    assert project() == ["one.cu"]
    monkeypatch.setattr(build.subprocess, "Popen", popen)
    assert project() == ["one.cu"]


def test_the_file_that_holds_the_flags_counts_as_a_source(tmp_path, monkeypatch):
    later = tmp_path / "build.py"
    later.write_text("")
    at = build._newest_source_mtime() + 1000.0
    os.utime(later, (at, at))
    monkeypatch.setattr(build, "__file__", str(later))
    assert build._newest_source_mtime() == at
