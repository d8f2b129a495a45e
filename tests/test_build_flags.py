"""Which sources the build compiles under the assumption that no value is a NaN."""
import os

from paper_2607_20125_amd import build


def commands(monkeypatch):
    """Compiler command of every source, without running one."""
    found = {}

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def record(cmd, **_):
        if "-c" in cmd:
            found[os.path.basename(cmd[cmd.index("-c") + 1])] = cmd
        return Done

    monkeypatch.setattr(build.subprocess, "run", record)
    monkeypatch.setattr(build.os, "replace", lambda *_: None)
    build.build_library()
    assert sorted(found) == sorted(build.SOURCES)
    return found


def test_no_source_that_meets_nan_is_compiled_without_it(monkeypatch):
    """The operators beside the routed attention pass a NaN on (a cache's groups, a sequence's keys), and the entry
    points look for it in their arguments."""
    for src, cmd in commands(monkeypatch).items():
        if src in ("hc_ops.cpp", "hc_runtime.cpp", "hc_rotate.hip", "hc_qcache.hip", "hc_seq.hip", "hc_seq128.hip",
                   "hc_decode.hip"):
            bad = [f for f in cmd if f in ("-fno-honor-nans", "-ffinite-math-only", "-ffast-math", "-Ofast")]
            assert not bad, (src, bad)


def test_every_source_is_kept_from_packed_fp32(monkeypatch):
    for src, cmd in commands(monkeypatch).items():
        assert "-packed-fp32-ops" in cmd, src
