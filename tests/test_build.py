"""What the build hands to the compiler, by a stand-in for hipcc that writes its arguments down; nothing is compiled."""
import os
import stat
import sys

from paper_2408_12588_amd import build as pab_build

STAND_IN = """#!%s
import os, sys
with open(os.environ["ARGUMENTS"], "a") as f:
    f.write("\\t".join(sys.argv[1:]) + "\\n")
open(sys.argv[sys.argv.index("-o") + 1], "w").close()
"""


def calls(tmp_path, monkeypatch, run):
    tool, log = tmp_path / "hipcc", tmp_path / "arguments"
    tool.write_text(STAND_IN % sys.executable)
    tool.chmod(tool.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("HIPCC", str(tool))
    monkeypatch.setenv("ARGUMENTS", str(log))
    run()
    return [line.split("\t") for line in log.read_text().splitlines()]


def test_extra_flags_reach_every_step(tmp_path, monkeypatch):
    """A sanitizer or a library is as much the link's as the compiler's."""
    monkeypatch.setattr(pab_build, "LIB", str(tmp_path / "libpab.so"))
    got = calls(tmp_path, monkeypatch, lambda: pab_build.build_lib(extra_flags=["-Xsome", "--flag"]))
    compiled = [a for a in got if "-c" in a]
    linked = [a for a in got if "-shared" in a]
    assert sorted(a[-1] for a in compiled) == sorted(pab_build.SOURCES + pab_build.SOURCES_NAN) and len(linked) == 1 and len(got) == len(compiled) + 1
    assert all(a[a.index("-Xsome") + 1] == "--flag" for a in got)
    assert all("-packed-fp32-ops" in a for a in compiled)
    assert os.listdir(tmp_path).count("libpab.so") == 1 and not [f for f in os.listdir(tmp_path) if f.endswith(".o")]


def test_assembly_is_of_every_source(tmp_path, monkeypatch):
    """... so that what is held of the generated code is held of all kernels, compiled as they are for the library."""
    path = str(tmp_path / "out" / "pab.s")
    os.mkdir(tmp_path / "out")
    got = calls(tmp_path, monkeypatch, lambda: pab_build.device_asm(path, ["--flag"]))
    assert sorted(a[-1] for a in got) == sorted(pab_build.SOURCES + pab_build.SOURCES_NAN)
    assert all("-S" in a and "--flag" in a and ("-fno-honor-nans" in a) == (a[-1] in pab_build.SOURCES) for a in got)
    assert os.listdir(tmp_path / "out") == ["pab.s"]
