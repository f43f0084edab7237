"""What the build runs (nothing is compiled here)."""
import subprocess

from paper_2503_04424_amd import build


def test_further_flags_reach_every_command(monkeypatch):
    """Flags of the caller's (a library, a host sanitizer, debug information) are for compiling and for linking."""
    commands = []
    monkeypatch.setattr(subprocess, "run", lambda cmd, **_: commands.append(cmd))
    build.build(extra=["-g", "-lm"])
    assert len(commands) == len(build.SOURCES) + 1
    link = commands[-1]
    assert "-shared" in link and link[link.index("-o") + 1] == build.LIB
    assert all("-g" in c and "-lm" in c for c in commands)
    objects = [c[c.index("-o") + 1] for c in commands[:-1]]
    assert [a for a in link if a.endswith(".o")] and set(objects) == {a for a in link if a.endswith(".o")}
    for c in commands[:-1]:
        assert "-c" in c and "-shared" not in c and all(f in c for f in build.FLAGS if f != "-shared")
