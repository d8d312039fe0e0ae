"""How the library is put together (paper_2311_17410_amd/build.py): what every command is given.  Nothing is compiled."""
from paper_2311_17410_amd import build


def test_options_reach_every_compile_and_the_link(monkeypatch):
    """Options that a caller adds may be the link's (-l, -L, -Wl, sanitizers) as well as the compiler's."""
    commands, moved = [], []
    monkeypatch.setattr(build.subprocess, "check_call", commands.append)
    monkeypatch.setattr(build.os, "replace", lambda a, b: moved.append((a, b)))
    extra = ["-DSOME=1", "-Wl,--no-undefined"]
    assert build.build(extra=extra) == build.LIB
    compiled, (link,) = [c for c in commands if "-c" in c], [c for c in commands if "-c" not in c]
    assert sorted(c[c.index("-c") + 1].rsplit("/", 1)[1] for c in compiled) == sorted(build.SOURCES)
    assert all(e in c for c in commands for e in extra)
    assert "-shared" in link and not any("-shared" in c for c in compiled)
    assert sorted(o for o in link if o.endswith(".o")) == sorted(c[c.index("-o") + 1] for c in compiled)
    assert moved == [(link[link.index("-o") + 1], build.LIB)]
