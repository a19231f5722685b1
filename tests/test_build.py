"""How the library is put together."""
from types import SimpleNamespace

from paper_2210_08804_amd import build


def test_flags_of_a_build_reach_the_link(monkeypatch):
    """Some are the linker's alone (-L, -l, -Wl), and some are needed by both (-Xarch_host -fsanitize=...)."""
    commands = []
    monkeypatch.setattr(build, "subprocess", SimpleNamespace(run=lambda cmd, check: commands.append(cmd)))
    extra = ["-L/somewhere", "-Wl,-z,now"]
    assert build.build(extra) == build.LIB
    links = [c for c in commands if "-shared" in c]
    assert len(links) == 1 and len(commands) == len(build.SRCS) + 1
    for c in commands:
        at = c.index(extra[0])
        assert c[at:at + len(extra)] == extra
