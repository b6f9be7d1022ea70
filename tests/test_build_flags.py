"""Flags that a caller gives to the build reach every command of it (nothing is compiled here)."""
from paper_2412_16112_amd import build as hip_build


def test_flags_reach_compiler_and_linker(monkeypatch, tmp_path):
    made = []

    def run(cmd):
        made.append(cmd)
        open(cmd[cmd.index("-o") + 1], "wb").close()
        return ""
    lib = tmp_path / "lib.so"
    monkeypatch.setattr(hip_build, "_run", run)
    monkeypatch.setattr(hip_build, "LIB", str(lib))
    flags = ["-DSOME=1", "-L/some/folder", "-lsome", "-Wl,-z,now"]
    assert hip_build.build(extra_flags=flags) == str(lib) and lib.exists()
    compiles, links = [c for c in made if "-c" in c], [c for c in made if "-c" not in c]
    assert len(compiles) == len(hip_build.SOURCES) and len(links) == 1 and "-shared" in links[0]
    for cmd in made:
        at = cmd.index(flags[0])
        assert cmd[at:at + len(flags)] == flags
    assert all(c[c.index("-o") + 1] in links[0] for c in compiles)
