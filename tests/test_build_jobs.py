"""What is compiled for the two builds of the library."""
import os
import subprocess

from paper_2604_11001_b200 import build as b


def commands(monkeypatch, tmp_path, checked, stale):
    """The compilers' command lines of a build, none of them run."""
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        if "-shared" in cmd:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(b.subprocess, "run", run)
    monkeypatch.setattr(b, "_stale", lambda path=b.LIB: stale)
    monkeypatch.setattr(b, "OBJ_DIR", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(b, "LIB_CHECKED", str(tmp_path / "lib_checked.so"))
    b.build(force=True, checked=checked)
    return [c for c in ran if "-c" in c], next(c for c in ran if "-shared" in c)


def test_the_checked_build_takes_the_caches_objects_as_they_are(monkeypatch, tmp_path):
    plain, link = commands(monkeypatch, tmp_path, False, True)
    checked, link_checked = commands(monkeypatch, tmp_path, True, False)
    again, _ = commands(monkeypatch, tmp_path, True, True)      # where they are missing or old they are compiled
    kv = lambda cs: [c for c in cs if "fcsim_kv" in os.path.basename(c[c.index("-c") + 1])]  # noqa: E731
    assert len(kv(plain)) == 1 + b.N_KV_TYPES and len(plain) == len(kv(plain)) + 1 + b.N_KERNEL_POLICIES
    assert kv(checked) == [] and len(checked) == 1 + b.N_KERNEL_POLICIES and all("-DFCSIM_CHECKED" in c for c in checked)
    assert kv(again) == kv(plain) and not any("-DFCSIM_CHECKED" in c for c in kv(again) + plain)
    objects = lambda c: {os.path.basename(x) for x in c if x.endswith(".o")}  # noqa: E731
    assert len(objects(link)) == len(objects(link_checked)) == len(plain)
    assert {"kv.o", "kv_attend0.o"} <= objects(link) & objects(link_checked)
