"""The native module beside the library (CPU): one that cannot be loaded, or was built for another Python or torch, is not
needed, and a build makes up for one that is missing."""
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

import pytest

torch = pytest.importorskip("torch")

from paper_2403_00835_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("content", [b"", b"not a shared object", b"\x7fELF\x02\x01\x01" + bytes(200)], ids=["empty", "text", "header"])
def test_a_damaged_file_is_none(content, tmp_path, monkeypatch, capfd):
    path = tmp_path / "_marshal.so"
    path.write_bytes(content)
    monkeypatch.setattr(build, "MARSHAL", str(path))
    assert build.load_marshal() is None
    assert "in Python" in capfd.readouterr().err


def test_an_absent_file_is_none(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    assert build.load_marshal() is None


def test_the_package_works_beside_a_damaged_file(tmp_path):
    path = tmp_path / "_marshal.so"
    path.write_bytes(b"not a shared object")
    code = f"""
from paper_2403_00835_gb300 import build
build.MARSHAL = {str(path)!r}
from paper_2403_00835_gb300 import paged, verify
verify.load()
assert paged._marshal is None
for bad in (dict(positions=-1), dict(positions=1, first=2 ** 31)):
    try:
        paged.rope_table(frequencies=[1.0], **bad)
    except ValueError:
        continue
    raise SystemExit("not refused")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_the_name_tells_what_it_was_built_for():
    name = os.path.basename(build.MARSHAL)
    assert name.startswith("_marshal") and name.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert importlib.metadata.version("torch") in name


def test_a_build_makes_up_for_a_missing_one(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libcllm.so"))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    calls = []
    monkeypatch.setattr(build, "_build_marshal", lambda: calls.append(1))
    monkeypatch.setattr(build, "_nvcc", lambda: pytest.fail("the library is built"))
    (tmp_path / "libcllm.so").write_bytes(b"")
    (tmp_path / "stamp").write_text(build._fingerprint())
    build.build()
    assert calls == [1]
    (tmp_path / "_marshal.so").write_bytes(b"")
    build.build()
    assert calls == [1]


def test_one_of_the_sources_before_does_not_stay(tmp_path, monkeypatch):
    """Another interpreter's too: it would read arguments of another layout.  One that another process is building does."""
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libcllm.so"))
    monkeypatch.setattr(build, "_build_marshal", lambda: None)
    monkeypatch.setattr(build, "_sources", lambda: [str(tmp_path / "none.cu")])
    for f in ("libcllm.so", "_marshal.so", "_marshal-torch0.cpython-30.so", "_marshal.so.tmp1"):
        (tmp_path / f).write_bytes(b"")
    (tmp_path / "stamp").write_text("another")
    with pytest.raises(RuntimeError, match="none.cu"):
        build.build()
    assert sorted(f for f in os.listdir(tmp_path) if f.startswith("_marshal")) == ["_marshal.so.tmp1"]
