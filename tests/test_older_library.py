"""A library of the same ABI built before the cache operators: the binding says
what to do."""
import re
import shutil
import subprocess

import pytest

import paper_2503_10571_amd as radar
from paper_2503_10571_amd import _build


def test_a_library_without_the_cache_operators(tmp_path, monkeypatch):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    text = re.sub(r"/\*.*?\*/", "", open(f"{_build.INCLUDE}/radar.h").read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(radar_[a-z_]+)\s*\(", text)) - {"radar_abi_version"})
    src, so = tmp_path / "old.c", tmp_path / "old.so"
    src.write_text(f"int radar_abi_version(void) {{ return {radar.ABI_VERSION}; }}\n" +
                   "".join(f"int {n}(void) {{ return 1; }}\n" for n in names))
    subprocess.run([gcc, "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    monkeypatch.setattr(radar, "_lib", None)
    monkeypatch.setattr(radar, "LIB_PATH", str(so))
    for _ in range(2):
        with pytest.raises(RuntimeError, match="rebuild it.*radar_"):
            radar.lib()
    assert radar._lib is None
