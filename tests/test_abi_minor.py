"""The ABI's minor number: entry points that were added to a version (CPU)."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2608_28511_amd import _lib as L

HEADER = (Path(__file__).resolve().parents[1] / "include" / "moe.h").read_text()


def defined(name):
    return int(re.search(rf"^#define {name} (\d+)$", HEADER, re.M).group(1))


def test_library_header_and_binding_agree():
    L.load(build_if_missing=True)
    want = (defined("MOE_ABI_VERSION"), defined("MOE_ABI_MINOR"))
    assert L.ABI == want == (L.moe_abi_version(), L.moe_abi_minor()) and want[1] >= 1


@pytest.mark.parametrize("source", ["int moe_abi_version(void) { return 5; }",
                                    "int moe_abi_version(void) { return 5; } int moe_abi_minor(void) { return 0; }",
                                    "int moe_abi_version(void) { return 4; } int moe_abi_minor(void) { return 9; }"])
def test_an_older_library_is_refused(tmp_path, monkeypatch, source):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    (tmp_path / "old.c").write_text(source)
    subprocess.run(["gcc", "-shared", "-fPIC", str(tmp_path / "old.c"), "-o", str(tmp_path / "old.so")], check=True)
    monkeypatch.setattr(L, "_lib", None)
    monkeypatch.setattr(L, "LIB_PATH", tmp_path / "old.so")
    with pytest.raises(RuntimeError, match="needs 5.1"):
        L.load()
