"""Shared-memory arrays of bytes are accessed 8 and 16 bytes at a time, which their element
type does not promise to be aligned for: each declaration has to (CPU, reads the sources)."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parents[1] / "paper_2608_28511_amd" / "csrc"
DECL = re.compile(r"^[^/\n]*__shared__[^;\n]*?\b(?:u?int8_t|char)\s+\w+\s*\[[^;]*;", re.M)


def test_byte_arrays_in_lds_are_aligned():
    found = [(f.name, m.group(0).strip()) for f in sorted(CSRC.iterdir()) if f.suffix in (".h", ".hip")
             for m in DECL.finditer(f.read_text())]
    assert len(found) >= 4
    assert [d for d in found if not re.search(r"aligned\((16|1024)\)", d[1])] == []
