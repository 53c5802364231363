"""Inline assembly names every register that it changes (runs without a GPU)."""
import re

import host_shim


def statements():
    for path in sorted(host_shim.CSRC.glob("*.h*")):
        for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", path.read_text(), flags=re.S):
            text = m.group(1)
            yield path.name, "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.split(":")[0])), text


def test_m0_is_named_where_it_is_written():
    """m0 is set by hand for copies from memory to LDS: the compiler has to know, or it may keep a value of its own there."""
    writes = [(name, text) for name, code, text in statements() if re.search(r"\bs_\w+\s+m0\b", code)]
    assert writes
    assert [name for name, text in writes if '"m0"' not in text.split(":")[-1]] == []
