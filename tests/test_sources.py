"""Rules on the kernels' sources that no run can show."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_17475_gb300", "csrc")
KV8 = sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "kv8*.cu*")))


def arguments(text, name):
    """The argument texts of the calls of `name`, comments taken out."""
    text = re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))
    out = []
    for m in re.finditer(r"\b%s\s*\(" % name, text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        out.append(text[m.end():i - 1])
    return out


@pytest.mark.parametrize("name", KV8)
def test_pool_bytes_are_not_read_as_constant(name):
    """Read-only loads ask that the memory keep its value for as long as the kernel lives.  The kernels of the 8-bit
    cache may be resident while an append or an eviction before them still writes codes and scales, so only page
    tables, which no kernel writes, are read that way."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert "ld.global.nc" not in text and "__restrict__" not in text
    for arg in arguments(text, "__ldg"):
        assert re.match(r"(a\.page_table|pt)\b", arg.strip()), arg


def test_the_files_are_found():
    assert {"kv8.cu", "kv8_decode.cu", "kv8_prefill.cu", "kv8_evict.cu"} <= set(KV8)
    assert arguments("x = __ldg(a + (b * c)); // __ldg(q)\n", "__ldg") == ["a + (b * c)"]
