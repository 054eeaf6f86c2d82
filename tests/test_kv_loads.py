"""Kernels of the key-value cache and the norm may start while the kernel ahead of them on the stream still
writes what they are going to read (programmatic dependent launch). Non-coherent loads are defined only for
memory that nobody writes while a kernel lives, so the sources use none (checked by reading them, no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_12876_gb300", "csrc")
FILES = ["kv.cuh", "kv_pages.cu", "kv_attend.cu", "norm.cu"]


def code(name):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, name)).read(), flags=re.S)


def noncoherent_helpers():
    """Functions of the shared headers whose body has a non-coherent load."""
    text = code("aq_internal.cuh")
    found = set()
    for m in re.finditer(r"__forceinline__\s+\w+\s+(\w+)\([^)]*\)\s*\{(.*?)\n\}", text, re.S):
        if "ld.global.nc" in m.group(2) or "__ldg" in m.group(2):
            found.add(m.group(1))
    return found


def test_no_noncoherent_loads_of_what_earlier_kernels_write():
    helpers = noncoherent_helpers()
    assert helpers == {"ld_stream_v4"}
    for name in FILES:
        text = code(name)
        for word in ["ld.global.nc", "__ldg", "__restrict__"] + sorted(helpers):
            assert word not in text, (name, word)
