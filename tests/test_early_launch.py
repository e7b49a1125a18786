"""Kernels that are launched while the one before them ends read nothing through the read-only path, checked on their source."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_08537_b200", "csrc")


def code(path):
    """A file without its comments."""
    text = re.sub(r"/\*.*?\*/", " ", open(path).read(), flags=re.S)
    return re.sub(r"//[^\n]*", " ", text)


def with_headers(path, seen):
    if path in seen:
        return
    seen.add(path)
    for name in re.findall(r'#include "([^"]+)"', open(path).read()):
        header = os.path.join(CSRC, name)
        if os.path.dirname(name) == "" and os.path.exists(header):
            with_headers(header, seen)


def test_no_read_only_loads_where_kernels_are_launched_early():
    """__ldg, ld.global.nc and __restrict__ promise data that does not change while the kernel runs; the logits are written by the kernel before
    it, and a gradient may be written in their place."""
    files = set()
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        if "launch_early(" in code(path):
            with_headers(path, files)
    assert {"sample.cu", "distill.cu", "pages.cu", "rows.cuh"} <= {os.path.basename(p) for p in files}
    for path in files:
        found = re.findall(r"__ldg\w*|ld\.global\.nc|__restrict__", code(path))
        assert not found, (os.path.basename(path), found)


def test_kernels_that_are_launched_early_begin_with_the_wait():
    """begin_kernel() is a kernel's first statement but for declarations and what forms addresses: nothing is read or written before it."""
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        text = code(path)
        names = set(re.findall(r"launch_early\(\s*(\w+)", text))
        for name in names:
            body = re.search(r"__global__[^;{]*\b" + name + r"\s*\([^{]*\)\s*\{(.*?)begin_kernel\(\);", text, flags=re.S)
            assert body, name
            assert not re.search(r"__sync|\ba\.\w+\[|args\.\w+\[|\*a\.", body.group(1)), (name, body.group(1))
