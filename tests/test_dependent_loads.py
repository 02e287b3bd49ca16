"""Kernels that are started as programmatic dependents are resident while the kernels before them still write. What those
write is read with ordinary loads behind the wait: a read-only load (`__ldg`, `ld.global.nc`, or one that the compiler makes of a
`const ... __restrict__` parameter) promises that its data do not change while the kernel lives, and may move above the wait."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_08522_b200", "csrc")
FILES = sorted(p for e in ("*.cu", "*.cuh") for p in glob.glob(os.path.join(CSRC, e)))
HOST_WRITES = ("Tensor", "Chunk")        # tables that the host fills before any kernel reads them


def code(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", lambda m: "\n" * m.group(0).count("\n"), f.read(), flags=re.S)


def kernels(text):
    """(signature, body) of every kernel"""
    for m in re.finditer(r"__global__", text):
        start = text.index("{", m.end())
        depth, end = 0, start
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            if depth == 0:
                break
            end += 1
        yield text[m.start():start], text[start:end]


def test_no_read_only_loads():
    found = []
    for path in FILES:
        for i, line in enumerate(code(path).split("\n"), 1):
            if re.search(r"__ldg\s*\(|\.nc\b", line):
                found.append("%s:%d" % (os.path.basename(path), i))
    assert not found, found


def test_dependents_promise_nothing_about_their_inputs():
    seen, found = 0, []
    for path in FILES:
        for signature, body in kernels(code(path)):
            if not re.search(r"griddepcontrol\.wait|wait_for_previous\(\)", body):
                continue
            seen += 1
            for kind in re.findall(r"const\s+(\w+)\s*\*\s*__restrict__", signature):
                if kind not in HOST_WRITES:
                    found.append((os.path.basename(path), re.findall(r"(\w+)\s*\(", signature)[-1], kind))
    assert seen >= 20, seen
    assert not found, found
