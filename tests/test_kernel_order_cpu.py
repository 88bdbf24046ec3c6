"""Every library kernel waits for the kernel before it.

Kernels of a call may be launched while their predecessor drains, and that a
launch is the first of its call is up to the host code: a kernel without the
wait would read unfinished data as soon as it is launched second."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_04910_gb300", "csrc")


def body(src, start):
    """The text from the first brace at or after ``start`` to the one that closes it."""
    i = start = src.index("{", start)
    depth = 0
    while True:
        depth += {"{": 1, "}": -1}.get(src[i], 0)
        i += 1
        if depth == 0:
            return src[start:i]


def kernels():
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(CSRC, name), encoding="utf-8") as f:
            src = re.sub(r"//[^\n]*", "", f.read())
        # Device functions of the file that wait for their callers.
        waits = {"pdl_wait"}
        for m in re.finditer(r"__forceinline__ [\w<> ]+?(\w+)\(", src):
            if "pdl_wait()" in body(src, m.end()):
                waits.add(m.group(1))
        for m in re.finditer(r"__global__ void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\(", src):
            yield name, m.group(1), body(src, m.end()), waits


def test_every_kernel_waits_for_its_predecessor():
    seen, idle = [], []
    for name, kernel, text, waits in kernels():
        if kernel.endswith("_probe_kernel"):
            continue            # (launched on their own, and timed: they read nothing)
        seen.append(kernel)
        calls = [m.start() for w in waits for m in re.finditer(rf"\b{w}(<\w+>)?\(", text)]
        if not calls:
            idle.append(f"{name}: {kernel}")
    assert len(seen) >= 30 and "rotary_kernel" in seen and "attn_rows_kernel" in seen, seen
    assert not idle, idle
