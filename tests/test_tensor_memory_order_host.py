"""In the kernels' sources: no kernel holds tensor memory while it waits for the kernel before it, which may be waiting for that memory."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_09103_b200", "csrc")


def _kernels(text):
    """(name, body) of every __global__ function that has one."""
    for m in re.finditer(r"__global__[^;{]*?(\w+_kernel)\s*\(", text):
        start, depth = text.index("{", m.end()), 0
        for i in range(start, len(text)):
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            if depth == 0:
                yield m.group(1), text[start:i]
                break


def test_tensor_memory_is_allocated_behind_the_wait_for_the_kernel_before():
    found = []
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for kernel, body in _kernels(text):
            at = re.search(r"\btmem_alloc\b", body)
            if not at:
                continue
            found.append(kernel)
            wait = re.search(r"\b(wait_for_previous_kernel|wait_for_what_is_before)\(\)", body)
            assert wait and wait.start() < at.start(), (name, kernel)
    assert {"linear8_kernel", "linear8_strip_kernel", "head_items_kernel", "tc_items_kernel", "tc_apply_kernel"} <= set(found)
