"""Kernels with tensor memory launch their dependents behind their allocation: read from the sources, since a kernel that does it the
other way round may never end.  (Dependents allocate before they wait for the kernel, and an allocation waits without a limit.)"""
import os
import re

from paper_2110_14871_b200 import build as gbuild


def kernels(text):
    """(name, body) of every __global__ function, without comments."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    for m in re.finditer(r"__global__", text):
        start = text.index("{", m.end())
        if ";" in text[m.end():start]:
            continue                                     # a declaration
        depth, end = 0, start
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if depth == 0:
                break
        yield re.findall(r"(\w+)\s*\(", text[m.end():start])[-1], text[start:end]


def block_of(body, at):
    """What follows position `at` in the innermost braces around it."""
    depth, end = 0, at
    while depth >= 0:
        depth += {"{": 1, "}": -1}.get(body[end], 0)
        end += 1
    return body[at:end]


def faults(text):
    found, wrong = [], []
    for name, body in kernels(text):
        if "tmem_alloc" not in body:
            continue
        found.append(name)
        alloc = body.index("tmem_alloc")
        trigger = [m.start() for m in re.finditer(r"grid_launch_dependents|griddepcontrol\.launch_dependents", body)]
        # one, and by the warp that allocates: no other warp's may come first
        if len(trigger) != 1 or trigger[0] < alloc or "grid_launch_dependents" not in block_of(body, alloc):
            wrong.append(name)
    return found, wrong


def test_tensor_memory_comes_before_the_dependents():
    found, wrong = [], []
    for source in gbuild.SOURCES:
        with open(os.path.join(gbuild.CSRC, source)) as f:
            a, b = faults(f.read())
        found += a
        wrong += b
    assert {"p8_slices_kernel", "p8_pairs_kernel", "fold_kernel", "fold_split_kernel", "fused_bf16_kernel", "fused_tc_kernel", "gdw_tc_kernel", "pw_bf16_tc_kernel", "f32_tc_kernel"} <= set(found), found
    assert not wrong, wrong


def test_the_order_is_told_apart():
    kernel = "__global__ void __launch_bounds__(64) k(int n)\n{\n%s\n}\n"
    good = "if (warp == 2) {\n tmem_alloc(a, 32);\n grid_launch_dependents();\n}\n__syncthreads();"
    assert faults(kernel % good) == (["k"], [])
    for bad in ("grid_launch_dependents();\nif (warp == 2) tmem_alloc(a, 32);", "if (warp == 2) { tmem_alloc(a, 32); }\ngrid_launch_dependents();", "if (warp == 2) tmem_alloc(a, 32); // grid_launch_dependents()",
                "grid_launch_dependents();\n" + good):
        assert faults(kernel % bad) == (["k"], ["k"]), bad
