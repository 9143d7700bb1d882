"""Kernels that are set up while the one before them still runs (after_previous) read what that one writes.  Loads through the
read-only path are only defined for memory that nothing writes during the whole kernel, and nothing holds them behind the wait,
so such a kernel has neither `const ... __restrict__` pointers nor __ldg.  Read from the sources; no GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_23087_b200", "csrc")


def functions(text):
    """(name, text) of every kernel: its head from __global__ on and its body, by matching braces."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"__global__", text):
        at = text.index("{", m.end())
        depth, end = 1, at + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        head = text[m.start():at]
        yield re.findall(r"(\w+)\s*\(", re.sub(r"__\w+__\s*\([^()]*\)", "", head))[0], text[m.start():end]


def test_chained_kernels_read_nothing_through_the_read_only_path():
    chained = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        for name, text in functions(open(path).read()):
            if "after_previous()" in text:
                chained[name] = re.findall(r"const[^;,(]*__restrict__\s*\w+|__ldg|ld\.global\.nc", text)
    assert {"k_logits", "k_join", "k_finish", "k_dx", "k_dx_join", "k_dw", "k_norm_join"} <= set(chained), sorted(chained)
    assert not {k: v for k, v in chained.items() if v}
