"""The bench quotes recorded HBM counters only for the code that they were taken on: its hash covers every file that the
reshard's kernels are made of. No GPU needed."""
import os
import re

import bench


def own_includes(path, seen):
    """The files beside `path` that it includes, and theirs."""
    for name in re.findall(r'#include "([^"]+)"', open(path).read()):
        at = os.path.join(os.path.dirname(path), name)
        if os.path.exists(at) and at not in seen:
            seen.add(at)
            own_includes(at, seen)
    return seen


def test_the_hash_covers_the_kernels_and_what_they_include():
    kernels = next(p for p in bench.KERNEL_SRCS if p.endswith("emu_exec.hip"))
    assert own_includes(kernels, {kernels}) <= set(bench.KERNEL_SRCS)


def test_a_change_of_any_of_them_changes_the_hash_and_a_comment_does_not():
    texts = [open(p).read() for p in bench.KERNEL_SRCS]
    now = bench.kernel_hash(texts)
    for i in range(len(texts)):
        assert bench.kernel_hash(texts[:i] + [texts[i] + "\nint x;\n"] + texts[i + 1:]) != now
        assert bench.kernel_hash(texts[:i] + [texts[i] + "\n// x\n"] + texts[i + 1:]) == now
