"""Which calls on an LM head's logits share rows among workgroups, read from the workspaces that they need: the k largest
need one for shared rows alone. No GPU needed."""
import ctypes

import pytest

from paper_2609_34645_amd import emu


def workspace(V, rows, k, dtype=emu.BF16, tp=1):
    lay, n = emu.Layout(emu.Model(2, 256, 8, 64, 8, 512, V), tp, 1), ctypes.c_uint64()
    ptrs = (ctypes.c_void_p * tp)(*[1 << 20] * tp)
    c = emu.c_logits(ctypes.pointer(lay.c()), dtype, tp, rows, V, ptrs)
    emu.check(emu.load().emu_logits_workspace(ctypes.addressof(c), k, ctypes.addressof(n)))
    return n.value


@pytest.mark.parametrize("V", [8192, 32768, 128256])
def test_rows_are_shared_below_a_line(V):
    for dtype in (emu.BF16, emu.FP32):
        assert all(workspace(V, rows, 4, dtype) > 0 for rows in (1, 2, 95))
        assert all(workspace(V, rows, 4, dtype) == 0 for rows in (96, 255, 511, 5000))
        # a distillation keeps its teachers there, too: a part more or less shows in the bytes of a row
        assert workspace(V, 95, 0, dtype) / 95 > workspace(V, 96, 0, dtype) / 96


def test_rows_of_one_unit_are_never_shared():
    assert workspace(4096, 1, 4) == 0 and workspace(4097, 1, 4) > 0
    assert workspace(2048, 1, 4, emu.FP32) == 0 and workspace(2049, 1, 4, emu.FP32) > 0


def test_the_widest_rows_are_always_shared():
    assert workspace(1 << 18, 5000, 4) == 0 and workspace((1 << 18) + 8, 5000, 4) > 0


def test_few_rows_fill_the_device_and_no_more():
    per_part = 64 * 8 + 8  # a sorted wave of keys, and the statistics
    assert [workspace(128256, rows, 4) // per_part for rows in (1, 16, 64, 95)] == [32, 16 * 32, 64 * 16, 95 * 11]
    assert workspace(1 << 20, 1, 4) // per_part == 64
