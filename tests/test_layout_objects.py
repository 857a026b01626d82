"""Layouts are plain values: what a call keeps with one never shows in its fields, copies and pickles. No GPU needed."""
import copy
import dataclasses
import pickle

from paper_2609_34645_amd import emu

MODEL = emu.Model(2, 256, 8, 64, 8, 512, 1000)


def test_a_layout_used_with_logits_stays_a_value():
    fresh, used = emu.Layout(MODEL, 2, 1, pad=64), emu.Layout(MODEL, 2, 1, pad=64)
    plain, columns = pickle.dumps(fresh), emu.shard_columns(used)
    assert pickle.dumps(used) == plain and vars(used) == vars(fresh) and dataclasses.asdict(used) == dataclasses.asdict(fresh)
    assert used == fresh and hash(used) == hash(fresh) and repr(used) == repr(fresh)
    copies = [copy.copy(used), copy.deepcopy(used), emu.Layout(**vars(used)), dataclasses.replace(used),
              *(pickle.loads(pickle.dumps(used, p)) for p in range(pickle.HIGHEST_PROTOCOL + 1))]
    for c in copies:
        assert c == used and type(c) is emu.Layout and emu.shard_columns(c) == columns
    assert emu.shard_columns(dataclasses.replace(used, pad=0)) == 500
    assert emu.shard_columns(used) == columns
