"""Loss and gradient of rows that stay in registers between the two (many aligned rows): bit for bit what the same rows
give off the vectors' alignment, where they are read again, and against the definition."""
import numpy as np
import pytest

from oracle import logits as ol
from paper_2609_34645_amd import emu
from tests.test_gpu_logits import check_distill, close, dev, layout, lse_tol, place, same_bits, teacher, torch_type

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def stays(lay, *sets):
    """Whether the sets' rows stay in registers: whole aligned vectors in every shard, shards of a tile at least, no tile of
    pads alone, and no more tiles than 16 waves hold."""
    V, cols = lay.model.vocab, emu.shard_columns(lay)
    size = sets[0].tensors[0].element_size()
    tile = 1024 // size
    aligned = all(t.data_ptr() % 16 == 0 and t.stride(0) * t.element_size() % 16 == 0 for s in sets for t in s.tensors)
    return aligned and cols * size % 16 == 0 and cols >= tile and -(-V // tile) == -(-cols * lay.tp // tile) <= 256


def held(z, lay, din, dout, index, value, w, tau, tail):
    """(loss, statistics, gradient's set) of the aligned rows, after comparing them with the same rows off alignment and,
    in one type, in place."""
    import torch

    ti, tv, tw = dev(index, np.int32), dev(value, np.float32), dev(w, np.float32)
    wide, runs = -emu.shard_columns(lay) % 8, []
    for skip in (0, 1):
        student = place(z, lay, din, wide=wide, skip=skip)
        grad = place(np.zeros((len(z), 1)), lay, dout, wide=wide, skip=skip, fill=7.0)
        assert stays(lay, student, grad) == (skip == 0)
        loss, stats = emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=grad)
        runs.append((loss, stats, grad))
        if din == dout:
            emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=student)
            assert same_bits(student.tensors, grad.tensors), "in place"
    (a, b), names = runs, ("loss", "stats")
    for x, y, name in zip(a, b, names):
        assert same_bits([x], [y]), name
    assert same_bits(a[2].tensors, b[2].tensors), "gradient"
    if wide:  # what lies between the rows
        cols = emu.shard_columns(lay)
        assert all((t.as_strided((len(z) - 1, wide), (t.stride(0), 1), t.storage_offset() + cols) == 7.0).all() for t in a[2].tensors)
    torch.cuda.synchronize()
    return a


@pytest.mark.parametrize("V,tp,dtype", [(1024, 2, "bf16"), (4096, 4, "fp32"), (50304, 4, "bf16"), (128256, 4, "bf16")])
@pytest.mark.parametrize("tail", [False, True])
def test_rows_without_an_entry_and_far_from_zero(gpu_lib, V, tp, dtype, tail):
    """Rows summed the careful way whose teachers have no entry: nothing stands between the sum and the row's end."""
    rows, k = 600, 8
    rng = np.random.default_rng(V)
    z = np.tile(rng.normal(0, 3, (6, V)), (rows // 6, 1))
    z[::3] = z[::3] * 1e4 + 3e7
    z[1::3] *= 1e7
    z = np.asarray(place(z, layout(V, 1, 0), dtype).tensors[0].double().cpu())
    index, value = teacher(V, rows, V, k, mess=False)
    index[rng.random(rows) < 0.8] = -1
    loss, stats, grad = held(z, layout(V, tp, 0), dtype, dtype, index, value, np.ones(rows), 1.0, tail)
    lse = ol.log_sum_exp(z)
    got = stats.double().cpu().numpy()
    close(got[:, 0], lse, lse_tol(V) + 16 * U * np.abs(lse), "lse")
    close(got[:, 2], z.max(1), 0, "largest")
    far = index.max(1) < 0
    if not tail:
        assert (loss.cpu().numpy()[far] == 0).all()
        assert all((t[dev(far, bool)] == 0).all() for t in grad.tensors)
    if V < 5000 and not tail:  # with a tail these rows' losses pass what 64 bits hold of the unlisted mass
        check_distill(z, index, value, np.ones(rows), 1.0, tail, loss, stats, grad, dtype)
