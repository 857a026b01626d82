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


# (vocabulary, tp, pad, rows, dtypes of the logits): what 4 waves hold at 4 tiles and at 16 each, with more rows than
# there are workgroups; 8 waves; 16 waves, up to the last tile; borders on tiles, inside them and a little more than a tile apart; pads in
# the vocabulary's last vector and behind it
KEPT = [(1024, 2, 0, 2600, "bf16 fp32"), (1000, 2, 4, 1500, "fp32"), (4001, 2, 64, 1300, "bf16 fp32"), (4352, 8, 0, 1300, "bf16 fp32"),
        (16000, 3, 8, 700, "bf16 fp32"), (40000, 8, 8, 300, "bf16 fp32"), (50304, 4, 8, 300, "bf16"), (65536, 4, 0, 300, "bf16 fp32"),
        (128256, 4, 0, 300, "bf16"), (128256, 1, 0, 270, "bf16"), (131072, 8, 0, 270, "bf16"), (131000, 2, 8, 270, "bf16")]


@pytest.mark.parametrize("V,tp,pad,rows,din", [(*head[:4], t) for head in KEPT for t in head[4].split()])
@pytest.mark.parametrize("dout", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [False, True])
def test_every_held_form(gpu_lib, V, tp, pad, rows, din, dout, tail):
    """Every number of waves and tiles, every pair of types; small ones, and parts of the others, against the definition."""
    import torch

    k, tau = 24, 1.3
    rng = np.random.default_rng(V + tp)
    lay = layout(V, tp, pad)
    torch.manual_seed(V)
    z = torch.randn(rows, V, device="cuda") * 3
    z[3], z[5], z[9, ::2] = -float("inf"), 2e7, -3.38e38
    z[8] = z[8] * 1e6
    z[11, 7] = float("nan")
    z[-1, : V // 2] = -float("inf")
    z = z.to(torch_type(din)).double().cpu().numpy()
    index, value = teacher(V, rows, V, k)
    index[20], value[21] = -1, -np.inf
    index[22] = V - 1 - np.arange(k)                 # the last tile's
    border = emu.shard_columns(lay)
    index[23] = np.clip(border - k // 2 + np.arange(k), 0, V - 1)  # around a border
    w = np.float32(rng.uniform(-1, 1, rows))
    w[rng.random(rows) < 0.3] = 0
    w[[3, 5, 8, 9, 11, 20, 21, 22, 23]] = 0.5
    loss, stats, grad = held(z, lay, din, dout, index, value, w, tau, tail)
    n = rows if V < 5000 else 32
    part = emu.LogitShards(lay, [t[:n] for t in grad.tensors])
    check_distill(z[:n], index[:n], value[:n], w[:n], tau, tail, loss[:n], stats[:n], part, dout)
    for t in grad.tensors:
        assert (t[dev(w == 0, bool)] == 0).all()


@pytest.mark.parametrize("V,tp,din,dout", [(4096, 2, "bf16", "fp32"), (4096, 4, "fp32", "bf16"), (50304, 4, "bf16", "bf16")])
@pytest.mark.parametrize("k", [1, 64, 256])
@pytest.mark.parametrize("tail", [False, True])
def test_held_rows_whose_entries_lie_together(gpu_lib, V, tp, din, dout, k, tail):
    """All of a row's entries in one or two tiles, as frequent tokens' numbers are, and lists of 1 and of 256."""
    rows = 300
    rng = np.random.default_rng(k)
    z = np.asarray(place(rng.normal(0, 2, (rows, V)), layout(V, 1, 0), din).tensors[0].double().cpu())
    _, value = teacher(k, rows, V, k, mess=False)
    first = rng.integers(0, V - 300, rows)
    first[::2] = 0
    index = first[:, None] + np.stack([rng.permutation(k) for _ in range(rows)])
    w = np.float32(rng.uniform(0.5, 1, rows))
    lay, n = layout(V, tp, 0), 40
    loss, stats, grad = held(z, lay, din, dout, index, value, w, 1.0, tail)
    part = emu.LogitShards(lay, [t[:n] for t in grad.tensors])
    check_distill(z[:n], index[:n], value[:n], w[:n], 1.0, tail, loss[:n], stats[:n], part, dout)


def test_more_held_rows_than_a_launch_takes(gpu_lib):
    """The second launch's rows, of which there are fewer, with every seventh without a weight."""
    V, tp, rows, k = 1024, 2, 32768 + 4100, 12
    rng = np.random.default_rng(4)
    base = np.asarray(place(rng.normal(0, 3, (1024, V)), layout(V, 1, 0), "bf16").tensors[0].double().cpu())
    index, value = teacher(5, 1024, V, k)
    at = np.arange(rows) % 1024
    w = np.float32(rng.uniform(0.5, 1, 1024))
    w[::7] = 0
    loss, stats, grad = held(base[at], layout(V, tp, 0), "bf16", "bf16", index[at], value[at], w[at], 1.0, True)
    part = emu.LogitShards(grad.layout, [t[:1024] for t in grad.tensors])
    check_distill(base, index, value, w, 1.0, True, loss[:1024], stats[:1024], part, "bf16")
    for r in range(1024, rows, 1024):
        n = min(1024, rows - r)
        assert all(same_bits([t[r:r + n]], [t[:n]]) for t in (loss, stats, *grad.tensors))


def test_held_rows_without_any_weight(gpu_lib):
    import torch

    lay, rows = layout(4096, 2, 0), 300
    z = np.full((rows, 4096), np.nan)  # not read
    index, value = teacher(1, rows, 4096, 8)
    loss, stats, grad = held(z, lay, "bf16", "bf16", index, value, np.zeros(rows), 1.0, False)
    assert (loss == 0).all() and torch.isnan(stats).all() and all((t == 0).all() for t in grad.tensors)


def step(student, ti, tv, w, grads, stream=None):
    """A training step's calls: loss with gradient, then the gradient alone from its statistics."""
    loss, stats = emu.distill_loss(student, ti, tv, weight=w, tail=True, grad=grads[0], stream=stream)
    emu.distill_backward(student, ti, tv, stats, w, grads[1], tail=True, stream=stream)
    return loss, stats


@pytest.mark.parametrize("V,tp,rows", [(4096, 2, 1200), (128256, 4, 300)])
def test_held_rows_captured_and_on_two_streams_at_once(gpu_lib, V, tp, rows):
    """Two steps that run at the same time, eagerly and as graphs replayed with new inputs and eager work between; every
    result is what the step gives by itself."""
    import torch

    lay = layout(V, tp, 0)
    sets = []
    for i in range(2):
        index, value = teacher(i, rows, V, 20, mess=False)
        student = emu.LogitShards.alloc(lay, rows, torch.bfloat16)
        grads = [emu.LogitShards.alloc(lay, rows, torch.bfloat16) for _ in range(2)]
        assert stays(lay, student, grads[0])
        w = torch.rand(rows, device="cuda")
        w[::5] = 0
        sets.append((student, dev(index, np.int32), dev(value, np.float32), w, grads))

    def renew():
        for student, _, _, _, grads in sets:
            for t in student.tensors:
                t.normal_(0, 3)
            for t in grads[0].tensors + grads[1].tensors:
                t.fill_(7)
        torch.cuda.synchronize()

    def results(outs):
        torch.cuda.synchronize()
        return [t.clone() for out, one in zip(outs, sets) for t in (*out, *one[4][0].tensors, *one[4][1].tensors)]

    streams = [torch.cuda.Stream() for _ in range(2)]
    renew()
    alone = []
    for one in sets:
        alone.append(step(*one))
        torch.cuda.synchronize()
    want = results(alone)
    for _ in range(3):
        outs = [step(*one, stream=s) for one, s in zip(sets, streams)]
        assert same_bits(results(outs), want)
    graphs, outs = [], []
    for one in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(*one))
        graphs.append(g)
    for replay in range(4):
        renew()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        got = results(outs)
        eager = []
        for one in sets:
            eager.append(step(*one))
            torch.cuda.synchronize()
        assert same_bits(results(eager), got), f"replay {replay}"
