"""The operators on an LM head's logits against their 64-bit definitions (oracle/logits.py), and with themselves under
other layouts, strides, streams and captures.

Tolerances, in u = 2^-24 (half a step of fp32). A sum over V columns in any grouping of at least 64 lanes adds at most
V / 64 + 8 terms to one partial sum, each addition off by u; an exponential's argument (x - m) / tau is off by 4u of its
size (subtraction, two roundings of log2(e) / tau, product) and the function by 2u. Weighted with the probabilities
the arguments' sizes average below log V, so log sum exp is off by (V / 64 + 64 + 4 log V) u beside what its largest
term's own rounding gives (4u of its size). An output in bf16 is off by 2^-8 of its value more."""
import numpy as np
import pytest

from oracle import logits as ol
from paper_2609_34645_amd import emu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}

# (vocabulary, tp, pad multiple): one column, less than a vector, one odd, shards that end inside a vector, a shard of
# pads alone, the decoders of the tests and the bench
HEADS = [(1, 1, 0), (5, 1, 0), (17, 2, 1), (1000, 8, 0), (1003, 4, 1), (1024, 2, 0), (2500, 8, 128), (4099, 3, 1),
         (50257, 2, 1), (128256, 8, 128)]
SMALL = [h for h in HEADS if h[0] < 5000]


def torch_type(name):
    import torch

    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def layout(V, tp, pad):
    return emu.Layout(emu.Model(2, 256, 24, 64, 24, 768, V), tp, 1, pad=pad)


def place(x, lay, dtype, wide=0, skip=0, fill=float("nan")):
    """x [rows, V] (float64) as shards: pads and everything around the shards hold `fill`, rows are `wide` elements
    longer than a shard and start `skip` elements into their buffer."""
    import torch

    cols, shards = emu.shard_columns(lay), []
    for t in range(lay.tp):
        buf = torch.full((x.shape[0] * (cols + wide) + skip + 8,), fill, dtype=torch_type(dtype), device="cuda")
        s = buf[skip:skip + x.shape[0] * (cols + wide)].view(x.shape[0], cols + wide)[:, :cols]
        part = torch.from_numpy(np.ascontiguousarray(x[:, t * cols:(t + 1) * cols]))
        s[:, :part.shape[1]] = part.to(torch_type(dtype)).cuda()
        shards.append(s)
    return emu.LogitShards(lay, shards)


def whole(logits):
    """(columns of the vocabulary as float64, pad columns)."""
    import torch

    x = torch.cat(logits.tensors, 1).double().cpu().numpy()
    V = logits.layout.model.vocab
    return x[:, :V], x[:, V:]


def rounded(x, dtype):
    import torch

    return torch.from_numpy(np.asarray(x)).to(torch_type(dtype)).double().numpy()


def dev(a, dtype):
    import torch

    return None if a is None else torch.from_numpy(np.asarray(a, dtype)).cuda()


def close(got, want, tol, label=""):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    same |= (got == np.where(want > 0, np.inf, -np.inf)) & (np.abs(want) > 3.3895e38)  # beyond the type's largest: rounds to infinity
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    at = np.argwhere(bad)
    assert not len(at), f"{label}: {len(at)} of {bad.size} off, first at {at[0]}: {got[tuple(at[0])]} for {want[tuple(at[0])]}"


def bits(*tensors):
    import torch

    return [t.contiguous().view(torch.uint8).cpu() for t in tensors]


def same_bits(a, b):
    import torch

    return all(torch.equal(x, y) for x, y in zip(bits(*a), bits(*b)))


# ----------------------------------------------------------------------------------------------------
# constraints
# ----------------------------------------------------------------------------------------------------

def constraints(seed, rows, V, capacity):
    """Histories with repeats, tokens outside the vocabulary and lengths outside the buffer; biases with repeats and
    tokens outside; masks that allow nothing, one token, and most."""
    rng = np.random.default_rng(seed)
    c = {}
    tokens = np.minimum((V * rng.random((rows, capacity)) ** 3).astype(np.int64), V - 1)
    tokens[rng.random(tokens.shape) < 0.05] = -1
    tokens[rng.random(tokens.shape) < 0.05] = V
    tokens[rng.random(tokens.shape) < 0.02] = 2 ** 31 - 1
    c["tokens"] = tokens
    c["seq_len"] = rng.integers(0, capacity + 1, rows)
    c["seq_len"][0], c["seq_len"][-1] = capacity + 1000, -3 if rows > 1 else capacity
    c["prompt_len"] = (np.clip(c["seq_len"], 0, capacity) * rng.random(rows) * 1.2).astype(np.int64)
    c["repetition"] = np.float32(rng.uniform(0.8, 1.5, rows))
    c["frequency"] = np.float32(rng.uniform(-0.5, 0.5, rows))
    c["presence"] = np.float32(rng.uniform(-0.5, 0.5, rows))
    n = rng.integers(0, 40, rows)
    c["first"] = np.concatenate([[0], np.cumsum(n)])
    c["token"] = rng.integers(-1, V + 1, n.sum())
    c["value"] = np.float32(rng.normal(0, 3, n.sum()))
    allowed = rng.random((4, V)) < np.array([0.0, 0.0, 0.9, 0.5])[:, None]
    allowed[1, rng.integers(V)] = True
    c["allowed"] = allowed
    c["mask_row"] = rng.integers(-1, 5, rows)  # -1: none, 4: beyond the last, none as well
    return c


def packed(allowed, spare=0):
    n, V = allowed.shape
    b = np.zeros((n, (V + 31) // 32 * 32 + 32 * spare), np.uint8)
    b[:, :V] = allowed
    return np.packbits(b, axis=1, bitorder="little").view(np.uint32).view(np.int32)


def apply(x, out, c, **more):
    bias = (dev(c["first"], np.int32), dev(c["token"], np.int32), dev(c["value"], np.float32))
    return emu.constrain_logits(x, out, tokens=dev(c["tokens"], np.int32), seq_len=dev(c["seq_len"], np.int32),
                                prompt_len=dev(c["prompt_len"], np.int32), repetition=dev(c["repetition"], np.float32),
                                frequency=dev(c["frequency"], np.float32), presence=dev(c["presence"], np.float32),
                                bias=bias, mask=dev(packed(c["allowed"], 2), np.int32),
                                mask_row=dev(c["mask_row"], np.int32), **more)


def constrained(x, c):
    """(the definition's result, a bound on fp32's error per element)."""
    rows, capacity = c["tokens"].shape
    history = [c["tokens"][r][:max(0, min(capacity, int(c["seq_len"][r])))].tolist() for r in range(rows)]
    biases = [list(zip(c["token"][a:b].tolist(), c["value"][a:b].astype(np.float64).tolist()))
              for a, b in zip(c["first"][:-1], c["first"][1:])]
    allowed = [c["allowed"][m] if 0 <= m < len(c["allowed"]) else None for m in c["mask_row"]]
    args = dict(history=history, prompt_len=c["prompt_len"], theta=c["repetition"].astype(np.float64),
                frequency=c["frequency"].astype(np.float64), presence=c["presence"].astype(np.float64))
    want = ol.constrain(x, biases=biases, allowed=allowed, **args)
    # each of penalty (two roundings), its sum, the subtraction, the biases' sums and the last sum is off by u of a
    # partial result; those are bounded by the sum of the terms' sizes
    size = np.abs(np.where(np.isfinite(x), x, 0)) * 1.6
    most = ol.constrain(np.zeros_like(x), history, c["prompt_len"], None, -np.abs(args["frequency"]), -np.abs(args["presence"]),
                        [[(v, abs(b)) for v, b in row] for row in biases])
    return want, U * (6 + 40) * (size + most)


@pytest.mark.parametrize("V,tp,pad", HEADS)
@pytest.mark.parametrize("din,dout", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
def test_constrain(gpu_lib, V, tp, pad, din, dout):
    rows = 6
    rng = np.random.default_rng(V + tp)
    x = rounded(rng.normal(0, 4, (rows, V)), din)
    x[0, ::7], x[1, ::3], x[2, ::5] = -np.inf, rounded(-3.3e38, din), np.nan
    lay, c = layout(V, tp, pad), constraints(V, rows, V, 300)
    src, out = place(x, lay, din, wide=3, skip=1), place(np.zeros_like(x), lay, dout, wide=5, skip=3, fill=7.0)
    apply(src, out, c)
    want, tol = constrained(x, c)
    got, pads = whole(out)
    close(got, want, tol + np.where(np.isfinite(want), HALF_STEP[dout] * (np.abs(want) + tol), 0), "out of place")
    assert (pads == -np.inf).all()
    assert all((t.as_strided((rows - 1, 5), (t.stride(0), 1), t.storage_offset() + t.shape[1]) == 7.0).all() for t in out.tensors)
    kept, _ = whole(src)
    assert np.array_equal(kept, x, equal_nan=True)
    if din == dout:
        apply(src, None, c)
        assert same_bits(src.tensors, out.tensors), "in place gives what out of place gives"


def test_constrain_one_operand_at_a_time(gpu_lib):
    V, rows = 3001, 3
    rng = np.random.default_rng(5)
    x, lay, c = rng.normal(0, 3, (rows, V)).astype(np.float32).astype(np.float64), layout(V, 2, 1), constraints(9, rows, V, 50)
    hist = [c["tokens"][r][:max(0, min(50, int(c["seq_len"][r])))].tolist() for r in range(rows)]
    tokens = dict(tokens=dev(c["tokens"], np.int32), seq_len=dev(c["seq_len"], np.int32))
    f32 = np.float32
    runs = [({}, {}),
            (dict(tokens, repetition=dev(c["repetition"], f32)), dict(history=hist, theta=c["repetition"].astype(float))),
            (dict(tokens, frequency=dev(c["frequency"], f32)), dict(history=hist, frequency=c["frequency"].astype(float))),
            (dict(tokens, presence=dev(c["presence"], f32)), dict(history=hist, presence=c["presence"].astype(float))),
            (tokens, dict(history=hist)), (dict(repetition=dev(c["repetition"], f32)), {}),
            (dict(mask=dev(packed(c["allowed"][[0, 1, 3]]), np.int32)), dict(allowed=list(c["allowed"][[0, 1, 3]])))]
    for call, definition in runs:
        out = place(np.zeros_like(x), lay, "fp32")
        emu.constrain_logits(place(x, lay, "fp32"), out, **call)
        close(whole(out)[0], ol.constrain(x, **definition), 40 * U * (1 + np.abs(x)) * 8, str(list(call)))


def test_constrain_long_history_and_one_token_many_times(gpu_lib):
    V, n = 128256, 200000
    lay = layout(V, 4, 0)
    x = np.random.default_rng(3).normal(0, 3, (2, V)).astype(np.float32).astype(np.float64)
    tokens = np.random.default_rng(4).integers(0, V, (2, n))
    tokens[0] = 77  # one counter takes every token of the row
    token = np.concatenate([np.full(500, 11), np.arange(0, V, 97)])
    value = np.float32(np.random.default_rng(6).normal(0, 1, len(token)))
    out = place(np.zeros_like(x), lay, "fp32")
    freq = np.float32([1e-3, 0.1])
    emu.constrain_logits(place(x, lay, "fp32"), out, tokens=dev(tokens, np.int32), seq_len=dev([n, n - 1], np.int32),
                         frequency=dev(freq, np.float32),
                         bias=(dev([0, 0, len(token)], np.int32), dev(token, np.int32), dev(value, np.float32)))
    want = ol.constrain(x, [tokens[0].tolist(), tokens[1, :n - 1].tolist()], frequency=freq.astype(float),
                        biases=[[], list(zip(token.tolist(), value.astype(float).tolist()))])
    # at most 500 additions of biases whose sizes sum to less than 600
    close(whole(out)[0], want, U * (8 * np.abs(want) + 8 * np.abs(x)) + np.where(np.arange(V) == 11, U * 500 * 600, 0))


def test_constrain_bad_list_ends_are_cut(gpu_lib):
    import torch

    V = 100
    lay = layout(V, 1, 0)
    x = np.zeros((3, V))
    first = dev([-5, 2, 1, 50], np.int32)  # a negative start, an end before the start, an end behind the list
    token, value = dev([3, 3, 4], np.int32), dev([1.0, 2.0, 4.0], np.float32)
    got = whole(emu.constrain_logits(place(x, lay, "fp32"), bias=(first, token, value)))[0]
    want = np.zeros((3, V))
    want[0, 3], want[2, 3], want[2, 4] = 3, 2, 4
    assert np.array_equal(got, want)
    assert torch.cuda.is_available()


# ----------------------------------------------------------------------------------------------------
# the k largest
# ----------------------------------------------------------------------------------------------------

def lse_tol(V):
    return U * (V / 64 + 64 + 4 * np.log(V + 1))


def check_topk(x, got, k, tau):
    rows, V = x.shape
    index, logp, lse = (t.double().cpu().numpy() for t in got)
    wi, wp, wl = ol.topk(x, k, tau)
    bad = np.argwhere(index != wi)
    assert not len(bad), f"index {bad[0]}: {index[tuple(bad[0])]} for {wi[tuple(bad[0])]}"
    with np.errstate(invalid="ignore"):
        top = np.nanmax(np.where(np.isnan(x), -np.inf, x), axis=1) / tau
        close(lse, wl, lse_tol(V) + 8 * U * (np.abs(top) + np.abs(wl)), "lse")
        far = np.abs(np.where(np.isfinite(wp), wp, 0)) + np.log(V)
        close(logp, wp, lse_tol(V) + 8 * U * far, "logprob")


@pytest.mark.parametrize("V,tp,pad", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("k,tau", [(1, 1.0), (5, 0.6), (20, 2.0), (33, 1.3), (64, 1.0)])
def test_topk(gpu_lib, V, tp, pad, dtype, k, tau):
    if k > V:
        with pytest.raises(emu.EmuError) as e:
            emu.top_logprobs(place(np.zeros((2, V)), layout(V, tp, pad), dtype), k, tau)
        assert e.value.code == emu.STATUS_CODE["EMU_ERR_RANGE"]
        return
    rng = np.random.default_rng(V * 7 + k)
    x = rounded(rng.normal(0, 3, (5, V)), dtype)
    x[1] = rounded(np.sort(x[1]), dtype)          # ascending: every column beats all before it
    x[2] = rng.integers(-2, 3, V)                 # five values: ties everywhere
    x[3, rng.random(V) < 0.97] = -np.inf          # a mask that leaves few, perhaps fewer than k
    x[4] = rounded(x[4] * 1e-30, dtype)
    check_topk(x, emu.top_logprobs(place(x, layout(V, tp, pad), dtype, wide=2, skip=1), k, tau), k, tau)


@pytest.mark.parametrize("V,tp,pad", SMALL)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_topk_rows_with_extreme_values(gpu_lib, V, tp, pad, dtype):
    lowest = rounded(-3.4e38 if dtype == "fp32" else -3.38e38, dtype)
    rng = np.random.default_rng(V)
    x = rounded(rng.normal(0, 2, (12, V)), dtype)
    x[0] = -np.inf
    x[1] = lowest                                   # uniform
    x[2, 1:] = lowest                               # one token left by a mask of the lowest value
    x[3, : V // 2] = lowest
    x[4] = -lowest                                  # uniform at the other end
    x[5, -1] = np.nan
    x[6, V // 2] = np.inf
    x[7] = np.where(np.arange(V) % 2 == 0, 0.0, -0.0)
    x[8, :] = -np.inf
    x[8, -1] = 1.0
    x[9] = rounded(x[9] * 1e6, dtype)
    x[10] = rounded(x[10] * 1e6 - 1e7, dtype)
    x[11] = rounded(2e6 + 1e6 * (np.arange(V) % 3), dtype)
    for tau in (1.0, 0.3):
        if tau == 0.3:
            x[[1, 4]] = 0.0  # lowest / 0.3 passes fp32
        check_topk(x, emu.top_logprobs(place(x, layout(V, tp, pad), dtype), min(V, 7), tau), min(V, 7), tau)


@pytest.mark.parametrize("rows", [1, 2, 7, 300, 1000])
def test_topk_rows(gpu_lib, rows):
    V, lay = 5003, layout(5003, 2, 1)
    x = rounded(np.random.default_rng(rows).normal(0, 3, (rows, V)), "bf16")
    check_topk(x, emu.top_logprobs(place(x, lay, "bf16"), 16), 16, 1.0)


# ----------------------------------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------------------------------

def teacher(seed, rows, V, k, mess=True):
    rng = np.random.default_rng(seed)
    index = np.stack([rng.permutation(V)[:k] if k <= V else rng.integers(0, V, k) for _ in range(rows)])
    value = np.log(rng.dirichlet(np.ones(k + 1) * 0.4, rows)[:, :k] + 1e-12)
    if mess:
        index[0, k // 2] = -1
        index[0, 0] = V
        index[1 % rows, k - 1] = index[1 % rows, 0]  # a column listed twice
        value[2 % rows, k // 3] = -np.inf
        index[3 % rows] = -1                         # a row without an entry
    return index, np.float32(value)


def distill_bounds(z, d, w, tau, tail):
    """(loss, gradient, factor) bounds beside the outputs' own rounding."""
    rows, V = z.shape
    m = np.max(np.where(np.isfinite(z), z, -1e30), axis=1)
    base = lse_tol(V)
    with np.errstate(invalid="ignore", divide="ignore"):
        far = np.where(np.isfinite(z), np.abs(z - m[:, None]) / tau, 0) + np.log(V + 1)
        log_p = np.where(d["p"] > 0, np.abs(np.log(np.where(d["p"] > 0, d["p"], 1))), 0)
        rest = np.clip(1 - d["p"].sum(1), 0, 1) if tail else np.zeros(rows)
        log_rest = np.abs(np.log(np.where(rest > 0, rest, 1)))
        # of each term p (log p - log q): p is off by 8u, the logs by their own; 64 terms' additions by 16u of their sizes
        term = (d["p"] * (base + 8 * U * far + 32 * U * (1 + log_p + far))).sum(1)
        # the rest: 1 - sum p is off by 4u, which its log magnifies
        term = term + rest * (2 * base + 32 * U * (log_rest + far.max(1) + 2)) + 8 * U * (1 + log_rest + far.max(1)) * (rest > 0)
        ratio = np.abs(1 - d["factor"])
        factor = ratio * (2 * base + 16 * U * (2 + far.max(1))) + 2 * U + np.where(rest > 0, ratio / np.where(rest > 0, rest, 1) * 8 * U, 0)
        q = d["q"]
        grad = (q * (base + 8 * U * far) * np.maximum(1, np.abs(d["factor"]))[:, None] + q * factor[:, None]
                + 16 * U * (d["p"] + q * np.maximum(1, np.abs(d["factor"]))[:, None]))
    scale = np.abs(w)
    return scale * term, grad * (scale / tau)[:, None] + 1e-37, factor


def check_distill(z, index, value, w, tau, tail, loss, stats, grad, dtype, label=""):
    d = ol.distill(z, index, value, w, tau, tail)
    weight = np.ones(z.shape[0]) if w is None else np.asarray(w, np.float64)
    tl, tg, tf = distill_bounds(z, d, weight, tau, tail)
    if loss is not None:
        close(loss.double().cpu().numpy(), d["loss"], tl + HALF_STEP["fp32"] * np.abs(d["loss"]), label + " loss")
        live = weight != 0
        s = stats.double().cpu().numpy()
        assert np.isnan(s[~live]).all(), label
        big = np.abs(np.where(np.isfinite(d["lse"]), d["lse"], 0))
        close(s[live, 0], d["lse"][live], (lse_tol(z.shape[1]) + 16 * U * big)[live], label + " lse")
        close(s[live, 1], d["factor"][live], tf[live] + HALF_STEP["fp32"] * np.abs(d["factor"][live]), label + " factor")
    if grad is not None:
        got, pads = whole(grad)
        close(got, d["grad"], tg + HALF_STEP[dtype] * (np.abs(d["grad"]) + tg), label + " grad")
        assert (pads == 0).all()


@pytest.mark.parametrize("V,tp,pad", HEADS)
@pytest.mark.parametrize("din,dout", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("tail", [False, True])
def test_distill(gpu_lib, V, tp, pad, din, dout, tail):
    import torch

    rows, k, tau = 7, min(V, 37), 1.7 if tail else 0.8
    rng = np.random.default_rng(V + 3)
    z = rounded(rng.normal(0, 3, (rows, V)), din)
    index, value = teacher(V, rows, V, k, mess=V > 4)
    z[4, rng.random(V) < 0.5] = -np.inf
    z[4, index[4][index[4] >= 0]] = 1.5
    w = np.float32(rng.uniform(-1, 1, rows))
    w[5] = 0.0
    z[5] = np.nan  # a padded position: not read
    lay = layout(V, tp, pad)
    ti, tv, tw = dev(index, np.int32), dev(value, np.float32), dev(w, np.float32)
    student, grad = place(z, lay, din, wide=3, skip=1), place(np.zeros_like(z), lay, dout, wide=1, skip=5, fill=7.0)
    if V == 1 and tail:
        value[:] = 0.0  # the one column has all the mass
        tv = dev(value, np.float32)
    loss, stats = emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=grad)
    z[5] = 0.0
    check_distill(z, index, value, w, tau, tail, loss, stats, grad, dout, "one call")
    assert all((t.as_strided((rows - 1, 1), (t.stride(0), 1), t.storage_offset() + t.shape[1]) == 7.0).all() for t in grad.tensors)
    alone = emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail)
    check_distill(z, index, value, w, tau, tail, *alone, None, dout, "loss alone")
    back = emu.distill_backward(student, ti, tv, stats, tw, place(np.zeros_like(z), lay, dout), temperature=tau, tail=tail)
    check_distill(z, index, value, w, tau, tail, None, None, back, dout, "backward")
    if din == dout:
        again = emu.LogitShards(lay, [t.clone() for t in student.tensors])
        emu.distill_backward(again, ti, tv, stats, tw, again, temperature=tau, tail=tail)
        assert same_bits(again.tensors, back.tensors), "backward in place"
        l2, _ = emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=student)
        assert same_bits(student.tensors, grad.tensors) and torch.equal(l2, loss), "in place"


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("k", [1, 2, 63, 64, 65, 255, 256])
def test_distill_list_lengths(gpu_lib, k, tail):
    V, rows = 2011, 4
    z = rounded(np.random.default_rng(k).normal(0, 2, (rows, V)), "fp32")
    index, value = teacher(k, rows, V, k, mess=k > 4)
    lay = layout(V, 2, 1)
    grad = place(np.zeros_like(z), lay, "fp32")
    wide_i, wide_v = dev(np.pad(index, ((0, 0), (0, 5))), np.int32)[:, :k], dev(np.pad(value, ((0, 0), (0, 3))), np.float32)[:, :k]
    loss, stats = emu.distill_loss(place(z, lay, "fp32"), wide_i, wide_v, tail=tail, grad=grad)
    check_distill(z, index, value, None, 1.0, tail, loss, stats, grad, "fp32")


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_distill_rows_with_extreme_values(gpu_lib, tail, dtype):
    V, rows, k = 1003, 10, 9
    lowest = rounded(-3.4e38 if dtype == "fp32" else -3.38e38, dtype)
    rng = np.random.default_rng(8)
    z = rounded(rng.normal(0, 2, (rows, V)), dtype)
    index, value = teacher(11, rows, V, k, mess=False)
    z[0] = -np.inf
    z[1] = lowest
    z[2, index[2, 0] + 1 if index[2, 0] < V - 1 else 0] = np.nan
    z[3, index[3, 0]] = np.inf
    z[4] = 3e6 + rounded(1e6 * rng.integers(0, 2, V), dtype)
    z[5, index[5, 2]] = -np.inf                       # p > 0 meets q = 0
    z[6] = rounded(np.where(rng.random(V) < 0.5, lowest, z[6]), dtype)
    z[6, index[6]] = 1.0
    outside = np.ones(V, bool)
    outside[index[7]] = False
    z[7, outside] = -np.inf                           # nothing outside the list, which sums to 1 but for rounding
    value[7] = np.float32(value[7] - np.log(np.exp(value[7].astype(np.float64)).sum()))
    z[8] = rounded(z[8] - 30, dtype)
    z[8, index[8]] = 30                               # a mass of e^-60 outside
    value[9] = -np.inf
    z = rounded(z, dtype)                             # what the kernel gets
    lay = layout(V, 4, 1)
    grad = place(np.zeros_like(z), lay, "fp32")
    loss, stats = emu.distill_loss(place(z, lay, dtype), dev(index, np.int32), dev(value, np.float32), tail=tail, grad=grad)
    check_distill(z, index, value, None, 1.0, tail, loss, stats, grad, "fp32")
    back = emu.distill_backward(place(z, lay, dtype), dev(index, np.int32), dev(value, np.float32), stats,
                                dev(np.ones(rows), np.float32), place(np.zeros_like(z), lay, "fp32"), tail=tail)
    check_distill(z, index, value, None, 1.0, tail, None, None, back, "fp32")


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(gpu_lib, tail):
    V, rows, k, tau = 301, 3, 12, 1.4
    rng = np.random.default_rng(2)
    z = rounded(rng.normal(0, 2, (rows, V)), "fp32")
    index, value = teacher(3, rows, V, k, mess=False)
    grad = place(np.zeros_like(z), layout(V, 1, 0), "fp32")
    emu.distill_loss(place(z, layout(V, 1, 0), "fp32"), dev(index, np.int32), dev(value, np.float32), temperature=tau,
                     tail=tail, grad=grad)
    g = whole(grad)[0]
    eps = 1e-4
    for _ in range(8):
        d = rng.normal(0, 1, z.shape)
        up, down = (ol.distill(z + s * eps * d, index, value, None, tau, tail)["loss"] for s in (1, -1))
        # third derivatives of the loss along d stay below 100 here: eps^2 / 6 * 100, and fp32's error of the sum
        assert np.allclose((up - down) / (2 * eps), (g * d).sum(1), rtol=0, atol=1e-6 + 64 * U * np.abs(g * d).sum())


@pytest.mark.parametrize("rows", [1, 2, 9, 300, 1500])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_rows(gpu_lib, rows, tail):
    V = 5003
    z = rounded(np.random.default_rng(rows).normal(0, 2, (rows, V)), "bf16")
    index, value = teacher(rows, rows, V, 20, mess=rows > 4)
    lay = layout(V, 2, 1)
    grad = place(np.zeros_like(z), lay, "bf16")
    loss, stats = emu.distill_loss(place(z, lay, "bf16"), dev(index, np.int32), dev(value, np.float32), tail=tail, grad=grad)
    check_distill(z, index, value, None, 1.0, tail, loss, stats, grad, "bf16")


# (vocabulary, tp, pad, dtype): what 4 waves hold at a tile or at 16 each, 8 waves, 16 waves; borders inside tiles, pads
HELD = [(1024, 2, 0, "bf16"), (4096, 2, 64, "bf16"), (4001, 2, 64, "fp32"), (16000, 3, 8, "bf16"), (40000, 8, 8, "fp32"),
        (50304, 4, 8, "bf16"), (128256, 8, 128, "bf16")]


@pytest.mark.parametrize("V,tp,pad,dtype", HELD)
@pytest.mark.parametrize("tail", [False, True])
def test_distill_rows_held_in_registers(gpu_lib, V, tp, pad, dtype, tail):
    """Many aligned rows, which stay in registers between loss and gradient: bit for bit what the same rows give off
    the vectors' alignment, where they are read again; the small ones against the definition, too."""
    import torch

    rows, k, tau = 601, 24, 1.3
    rng = np.random.default_rng(V)
    lay = layout(V, tp, pad)
    z = torch.randn(rows, V, device="cuda") * 3
    z[3], z[5], z[9, ::2] = -float("inf"), 2e7, -3.38e38
    z[8] = z[8] * 1e6
    z[11, 7] = float("nan")
    z[-1, : V // 2] = -float("inf")
    z = z.to(torch_type(dtype)).double().cpu().numpy()
    index, value = teacher(V, rows, V, k)
    index[20], value[21], value[3] = -1, -np.inf, value[3]
    w = np.float32(rng.uniform(-1, 1, rows))
    w[rng.random(rows) < 0.3] = 0
    w[[3, 5, 8, 9, 11, 20, 21]] = 0.5
    ti, tv, tw = dev(index, np.int32), dev(value, np.float32), dev(w, np.float32)
    wide = -emu.shard_columns(lay) % 8
    got = []
    for skip in (0, 1):
        student = place(z, lay, dtype, wide=wide, skip=skip)
        grad = place(np.zeros_like(z), lay, dtype, wide=wide, skip=skip, fill=7.0)
        loss, stats = emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=grad)
        got.append([loss, stats] + [t.clone() for t in grad.tensors])
        if skip == 0:
            held = grad
        emu.distill_loss(student, ti, tv, weight=tw, temperature=tau, tail=tail, grad=student)
        assert same_bits(student.tensors, grad.tensors), "in place"
    assert same_bits(*got)
    if V < 5000:
        check_distill(z, index, value, w, tau, tail, got[0][0], got[0][1], held, dtype)


@pytest.mark.parametrize("V,tp,pad", [(266240, 2, 0), (300007, 4, 64), (262100, 2, 65536)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [2, 270])
def test_wide_vocabularies(gpu_lib, V, tp, pad, dtype, rows):
    """Rows that no single workgroup takes, and rows whose pads reach beyond what one does."""
    rng = np.random.default_rng(V)
    x = rounded(np.tile(rng.normal(0, 3, (2, V)), (rows // 2, 1)), dtype)
    lay = layout(V, tp, pad)
    student, grad = place(x, lay, dtype), place(np.zeros_like(x), lay, dtype)
    top = emu.top_logprobs(student, 64)
    check_topk(x[:2], [t[:2] for t in top], 64, 1.0)
    index, value = teacher(V, 2, V, 256, mess=False)
    index, value = np.tile(index, (rows // 2, 1)), np.tile(value, (rows // 2, 1))
    loss, stats = emu.distill_loss(student, dev(index, np.int32), dev(value, np.float32), tail=True, grad=grad)
    part = emu.LogitShards(lay, [t[:2] for t in grad.tensors])
    check_distill(x[:2], index[:2], value[:2], None, 1.0, True, loss[:2], stats[:2], part, dtype)
    for t in (*top, loss, stats, *grad.tensors):  # the same two rows again and again
        assert same_bits([t[-2:]], [t[:2]])
    c = constraints(1, 2, V, 20)
    got = place(x[:2], lay, dtype)
    want, tol = constrained(x[:2], c)
    apply(got, None, c)
    close(whole(got)[0], want, tol + np.where(np.isfinite(want), HALF_STEP[dtype] * (np.abs(want) + tol), 0))


def test_more_rows_than_a_launch_takes(gpu_lib):
    import torch

    V, rows, lay = 70, 70001, layout(70, 2, 0)
    x = rounded(np.random.default_rng(0).normal(0, 3, (1000, V)), "fp32")
    X = torch.from_numpy(x).float().cuda().repeat(71, 1)[:rows]
    student = emu.LogitShards(lay, [X[:, :35], X[:, 35:]])
    index, logp, lse = emu.top_logprobs(student, 9)
    check_topk(x, (index[:1000], logp[:1000], lse[:1000]), 9, 1.0)
    grad = emu.LogitShards.alloc(lay, rows, torch.float32)
    loss, stats = emu.distill_loss(student, index, logp, tail=True, grad=grad)
    out = emu.LogitShards.alloc(lay, rows, torch.float32)
    emu.constrain_logits(student, out, tokens=index, seq_len=dev(np.full(rows, 9), np.int32), presence=lse)
    head = [t[:1000] for t in (index, logp, lse, loss, stats, *grad.tensors, *out.tensors)]
    for at in (32000, 65000, 69000):
        assert same_bits(head, [t[at:at + 1000] for t in (index, logp, lse, loss, stats, *grad.tensors, *out.tensors)])
    d = ol.distill(x, index[:1000].cpu().numpy(), logp[:1000].cpu().numpy(), None, 1.0, True)
    assert np.abs(loss[:1000].double().cpu().numpy() - d["loss"]).max() < 1e-5  # 0 but for rounding: student and teacher agree


@pytest.mark.parametrize("rows", [3, 600])
def test_topk_many_ties(gpu_lib, rows):
    """More logits at the bound than the list holds, in rows shared by workgroups and in rows of their own."""
    V, lay = 20003, layout(20003, 2, 1)
    rng = np.random.default_rng(rows)
    x = np.tile(np.stack([rng.integers(0, 2, V), np.full(V, -1.5), np.arange(V) // 64 * 0.5]).astype(float), (rows // 3, 1))
    got = emu.top_logprobs(place(x, lay, "fp32"), 64)
    check_topk(x[:3], [t[:3] for t in got], 64, 1.0)
    assert same_bits([t[-3:] for t in got], [t[:3] for t in got])


@pytest.mark.parametrize("tau", [1e-6, 1e-3, 1e6])
@pytest.mark.parametrize("tail", [False, True])
def test_far_temperatures(gpu_lib, tau, tail):
    V, rows, k = 1500, 4, 10
    z = rounded(np.random.default_rng(5).normal(0, 3, (rows, V)), "fp32")
    index, value = teacher(6, rows, V, k, mess=False)
    lay = layout(V, 2, 0)
    check_topk(z, emu.top_logprobs(place(z, lay, "fp32"), k, tau), k, tau)
    if tail and tau < 1:  # a q of e^-1000 and less is 0 in the row's sum, and the loss infinite by definition of the tail's log
        return
    grad = place(np.zeros_like(z), lay, "fp32")
    loss, stats = emu.distill_loss(place(z, lay, "fp32"), dev(index, np.int32), dev(value, np.float32), temperature=tau, tail=tail, grad=grad)
    check_distill(z, index, value, None, tau, tail, loss, stats, grad, "fp32")


# ----------------------------------------------------------------------------------------------------
# together, and how they are called
# ----------------------------------------------------------------------------------------------------

def pipeline(lay, x, z, c, w, tail, stream=None):
    """A generation stage's constraints, the teacher's top of them, a student's loss and gradient: every output."""
    raw = place(x, lay, "bf16")
    out = apply(raw, None, c, stream=stream)
    index, logp, lse = emu.top_logprobs(out, 24, temperature=1.3, stream=stream)
    grad = emu.LogitShards.alloc(lay, x.shape[0], torch_type("bf16"))
    student = place(z, lay, "bf16")
    loss, stats = emu.distill_loss(student, index, logp, weight=w, temperature=1.3, tail=tail, grad=grad, stream=stream)
    back = emu.distill_backward(student, index, logp, stats, w, emu.LogitShards.alloc(lay, x.shape[0], torch_type("fp32")),
                                temperature=1.3, tail=tail, stream=stream)
    return out, index, logp, lse, loss, stats, grad, back


@pytest.mark.parametrize("V,rows", [(1024, 3), (1003, 40), (50257, 2), (50257, 400), (128256, 5)])
@pytest.mark.parametrize("tail", [False, True])
def test_one_result_under_every_layout(gpu_lib, V, rows, tail):
    """The run of a step's operators, bit for bit the same before and after a Split or Merge."""
    import torch

    rng = np.random.default_rng(V + rows)
    x, z = rounded(rng.normal(0, 3, (rows, V)), "bf16"), rounded(rng.normal(0, 3, (rows, V)), "bf16")
    c = constraints(V, rows, V, 200)
    c["allowed"][0, :30] = True
    w = dev(rng.uniform(0.1, 1, rows), np.float32)
    first = None
    for tp, pad in ((1, 0), (2, 1), (3, 1), (4, 64), (8, 128), (24, 7)):
        out, index, logp, lse, loss, stats, grad, back = pipeline(layout(V, tp, pad), x, z, c, w, tail)
        parts = [torch.cat(s.tensors, 1)[:, :V] for s in (out, grad, back)] + [index, logp, lse, loss, stats]
        first = first or parts
        assert same_bits(first, parts), f"tp={tp} pad={pad}"
    # each stage against the definition, from the inputs it had
    got = whole(out)[0]
    want, tol = constrained(x, c)
    close(got, want, tol + np.where(np.isfinite(want), HALF_STEP["bf16"] * (np.abs(want) + tol), 0), "constraints")
    if rows <= 40:
        check_topk(got, (index, logp, lse), 24, 1.3)
        check_distill(z, index.cpu().numpy(), logp.cpu().numpy(), w.cpu().numpy(), 1.3, tail, loss, stats, grad, "bf16")


def test_other_streams(gpu_lib):
    """The given stream's order: inputs written there, late, are what the calls read."""
    import torch

    V, rows, lay = 50257, 6, layout(50257, 2, 1)
    rng = np.random.default_rng(1)
    x, z = rounded(rng.normal(0, 3, (rows, V)), "bf16"), rounded(rng.normal(0, 3, (rows, V)), "bf16")
    c, w = constraints(4, rows, V, 100), dev(np.ones(rows), np.float32)
    c["allowed"][:, :40] = True
    want = pipeline(lay, x, z, c, w, True)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 1e-3
        got = pipeline(lay, x, z, c, w, True)
    b.wait_stream(torch.cuda.current_stream())
    other = pipeline(lay, x, z, c, w, True, stream=None)
    a.synchronize()
    for run in (got, other):
        for p, q in zip(want, run):
            p, q = (t.tensors if hasattr(t, "tensors") else [t] for t in (p, q))
            assert same_bits(p, q)
    # an explicit stream, with its inputs ready
    src = place(x, lay, "bf16")
    torch.cuda.synchronize()
    index, logp, lse = emu.top_logprobs(src, 9, stream=b)
    b.synchronize()
    assert same_bits((index, logp, lse), emu.top_logprobs(src, 9))


def test_captured_and_replayed(gpu_lib):
    """A decode step's and a training step's calls in two graphs, replayed in turn with new inputs and eager work
    between; every replay equals the eager result."""
    import torch

    V, lay = 50257, layout(50257, 2, 1)
    rng = np.random.default_rng(7)
    for rows in (2, 300):
        raw, student = place(np.zeros((rows, V)), lay, "bf16"), place(np.zeros((rows, V)), lay, "bf16")
        out, grad = (emu.LogitShards.alloc(lay, rows, torch.bfloat16) for _ in range(2))
        c = constraints(rows, rows, V, 64)
        c["allowed"][:, :40] = True
        w = dev(rng.uniform(0.5, 1, rows), np.float32)
        ops = dict(tokens=dev(c["tokens"], np.int32), seq_len=dev(c["seq_len"], np.int32),
                   repetition=dev(c["repetition"], np.float32), mask=dev(packed(c["allowed"]), np.int32),
                   mask_row=dev(c["mask_row"], np.int32))
        index, logp, lse = emu.top_logprobs(emu.constrain_logits(raw, out, **ops), 20)
        emu.distill_loss(student, index, logp, weight=w, tail=True, grad=grad)
        torch.cuda.synchronize()
        decode, train = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(decode):
            emu.constrain_logits(raw, out, **ops)
            gi, gp, gl = emu.top_logprobs(out, 20)
        with torch.cuda.graph(train):
            loss, stats = emu.distill_loss(student, gi, gp, weight=w, tail=True, grad=grad)
        for replay in range(4):
            for s in (raw, student):
                for t in s.tensors:
                    t.normal_(0, 3)
            torch.cuda.synchronize()
            decode.replay()
            train.replay()
            torch.cuda.synchronize()
            kept = [t.clone() for t in (gi, gp, gl, loss, stats, *grad.tensors, *out.tensors)]
            o2, g2 = (emu.LogitShards.alloc(lay, rows, torch.bfloat16) for _ in range(2))
            top = emu.top_logprobs(emu.constrain_logits(raw, o2, **ops), 20)
            eager = emu.distill_loss(student, top[0], top[1], weight=w, tail=True, grad=g2)
            V_cols = [t for t in (*top, *eager, *g2.tensors, *o2.tensors)]
            assert same_bits(kept, V_cols), f"{rows} rows, replay {replay}"


def test_rows_beyond_32_bit_offsets(gpu_lib):
    """Rows that start behind 2^32 elements of a shard."""
    import torch

    V, lay = 1003, layout(1003, 1, 0)
    stride, rows = 1 << 31, 3
    buf = torch.zeros(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    x = rounded(np.random.default_rng(1).normal(0, 3, (rows, V)), "bf16")
    s = buf.as_strided((rows, V), (stride, 1))
    s.copy_(torch.from_numpy(x).to(torch.bfloat16))
    far, near = emu.LogitShards(lay, [s]), place(x, lay, "bf16")
    assert same_bits(emu.top_logprobs(far, 8), emu.top_logprobs(near, 8))
    index, value = teacher(1, rows, V, 8, mess=False)
    ti, tv = dev(index, np.int32), dev(value, np.float32)
    g = place(np.zeros_like(x), lay, "bf16")
    emu.distill_loss(near, ti, tv, grad=g)
    emu.distill_loss(far, ti, tv, grad=far)
    assert same_bits([s], g.tensors)


def test_binding_on_the_device(gpu_lib):
    import torch

    lay, rows = layout(1000, 2, 0), 3
    x = place(np.zeros((rows, 1000)), lay, "fp32")
    i32 = dict(dtype=torch.int32, device="cuda")
    for bad in (dict(tokens=torch.zeros(rows, 4, **i32)), dict(seq_len=torch.zeros(rows, **i32)),
                dict(tokens=torch.zeros(rows, 4, dtype=torch.int64, device="cuda"), seq_len=torch.zeros(rows, **i32)),
                dict(tokens=torch.zeros(rows + 1, 4, **i32), seq_len=torch.zeros(rows, **i32)),
                dict(repetition=torch.zeros(rows, device="cuda").double()), dict(repetition=torch.zeros(rows)),
                dict(mask=torch.zeros(2, 32, **i32)), dict(mask=torch.zeros(rows, 31, **i32)),
                dict(mask_row=torch.zeros(rows, **i32)),
                dict(bias=(torch.zeros(rows, **i32), torch.zeros(1, **i32), torch.zeros(1, device="cuda")))):
        with pytest.raises((ValueError, emu.EmuError)):
            emu.constrain_logits(x, **bad)
    index, value = torch.zeros(rows, 4, **i32), torch.zeros(rows, 4, device="cuda")
    for bad in ((index.long(), value), (index, value.double()), (index[:2], value), (index, value[:, :3]),
                (index.cpu(), value)):
        with pytest.raises((ValueError, emu.EmuError)):
            emu.distill_loss(x, *bad)
    with pytest.raises(ValueError):
        emu.distill_backward(x, index, value, torch.zeros(rows, 2, device="cuda"), None, x)
    empty = emu.LogitShards(lay, [torch.zeros(0, 500, device="cuda") for _ in range(2)])
    assert [tuple(t.shape) for t in emu.top_logprobs(empty, 3)] == [(0, 3), (0, 3), (0,)]
    loss, stats = emu.distill_loss(empty, index[:0], value[:0], grad=empty)
    assert loss.shape == (0,) and stats.shape == (0, 4)
