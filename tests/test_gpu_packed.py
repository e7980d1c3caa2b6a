"""Packed sequences on the GPU: row maps, attention, normed and rotated queries and keys, against 64 bits (packed_reference.py derives the
bounds)."""
import math
import random

import pytest
import torch

import packed_reference as ref
from paper_2503_01328_amd import binding as po

pytestmark = pytest.mark.gpu

DT = {"f32": (po.PO_F32, torch.float32), "bf16": (po.PO_BF16, torch.bfloat16)}
MARK = 7.0  # what untouched rows hold


def _gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _plan(lengths, rows, dev, maps=False):
    t = torch.tensor(lengths, dtype=torch.int32, device=dev)
    plan = torch.empty(po.po_op_packed_plan_bytes(rows) // 4, dtype=torch.int32, device=dev)
    new = lambda n: torch.full((n,), -9, dtype=torch.int32, device=dev)
    out = (new(len(lengths) + 1), new(rows), new(rows)) if maps else (None, None, None)
    po.po_op_packed_plan(t, len(lengths), rows, *out, plan)
    return (plan, *out) if maps else plan


def _within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    bad &= ~(want.isnan() & (got.float() == MARK))  # rows of no sequence keep what they held
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])} for {float(want[i])} +- {float(tol[i])}")


# ---- maps ---------------------------------------------------------------------------------------------------------
def _random_lengths(seed, n, most):
    rng = random.Random(seed)
    return [rng.choice([0, 1, rng.randrange(most + 1)]) for _ in range(n)]


LENGTHS = [([1], 1), ([5], 9), ([0, 3, 0, 1, 0], 4), ([0], 3), ([-4, 6, -1, 2], 20), ([10, 2000, 5], 700), ([2 ** 31 - 1] * 3, 200),
           ([128, 128], 256), ([127, 1, 129, 64], 400), (_random_lengths(1, 1500, 9), 4500), (_random_lengths(2, 16384, 40), 200000),
           (_random_lengths(3, 1024, 5), 1024), (_random_lengths(4, 1025, 5), 2000), ([1] * 5000, 5000), ([2097152], 2097152),
           (_random_lengths(5, 16384, 100), 900001)]


@pytest.mark.parametrize("lengths,rows", LENGTHS, ids=lambda v: str(len(v)) if isinstance(v, list) else str(v))
def test_plan(gpu_device, lengths, rows):
    plan, starts, positions, sequence = _plan(lengths, rows, gpu_device, maps=True)
    want = ref.maps(lengths, rows)
    assert starts.tolist() == want[0]
    assert sequence.tolist() == want[1] and positions.tolist() == want[2]
    total, blocks = want[0][-1], -(-rows // 128)
    plan, padded = plan.cpu(), 128 * blocks
    assert plan[:2].tolist() == [total, rows]
    first, end = plan[16:16 + padded], plan[16 + padded:16 + 2 * padded]
    row = torch.arange(padded)
    held = torch.tensor(want[1] + [-1] * (padded - rows))
    s = torch.tensor(want[0])
    assert torch.equal(first, torch.where(held >= 0, s[held.clamp(min=0)], rows).int())
    assert torch.equal(end, torch.where(held >= 0, s[held.clamp(min=0) + 1], total).int())
    # the orders: the blocks by falling number of tiles of 64, lower ones first among equals
    b0 = torch.arange(blocks) * 128
    b1 = torch.clamp(b0 + 128, max=total)
    keys = torch.where(b0 < total, (b1 - first[b0] // 64 * 64 + 63) // 64, 0)
    queries = torch.where(b0 < total, (end[(b1 - 1).clamp(min=0)] - b0 + 63) // 64, 0)
    bounds = (torch.where(b0 < total, first[b0], 0), torch.where(b0 < total, end[(b1 - 1).clamp(min=0)], 0))
    for work, bound, order in zip((keys, queries), bounds, plan[16 + 2 * padded:].reshape(2, blocks, 2)):
        assert order[:, 0].tolist() == sorted(range(blocks), key=lambda b: (-int(work[b]), b))
        assert torch.equal(order[:, 1].long(), bound[order[:, 0].long()].long())


def test_plan_leaves_out_what_is_not_wanted(gpu_device):
    lengths = torch.tensor([3, 4], dtype=torch.int32, device=gpu_device)
    positions = torch.full((11,), -9, dtype=torch.int32, device=gpu_device)
    po.po_op_packed_plan(lengths, 2, 10, None, positions, None, None)
    assert positions.tolist() == [0, 1, 2, 0, 1, 2, 3, -1, -1, -1, -9]


# ---- attention ----------------------------------------------------------------------------------------------------
def _inputs(dev, dtype, rows, h, hkv, seed, used=None):
    g, tdt = _gen(dev, seed), DT[dtype][1]
    qkv = torch.randn(rows, h + 2 * hkv, generator=g, device=dev).to(tdt)
    d_o = torch.randn(rows, h, generator=g, device=dev).to(tdt)
    if used is not None:  # rows of no sequence: whatever memory holds
        qkv[used:] = math.nan
        d_o[used:] = math.nan
    return qkv, d_o


def _guarded(dev, dtype, *shape):
    """A tensor of MARK in the middle of a buffer of it."""
    n, edge = math.prod(shape), 1 << 16
    whole = torch.full((n + 2 * edge,), MARK, dtype=dtype, device=dev)
    return whole[edge:edge + n].view(shape), (whole[:edge], whole[edge + n:])


def _attention(dtype, qkv, d_o, plan, h, a, akv):
    code, rows, dev = DT[dtype][0], qkv.shape[0], qkv.device
    (o, edge_o), (lse, edge_lse), (dqkv, edge_d) = (_guarded(dev, t, *s) for t, s in ((qkv.dtype, (rows, h)), (torch.float32, (a, rows)),
                                                                                 (qkv.dtype, qkv.shape)))
    po.po_op_attention_packed_forward(code, qkv, plan, o, lse, rows, h, a, akv)
    size = po.po_op_attention_packed_backward_workspace(code, rows, h, a, akv)
    ws = torch.full((size + (1 << 16),), 255, dtype=torch.uint8, device=dev)  # NaN, and a margin to be left alone
    po.po_op_attention_packed_backward(code, qkv, plan, o, lse, d_o, dqkv, ws, rows, h, a, akv)
    assert bool((ws[size:] == 255).all())
    assert all(bool((t == MARK).all()) for edges in (edge_o, edge_lse, edge_d) for t in edges)
    return dict(o=o, lse=lse, dqkv=dqkv)


def _attention_case(dev, dtype, dh, a, akv, lengths, rows, seed=0):
    h, hkv = a * dh, akv * dh
    qkv, d_o = _inputs(dev, dtype, rows, h, hkv, seed, min(rows, sum(max(0, n) for n in lengths)))
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, dev), h, a, akv)
    want, tol = ref.attention(qkv, d_o, lengths, h, a, akv)
    for k in ("o", "lse", "dqkv"):
        _within(got[k], want[k], tol[k], k)


PACKS = [([1], 1), ([1, 1, 1], 5), ([7], 7), ([0, 3, 0, 1, 0], 6), ([31, 32, 33], 96), ([128], 128), ([127, 1, 129], 300),
         ([64] * 5, 320), ([5, 250, 3, 40], 333), ([300, 2, 500], 802), ([3] * 40 + [100] + [17] * 9, 400), ([700], 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh,a,akv", [(64, 1, 1), (64, 6, 2), (128, 3, 3), (128, 4, 1)])
@pytest.mark.parametrize("lengths,rows", PACKS, ids=lambda v: "x".join(map(str, v[:4])) if isinstance(v, list) else str(v))
def test_attention(gpu_device, dtype, dh, a, akv, lengths, rows):
    _attention_case(gpu_device, dtype, dh, a, akv, lengths, rows)


# launches that fill the chip, blocks that hold many sequences, and one that walks many tiles
MANY = [("bf16", 64, 16, 4, [700, 1, 0, 900, 64], 1700), ("bf16", 64, 8, 8, [130] * 12, 1560), ("bf16", 128, 20, 4, [400, 33, 300], 800),
        ("bf16", 128, 32, 8, [150] * 20 + [3] * 50, 3200), ("bf16", 64, 40, 40, [1000, 11, 2000], 3100), ("bf16", 128, 16, 2, [2500, 1, 90], 2600),
        ("bf16", 128, 7, 7, [4096], 4096), ("bf16", 64, 40, 8, [37] * 100, 3712), ("bf16", 128, 40, 40, [600, 70, 1400], 2071), ("f32", 64, 16, 4, [900, 20, 400], 1400)]


@pytest.mark.parametrize("dtype,dh,a,akv,lengths,rows", MANY, ids=lambda v: "" if isinstance(v, list) else str(v))
def test_attention_of_many_blocks(gpu_device, dtype, dh, a, akv, lengths, rows):
    _attention_case(gpu_device, dtype, dh, a, akv, lengths, rows)


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
def test_attention_gradient_is_that_of_differences(gpu_device, dtype, dh):
    """sum(w o) along random directions of qkv: central differences of the 64-bit definition against the kernels' gradient."""
    a, akv, lengths, rows = 4, 2, [40, 1, 90], 131
    h, hkv = a * dh, akv * dh
    qkv, w = _inputs(gpu_device, dtype, rows, h, hkv, 5)
    got = _attention(dtype, qkv, w, _plan(lengths, rows, gpu_device), h, a, akv)["dqkv"].double()
    _, tol = ref.attention(qkv, w, lengths, h, a, akv)
    loss = lambda x: float((ref.attention(x, w.double(), lengths, h, a, akv)[0]["o"] * w.double()).sum())
    g = _gen(gpu_device, 6)
    for cols in (slice(0, h), slice(h, h + hkv), slice(h + hkv, None)):
        v = torch.zeros_like(got)
        v[:, cols] = torch.randn(got[:, cols].shape, generator=g, device=gpu_device, dtype=torch.float64)
        step = 1e-5
        slope = (loss(qkv.double() + step * v) - loss(qkv.double() - step * v)) / (2 * step)
        # differences in 64 bits: step^2 of a third derivative of about the slope's size, 2^-53 of the loss over the step
        assert abs(float((got * v).sum()) - slope) <= float((tol["dqkv"] * v.abs()).sum()) + 1e-6 * (abs(slope) + 1)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["q", "k", "v", "d_o"])
@pytest.mark.parametrize("dtype,dh,a,akv,lengths", [("f32", 64, 2, 1, [10, 50, 20]), ("bf16", 64, 4, 2, [10, 50, 20]), ("f32", 128, 2, 2, [70, 90]),
                                                    ("bf16", 128, 2, 1, [33, 100, 200, 5]), ("bf16", 128, 32, 8, [300] * 10),
                                                    ("bf16", 64, 40, 40, [300] * 10), ("bf16", 64, 15, 15, [300] * 5),
                                                    ("bf16", 128, 20, 4, [250] * 5)])
def test_attention_non_finite_rows_stay_in_their_sequence(gpu_device, dtype, dh, a, akv, lengths, where, value):
    """One element that is not finite, in head 0 of a row in the middle of a sequence.  Every other sequence, and every other head, gets the
    results that it gets without; in key or value rows it reaches no row of o and dQ before it."""
    h, hkv, rows = a * dh, akv * dh, sum(lengths)
    qkv, d_o = _inputs(gpu_device, dtype, rows, h, hkv, 8)
    plan = _plan(lengths, rows, gpu_device)
    clean = _attention(dtype, qkv, d_o, plan, h, a, akv)
    want, tol = ref.attention(qkv, d_o, lengths, h, a, akv)
    j = len(lengths) // 2
    lo, hi = sum(lengths[:j]), sum(lengths[:j + 1])
    row = (lo + hi) // 2
    {"q": qkv[:, :h], "k": qkv[:, h:], "v": qkv[:, h + hkv:], "d_o": d_o}[where][row, 3] = value
    got = _attention(dtype, qkv, d_o, plan, h, a, akv)
    group = a // akv
    for k in ("o", "lse", "dqkv"):
        keep = torch.ones_like(want[k], dtype=torch.bool)
        if k == "lse":
            keep[:group if where != "q" else 1, lo if where == "q" else row:hi] = False
        elif k == "o":
            keep[row if where in "kv" else row:hi, :group * dh] = False
        else:
            keep[row if where in "kv" else row:hi, :group * dh] = False  # dQ of the rows that see it
            keep[lo:hi, h:h + dh] = False
            keep[lo:hi, h + hkv:h + hkv + dh] = False
        same = torch.where(keep, got[k].double(), want[k])
        _within(same, want[k], tol[k], k)
        outside = keep.clone()
        (outside[:, lo:hi] if k == "lse" else outside[lo:hi])[:] = False
        assert torch.isfinite(got[k][outside]).all()
    if where in "kv" and not math.isinf(value):
        assert got["o"][row, 3 if where == "v" else 0].isnan() and clean["o"][row].isfinite().all()


@pytest.mark.parametrize("where", ["q", "k", "v", "d_o"])
@pytest.mark.parametrize("dtype,dh,a,akv", [("f32", 64, 4, 2), ("bf16", 64, 4, 2), ("bf16", 128, 40, 8)])
def test_attention_of_nan_sequences(gpu_device, dtype, dh, a, akv, where):
    """A whole input NaN in one of three sequences: there everything that it reaches is NaN (dV of NaN values is not), elsewhere nothing."""
    h, hkv, lengths, rows = a * dh, akv * dh, [400, 300, 500], 1200
    qkv, d_o = _inputs(gpu_device, dtype, rows, h, hkv, 15)
    want, tol = ref.attention(qkv, d_o, lengths, h, a, akv)
    {"q": qkv[:, :h], "k": qkv[:, h:h + hkv], "v": qkv[:, h + hkv:], "d_o": d_o}[where][400:700] = math.nan
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, gpu_device), h, a, akv)
    inside = torch.zeros(rows, dtype=torch.bool, device=gpu_device)
    inside[400:700] = True
    for k in ("o", "lse", "dqkv"):
        x, w, t = (y.T if k == "lse" else y for y in (got[k], want[k], tol[k]))
        _within(x[~inside], w[~inside], t[~inside], k)
    if where != "d_o":
        assert got["o"][inside].isnan().all()
    nan = got["dqkv"][inside].isnan()
    assert nan[:, :h + hkv].all() and (where == "v" or nan[:, h + hkv:].all())
    if where == "v":
        _within(got["dqkv"][inside][:, h + hkv:], want["dqkv"][inside][:, h + hkv:], tol["dqkv"][inside][:, h + hkv:], "dV")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first,last", [(0, 40), (64, 128), (5, 70)])
def test_attention_keys_of_minus_infinity_add_nothing(gpu_device, dtype, first, last):
    """Scores of -inf for keys first .. last - 1 of a sequence: rows that see another key are as if these were not there."""
    dh, n, lead = 64, 160, 23
    qkv, _ = _inputs(gpu_device, dtype, lead + n, dh, dh, 9)
    qkv[:, 0] = 1.0
    qkv[:, dh] = 0.0
    qkv[lead + first:lead + last, dh] = -math.inf
    o = torch.full((lead + n, dh), MARK, dtype=qkv.dtype, device=gpu_device)
    lse = torch.empty(1, lead + n, device=gpu_device)
    po.po_op_attention_packed_forward(DT[dtype][0], qkv, _plan([lead, n], lead + n, gpu_device), o, lse, lead + n, dh, 1)
    x = qkv[lead:].double()
    q, k, v = x.split(dh, 1)
    seen = torch.ones(n, n, dtype=torch.bool, device=gpu_device).tril()
    seen[:, first:last] = False
    sc = (q @ torch.nan_to_num(k, neginf=0.0).T / 8).masked_fill(~seen, -math.inf)
    rows = seen.any(1)
    p = torch.softmax(sc[rows], 1)
    u = ref.half_step(qkv.dtype)
    _within(o[lead:][rows], p @ v, 2.1 * u * (p @ v.abs()) + 1e-4 * (p @ v.abs()), "o")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_large_scores(gpu_device, dtype):
    """Scores in the hundreds, one key ahead of all others: the sums stay exact."""
    dh, a, lengths, rows = 128, 2, [200, 60], 260
    qkv, d_o = _inputs(gpu_device, dtype, rows, a * dh, a * dh, 10)
    qkv[:, :2 * a * dh] *= 6
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, gpu_device), a * dh, a, a)
    want, tol = ref.attention(qkv, d_o, lengths, a * dh, a, a)
    for k in ("o", "lse", "dqkv"):
        _within(got[k], want[k], tol[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_equals_that_of_the_sequences_alone(gpu_device, dtype):
    """A sequence's results against po_op_attention_* of it by itself: both within their bounds of the same values."""
    dh, a, akv, lengths = 64, 4, 2, [65, 130, 1]
    h, hkv, rows = a * dh, akv * dh, sum(lengths)
    code, tdt = DT[dtype]
    qkv, d_o = _inputs(gpu_device, dtype, rows, h, hkv, 11)
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, gpu_device), h, a, akv)
    _, tol = ref.attention(qkv, d_o, lengths, h, a, akv)
    at = 0
    for n in lengths:
        s, at = slice(at, at + n), at + n
        o, lse = torch.empty(n, h, dtype=tdt, device=gpu_device), torch.empty(a, n, device=gpu_device)
        dqkv, delta = torch.empty(n, h + 2 * hkv, dtype=tdt, device=gpu_device), torch.empty(a, n, device=gpu_device)
        x, d = qkv[s].contiguous(), d_o[s].contiguous()
        po.po_op_attention_forward(code, x, o, lse, n, h, a, n_kv_heads=akv)
        po.po_op_attention_backward(code, x, o, lse, d, dqkv, delta, n, h, a, n_kv_heads=akv)
        _within(got["o"][s], o.double(), 2 * tol["o"][s], "o")
        _within(got["lse"][:, s], lse.double(), 2 * tol["lse"][:, s], "lse")
        _within(got["dqkv"][s], dqkv.double(), 2 * tol["dqkv"][s], "dqkv")


@pytest.mark.parametrize("dtype,dh,a,akv,rows", [("f32", 64, 4, 2, 500), ("bf16", 64, 4, 2, 500), ("bf16", 128, 32, 8, 2048)])
def test_attention_runs_alike_every_time(gpu_device, dtype, dh, a, akv, rows):
    lengths = [rows // 3, 1, rows // 2, rows // 12]
    qkv, d_o = _inputs(gpu_device, dtype, rows, a * dh, akv * dh, 12)
    plan = _plan(lengths, rows, gpu_device)
    one, two = (_attention(dtype, qkv, d_o, plan, a * dh, a, akv) for _ in range(2))
    assert all(torch.equal(one[k], two[k]) for k in one)


def test_attention_with_another_batchs_plan_computes_nothing(gpu_device):
    rows, dh = 300, 64
    qkv, d_o = _inputs(gpu_device, "bf16", rows, dh, dh, 13)
    got = _attention("bf16", qkv, d_o, _plan([100, 28], 128, gpu_device), dh, 1, 1)
    assert all(bool((t == MARK).all()) for t in got.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(gpu_device, dtype):
    """A batch of more than 2^31 elements: its last sequences, and its first."""
    dh, a = 128, 32
    rows = 2 ** 31 // (3 * a * dh) + 400 if dtype == "bf16" else 2 ** 30 // (3 * a * dh) + 400  # 4 GiB of qkv and more
    h, tdt = a * dh, DT[dtype][1]
    lengths = [150] + [1] * 9000 + [200] * ((rows - 9150 - 50) // 200)
    g = _gen(gpu_device, 14)
    qkv = torch.empty(rows, 3 * h, dtype=tdt, device=gpu_device).normal_(generator=g)
    d_o = torch.empty(rows, h, dtype=tdt, device=gpu_device).normal_(generator=g)
    plan, _, positions, _ = _plan(lengths, rows, gpu_device, maps=True)
    got = _attention(dtype, qkv, d_o, plan, h, a, a)
    used = sum(lengths)
    for s, n in ((slice(0, 150), [150]), (slice(used - 400, used), [200, 200])):
        want, tol = ref.attention(qkv[s], d_o[s], n, h, a, a)
        _within(got["o"][s], want["o"], tol["o"], "o")
        _within(got["lse"][:, s], want["lse"], tol["lse"], "lse")
        _within(got["dqkv"][s], want["dqkv"], tol["dqkv"], "dqkv")
    assert bool((got["dqkv"][used:] == MARK).all()) and bool((got["o"][used:] == MARK).all())
    inv_freq = (10000.0 ** (-torch.arange(64, device=gpu_device) / 64)).float()
    out = got["dqkv"]
    po.po_op_qk_norm_rotary_forward(DT[dtype][0], qkv, None, None, positions, inv_freq, [64], 0, out, rows, h, a)
    s = slice(used - 300, used)
    want, tol = ref.rotary(qkv[s], None, None, positions[None, s], inv_freq, [64], False, h, a, a, 0.0)
    _within(out[s], want["out"], tol["out"], "out")


# ---- norm and rotation --------------------------------------------------------------------------------------------
def _rotary_case(dev, dtype, dh, a, akv, rows, axis_pairs, neighbours, norm, far, in_place, seed=0):
    code, tdt = DT[dtype]
    h, hkv, g = a * dh, akv * dh, _gen(dev, seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=dev).to(tdt)
    qkv, d_out = rand(rows, h + 2 * hkv), rand(rows, h + 2 * hkv)
    gain_q, gain_k = (1 + 0.3 * rand(dh), 1 - 0.3 * rand(dh)) if norm else (None, None)
    positions = torch.randint(0, far + 1, (len(axis_pairs), rows), generator=g, device=dev, dtype=torch.int32)
    positions[1:] -= far // 2
    positions[0, ::5] = -1  # rows that hold nothing
    positions[0, :1] = far
    qkv[positions[0] < 0] = math.nan
    d_out[positions[0] < 0] = math.nan
    pairs = sum(axis_pairs)
    inv_freq = (10000.0 ** (-torch.arange(pairs, device=dev, dtype=torch.float64) / max(1, pairs))).float()
    want, tol = ref.rotary(qkv, gain_q, gain_k, positions, inv_freq, axis_pairs, neighbours, h, a, akv, 1e-6, d_out)
    layout = po.PO_ROTARY_NEIGHBOURS if neighbours else po.PO_ROTARY_HALVES
    held = positions[0] >= 0
    out = qkv.clone() if in_place else torch.full_like(qkv, MARK)
    po.po_op_qk_norm_rotary_forward(code, out if in_place else qkv, gain_q, gain_k, positions, inv_freq, axis_pairs, layout, out, rows, h, a,
                                    akv)
    size = po.po_op_qk_norm_rotary_backward_workspace(rows, h, a, akv)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device=dev)
    dqkv = d_out.clone() if in_place else torch.full_like(qkv, MARK)
    start = torch.randn(2, dh, generator=g, device=dev)
    dg = start.clone() if norm else (None, None)
    po.po_op_qk_norm_rotary_backward(code, dqkv if in_place else d_out, qkv if norm else None, gain_q, gain_k, positions, inv_freq, axis_pairs,
                                     layout, dqkv, dg[0], dg[1], ws if norm else None, rows, h, a, akv)
    for t in (out, dqkv):
        assert bool((t[~held].isnan() if in_place else t[~held] == MARK).all())
    _within(out[held], want["out"][held], tol["out"][held], "out")
    _within(dqkv[held], want["dqkv"][held], tol["dqkv"][held], "dqkv")
    if norm:
        assert bool((ws[size:] == 255).all())
        for i, k in enumerate(("dgain_q", "dgain_k")):
            _within(dg[i], start[i].double() + want[k], tol[k] + 2 * ref.E * (start[i].double().abs() + want[k].abs()), k)


ROTARY = [(64, 4, 4, 1, [32], False, True), (64, 4, 2, 7, [32], True, True), (128, 16, 8, 100, [64], False, True), (128, 3, 1, 33, [16, 24, 24], False, True),
          (128, 40, 8, 50, [10, 27, 27], True, True), (96, 6, 3, 40, [48], False, True), (96, 2, 1, 29, [9, 7, 8], True, False), (256, 4, 2, 21, [128], False, True),
          (256, 3, 3, 21, [30, 30, 30, 38], True, True), (32, 7, 7, 19, [16], False, True), (16, 5, 1, 11, [8], True, True), (48, 5, 5, 13, [16], False, True),
          (80, 2, 2, 12, [8, 16], False, True), (64, 40, 8, 65, [16], True, False), (64, 12, 4, 4200, [32], False, True), (128, 2, 2, 9, [0], False, True),
          (64, 1, 1, 9, [0, 8, 0, 24], False, False), (112, 2, 1, 9, [56], True, True), (240, 1, 1, 6, [40], False, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dh,a,akv,rows,axis_pairs,neighbours,norm", ROTARY, ids=lambda v: "-".join(map(str, v)) if isinstance(v, list) else str(v))
def test_norm_and_rotation(gpu_device, dtype, in_place, dh, a, akv, rows, axis_pairs, neighbours, norm):
    _rotary_case(gpu_device, dtype, dh, a, akv, rows, axis_pairs, neighbours, norm, 2 ** 20, in_place)


# one, two or four waves to a row, by rows and heads, with shares of them that have no heads
@pytest.mark.parametrize("rows", [511, 513, 1023, 1025, 4101])
@pytest.mark.parametrize("dtype,dh,a,akv,norm", [("bf16", 128, 40, 8, True), ("f32", 128, 9, 9, True), ("bf16", 64, 24, 8, False), ("bf16", 256, 10, 1, True),
                                                 ("f32", 32, 33, 1, True)])
def test_norm_and_rotation_of_shared_rows(gpu_device, dtype, dh, a, akv, norm, rows):
    _rotary_case(gpu_device, dtype, dh, a, akv, rows, [8, dh // 4], False, norm, 2 ** 20, True)


@pytest.mark.parametrize("far", [0, 1, 2 ** 31 - 1])
def test_rotation_of_the_first_and_the_last_positions(gpu_device, far):
    _rotary_case(gpu_device, "f32", 128, 2, 1, 40, [40, 24], False, True, far, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_and_rotation_gradient_is_that_of_differences(gpu_device, dtype):
    code, tdt = DT[dtype]
    dh, a, akv, rows = 64, 4, 2, 23
    h, hkv, g = a * dh, akv * dh, _gen(gpu_device, 3)
    rand = lambda *s: torch.randn(*s, generator=g, device=gpu_device).to(tdt)
    qkv, w, gq, gk = rand(rows, h + 2 * hkv), rand(rows, h + 2 * hkv), 1 + 0.2 * rand(dh), 1 + 0.2 * rand(dh)
    positions = torch.randint(0, 5000, (2, rows), generator=g, device=gpu_device, dtype=torch.int32)
    inv_freq = (10000.0 ** (-torch.arange(32, device=gpu_device) / 32)).float()
    dqkv, dg = torch.empty_like(qkv), torch.zeros(2, dh, device=gpu_device)
    ws = torch.empty(po.po_op_qk_norm_rotary_backward_workspace(rows, h, a, akv), dtype=torch.uint8, device=gpu_device)
    po.po_op_qk_norm_rotary_backward(code, w, qkv, gq, gk, positions, inv_freq, [8, 24], 0, dqkv, dg[0], dg[1], ws, rows, h, a, akv, 1e-6)
    args = (positions, inv_freq, [8, 24], False, h, a, akv, 1e-6)
    _, tol = ref.rotary(qkv, gq, gk, *args, w)
    loss = lambda x, p, r: float((ref.rotary(x, p, r, *args)[0]["out"] * w.double()).sum())
    x, p, r = qkv.double(), gq.double(), gk.double()
    vx, vp, vr = (torch.randn(t.shape, generator=g, device=gpu_device, dtype=torch.float64) for t in (x, p, r))
    for v, got, t in ((( vx, 0, 0), dqkv, tol["dqkv"]), ((0, vp, 0), dg[0], tol["dgain_q"]), ((0, 0, vr), dg[1], tol["dgain_k"])):
        step, moved = 1e-5, lambda s: (x + s * v[0], p + s * v[1], r + s * v[2])
        slope = (loss(*moved(step)) - loss(*moved(-step))) / (2 * step)
        d = next(t for t in v if torch.is_tensor(t))
        # differences in 64 bits, as above
        assert abs(float((got.double() * d).sum()) - slope) <= float((t * d.abs()).sum()) + 1e-6 * (abs(slope) + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("size,eps", [(1e15, 1e-6), (1e-15, 0.0), (0.0, 1e-30)])
def test_norm_gradient_where_r_cubed_is_out_of_range(gpu_device, dtype, dh, size, eps):
    """Heads so large or small that r^3 is no fp32 number, while x, r and the gradient are: within the bounds of any other head."""
    code, tdt = DT[dtype]
    a, akv, rows, g = 4, 2, 37, _gen(gpu_device, 4)
    h, hkv = a * dh, akv * dh
    rand = lambda *s: torch.randn(*s, generator=g, device=gpu_device)
    qkv, d_out = (size * rand(rows, h + 2 * hkv)).to(tdt), rand(rows, h + 2 * hkv).to(tdt)
    gq, gk = (1 + 0.2 * rand(dh)).to(tdt), (1 + 0.2 * rand(dh)).to(tdt)
    positions = torch.arange(rows, device=gpu_device, dtype=torch.int32)
    inv_freq = (10000.0 ** (-torch.arange(dh // 2, device=gpu_device) / (dh // 2))).float()
    rot = (gq, gk, positions, inv_freq, [dh // 2], 0)
    out, dqkv, dg = torch.empty_like(qkv), torch.empty_like(qkv), torch.zeros(2, dh, device=gpu_device)
    ws = torch.empty(po.po_op_qk_norm_rotary_backward_workspace(rows, h, a, akv), dtype=torch.uint8, device=gpu_device)
    po.po_op_qk_norm_rotary_forward(code, qkv, *rot, out, rows, h, a, akv, eps)
    po.po_op_qk_norm_rotary_backward(code, d_out, qkv, *rot, dqkv, dg[0], dg[1], ws, rows, h, a, akv, eps)
    want, tol = ref.rotary(qkv, gq, gk, positions[None], inv_freq, [dh // 2], False, h, a, akv, eps, d_out)
    for got, k in ((out, "out"), (dqkv, "dqkv"), (dg[0], "dgain_q"), (dg[1], "dgain_k")):
        _within(got, want[k], tol[k], k)


def test_a_gain_that_queries_and_keys_share(gpu_device):
    dh, a, akv, rows = 128, 8, 4, 300
    h, hkv, g = a * dh, akv * dh, _gen(gpu_device, 7)
    qkv, d_out = (torch.randn(rows, h + 2 * hkv, generator=g, device=gpu_device).bfloat16() for _ in range(2))
    gain, start = torch.rand(dh, generator=g, device=gpu_device).bfloat16(), torch.randn(dh, generator=g, device=gpu_device)
    positions = torch.arange(rows, device=gpu_device, dtype=torch.int32)
    inv_freq = torch.rand(64, generator=g, device=gpu_device)
    ws = torch.empty(po.po_op_qk_norm_rotary_backward_workspace(rows, h, a, akv), dtype=torch.uint8, device=gpu_device)
    dqkv, of_both = torch.empty_like(qkv), start.clone()
    po.po_op_qk_norm_rotary_backward(po.PO_BF16, d_out, qkv, gain, gain, positions, inv_freq, [64], 0, dqkv, of_both, of_both, ws, rows, h, a, akv)
    want, tol = ref.rotary(qkv, gain, gain, positions[None], inv_freq, [64], False, h, a, akv, 1e-6, d_out)
    both = want["dgain_q"] + want["dgain_k"]  # one sum of both, and the addition to what was there
    _within(of_both, start.double() + both, tol["dgain_q"] + tol["dgain_k"] + 2 * ref.E * (start.double().abs() + 2 * both.abs()), "dgain")


def test_rotation_keeps_what_is_not_rotated(gpu_device):
    """Elements behind the pairs pass bit for bit, infinities among them."""
    dh, rows = 128, 5
    x = torch.randn(rows, 3 * dh, device=gpu_device).bfloat16()
    x[2, 40] = math.inf
    x[3, 127] = -math.inf
    positions = torch.arange(rows, device=gpu_device, dtype=torch.int32)
    for layout in (0, 1):
        out = torch.zeros_like(x)
        po.po_op_qk_norm_rotary_forward(po.PO_BF16, x, None, None, positions, torch.ones(16, device=gpu_device), [16], layout, out, rows, dh, 1)
        q, got = x[:, :dh], out[:, :dh]
        assert torch.equal(got[:, 32:], q[:, 32:]) and torch.equal(out[:, 2 * dh:], x[:, 2 * dh:])


# ---- together -----------------------------------------------------------------------------------------------------
class _Layer:
    """Lengths to gradients: maps, norm and rotation, attention, and back, all in buffers made beforehand."""

    def __init__(self, dev, dtype, rows, dh, a, akv, lengths, seed=0):
        self.code, self.tdt = DT[dtype]
        self.rows, self.dh, self.a, self.akv, self.h, self.hkv = rows, dh, a, akv, a * dh, akv * dh
        g = _gen(dev, seed)
        rand = lambda *s: torch.randn(*s, generator=g, device=dev).to(self.tdt)
        new = lambda *s, t=self.tdt: torch.full(s, MARK, dtype=t, device=dev)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=dev)
        self.plan = torch.empty(po.po_op_packed_plan_bytes(rows) // 4, dtype=torch.int32, device=dev)
        self.positions = torch.empty(rows, dtype=torch.int32, device=dev)
        self.qkv, self.d_o, self.gains = rand(rows, self.h + 2 * self.hkv), rand(rows, self.h), 1 + 0.1 * rand(2, dh)
        self.inv_freq = (10000.0 ** (-torch.arange(dh // 2, device=dev) / (dh // 2))).float()
        self.turned, self.o, self.lse = new(*self.qkv.shape), new(rows, self.h), new(a, rows, t=torch.float32)
        self.d, self.dgains = new(*self.qkv.shape), torch.zeros(2, dh, device=dev)
        size = max(po.po_op_attention_packed_backward_workspace(self.code, rows, self.h, a, akv),
                   po.po_op_qk_norm_rotary_backward_workspace(rows, self.h, a, akv))
        self.ws = torch.empty(size, dtype=torch.uint8, device=dev)

    def run(self):
        shape = (self.rows, self.h, self.a, self.akv)
        po.po_op_packed_plan(self.lengths, self.lengths.numel(), self.rows, None, self.positions, None, self.plan)
        rot = (self.gains[0], self.gains[1], self.positions, self.inv_freq, [self.dh // 2], po.PO_ROTARY_HALVES)
        po.po_op_qk_norm_rotary_forward(self.code, self.qkv, *rot, self.turned, *shape)
        po.po_op_attention_packed_forward(self.code, self.turned, self.plan, self.o, self.lse, *shape)
        po.po_op_attention_packed_backward(self.code, self.turned, self.plan, self.o, self.lse, self.d_o, self.d, self.ws, *shape)
        self.dgains.zero_()
        po.po_op_qk_norm_rotary_backward(self.code, self.d, self.qkv, *rot, self.d, self.dgains[0], self.dgains[1], self.ws, *shape)

    def results(self):
        return [t.clone() for t in (self.positions, self.turned, self.o, self.lse, self.d, self.dgains)]

    def clear(self):
        for t in (self.turned, self.o, self.lse, self.d):
            t.fill_(MARK)

    def check(self):
        lengths = self.lengths.tolist()
        positions = torch.tensor([ref.maps(lengths, self.rows)[2]], dtype=torch.int32, device=self.qkv.device)
        assert torch.equal(self.positions, positions[0])
        rot = (self.gains[0], self.gains[1], positions, self.inv_freq, [self.dh // 2], False, self.h, self.a, self.akv, 1e-6)
        want, tol = ref.rotary(self.qkv, *rot)
        _within(self.turned, want["out"], tol["out"], "turned")
        # each step from what the one before it left
        want, tol = ref.attention(self.turned, self.d_o, lengths, self.h, self.a, self.akv)
        _within(self.o, want["o"], tol["o"], "o")
        _within(self.lse, want["lse"], tol["lse"], "lse")
        d, t = want["dqkv"], tol["dqkv"]
        held = positions[0] >= 0
        back, _ = ref.rotary(self.qkv, *rot, d_out=d.nan_to_num(0.0))
        # the gradient of the gradient's error: every element through the rotation and the norm's projection, at most gain and r times the
        # sum of three heads' worth of it (the mean of w xn over a head times xn, |xn| at most the root of the head size)
        x = self.qkv.double()[held][:, :self.h + self.hkv].reshape(-1, self.a + self.akv, self.dh)
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        gain = torch.cat([self.gains[0].double().expand(self.a, self.dh), self.gains[1].double().expand(self.akv, self.dh)]).abs()
        moved = t[held][:, :self.h + self.hkv].reshape(x.shape)
        worst = moved.amax(-1, keepdim=True) * 2 * gain.max()
        through = r * worst * (1 + (x * r).abs().amax(-1, keepdim=True) * (x * r).abs().mean(-1, keepdim=True))
        u = ref.half_step(self.tdt)
        bound = torch.cat([through.expand_as(x).flatten(1), t[held][:, self.h + self.hkv:]], 1) + 4 * u * back["dqkv"][held].abs() + 1e-5
        _within(self.d[held], back["dqkv"][held], bound, "d")
        assert bool((self.d[~held] == MARK).all())
        n = (x * r).abs()
        for i, (k, heads) in enumerate((("dgain_q", slice(0, self.a)), ("dgain_k", slice(self.a, None)))):
            off = (2 * moved.amax(-1, keepdim=True) * n)[:, heads].sum((0, 1)) + 1e-4
            _within(self.dgains[i], back[k], off, k)


@pytest.mark.parametrize("dtype,rows,dh,a,akv,lengths", [("f32", 300, 64, 4, 2, [100, 1, 0, 150, 40]), ("bf16", 300, 128, 4, 1, [100, 1, 0, 150, 40]),
                                                         ("bf16", 2048, 128, 16, 16, [900, 30, 1100])])
def test_a_layers_operators_together(gpu_device, dtype, rows, dh, a, akv, lengths):
    layer = _Layer(gpu_device, dtype, rows, dh, a, akv, lengths)
    layer.run()
    layer.check()


@pytest.mark.parametrize("dtype,rows,dh,a,akv", [("f32", 400, 64, 4, 2), ("bf16", 400, 64, 4, 2), ("bf16", 2048, 128, 16, 8)])
def test_captured_and_replayed_with_other_lengths(gpu_device, dtype, rows, dh, a, akv):
    """A graph of the whole run, replayed over new inputs and lengths, with eager runs of another batch between the replays."""
    layer, other = (_Layer(gpu_device, dtype, rows, dh, a, akv, [rows // 4] * 3, seed) for seed in (1, 2))
    layer.run()
    other.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run()
    for k, lengths in enumerate(([rows, 0, 0], [1, rows // 2, 7], [0, 0, 0], [rows // 3] * 3)):
        layer.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        layer.qkv.normal_(generator=_gen(gpu_device, 20 + k))
        layer.clear()
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        replayed = layer.results()
        layer.clear()
        layer.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(replayed, layer.results()))


def test_on_two_streams_at_once(gpu_device):
    """Two batches on streams of their own, again and again beside each other, give what they give alone."""
    layers = [_Layer(gpu_device, "bf16", 700, 128, 8, 2, lengths, seed) for lengths, seed in (([300, 20, 300], 3), ([1, 650], 4))]
    alone = []
    for layer in layers:
        layer.run()
        torch.cuda.synchronize()
        alone.append(layer.results())
        layer.clear()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for layer, stream in zip(layers, streams):
            with torch.cuda.stream(stream):
                layer.run()
    torch.cuda.synchronize()
    for layer, want in zip(layers, alone):
        assert all(torch.equal(x, y) for x, y in zip(layer.results(), want))


def test_calls_without_a_stream_go_to_the_current_one(gpu_device):
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            assert po._stream(None) == torch.cuda.current_stream().cuda_stream == stream.cuda_stream


@pytest.mark.parametrize("rows,largest", [(512, 513), (1000, 1025), (1024, 1400)])
def test_a_workspace_kept_from_a_larger_batch(gpu_device, rows, largest):
    """Both backward calls in fp32, in a workspace of the size that a larger batch asks for, with nothing written behind it: as in one of their own."""
    dh, a, akv = 128, 16, 4
    layer = _Layer(gpu_device, "f32", rows, dh, a, akv, [rows // 2, rows // 3])
    layer.run()
    torch.cuda.synchronize()
    want = layer.results()
    layer.clear()
    size = max(po.po_op_attention_packed_backward_workspace(layer.code, largest, a * dh, a, akv),
               po.po_op_qk_norm_rotary_backward_workspace(largest, a * dh, a, akv))
    layer.ws = torch.full((size + (1 << 16),), 255, dtype=torch.uint8, device=gpu_device)
    layer.run()
    torch.cuda.synchronize()
    assert bool((layer.ws[size:] == 255).all())
    assert all(torch.equal(x, y) for x, y in zip(layer.results(), want))


@pytest.mark.parametrize("rows,largest", [(512, 513), (1024, 1025), (300, 2048)])
def test_a_rotation_workspace_kept_from_a_larger_batch(gpu_device, rows, largest):
    dh, a, akv = 128, 40, 8
    h, hkv, g = a * dh, akv * dh, _gen(gpu_device, 31)
    qkv, d_out = (torch.randn(rows, h + 2 * hkv, generator=g, device=gpu_device).bfloat16() for _ in range(2))
    gains = 1 + 0.1 * torch.randn(2, dh, generator=g, device=gpu_device).bfloat16()
    positions = torch.arange(rows, device=gpu_device, dtype=torch.int32)
    inv_freq = torch.rand(64, generator=g, device=gpu_device)
    results = []
    for asked in (rows, largest):
        size = po.po_op_qk_norm_rotary_backward_workspace(asked, h, a, akv)
        ws = torch.full((size + (1 << 20),), 255, dtype=torch.uint8, device=gpu_device)
        dqkv, dg = torch.empty_like(qkv), torch.zeros(2, dh, device=gpu_device)
        po.po_op_qk_norm_rotary_backward(po.PO_BF16, d_out, qkv, gains[0], gains[1], positions, inv_freq, [64], 0, dqkv, dg[0], dg[1], ws, rows, h, a, akv)
        assert bool((ws[size:] == 255).all())
        results.append((dqkv, dg))
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_inputs_are_left_alone(gpu_device):
    layer = _Layer(gpu_device, "bf16", 200, 64, 4, 2, [90, 100])
    kept = [t.clone() for t in (layer.lengths, layer.qkv, layer.d_o, layer.gains, layer.inv_freq)]
    layer.run()
    assert all(torch.equal(x, y) for x, y in zip(kept, (layer.lengths, layer.qkv, layer.d_o, layer.gains, layer.inv_freq)))
