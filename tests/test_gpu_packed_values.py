"""Special values in packed attention, in every form of its kernels: what one element that is not finite leaves as it was inside its own
sequence, and keys whose scores are -inf.  Bounds: packed_reference.py."""
import math

import pytest
import torch

import packed_reference as ref
from test_gpu_packed import _attention, _inputs, _plan, _within

pytestmark = pytest.mark.gpu

# heads, and sequences of these lengths, for blocks of 32, 64 and 128 rows, forward and backward, and for fp32 with and without parts
FORMS = [("bf16", 64, 4, 2, [33, 150]), ("bf16", 128, 4, 2, [33, 150]), ("bf16", 64, 40, 40, [70, 400]), ("bf16", 128, 40, 8, [70, 400]),
         ("bf16", 64, 52, 52, [23, 700, 600]), ("bf16", 128, 40, 40, [23, 700, 600]), ("f32", 64, 4, 2, [33, 150, 200]), ("f32", 128, 3, 3, [33, 300])]


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("where", ["q", "v", "d_o"])
@pytest.mark.parametrize("at", [0.1, 0.9])
@pytest.mark.parametrize("dtype,dh,a,akv,lengths", FORMS, ids=str)
def test_what_a_row_that_is_not_finite_does_not_reach(gpu_device, dtype, dh, a, akv, lengths, where, value, at):
    """Column 3 of head 0 of one row.  In q: o, lse and dQ of that row and, through its probabilities, dK and dV of the keys that it sees; in d_o: its
    dQ, those keys' dK and column 3 of their dV; in v: column 3 of o and all of dQ from the row on, dK of the sequence.  All else is as without it."""
    h, hkv, rows, group = a * dh, akv * dh, sum(lengths), a // akv
    qkv, d_o = _inputs(gpu_device, dtype, rows, h, hkv, 21)
    want, tol = ref.attention(qkv, d_o, lengths, h, a, akv)
    lo, hi = rows - lengths[-1], rows
    row = lo + int(at * lengths[-1])
    {"q": qkv[:, :h], "v": qkv[:, h + hkv:], "d_o": d_o}[where][row, 3] = value
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, gpu_device), h, a, akv)
    keep = {k: torch.ones_like(v, dtype=torch.bool) for k, v in want.items()}
    dq, dk, dv = keep["dqkv"][:, :h], keep["dqkv"][:, h:h + hkv], keep["dqkv"][:, h + hkv:]
    if where == "q":
        keep["o"][row, :dh] = keep["lse"][0, row] = False
        dq[row, :dh] = dk[lo:row + 1, :dh] = dv[lo:row + 1, :dh] = False
    elif where == "d_o":
        dq[row, :dh] = dk[lo:row + 1, :dh] = dv[lo:row + 1, 3] = False
    else:
        for head in range(group):
            keep["o"][row:, head * dh + 3] = False
        dq[row:, :group * dh] = dk[lo:, :dh] = False
    for k in want:
        _within(torch.where(keep[k], got[k].double(), want[k]), want[k], tol[k], k)
    if where == "v":  # and there it is
        assert not got["o"][row:, 3].isfinite().any()


@pytest.mark.parametrize("first,last", [(0, 40), (64, 128), (5, 70), (0, 130), (31, 149)])
@pytest.mark.parametrize("dtype,dh,a,akv,lengths", FORMS, ids=str)
def test_keys_whose_scores_are_minus_infinity(gpu_device, dtype, dh, a, akv, lengths, first, last):
    """Keys first .. last - 1 of the last sequence have scores of -inf, in every head.  Rows that see another key have the o, lse and dQ (but for
    the element that multiplies the infinity itself) that they have without these keys, and they give these keys no gradient."""
    h, hkv, rows = a * dh, akv * dh, sum(lengths)
    qkv, d_o = _inputs(gpu_device, dtype, rows, h, hkv, 22)
    lo = rows - lengths[-1]
    qkv[:, 0:h:dh] = 1.0
    qkv[:, h:h + hkv:dh] = 0.0
    absent = torch.zeros(rows, dtype=torch.bool, device=gpu_device)
    absent[lo + first:lo + last] = True
    want, tol = ref.attention(qkv, d_o, lengths, h, a, akv, absent=absent)
    qkv[lo + first:lo + last, h:h + hkv:dh] = -math.inf
    got = _attention(dtype, qkv, d_o, _plan(lengths, rows, gpu_device), h, a, akv)
    keep = {k: torch.ones_like(v, dtype=torch.bool) for k, v in want.items()}
    if first == 0:  # rows that see nothing else, and the keys that they see
        keep["o"][lo:lo + last] = keep["lse"][:, lo:lo + last] = keep["dqkv"][lo:lo + last] = False
    for head in range(a):  # 0 times an infinity
        keep["dqkv"][lo + first:, head * dh] = False
    for k in want:
        _within(torch.where(keep[k], got[k].double(), want[k]), want[k], tol[k], k)
    if first > 0:
        assert not got["dqkv"][lo + first:lo + last, h:].any()
