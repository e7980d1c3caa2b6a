"""Packed sequences, host side: what the entry points refuse, without a GPU; the 64-bit reference against autograd."""
import ctypes
import math

import pytest
import torch

import packed_reference as ref
from paper_2503_01328_amd import binding as po

AT = ctypes.addressof((ctypes.c_char * 4096).from_buffer(bytearray(4096)))
AT += -AT % 16  # an aligned address that no launch is to see


def _refused(call, match, *args, **kw):
    with pytest.raises(po.PipeOffloadError, match=match) as e:
        call(*args, **kw)
    assert e.value.code == po.PO_E_INVAL


@pytest.mark.parametrize("rows,bytes_", [(0, 0), (-5, 0), (1, 4 * (16 + 256 + 4)), (128, 4 * (16 + 256 + 4)), (129, 4 * (16 + 512 + 8)),
                                         (2097152, 4 * (16 + 2 * 2097152 + 4 * 16384)), (2097153, 0)])
def test_plan_bytes(rows, bytes_):
    assert po.po_op_packed_plan_bytes(rows) == bytes_


@pytest.mark.parametrize("lengths,n,rows,plan", [(None, 1, 8, AT), (AT, 0, 8, AT), (AT, -1, 8, AT), (AT, 16385, 8, AT), (AT, 1, 0, AT), (AT, 1, 2097153, AT),
                                                 (AT, 1, 8, AT + 4)], ids=[str(i) for i in range(7)])
def test_plan_refuses(lengths, n, rows, plan):
    _refused(po.po_op_packed_plan, "packed_plan", lengths, n, rows, None, None, None, plan, stream=0)


OVERLAPS = [dict(starts=AT), dict(starts=AT - 16), dict(positions=AT + 8), dict(sequence=AT), dict(plan=AT), dict(starts=AT + 64, positions=AT + 72),
            dict(positions=AT + 64, sequence=AT + 64), dict(positions=AT + 64, plan=AT + 80), dict(starts=AT + 1024, plan=AT + 48)]
ASKEW = [dict(starts=AT + 66), dict(positions=AT + 65), dict(sequence=AT + 67), dict(lengths=AT + 2)]


@pytest.mark.parametrize("given", OVERLAPS + ASKEW, ids=[str(i) for i in range(13)])
def test_plan_refuses_arrays_that_overlap_or_lie_askew(given):
    """4 lengths at AT, 8 rows."""
    c = {**dict(lengths=AT, starts=None, positions=None, sequence=None, plan=None), **given}
    _refused(po.po_op_packed_plan, "none overlaps", c["lengths"], 4, 8, c["starts"], c["positions"], c["sequence"], c["plan"], stream=0)


GOOD = dict(qkv=AT, plan=AT, o=AT, lse=AT, d_o=AT, dqkv=AT, workspace=AT, rows=100, h=256, n_heads=4, n_kv_heads=2)
BAD_SHAPES = [dict(rows=0), dict(rows=-1), dict(rows=2097153), dict(h=0), dict(n_heads=0), dict(n_heads=-4), dict(n_heads=3), dict(n_kv_heads=3),
              dict(n_kv_heads=8), dict(h=128), dict(h=384), dict(h=1024), dict(h=2 ** 30, n_heads=2 ** 24, n_kv_heads=1),
              dict(rows=2097152, h=128 * 128, n_heads=128, n_kv_heads=128)]


def _forward(dtype, c):
    return po.po_op_attention_packed_forward, (dtype, c["qkv"], c["plan"], c["o"], c["lse"], c["rows"], c["h"], c["n_heads"], c["n_kv_heads"])


def _backward(dtype, c):
    return po.po_op_attention_packed_backward, (dtype, c["qkv"], c["plan"], c["o"], c["lse"], c["d_o"], c["dqkv"], c["workspace"], c["rows"], c["h"],
                                                c["n_heads"], c["n_kv_heads"])


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("bad", BAD_SHAPES, ids=str)
def test_attention_refuses_shapes(dtype, call, bad):
    f, args = call(dtype, {**GOOD, **bad})
    _refused(f, "attention_packed", *args, stream=0)


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
@pytest.mark.parametrize("call,names", [(_forward, ("qkv", "plan", "o", "lse")), (_backward, ("qkv", "plan", "o", "lse", "d_o", "dqkv", "workspace"))])
def test_attention_refuses_pointers(dtype, call, names):
    for name in names:
        for value in (None, AT + (2 if name == "lse" else 8)):
            f, args = call(dtype, {**GOOD, name: value})
            _refused(f, "attention_packed", *args, stream=0)


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
@pytest.mark.parametrize("other", ["qkv", "d_o"])
def test_attention_backward_refuses_its_inputs_as_output(dtype, other):
    f, args = _backward(dtype, {**GOOD, "qkv": AT, "d_o": AT + 256, "dqkv": AT if other == "qkv" else AT + 256})
    _refused(f, "another tensor", *args, stream=0)


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
def test_attention_forward_refuses_its_input_as_output(dtype):
    f, args = _forward(dtype, GOOD)
    _refused(f, "another tensor", *args, stream=0)


@pytest.mark.parametrize("call", [_forward, _backward])
def test_attention_refuses_types(call):
    f, args = call(2, GOOD)
    _refused(f, "unknown dtype", *args, stream=0)


def test_workspaces():
    for dtype in (po.PO_F32, po.PO_BF16):
        assert po.po_op_attention_packed_backward_workspace(dtype, 1000, 512, 8, 2) >= 4 * 8 * 1000
        for bad in ((dtype, 0, 512, 8, 2), (dtype, 1000, 0, 8, 2), (dtype, 1000, 512, 0, 2), (5, 1000, 512, 8, 2)):
            assert po.po_op_attention_packed_backward_workspace(*bad) == 0
    assert po.po_op_qk_norm_rotary_backward_workspace(1000, 512, 8, 2) >= 4 * 2 * 64
    for bad in ((0, 512, 8, 2), (1000, 0, 8, 2), (1000, 512, 0, 2)):
        assert po.po_op_qk_norm_rotary_backward_workspace(*bad) == 0


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
@pytest.mark.parametrize("dh,a,akv", [(64, 12, 4), (128, 40, 8), (64, 8, 1), (64, 3, 3), (128, 256, 128), (64, 400, 200)])
def test_attention_workspace_for_more_rows_serves_fewer(dtype, dh, a, akv):
    """A program keeps one workspace, of the size that its largest batch asks for."""
    sizes = [po.po_op_attention_packed_backward_workspace(dtype, rows, a * dh, a, akv) for rows in range(1, 5000)]
    assert all(x <= y for x, y in zip(sizes, sizes[1:]))
    assert po.po_op_attention_packed_backward_workspace(dtype, 2097152, a * dh, a, akv) >= sizes[-1]


ROT = dict(qkv=AT, gain_q=AT, gain_k=AT, positions=AT, inv_freq=AT, axis_pairs=[32], layout=0, out=AT, d_out=AT, dqkv=AT + 64, dgain_q=AT, dgain_k=AT,
           workspace=AT, rows=10, h=256, n_heads=4, n_kv_heads=2, eps=1e-6)
BAD_ROT = [dict(rows=0), dict(rows=2 ** 25 + 1), dict(h=0), dict(n_heads=0), dict(n_heads=3), dict(n_kv_heads=3), dict(h=4 * 24), dict(h=4 * 8), dict(h=4 * 272),
           dict(h=2 ** 30, n_heads=2 ** 22, n_kv_heads=2 ** 22), dict(axis_pairs=[]), dict(axis_pairs=[8] * 5), dict(axis_pairs=[36]), dict(axis_pairs=[40]),
           dict(axis_pairs=[12]), dict(axis_pairs=[40, -8]), dict(axis_pairs=[2 ** 31 - 1, 2 ** 31 - 1, 2]), dict(layout=2), dict(layout=-1), dict(eps=-1.0),
           dict(eps=math.nan), dict(eps=math.inf), dict(gain_q=None), dict(gain_k=None), dict(positions=None), dict(inv_freq=None), dict(gain_q=AT + 8),
           dict(gain_k=AT + 2), dict(positions=AT + 2), dict(inv_freq=AT + 1)]


def _rot_forward(dtype, c):
    return po.po_op_qk_norm_rotary_forward, [dtype] + [c[k] for k in ("qkv", "gain_q", "gain_k", "positions", "inv_freq", "axis_pairs", "layout", "out",
                                                                     "rows", "h", "n_heads", "n_kv_heads", "eps")]


def _rot_backward(dtype, c):
    return po.po_op_qk_norm_rotary_backward, [dtype] + [c[k] for k in ("d_out", "qkv", "gain_q", "gain_k", "positions", "inv_freq", "axis_pairs", "layout",
                                                                      "dqkv", "dgain_q", "dgain_k", "workspace", "rows", "h", "n_heads", "n_kv_heads", "eps")]


@pytest.mark.parametrize("dh,a,akv", [(128, 40, 8), (64, 8, 2), (64, 40, 8), (128, 16, 16), (32, 33, 1), (256, 10, 1), (16, 1, 1)])
def test_rotary_workspace_for_more_rows_serves_fewer(dh, a, akv):
    sizes = [po.po_op_qk_norm_rotary_backward_workspace(rows, a * dh, a, akv) for rows in range(1, 9000)]
    assert all(x <= y for x, y in zip(sizes, sizes[1:]))
    assert po.po_op_qk_norm_rotary_backward_workspace(2 ** 25, a * dh, a, akv) >= sizes[-1]


@pytest.mark.parametrize("dtype", [po.PO_F32, po.PO_BF16])
@pytest.mark.parametrize("call,more", [(_rot_forward, [dict(qkv=None), dict(out=None), dict(qkv=AT + 8), dict(out=AT + 4)]),
                                       (_rot_backward, [dict(d_out=None), dict(dqkv=None), dict(qkv=None), dict(dgain_q=None), dict(dgain_k=None),
                                                        dict(workspace=None), dict(dqkv=AT), dict(dgain_q=AT + 2), dict(workspace=AT + 2), dict(qkv=AT + 8)])])
def test_rotary_refuses(dtype, call, more):
    for bad in BAD_ROT + more:
        f, args = call(dtype, {**ROT, **bad})
        _refused(f, "qk_norm_rotary", *args, stream=0)


@pytest.mark.parametrize("call", [_rot_forward, _rot_backward])
def test_rotary_refuses_types(call):
    f, args = call(7, ROT)
    _refused(f, "unknown dtype", *args, stream=0)


# ---- the reference ------------------------------------------------------------------------------------------------
def test_reference_attention_is_autograds():
    a, akv, dh, lengths = 4, 2, 8, [5, 0, 1, 7]
    h, hkv, rows = a * dh, akv * dh, 15
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(rows, h + 2 * hkv, generator=g, dtype=torch.float64, requires_grad=True)
    d_o = torch.randn(rows, h, generator=g, dtype=torch.float64)
    want, _ = ref.attention(qkv.detach(), d_o, lengths, h, a, akv)
    outs, at = [], 0
    for n in lengths:
        x = qkv[at:at + n]
        at += n
        q, k, v = x[:, :h].reshape(n, a, dh), x[:, h:h + hkv].reshape(n, akv, dh), x[:, h + hkv:].reshape(n, akv, dh)
        for i in range(n):
            for t in range(a):
                s = k[:i + 1, t // 2] @ q[i, t] / math.sqrt(dh)
                outs.append(torch.softmax(s, 0) @ v[:i + 1, t // 2])
    o = torch.stack(outs).reshape(13, h)
    (o * d_o[:13]).sum().backward()
    assert torch.allclose(want["o"][:13], o.detach(), atol=1e-12) and want["o"][13:].isnan().all()
    assert torch.allclose(want["dqkv"][:13], qkv.grad[:13], atol=1e-12) and want["dqkv"][13:].isnan().all()


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_reference_rotary_is_autograds(neighbours, norm):
    a, akv, dh, rows, axis_pairs = 2, 1, 16, 6, [3, 5]
    h, hkv = a * dh, akv * dh
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True)
    qkv, gq, gk, d = rand(rows, h + 2 * hkv), rand(dh), rand(dh), rand(rows, h + 2 * hkv).detach()
    positions = torch.randint(0, 100, (2, rows), generator=g, dtype=torch.int32)
    inv_freq = torch.rand(8, generator=g)
    want, _ = ref.rotary(qkv.detach(), gq.detach() if norm else None, gk.detach() if norm else None, positions, inv_freq, axis_pairs, neighbours, h, a, akv,
                         1e-6, d)
    rows_out = []
    for r in range(rows):
        heads = []
        for t in range(a + akv):
            x = qkv[r, t * dh:(t + 1) * dh]
            if norm:
                x = x / (x.square().mean() + 1e-6).sqrt() * (gq if t < a else gk)
            y = list(x)
            for p in range(8):
                i, j = (2 * p, 2 * p + 1) if neighbours else (p, p + 8)
                angle = float(positions[0 if p < 3 else 1, r]) * float(inv_freq[p])
                y[i], y[j] = x[i] * math.cos(angle) - x[j] * math.sin(angle), x[i] * math.sin(angle) + x[j] * math.cos(angle)
            heads.append(torch.stack(y))
        rows_out.append(torch.cat(heads + [qkv[r, h + hkv:]]))
    out = torch.stack(rows_out)
    (out * d).sum().backward()
    assert torch.allclose(want["out"], out.detach(), atol=1e-12) and torch.allclose(want["dqkv"], qkv.grad, atol=1e-12)
    if norm:
        assert torch.allclose(want["dgain_q"], gq.grad, atol=1e-12) and torch.allclose(want["dgain_k"], gk.grad, atol=1e-12)


def test_kernels_keep_their_accumulators_in_registers():
    """The compiler's resource report: no kernel of packed sequences uses scratch memory."""
    import json
    import os

    from paper_2503_01328_amd import build as b

    if not os.path.exists(b.RESOURCES):
        b.build(verbose=False)
    usage = {k: v for k, v in json.load(open(b.RESOURCES)).items() if "packed_" in k or "rotary" in k}
    assert len(usage) >= 30
    for name, v in usage.items():
        assert v["ScratchSize"] == 0, (name, v)
