"""The operators of training on packed sequences, measured: several sequences back to back in one [rows, ...] tensor, none
of which sees another, and behind the last one rows that hold nothing and are left as they were.

Three kinds of case.
  plan       the maps of a packed batch built on the GPU from its lengths: where each sequence starts, each row's sequence
             and its position there (po_op_packed_plan)
  rotary     queries and keys normed head by head (root mean square) and rotated by their positions of one to three axes, in
             one pass over q | k | v; a training pass takes the gradients of input and gains too (po_op_qk_norm_rotary_*)
  attention  the maps, and causal grouped-query attention within each sequence, forward or forward and backward
             (po_op_attention_packed_*)

With `own` false everything is computed from elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"


# ---- cases --------------------------------------------------------------------------------------------------------
def _rotary(name=None, **kw):
    case = dict(kind="rotary", rows=0, used=0, sequences=1, spread=0, heads=1, kv_heads=1, head_size=64, pairs=32, axes=1,
                far=0, neighbours=False, norm=True, dtype="bf16", training=True)
    case.update(kw)
    return case if name is None else dict(name=name, **case)


def _attention(name=None, **kw):
    case = dict(kind="attention", rows=0, used=0, sequences=1, spread=0, heads=1, kv_heads=1, head_size=64, dtype="bf16",
                training=True)
    case.update(kw)
    return case if name is None else dict(name=name, **case)


def listed():
    return [
        # A microbatch of 2048 rows, packed from a few documents.
        dict(name="plan_small", kind="plan", rows=2048, used=2048, sequences=8, spread=1),
        # A large microbatch of chat turns: thousands of short sequences, some of them empty, and a padded end.
        dict(name="plan_many", kind="plan", rows=131072, used=131001, sequences=4000, spread=2),
        # The debugging configuration's width in fp32: a handful of rows, where only latency counts.
        _rotary("rotary_few_f32", rows=128, used=120, sequences=3, spread=3, heads=4, kv_heads=4, head_size=64, dtype="f32"),
        # A 2048-wide model's forward pass of one microbatch.
        _rotary("rotary_forward", rows=2048, used=2048, sequences=6, spread=4, heads=16, kv_heads=16, head_size=128, pairs=64,
                training=False),
        # Images and video among text: positions of time, height and width, a 5120-wide model's long microbatch, with gradients.
        _rotary("rotary_three_axes", rows=16384, used=16384, sequences=9, spread=5, heads=40, kv_heads=8, head_size=128, pairs=64,
                axes=3),
        # Rotation alone of half of each head, neighbouring elements as pairs, far into a long document; odd rows, a padded end.
        _rotary("rotary_far_half", rows=5001, used=4890, sequences=2, spread=6, heads=40, kv_heads=8, head_size=64, pairs=16,
                far=900000, neighbours=True, norm=False),
        # A few short samples, the size at which a model is brought up.
        _attention("attention_few", rows=128, used=100, sequences=5, spread=7, heads=8, kv_heads=8, head_size=64),
        # Numerical debugging in fp32.
        _attention("attention_f32", rows=1000, used=977, sequences=4, spread=8, heads=12, kv_heads=4, head_size=64, dtype="f32"),
        # A 2048-wide model's microbatch of documents.
        _attention("attention_documents", rows=2048, used=2048, sequences=6, spread=9, heads=16, kv_heads=16, head_size=128),
        # A 4096-wide model with grouped heads, documents of all lengths and a padded end.
        _attention("attention_grouped", rows=4096, used=4001, sequences=21, spread=10, heads=32, kv_heads=8, head_size=128),
        # Many short samples in one long microbatch: instruction tuning.
        _attention("attention_many_short", rows=8192, used=8192, sequences=170, spread=11, heads=40, kv_heads=8, head_size=64),
        # Evaluation of a 5120-wide model on long documents, forward alone.
        _attention("attention_long", rows=16384, used=16384, sequences=3, spread=12, heads=40, kv_heads=40, head_size=128,
                   training=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["plan", "rotary", "attention"], [1, 3, 5])[0]
    spread = rng.randrange(1 << 20)
    if kind == "plan":
        rows = _log_int(rng, 100, 131072)
        return dict(kind="plan", rows=rows, used=rows - rng.choice([0, rng.randrange(rows // 4)]),
                    sequences=_log_int(rng, 1, min(4000, rows)), spread=spread)
    group = rng.choice([1, 1, 2, 4, 8])
    dtype = rng.choices(["bf16", "f32"], [4, 1])[0]
    if kind == "rotary":
        head_size = rng.choice([64, 96, 128])
        kv_heads = _log_int(rng, 1, 40 // group)
        heads = kv_heads * group
        rows = _log_int(rng, 50, min(16384, 16384 * 48 * 128 * 2 // ((heads + 2 * kv_heads) * head_size * (2 if dtype == "bf16" else 4))))
        return _rotary(rows=rows, used=rows - rng.choice([0, rng.randrange(rows // 4)]), sequences=_log_int(rng, 1, min(100, rows)),
                       spread=spread, heads=heads, kv_heads=kv_heads, head_size=head_size,
                       pairs=rng.choice([head_size // 2, head_size // 2, head_size // 4]), axes=rng.choice([1, 1, 2, 3]),
                       far=rng.choice([0, 0, 100000, 900000]), neighbours=rng.random() < 0.4, norm=rng.random() < 0.7, dtype=dtype,
                       training=rng.random() < 0.7)
    head_size = rng.choice([64, 128])
    training = rng.random() < 0.7
    kv_heads = _log_int(rng, 1, 40 // group)
    heads = kv_heads * group
    # the plain form's scores, and the fp32 matrix rate, bound what is drawn: no more than the largest listed case
    most = math.sqrt(40 * 16384.0 ** 2 / heads / (8 if training else 1) / (4 if dtype == "f32" else 1))
    rows = _log_int(rng, 50, int(min(16384, most)))
    return _attention(rows=rows, used=rows - rng.choice([0, rng.randrange(rows // 4)]), sequences=_log_int(rng, 1, min(200, rows)),
                      spread=spread, heads=heads, kv_heads=kv_heads, head_size=head_size, dtype=dtype, training=training)


def _lengths(case):
    """The case's sequence lengths: `sequences` of them, spread over about a factor of twenty, some empty where there are many;
    they add up to `used`."""
    rng, n, used = random.Random(case["spread"]), case["sequences"], case["used"]
    weights = [0.0 if n > 100 and rng.random() < 0.02 else math.exp(rng.uniform(0, 3)) for _ in range(n)]
    weights[0] = max(weights[0], 1.0)
    total, at, done, out = sum(weights), 0.0, 0, []
    for w in weights:
        at += w
        end = min(used, int(round(used * at / total)))
        out.append(end - done)
        done = end
    out[-1] += used - done
    return out


# ---- inputs -------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _widths(case):
    return case["heads"] * case["head_size"], case["kv_heads"] * case["head_size"]


def _axis_pairs(case):
    """How many of the pairs turn by each axis: with three, a quarter by time and the rest by height and width."""
    pairs, axes = case["pairs"], case["axes"]
    if axes == 3:
        return [pairs - 2 * (3 * pairs // 8)] + [3 * pairs // 8] * 2
    return [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    lengths = _lengths(case)
    random.Random(seed).shuffle(lengths)  # the same work in another order
    state = dict(case=case, lengths=torch.tensor(lengths, dtype=torch.int32, device=DEVICE))
    rows = case["rows"]
    if case["kind"] == "plan":
        state["starts"] = torch.zeros(case["sequences"] + 1, dtype=torch.int32, device=DEVICE)
        state["positions"] = torch.zeros(rows, dtype=torch.int32, device=DEVICE)
        state["sequence"] = torch.zeros(rows, dtype=torch.int32, device=DEVICE)
        return state
    dt, (h, hkv), dh = _dtype(case), _widths(case), case["head_size"]
    rand = lambda *size: torch.randn(*size, generator=g, device=DEVICE).to(dt)
    zeros = lambda *size, t=dt: torch.zeros(*size, dtype=t, device=DEVICE)
    state["qkv"] = rand(rows, h + 2 * hkv)
    if case["kind"] == "attention":
        state.update(o=zeros(rows, h), lse=zeros(case["heads"], rows, t=torch.float32))
        if case["training"]:
            state.update(d_o=rand(rows, h), dqkv=zeros(rows, h + 2 * hkv))
        return state
    # rotary: each row's position in its sequence, from `far` on; further axes walk an image 24 rows of 24 wide.  Rows behind the
    # last sequence have the position -1.
    at = torch.cat([torch.arange(n) for n in lengths]).to(torch.int32)
    positions = torch.full((case["axes"], rows), -1, dtype=torch.int32)
    positions[0, :case["used"]] = at + case["far"]
    for axis in range(1, case["axes"]):
        positions[axis, :case["used"]] = at // 24 % 24 if axis == 1 else at % 24
    pairs = case["pairs"]
    state.update(positions=positions.to(DEVICE), axis_pairs=_axis_pairs(case),
                 axis=torch.tensor([i for i, n in enumerate(_axis_pairs(case)) for _ in range(n)], device=DEVICE),
                 inv_freq=(10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).to(torch.float32).to(DEVICE),
                 gain_q=(1 + 0.1 * rand(dh)).to(dt) if case["norm"] else None,
                 gain_k=(1 + 0.1 * rand(dh)).to(dt) if case["norm"] else None, out=zeros(rows, h + 2 * hkv))
    if case["training"]:
        state.update(d_out=rand(rows, h + 2 * hkv), dqkv=zeros(rows, h + 2 * hkv),
                     dgains=zeros(2, dh, t=torch.float32) if case["norm"] else None)
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    return {"plan": _plan, "rotary": _qk_norm_rotary, "attention": _attention_packed}[state["case"]["kind"]](state)


def _maps(lengths, rows):
    """starts [n + 1], and per row its sequence (-1 behind the last one) and its position there (-1)."""
    ends = torch.cumsum(lengths, 0, dtype=torch.int32)
    starts = torch.cat([torch.zeros_like(ends[:1]), ends])
    row = torch.arange(rows, device=lengths.device, dtype=torch.int32)
    sequence = torch.searchsorted(ends, row, right=True).to(torch.int32)
    held = row < ends[-1]
    positions = torch.where(held, row - starts[sequence.long().clamp_(max=lengths.numel() - 1)], -1)
    return starts, torch.where(held, sequence, -1), positions


def _own_plan(state):
    """The maps and the plan that the attention calls read, in a buffer that the state keeps."""
    from paper_2503_01328_amd import binding as po

    rows = state["case"]["rows"]
    if "plan" not in state:
        state["plan"] = torch.empty(po.po_op_packed_plan_bytes(rows) // 4, dtype=torch.int32, device=DEVICE)
    po.po_op_packed_plan(state["lengths"], state["lengths"].numel(), rows, state.get("starts"), state.get("positions"),
                         state.get("sequence"), state["plan"])
    return state["plan"]


def _plan(state):
    if own:
        _own_plan(state)
        return {"starts": state["starts"], "sequence": state["sequence"], "positions": state["positions"]}
    starts, sequence, positions = _maps(state["lengths"], state["case"]["rows"])
    return {"starts": starts, "sequence": sequence, "positions": positions}


def _workspace(state, size):
    """Scratch memory that a program keeps from pass to pass."""
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=DEVICE)
    return state["workspace"]


def _own_qk_norm_rotary(state):
    from paper_2503_01328_amd import binding as po

    case, (h, _) = state["case"], _widths(state["case"])
    code = po.PO_BF16 if case["dtype"] == "bf16" else po.PO_F32
    layout = po.PO_ROTARY_NEIGHBOURS if case["neighbours"] else po.PO_ROTARY_HALVES
    shape = dict(rows=case["rows"], h=h, n_heads=case["heads"], n_kv_heads=case["kv_heads"], eps=1e-6)
    po.po_op_qk_norm_rotary_forward(code, state["qkv"], state["gain_q"], state["gain_k"], state["positions"], state["inv_freq"],
                                    state["axis_pairs"], layout, state["out"], **shape)
    if not case["training"]:
        return {"out": state["out"]}
    dgains = state["dgains"]
    if case["norm"]:
        dgains.zero_()
    workspace = _workspace(state, po.po_op_qk_norm_rotary_backward_workspace(case["rows"], h, case["heads"], case["kv_heads"]))
    po.po_op_qk_norm_rotary_backward(code, state["d_out"], state["qkv"], state["gain_q"], state["gain_k"], state["positions"],
                                     state["inv_freq"], state["axis_pairs"], layout, state["dqkv"],
                                     dgains[0] if case["norm"] else None, dgains[1] if case["norm"] else None, workspace, **shape)
    return {"out": state["out"], "dqkv": state["dqkv"], "dgains": dgains}


def _turn(x, cos, sin, pairs, neighbours):
    """The first 2 pairs elements of every head of x [rows, heads, head size] turned by the angles [rows, 1, pairs]."""
    a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if neighbours else (x[..., :pairs], x[..., pairs:2 * pairs])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([y, z], -1).flatten(-2) if neighbours else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _qk_norm_rotary(state):
    if own:
        return _own_qk_norm_rotary(state)
    case, (h, hkv), dh, dt = state["case"], _widths(state["case"]), state["case"]["head_size"], _dtype(state["case"])
    pairs, used = case["pairs"], case["used"]
    angle = state["positions"][:, :used].to(torch.float64).T[:, state["axis"]] * state["inv_freq"].to(torch.float64)
    cos, sin = torch.cos(angle).to(torch.float32)[:, None], torch.sin(angle).to(torch.float32)[:, None]
    x = state["qkv"][:used].to(torch.float32)
    qk = x[:, :h + hkv].reshape(used, -1, dh)
    if case["norm"]:  # one gain for all query heads, one for all key heads
        gain = torch.cat([state["gain_q"].to(torch.float32).expand(case["heads"], dh), state["gain_k"].to(torch.float32).expand(case["kv_heads"], dh)])
        r = torch.rsqrt((qk * qk).mean(-1, keepdim=True) + 1e-6)
        normed = qk * r
        y = normed * gain
    else:
        y = qk
    out = torch.zeros_like(state["out"])
    out[:used] = torch.cat([_turn(y, cos, sin, pairs, case["neighbours"]).reshape(used, -1), x[:, h + hkv:]], 1).to(dt)
    if not case["training"]:
        return {"out": out}
    d = state["d_out"][:used].to(torch.float32)
    g = _turn(d[:, :h + hkv].reshape(used, -1, dh), cos, -sin, pairs, case["neighbours"])
    dgains = None
    if case["norm"]:
        t = g * normed
        dgains = torch.stack([t[:, :case["heads"]].sum((0, 1)), t[:, case["heads"]:].sum((0, 1))])
        g = g * gain
        g = r * (g - normed * (g * normed).mean(-1, keepdim=True))
    dqkv = torch.zeros_like(state["dqkv"])
    dqkv[:used] = torch.cat([g.reshape(used, -1), d[:, h + hkv:]], 1).to(dt)
    return {"out": out, "dqkv": dqkv, "dgains": dgains}


def _own_attention_packed(state):
    from paper_2503_01328_amd import binding as po

    case, (h, _) = state["case"], _widths(state["case"])
    code = po.PO_BF16 if case["dtype"] == "bf16" else po.PO_F32
    plan = _own_plan(state)
    po.po_op_attention_packed_forward(code, state["qkv"], plan, state["o"], state["lse"], case["rows"], h, case["heads"], case["kv_heads"])
    if not case["training"]:
        return {"o": state["o"], "lse": state["lse"]}
    workspace = _workspace(state, po.po_op_attention_packed_backward_workspace(code, case["rows"], h, case["heads"], case["kv_heads"]))
    po.po_op_attention_packed_backward(code, state["qkv"], plan, state["o"], state["lse"], state["d_o"], state["dqkv"], workspace,
                                       case["rows"], h, case["heads"], case["kv_heads"])
    return {"o": state["o"], "lse": state["lse"], "dqkv": state["dqkv"]}


def _attention_packed(state):
    if own:
        return _own_attention_packed(state)
    case, (h, hkv), dh, dt = state["case"], _widths(state["case"]), state["case"]["head_size"], _dtype(state["case"])
    rows, used, a, group = case["rows"], case["used"], case["heads"], case["heads"] // case["kv_heads"]
    starts, sequence, _ = _maps(state["lengths"], rows)
    first, row = starts[sequence[:used].long()], torch.arange(used, device=DEVICE)
    hidden = (row[None, :] > row[:, None]) | (row[None, :] < first[:, None])
    heads = lambda t, n: t[:used].to(torch.float32).reshape(used, n, dh).transpose(0, 1).contiguous()
    q = heads(state["qkv"][:, :h], a)
    k, v = (heads(t, case["kv_heads"]).repeat_interleave(group, 0) for t in state["qkv"][:, h:].split(hkv, 1))
    p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(dh)).masked_fill_(hidden, -math.inf)
    m = p.amax(-1, keepdim=True)
    total = p.sub_(m).exp_().sum(-1, keepdim=True)
    p.div_(total)
    o32 = torch.bmm(p, v)
    o, lse = torch.zeros_like(state["o"]), torch.zeros_like(state["lse"])
    o[:used] = o32.transpose(0, 1).reshape(used, h).to(dt)
    lse[:, :used] = (m + torch.log(total))[..., 0]
    if not case["training"]:
        return {"o": o, "lse": lse}
    d = heads(state["d_o"], a)
    shared = lambda t: t.reshape(-1, group, used, dh).sum(1)  # the heads of a group share a key/value head
    flat = lambda t: t.transpose(0, 1).reshape(used, -1)
    dv = shared(torch.bmm(p.transpose(1, 2).contiguous(), d))
    ds = torch.bmm(d, v.transpose(1, 2).contiguous()).sub_((d * o32).sum(-1, keepdim=True)).mul_(p).mul_(1 / math.sqrt(dh))
    dq, dk = torch.bmm(ds, k), shared(torch.bmm(ds.transpose(1, 2).contiguous(), q))
    dqkv = torch.zeros_like(state["dqkv"])
    dqkv[:used] = torch.cat([flat(dq), flat(dk), flat(dv)], 1).to(dt)
    return {"o": o, "lse": lse, "dqkv": dqkv}


# ---- the operators' definitions in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "plan":
        return None  # whole numbers
    state = prepare(case, seed)
    with torch.no_grad():
        return (_exact_rotary if case["kind"] == "rotary" else _exact_attention)(case, state)


def _exact_rotary(case, state):
    """The rotation as a product of complex numbers; the norm's gradients from its Jacobian, head by head."""
    (h, hkv), dh, pairs, used = _widths(case), case["head_size"], case["pairs"], case["used"]
    n = case["heads"] + case["kv_heads"]
    out = torch.zeros(case["rows"], h + 2 * hkv, dtype=torch.float64, device=DEVICE)
    out[:used, h + hkv:] = state["qkv"][:used, h + hkv:].double()
    grads = torch.zeros_like(out) if case["training"] else None
    dgains = torch.zeros(2, dh, dtype=torch.float64, device=DEVICE)
    first, angle = 0, torch.empty(used, pairs, dtype=torch.float64, device=DEVICE)
    for axis, count in enumerate(state["axis_pairs"]):
        angle[:, first:first + count] = torch.outer(state["positions"][axis, :used].double(), state["inv_freq"][first:first + count].double())
        first += count
    unit = torch.polar(torch.ones_like(angle), angle)
    index = torch.arange(2 * pairs, device=DEVICE)
    re, im = (index[0::2], index[1::2]) if case["neighbours"] else (index[:pairs], index[pairs:])

    def turned(x, by):
        z = torch.complex(x[:, re], x[:, im]) * by
        x = x.clone()
        x[:, re], x[:, im] = z.real, z.imag
        return x

    for i in range(n):
        cols, kind = slice(i * dh, (i + 1) * dh), int(i >= case["heads"])
        x = state["qkv"][:used, cols].double()
        norm = torch.sqrt(x.square().sum(1, keepdim=True) / dh + 1e-6)
        gain = state["gain_k" if kind else "gain_q"].double() if case["norm"] else None
        out[:used, cols] = turned(x / norm * gain if case["norm"] else x, unit)
        if case["training"]:
            g = turned(state["d_out"][:used, cols].double(), unit.conj())
            if case["norm"]:
                dgains[kind] += (g * x / norm).sum(0)
                g = g * gain
                g = g / norm - x * (g * x).sum(1, keepdim=True) / (dh * norm ** 3)
            grads[:used, cols] = g
    if not case["training"]:
        return {"out": out}
    grads[:used, h + hkv:] = state["d_out"][:used, h + hkv:].double()
    return {"out": out, "dqkv": grads, "dgains": dgains if case["norm"] else None}


def _exact_attention(case, state):
    """Sequence by sequence and head by head, the gradients through the softmax's Jacobian."""
    (h, hkv), dh, a = _widths(case), case["head_size"], case["heads"]
    o = torch.zeros(case["rows"], h, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(a, case["rows"], dtype=torch.float64, device=DEVICE)
    grads = torch.zeros(case["rows"], h + 2 * hkv, dtype=torch.float64, device=DEVICE) if case["training"] else None
    lengths, at = state["lengths"].tolist(), 0
    if len(lengths) * a > 20000:
        return None
    for n in lengths:
        rows, at = slice(at, at + n), at + n
        if n == 0:
            continue
        x = state["qkv"][rows].double()
        visible = torch.ones(n, n, dtype=torch.bool, device=DEVICE).tril()
        for i in range(a):
            kv = i * case["kv_heads"] // a
            qs, ks, vs = slice(i * dh, (i + 1) * dh), slice(h + kv * dh, h + (kv + 1) * dh), slice(h + hkv + kv * dh, h + hkv + (kv + 1) * dh)
            scores = torch.where(visible, x[:, qs] @ x[:, ks].T / dh ** 0.5, -math.inf)
            lse[i, rows] = torch.logsumexp(scores, 1)
            p = torch.exp(scores - lse[i, rows, None])
            o[rows, qs] = p @ x[:, vs]
            if case["training"]:
                d = state["d_o"][rows, qs].double()
                dp = d @ x[:, vs].T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / dh ** 0.5
                grads[rows, qs] = ds @ x[:, ks]
                grads[rows, ks] += ds.T @ x[:, qs]
                grads[rows, vs] += p.T @ d
    return {"o": o, "lse": lse, "dqkv": grads} if case["training"] else {"o": o, "lse": lse}


# ---- work ---------------------------------------------------------------------------------------------------------
def work(case):
    rows, used = case["rows"], case["used"]
    if case["kind"] == "plan":
        return {"bytes": 4 * (2 * case["sequences"] + 1 + 2 * rows), "flops": 2 * rows}
    (h, hkv), size = _widths(case), 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rotary":
        # forward: q, k, v in and out; backward: the upstream gradient, q and k (for the norm) in, the gradient out
        qk, v = used * (h + hkv) * size, used * hkv * size
        training = (2 * (qk + v) + (qk if case["norm"] else 0)) if case["training"] else 0
        return {"bytes": 2 * (qk + v) + training + 4 * rows * case["axes"],
                "flops": used * (h + hkv) * ((8 if case["norm"] else 4) + (case["training"] and (14 if case["norm"] else 4)))}
    pairs = sum(n * (n + 1) // 2 for n in _lengths(case))
    forward = used * (2 * h + 2 * hkv) * size + 4 * case["heads"] * used
    training = used * (2 * h + 2 * hkv) * size if case["training"] else 0
    return {"bytes": forward + training, "flops": (12 if case["training"] else 4) * pairs * h}
