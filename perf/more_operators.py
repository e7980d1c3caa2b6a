"""The operators of 8-bit activation checkpoints, measured: what a layer keeps for its backward pass in one byte a value and a
power of two for every 32, written by the passes that have the values in hand and read by the backward pass as it is.

Four kinds of case.
  save        tensors into their 8-bit form and back, several a call (po_op_save8, po_op_restore8)
  join        a block's output normed, gated, scaled and added to the residual stream, and the norm in front of the next block; the
              forward leaves checkpoints, the backward reads them (po_op_norm_join_*)
  activation  GeLU or SiLU, gated or not, forward with the checkpoint of its input and backward from it (po_op_activation_*)
  weights     a weight's gradient from its input's checkpoint (po_op_weight_grad_saved8)

With `own` false everything is computed from elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
SKIP, BRANCH = 0.9, 0.35  # what the residual stream and the block's output are multiplied by
BLOCK = 32


# ---- cases --------------------------------------------------------------------------------------------------------
def _named(name, case, kw):
    case.update(kw)
    return case if name is None else dict(name=name, **case)


def _save(name=None, **kw):
    return _named(name, dict(kind="save", rows=0, h=0, f=0, apart=False, dtype="bf16"), kw)


def _join(name=None, **kw):
    return _named(name, dict(kind="join", rows=0, h=0, rms=False, post=False, gate="none", backward=False, again=False, dtype="bf16"), kw)


def _activation(name=None, **kw):
    return _named(name, dict(kind="activation", rows=0, f=0, silu=False, gated=False, training=True, dtype="bf16"), kw)


def _weights(name=None, **kw):
    return _named(name, dict(kind="weights", rows=0, k=0, n=0, add=False, dtype="bf16"), kw)


def listed():
    return [
        # The saved set of a small fp32 layer: five tensors, latency counts.
        _save("save_few", rows=128, h=256, f=1024, dtype="f32"),
        # The saved set of a 4096-wide layer, 4096 rows: what travels to the host.
        _save("save_layer", rows=4096, h=4096, f=16384),
        # A small fp32 layer in the stage's own arrangement: residual sum and LayerNorm.
        _join("join_few", rows=128, h=256, dtype="f32"),
        # A 2048-wide model with norms on both sides of its blocks and a learned gate per column.
        _join("join_gated", rows=2048, h=2048, rms=True, post=True, gate="columns"),
        # The stage's own arrangement backward, with the normed values that the weight gradient needs computed again.
        _join("join_backward", rows=4096, h=4096, backward=True, again=True),
        # Norms on both sides and a gate of the block's own for every value, a long microbatch of a 5120-wide model.
        _join("join_backward_sandwich", rows=16384, h=5120, rms=True, post=True, gate="values", backward=True),
        # A small fp32 feed-forward, forward and backward.
        _activation("activation_few", rows=128, f=1024, dtype="f32"),
        # A gated feed-forward of a 4096-wide model, forward and backward.
        _activation("activation_gated", rows=4096, f=8192, silu=True, gated=True),
        # A small fp32 projection.
        _weights("weights_few", rows=128, k=256, n=1024, dtype="f32"),
        # A 2048-wide projection, a ragged microbatch, added to the gradient of earlier microbatches.
        _weights("weights_ragged", rows=1733, k=2048, n=2048, add=True),
        # A narrow projection of a long microbatch: few results, many rows.
        _weights("weights_long", rows=16384, k=640, n=256),
        # The wide projection of a 4096-wide feed-forward.
        _weights("weights_wide", rows=4096, k=4096, n=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: most are whole vectors, some are odd."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.25 else max(8, n // 8 * 8)


def draw(rng):
    kind = rng.choices(["save", "join", "activation", "weights"], [2, 5, 3, 5])[0]
    dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
    size = 2 if dtype == "bf16" else 4
    if kind == "save":
        h = _width(rng, 64, 5120)
        f = _width(rng, h, 4 * h)
        return _save(rows=_log_int(rng, 1, min(16384, 300_000_000 // ((6 * h + f) * size))), h=h, f=f, apart=rng.random() < 0.4, dtype=dtype)
    if kind == "join":
        h = _width(rng, 64, 8192)
        return _join(rows=_log_int(rng, 1, min(16384, 150_000_000 // (h * size))), h=h, rms=rng.random() < 0.5, post=rng.random() < 0.5,
                     gate=rng.choice(["none", "columns", "values"]), backward=rng.random() < 0.6, again=rng.random() < 0.4, dtype=dtype)
    if kind == "activation":
        gated = rng.random() < 0.5
        f = _width(rng, 64, 16384)
        return _activation(rows=_log_int(rng, 1, min(16384, 130_000_000 // (f * size * (2 if gated else 1)))), f=f, silu=rng.random() < 0.5,
                           gated=gated, training=rng.random() < 0.7, dtype=dtype)
    k, n = _width(rng, 64, 8192), _width(rng, 64, 8192)
    return _weights(rows=_log_int(rng, 1, min(16384, 130_000_000_000 // (k * n))), k=k, n=n, add=rng.random() < 0.4, dtype=dtype)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- the 8-bit form -----------------------------------------------------------------------------------------------
def _padded(cols):
    return -(-cols // BLOCK) * BLOCK


def _blocks(x):
    """x [rows, cols] in fp32 as [rows, blocks, 32], zeros behind the last column."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x.float(), (0, _padded(cols) - cols)).view(rows, -1, BLOCK)


def _power(e):
    """2^e in fp32 for whole e of normal numbers, from its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(x):
    """(codes, exponents + 127) of x: a block's exponent is the least e with its largest magnitude at most 448 * 2^e, a code the e4m3
    number nearest to x / 2^e."""
    b = _blocks(x)
    m, e = torch.frexp(b.abs().amax(-1))  # m * 2^e, m in [0.5, 1): 448 is 0.875 * 2^9
    e = (e - 9 + (m > 0.875)).clamp_(min=-117)
    codes = (b * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8).flatten(1), (e + 127).to(torch.uint8)


def _buffer(x):
    """The checkpoint of x as the operators keep it: codes, behind them the exponents, in whole 16 bytes."""
    codes, scales = _encode(x)
    flat = torch.cat([codes.reshape(-1), scales.reshape(-1)])
    return torch.nn.functional.pad(flat, (0, -flat.numel() % 16))


def _values(codes, scales, cols):
    """What the codes stand for, in fp32."""
    b = codes.view(torch.float8_e4m3fn).float().view(codes.shape[0], -1, BLOCK)
    return (b * _power(scales.int() - 127)[..., None]).flatten(1)[:, :cols]


def _restored(buffer, rows, cols):
    n = rows * _padded(cols)
    return _values(buffer[:n].view(rows, -1), buffer[n:n + n // BLOCK].view(rows, -1), cols)


def _room(rows, cols):
    n = rows * _padded(cols)
    return torch.zeros((n + n // BLOCK + 15) // 16 * 16, dtype=torch.uint8, device=DEVICE)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _shapes(case):
    """Columns of the tensors of a layer's saved set: x, q | k | v, attention output, x1, u."""
    return [case["h"], 3 * case["h"], case["h"], case["h"], case["f"]]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dt, rows = _dtype(case), case["rows"]
    rand = lambda *size: torch.randn(*size, generator=g, device=DEVICE).to(dt)
    zeros = lambda *size, t=dt: torch.zeros(*size, dtype=t, device=DEVICE)

    def activations(cols):  # a few columns of a residual stream are much larger than the rest
        large = 1 + 15 * (torch.rand(cols, generator=g, device=DEVICE) < 0.01)
        return (torch.randn(rows, cols, generator=g, device=DEVICE) * large).to(dt)

    state = dict(case=case)
    if case["kind"] == "save":
        cols = _shapes(case)
        if case["apart"]:  # columns of one wide tensor
            wide = activations(sum(cols) + 5)
            state["tensors"] = list(wide[:, :sum(cols)].split(cols, 1))
        else:
            state["tensors"] = [activations(c) for c in cols]
        state.update(saved=[_room(rows, c) for c in cols], out=[zeros(rows, c) for c in cols])
    elif case["kind"] == "join":
        h = case["h"]
        vector = lambda mean, spread: (mean + spread * torch.randn(h, generator=g, device=DEVICE)).to(dt)
        x, f = activations(h), rand(rows, h)
        state.update(gains=[vector(1, 0.02) if case["post"] else None, vector(1, 0.02)],
                     shifts=[None if case["rms"] or not case["post"] else vector(0, 0.02), None if case["rms"] else vector(0, 0.02)],
                     gate={"none": None, "columns": vector(0.5, 0.1), "values": torch.sigmoid(rand(rows, h).float()).to(dt)}[case["gate"]])
        if case["backward"]:
            state.update(y_saved=_buffer(x), f_saved=_buffer(f), dy=(0.01 * rand(rows, h)).to(dt), dn=(0.01 * rand(rows, h)).to(dt),
                         dx=zeros(rows, h), df=zeros(rows, h), dgate=zeros(rows, h) if case["gate"] == "values" else None,
                         sums=zeros(5, h, t=torch.float32), n=zeros(rows, h) if case["again"] else None)
        else:
            state.update(x=x, f=f, y=zeros(rows, h), n=zeros(rows, h), y_saved=_room(rows, h), f_saved=_room(rows, h),
                         y8=zeros(rows, h, t=torch.bfloat16), f8=zeros(rows, h, t=torch.bfloat16))
    elif case["kind"] == "activation":
        cols = case["f"] * (2 if case["gated"] else 1)
        state.update(u=rand(rows, cols), saved=_room(rows, cols), out=zeros(rows, case["f"]))
        if case["training"]:
            state.update(d_out=(0.01 * rand(rows, case["f"])).to(dt), du=zeros(rows, cols), again=zeros(rows, case["f"]))
    else:
        state.update(saved=_buffer(activations(case["k"])), dy=(0.01 * rand(rows, case["n"])).to(dt),
                     dw=zeros(case["k"], case["n"], t=torch.float32))
        if case["add"]:
            state["before"] = torch.randn(case["k"], case["n"], generator=g, device=DEVICE)
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    return {"save": _run_save, "join": _run_join, "activation": _run_activation, "weights": _run_weights}[state["case"]["kind"]](state)


def _code(case):
    from paper_2503_01328_amd import binding as po

    return po.PO_BF16 if case["dtype"] == "bf16" else po.PO_F32


def _workspace(state, size):
    """Scratch memory that a program keeps from pass to pass."""
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEVICE)
    return state["workspace"]


def _run_save(state):
    """Into the 8-bit form, and back."""
    if own:
        return _own_save(state)
    dt = _dtype(state["case"])
    return {"out": [_values(*_encode(x), x.shape[1]).to(dt) for x in state["tensors"]]}


def _own_save(state):
    from paper_2503_01328_amd import binding as po

    code = _code(state["case"])
    po.po_op_save8(code, state["tensors"], state["saved"])
    po.po_op_restore8(code, state["saved"], state["out"])
    return {"out": state["out"]}


def _scales(v, rms):
    """Normed v, and what its gradient is multiplied by."""
    if not rms:
        v = v - v.mean(-1, keepdim=True)
    r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _affine(hat, gain, shift):
    v = hat * gain.float()
    return v if shift is None else v + shift.float()


def _through_norm(d, hat, r, gain, rms):
    """The gradient of a norm's input."""
    a = d * gain.float()
    back = a - hat * (a * hat).mean(-1, keepdim=True)
    return r * (back if rms else back - a.mean(-1, keepdim=True))


def _run_join(state):
    case = state["case"]
    if own:
        return _own_join_backward(state) if case["backward"] else _own_join(state)
    rms, dt, gate = case["rms"], _dtype(case), state["gate"]
    gate = 1.0 if gate is None else gate.float()
    (post, pre), (post_shift, pre_shift) = state["gains"], state["shifts"]
    if not case["backward"]:
        f = state["f"].float()
        z = _affine(_scales(f, rms)[0], post, post_shift) if case["post"] else f
        y = SKIP * state["x"].float() + BRANCH * gate * z
        n = _affine(_scales(y, rms)[0], pre, pre_shift).to(dt)
        y = y.to(dt)
        return {"y": y, "n": n, "y8": _values(*_encode(y), case["h"]).to(torch.bfloat16),
                "f8": _values(*_encode(state["f"]), case["h"]).to(torch.bfloat16)}
    y = _restored(state["y_saved"], case["rows"], case["h"])
    if case["post"] or case["gate"] != "none":
        f = _restored(state["f_saved"], case["rows"], case["h"])
    dn = state["dn"].float()
    hat, r = _scales(y, rms)
    t = state["dy"].float() + _through_norm(dn, hat, r, pre, rms)
    out = {"dx": (SKIP * t).to(dt), "dpre_gain": (dn * hat).sum(0)}
    if not rms:
        out["dpre_shift"] = dn.sum(0)
    if case["again"]:
        out["n"] = _affine(hat, pre, pre_shift).to(dt)
    w = BRANCH * t
    dz = w * gate
    if case["post"]:
        fhat, fr = _scales(f, rms)
    if case["gate"] != "none":
        dgate = w * (_affine(fhat, post, post_shift) if case["post"] else f)
        out["dgate"] = dgate.to(dt) if case["gate"] == "values" else dgate.sum(0)
    if case["post"]:
        out["dpost_gain"] = (dz * fhat).sum(0)
        if not rms:
            out["dpost_shift"] = dz.sum(0)
        dz = _through_norm(dz, fhat, fr, post, rms)
    out["df"] = dz.to(dt)
    return out


def _own_join(state):
    from paper_2503_01328_amd import binding as po

    case = state["case"]
    po.po_op_norm_join_forward(_code(case), po.PO_NORM_RMS if case["rms"] else po.PO_NORM_LAYER, state["x"], state["f"], state["gains"][0],
                               state["shifts"][0], state["gate"], int(case["gate"] == "values"), SKIP, BRANCH, state["gains"][1],
                               state["shifts"][1], state["y"], state["n"], state["f_saved"], state["y_saved"], case["rows"], case["h"], EPS)
    po.po_op_restore8(po.PO_BF16, [state["y_saved"], state["f_saved"]], [state["y8"], state["f8"]])
    return {k: state[k] for k in ("y", "n", "y8", "f8")}


def _own_join_backward(state):
    from paper_2503_01328_amd import binding as po

    case, sums = state["case"], state["sums"]
    sums.zero_()
    post, rms, gate = case["post"], case["rms"], case["gate"]
    dgate = {"none": None, "columns": sums[4], "values": state["dgate"]}[gate]
    workspace = _workspace(state, po.po_op_norm_join_backward_workspace(case["rows"], case["h"]))
    po.po_op_norm_join_backward(_code(case), po.PO_NORM_RMS if rms else po.PO_NORM_LAYER, state["dy"], state["dn"], state["y_saved"], 1,
                                state["f_saved"], 1, state["gains"][0], state["shifts"][0], state["gate"], int(gate == "values"), SKIP, BRANCH,
                                state["gains"][1], state["shifts"][1], state["dx"], state["df"], dgate, sums[0] if post else None,
                                sums[1] if post and not rms else None, sums[2], None if rms else sums[3], state["n"], workspace, case["rows"],
                                case["h"], EPS)
    out = {"dx": state["dx"], "df": state["df"], "dpre_gain": sums[2]}
    if not rms:
        out["dpre_shift"] = sums[3]
    if gate != "none":
        out["dgate"] = dgate
    if post:
        out["dpost_gain"] = sums[0]
        if not rms:
            out["dpost_shift"] = sums[1]
    if case["again"]:
        out["n"] = state["n"]
    return out


def _curve(a, silu):
    """The activation and its slope."""
    if silu:
        s = torch.sigmoid(a)
        return a * s, s * (1 + a * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * c * (1 + 3 * 0.044715 * a * a)


def _run_activation(state):
    case = state["case"]
    if own:
        return _own_activation(state)
    dt, f, gated = _dtype(case), case["f"], case["gated"]
    codes, scales = _encode(state["u"])
    u = state["u"].float()
    v = _curve(u[:, :f], case["silu"])[0]
    out = {"out": (v * u[:, f:] if gated else v).to(dt)}
    u = _values(codes, scales, u.shape[1])
    if not case["training"]:
        return {**out, "u8": u.to(dt)}
    v, slope = _curve(u[:, :f], case["silu"])
    d = state["d_out"].float()
    if gated:
        b = u[:, f:]
        return {**out, "again": (v * b).to(dt), "du": torch.cat([d * b * slope, d * v], 1).to(dt)}
    return {**out, "again": v.to(dt), "du": (d * slope).to(dt)}


def _own_activation(state):
    from paper_2503_01328_amd import binding as po

    case, code = state["case"], _code(state["case"])
    kind = po.PO_ACT_SILU if case["silu"] else po.PO_ACT_GELU
    po.po_op_activation_forward(code, kind, int(case["gated"]), state["u"], state["out"], state["saved"], case["rows"], case["f"])
    if not case["training"]:
        if "u8" not in state:
            state["u8"] = torch.empty_like(state["u"])
        po.po_op_restore8(code, [state["saved"]], [state["u8"]])
        return {"out": state["out"], "u8": state["u8"]}
    po.po_op_activation_backward(code, kind, int(case["gated"]), state["saved"], 1, state["d_out"], state["du"], state["again"], case["rows"],
                                 case["f"])
    return {"out": state["out"], "again": state["again"], "du": state["du"]}


def _run_weights(state):
    case = state["case"]
    if own:
        return _own_weights(state)
    x = _restored(state["saved"], case["rows"], case["k"])
    dw = torch.mm(x.t(), state["dy"].float())
    return {"dw": dw + state["before"] if case["add"] else dw}


def _own_weights(state):
    from paper_2503_01328_amd import binding as po

    case, code = state["case"], _code(state["case"])
    rows, k, n = case["rows"], case["k"], case["n"]
    if case["add"]:
        state["dw"].copy_(state["before"])
    workspace = _workspace(state, po.po_op_weight_grad_saved8_workspace(code, rows, k, n))
    po.po_op_weight_grad_saved8(code, state["saved"], state["dy"], n, state["dw"], n, int(case["add"]), workspace, rows, k, n)
    return {"dw": state["dw"]}


# ---- the operators' definitions in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"save": _exact_save, "join": _exact_join, "activation": _exact_activation, "weights": _exact_weights}[case["kind"]](case, state)


def _two(e):
    """2^e in 64 bits for whole e, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid(x):
    """x as its checkpoint holds it: of the multiples of 2^(e - 9) that e4m3 has, the nearest, in 64 bits."""
    rows, cols = x.shape
    b = torch.zeros(rows, _padded(cols), dtype=torch.float64, device=DEVICE)
    b[:, :cols] = x
    b = b.view(rows, -1, BLOCK)
    largest = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(largest / 448, min=2.0 ** -117)))
    e = torch.where(largest > 448 * _two(e), e + 1, e)  # should the logarithm have been rounded
    e = torch.where((largest <= 448 * _two(e - 1)) & (e > -117), e - 1, e)
    v = b / _two(e)
    step = _two(torch.frexp(v)[1].clamp_(min=-5) - 4)  # three bits behind the first, the smallest numbers evenly spaced
    return (torch.round(v / step) * step * _two(e)).flatten(1)[:, :cols]


def _stored(buffer, rows, cols):
    """A checkpoint's values from its bytes: sign, four bits of exponent, three of fraction."""
    n = rows * _padded(cols)
    byte = buffer[:n].view(rows, -1).long()
    exponent = byte >> 3 & 15
    fraction = torch.where(exponent > 0, 1 + (byte & 7) / 8.0, (byte & 7) / 8.0).double()
    v = torch.where(byte > 127, -fraction, fraction) * _two(exponent.clamp(min=1) - 7)
    scale = _two(buffer[n:n + n // BLOCK].long() - 127)
    return (v.view(rows, -1, BLOCK) * scale.view(rows, -1, 1)).flatten(1)[:, :cols].contiguous()


def _exact_save(case, state):
    return {"out": [_grid(x.double()) for x in state["tensors"]]}


def _normed(v, gain, shift, rms):
    var = v.square().mean(1) if rms else v.var(1, unbiased=False)
    centre = v if rms else v - v.mean(1)[:, None]
    out = centre / torch.sqrt(var + EPS)[:, None] * gain
    return out if shift is None else out + shift


def _exact_join(case, state):
    """The gradients by differentiating the definition."""
    wide = lambda t: None if t is None else t.double()
    rms, rows, h = case["rms"], case["rows"], case["h"]
    post, pre, post_shift, pre_shift, gate = (wide(t) for t in (*state["gains"], *state["shifts"], state["gate"]))

    def branch(f):
        z = _normed(f, post, post_shift, rms) if case["post"] else f
        return BRANCH * (z if gate is None else z * gate)

    if not case["backward"]:
        y = SKIP * state["x"].double() + branch(state["f"].double())
        return {"y": y, "n": _normed(y, pre, pre_shift, rms), "y8": None, "f8": _grid(state["f"].double())}
    y, f = (_stored(state[k], rows, h).requires_grad_() for k in ("y_saved", "f_saved"))
    for v in (post, pre, post_shift, pre_shift, gate):
        if v is not None:
            v.requires_grad_()
    n = _normed(y, pre, pre_shift, rms)
    out = {"n": n.detach()} if case["again"] else {}
    n.backward(state["dn"].double())
    t = state["dy"].double() + y.grad
    out.update(dx=SKIP * t, dpre_gain=pre.grad)
    branch(f).backward(t)
    out["df"] = f.grad
    for name, v in (("dpre_shift", pre_shift), ("dgate", gate), ("dpost_gain", post), ("dpost_shift", post_shift)):
        if v is not None:
            out[name] = v.grad
    return out


def _exact_activation(case, state):
    def curve(u):
        a = u[:, :case["f"]]
        if case["silu"]:
            v = a / (1 + torch.exp(-a))
        else:  # (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
            v = a / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a)))
        return v * u[:, case["f"]:] if case["gated"] else v

    u = _grid(state["u"].double())
    out = {"out": curve(state["u"].double())}
    if not case["training"]:
        return {**out, "u8": u}
    u.requires_grad_()
    again = curve(u)
    again.backward(state["d_out"].double())
    return {**out, "again": again.detach(), "du": u.grad}


def _exact_weights(case, state):
    dw = _stored(state["saved"], case["rows"], case["k"]).T @ state["dy"].double()
    return {"dw": dw + state["before"].double() if case["add"] else dw}


# ---- work ---------------------------------------------------------------------------------------------------------
def work(case):
    rows, size = case["rows"], 2 if case["dtype"] == "bf16" else 4
    saved = lambda cols: rows * _padded(cols) * (1 + 1 / BLOCK)
    if case["kind"] == "save":
        # in, checkpoint out; checkpoint in, out
        return {"bytes": sum(2 * (rows * c * size + saved(c)) for c in _shapes(case)), "flops": sum(4 * rows * c for c in _shapes(case))}
    if case["kind"] == "join":
        h = case["h"]
        one, gate = rows * h * size, {"none": 0, "columns": h * size, "values": rows * h * size}[case["gate"]]
        needs_f = case["post"] or case["gate"] != "none"
        if case["backward"]:
            given = 2 * one + saved(h) * (2 if needs_f else 1) + gate
            made = (3 if case["again"] else 2) * one + (gate if case["gate"] == "values" else 4 * h)
            return {"bytes": given + made, "flops": rows * h * (40 if case["post"] else 22)}
        # x and f in, sum and normed sum out, two checkpoints out and their values read back
        return {"bytes": 4 * one + gate + 4 * saved(h) + 2 * rows * h * 2, "flops": rows * h * (24 if case["post"] else 16)}
    if case["kind"] == "activation":
        cols, one = case["f"] * (2 if case["gated"] else 1), rows * case["f"] * size
        forward = rows * cols * size + one + saved(cols)
        backward = saved(cols) + (2 * one + rows * cols * size if case["training"] else rows * cols * size)
        return {"bytes": forward + backward, "flops": rows * case["f"] * (40 if case["training"] else 16)}
    k, n = case["k"], case["n"]
    return {"bytes": saved(k) + rows * n * size + 4 * k * n * (4 if case["add"] else 1), "flops": 2 * rows * k * n}
