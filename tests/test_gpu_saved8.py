"""8-bit checkpoints on the GPU and the operators that write and read them, against 64 bits (saved8_reference.py derives the bounds)."""
import math

import pytest
import torch

import saved8_reference as ref
from paper_2503_01328_amd import binding as po

pytestmark = pytest.mark.gpu

DT = {"f32": (po.PO_F32, torch.float32), "bf16": (po.PO_BF16, torch.bfloat16)}
MARK = 7.0  # what is to be left alone
EDGE = 4096


def _gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _rand(dev, seed, *shape, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(*shape, generator=_gen(dev, seed), device=dev)).to(dtype)


class Guarded:
    """A tensor of NaN or zeros between margins that are looked at afterwards."""

    def __init__(self, dev, dtype, *shape, offset=0, fill=math.nan):
        n = math.prod(shape)
        self.fill = 171 if dtype == torch.uint8 else MARK
        self.whole = torch.full((n + 2 * EDGE + offset,), self.fill, dtype=dtype, device=dev)
        self.t = self.whole[EDGE + offset:EDGE + offset + n].view(shape)
        self.t.fill_(0 if dtype == torch.uint8 else fill)
        self.ends = (self.whole[:EDGE + offset], self.whole[EDGE + offset + n:])

    def intact(self):
        return all(bool((e == self.fill).all()) for e in self.ends)


def _room(dev, rows, cols):
    return Guarded(dev, torch.uint8, po.po_op_saved8_bytes(rows, cols))


def _saved(x):
    """The checkpoint of x [rows, cols]."""
    buf = torch.empty(po.po_op_saved8_bytes(*x.shape), dtype=torch.uint8, device=x.device)
    po.po_op_save8(po.PO_F32 if x.dtype == torch.float32 else po.PO_BF16, [x], [buf])
    return buf


def _same(got, want):
    """Equal, NaN where there is NaN, zeros with their signs."""
    return bool((((got == want) & (torch.signbit(got) == torch.signbit(want))) | (got.isnan() & want.isnan())).all())


# ---- the form -----------------------------------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 31), (3, 32), (5, 33), (7, 100), (64, 256), (33, 1000), (2, 4099), (300, 24)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_save_and_restore(gpu_device, dtype, rows, cols):
    code, tdt = DT[dtype]
    # magnitudes over a wide range, so that every block has its own exponent and small codes
    x = (_rand(gpu_device, 1, rows, cols) * torch.exp2(torch.randint(-20, 21, (rows, cols), generator=_gen(gpu_device, 2), device=gpu_device).float() / 2)).to(tdt)
    room = _room(gpu_device, rows, cols)
    po.po_op_save8(code, [x], [room.t])
    codes, scales = ref.encode(x)
    got = ref.split(room.t, rows, cols)
    assert torch.equal(got[0].cpu(), codes) and torch.equal(got[1].cpu(), scales) and room.intact()
    want = ref.decode(codes, scales, cols).to(gpu_device)
    for c, t in DT.values():  # a checkpoint is restored in either type, the same numbers
        out = Guarded(gpu_device, t, rows, cols)
        po.po_op_restore8(c, [room.t], [out.t])
        assert torch.equal(out.t.double(), want) and out.intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_save_special_values(gpu_device, dtype):
    code, tdt = DT[dtype]
    big, tiny = torch.finfo(tdt).max, torch.finfo(tdt).tiny
    values = [0.0, -0.0, math.nan, math.inf, -math.inf, big, -big, 2.0 ** 127 * 1.875, 2.0 ** 127 * 1.75, 2.0 ** 127, tiny, -tiny, tiny / 8, 2.0 ** -126, 2.0 ** -127,
              2.0 ** -125, 1.5 * 2.0 ** -126, 448.0, 449.0, 464.0, 1.75, 1.7578125, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -10, 1.0, 17.0, 1.0625, 1.1875]
    rows = [values, [math.nan] * 32, [math.inf, 1.0], [0.0] * 32, [tiny / 4] * 5, [-big] * 32, [448 * 2.0 ** -117, 2.0 ** -126], [449 * 2.0 ** -117, 2.0 ** -126]]
    x = torch.zeros(len(rows) + len(values), 64, dtype=tdt)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, dtype=torch.float64).to(tdt)
    for i, v in enumerate(values):  # each as the largest of its block, and beside a one
        x[len(rows) + i, 3], x[len(rows) + i, 40], x[len(rows) + i, 50] = v, v, 1.0
    codes, scales = ref.encode(x)
    buf = _saved(x.to(gpu_device))
    got = [t.cpu() for t in ref.split(buf, *x.shape)]
    nan = (codes & 127) == 127
    assert torch.equal((got[0] & 127) == 127, nan) and torch.equal(got[0][~nan], codes[~nan]) and torch.equal(got[1], scales)
    out = torch.empty_like(x, device=gpu_device)
    po.po_op_restore8(code, [buf], [out])
    want = ref.decode(codes, scales, 64)
    assert _same(out.cpu().double(), want)
    assert not out.isinf().any()
    assert bool(((out == 0) | out.isnan() | (out.abs() >= torch.finfo(torch.float32).tiny)).all())  # nothing below the normal numbers


def test_every_code_is_restored(gpu_device):
    """All 256 codes under every scale byte that is written."""
    scales = torch.arange(10, 248, dtype=torch.uint8)
    rows = scales.numel()
    buf = torch.zeros(po.po_op_saved8_bytes(rows, 256), dtype=torch.uint8)
    buf[:rows * 256] = torch.arange(256).to(torch.uint8).repeat(rows)
    buf[rows * 256:rows * 264] = scales.repeat_interleave(8)
    want = ref.stored(buf, rows, 256)
    for c, t in DT.values():
        out = torch.empty(rows, 256, dtype=t, device=gpu_device)
        po.po_op_restore8(c, [buf.to(gpu_device)], [out])
        assert _same(out.cpu().double(), want.to(t).double())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_save_tensors_of_all_kinds_in_one_launch(gpu_device, dtype):
    """Eight: columns of a wide tensor, addresses off 16 bytes, one row, one column, whole blocks; restored into columns of another wide one."""
    code, tdt = DT[dtype]
    wide = _rand(gpu_device, 3, 40, 700, dtype=tdt)
    flat = _rand(gpu_device, 4, 5000, dtype=tdt)
    tensors = [wide[:, :96], wide[:, 96:200], wide[3:17, 201:300], flat[1:1 + 33 * 64].view(33, 64), flat[:4999].view(1, 4999), flat[:70].view(70, 1),
               flat[8:8 + 64 * 32].view(64, 32), wide[:, 320:321]]
    rooms = [_room(gpu_device, *t.shape) for t in tensors]
    po.po_op_save8(code, tensors, [r.t for r in rooms])
    for t, r in zip(tensors, rooms):
        codes, scales = ref.encode(t)
        got = ref.split(r.t, *t.shape)
        assert torch.equal(got[0].cpu(), codes) and torch.equal(got[1].cpu(), scales) and r.intact()
    back = torch.full((40, 500), MARK, dtype=tdt, device=gpu_device)
    outs = [back[:, :96], back[:, 101:205], back[:14, 300:399]]
    po.po_op_restore8(code, [rooms[0].t, rooms[1].t, rooms[2].t], outs)
    for t, o in zip(tensors, outs):
        assert torch.equal(o.double().cpu(), ref.decode(*ref.encode(t), t.shape[1]))
    assert bool((back[:, 96:101] == MARK).all()) and bool((back[:, 205:300] == MARK).all()) and bool((back[14:, 300:] == MARK).all())


def test_save_of_many_values(gpu_device):
    """2^31 of them: offsets past 32 bits, and enough of small and large launches' forms."""
    rows, cols = 65536, 32768
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=gpu_device)
    x.copy_(_rand(gpu_device, 5, 1, cols))
    x[-3:] = _rand(gpu_device, 6, 3, cols).to(torch.bfloat16)
    buf = _saved(x)
    some = torch.cat([x[:2], x[40000:40002], x[-4:]])
    codes, scales = ref.encode(some)
    got = ref.split(buf, rows, cols)
    pick = lambda t: torch.cat([t[:2], t[40000:40002], t[-4:]])
    assert torch.equal(pick(got[0]).cpu(), codes) and torch.equal(pick(got[1]).cpu(), scales)
    x.fill_(MARK)
    po.po_op_restore8(po.PO_BF16, [buf], [x])
    assert torch.equal(pick(x).double().cpu(), ref.decode(codes, scales, cols))


# ---- activations --------------------------------------------------------------------------------------------------
ACT_SHAPES = [(1, 1), (3, 7), (5, 32), (4, 100), (129, 1024), (2, 2056), (17, 96)]


def _activation(dev, dtype, silu, gated, u, d, offset=0):
    code, tdt = DT[dtype]
    rows, f = d.shape
    kind = po.PO_ACT_SILU if silu else po.PO_ACT_GELU
    out, room = Guarded(dev, tdt, rows, f, offset=offset), _room(dev, *u.shape)
    po.po_op_activation_forward(code, kind, int(gated), u, out.t, room.t, rows, f)
    du, again = Guarded(dev, tdt, *u.shape, offset=offset), Guarded(dev, tdt, rows, f, offset=offset)
    po.po_op_activation_backward(code, kind, int(gated), room.t, 1, d, du.t, again.t, rows, f)
    assert all(g.intact() for g in (out, room, du, again))
    return out.t, room.t, du.t, again.t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,f", ACT_SHAPES)
def test_activation(gpu_device, dtype, silu, gated, rows, f):
    tdt = DT[dtype][1]
    u = _rand(gpu_device, 7, rows, 2 * f if gated else f, dtype=tdt, scale=3.0)
    d = _rand(gpu_device, 8, rows, f, dtype=tdt)
    for offset in (0, 1):  # aligned tensors, and others
        out, saved, du, again = _activation(gpu_device, dtype, silu, gated, u, d, offset)
        ref.check(out, ref.activation_forward(u, silu, gated, tdt), "out")
        codes, scales = ref.encode(u)
        got = ref.split(saved, *u.shape)
        assert torch.equal(got[0].cpu(), codes) and torch.equal(got[1].cpu(), scales)
        want = ref.activation_backward(ref.stored(saved, *u.shape), d, silu, gated, tdt)
        ref.check(du, want["du"], "du")
        ref.check(again, want["out"], "out again")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("gated,f", [(False, 40), (True, 64), (True, 40)])
def test_activation_without_checkpoints_and_in_place(gpu_device, dtype, silu, gated, f):
    code, tdt = DT[dtype]
    kind = po.PO_ACT_SILU if silu else po.PO_ACT_GELU
    rows = 9
    u, d = _rand(gpu_device, 9, rows, 2 * f if gated else f, dtype=tdt, scale=3.0), _rand(gpu_device, 10, rows, f, dtype=tdt)
    want = ref.activation_backward(u, d, silu, gated, tdt)
    du = torch.empty_like(u)
    po.po_op_activation_backward(code, kind, int(gated), u, 0, d, du, None, rows, f)
    ref.check(du, want["du"], "du")
    out = torch.empty_like(d)
    po.po_op_activation_forward(code, kind, int(gated), u, out, None, rows, f)
    ref.check(out, ref.activation_forward(u, silu, gated, tdt), "out")
    if not gated:
        d2, u2 = d.clone(), u.clone()
        po.po_op_activation_backward(code, kind, 0, u, 0, d2, d2, None, rows, f)
        po.po_op_activation_forward(code, kind, 0, u2, u2, None, rows, f)
        assert torch.equal(d2, du) and torch.equal(u2, out)


@pytest.mark.parametrize("silu", [False, True])
def test_activation_far_out(gpu_device, silu):
    """The gate is 0 or 1 there: no NaN but from a NaN, whatever the magnitude."""
    kind = po.PO_ACT_SILU if silu else po.PO_ACT_GELU
    a = torch.tensor([0.0, -0.0, 5.0, -5.0, 20.0, -20.0, 90.0, -90.0, 200.0, -200.0, 1e10, -1e10, 1e20, -1e20, 3e38, -3e38, math.inf, -math.inf, math.nan],
                     device=gpu_device).view(1, -1)
    d = torch.ones_like(a)
    out, du = torch.empty_like(a), torch.empty_like(a)
    po.po_op_activation_forward(po.PO_F32, kind, 0, a, out, None, 1, a.shape[1])
    po.po_op_activation_backward(po.PO_F32, kind, 0, a, 0, d, du, None, 1, a.shape[1])
    assert out[0, -1].isnan() and du[0, -1].isnan()
    assert out[0, -3] == math.inf and out[0, -2] == 0 and du[0, -3] == 1 and du[0, -2] == 0
    want = ref.activation_backward(a[:, :-3], d[:, :-3], silu, False, torch.float32)
    ref.check(out[:, :-3], want["out"], "out")
    ref.check(du[:, :-3], want["du"], "du")


# ---- norms joined to the residual stream --------------------------------------------------------------------------
def _params(dev, tdt, h, rows, rms, post, gate, seed=20, shifts=True):
    v = lambda k, mean, spread: (mean + spread * _rand(dev, seed + k, h)).to(tdt)
    p = dict(rms=rms, eps=1e-5, skip=0.9, branch=-0.35, gate=None, post_gain=v(1, 1, 0.3) if post else None, pre_gain=v(2, 1, 0.3),
             post_shift=v(3, 0, 0.3) if post and not rms and shifts else None, pre_shift=v(4, 0, 0.3) if not rms and shifts else None)
    if gate == "columns":
        p["gate"] = v(5, 0.5, 0.3)
    elif gate == "values":
        p["gate"] = (0.5 + 0.3 * _rand(dev, seed + 6, rows, h)).to(tdt)
    return p


def _norm_kind(p):
    return po.PO_NORM_RMS if p["rms"] else po.PO_NORM_LAYER


def _per_value(p):
    return int(p["gate"] is not None and p["gate"].dim() == 2)


def _join_forward(dev, dtype, x, f, p, offset=0, save=True):
    code, tdt = DT[dtype]
    rows, h = x.shape
    pre = p["pre_gain"] is not None
    y, n = Guarded(dev, tdt, rows, h, offset=offset), Guarded(dev, tdt, rows, h, offset=offset)
    sf, sy = (_room(dev, rows, h) for _ in range(2))
    po.po_op_norm_join_forward(code, _norm_kind(p), x, f, p["post_gain"], p["post_shift"], p["gate"], _per_value(p), p["skip"], p["branch"], p["pre_gain"],
                               p["pre_shift"], y.t, n.t if pre else None, sf.t if save else None, sy.t if save else None, rows, h, p["eps"])
    assert all(g.intact() for g in (y, n, sf, sy))
    return y.t, n.t, sf.t, sy.t


NAMES = ("dgate", "dpost_gain", "dpost_shift", "dpre_gain", "dpre_shift")


def _join_backward(dev, dtype, dy, dn, y, f, p, rows, h, saved=True, again=True, offset=0, workspace=None, start=0.0):
    """All gradients; sums begin at `start`."""
    code, tdt = DT[dtype]
    sums = {k: Guarded(dev, torch.float32, h, fill=start) for k in NAMES if p[k[1:]] is not None and not (k == "dgate" and _per_value(p))}
    g = {k: Guarded(dev, tdt, rows, h, offset=offset) for k in ("dx", "df") + (("dgate",) if _per_value(p) else ()) + (("n",) if again else ())}
    g.update(sums)
    t = lambda k: g[k].t if k in g else None
    size = po.po_op_norm_join_backward_workspace(rows, h)
    if workspace is None:
        workspace = torch.full((size + EDGE,), 255, dtype=torch.uint8, device=dev)  # NaN, and a margin to be left alone
    po.po_op_norm_join_backward(code, _norm_kind(p), dy, dn, y, int(saved), f, int(saved), p["post_gain"], p["post_shift"], p["gate"], _per_value(p), p["skip"],
                                p["branch"], p["pre_gain"], p["pre_shift"], t("dx"), t("df"), t("dgate"), t("dpost_gain"), t("dpost_shift"), t("dpre_gain"),
                                t("dpre_shift"), t("n"), workspace, rows, h, p["eps"])
    assert bool((workspace[size:] == 255).all()) and all(v.intact() for v in g.values())
    return {k: v.t for k, v in g.items()}


def _join_case(dev, dtype, rows, h, p, offset=0, seed=30, scale=1.0):
    tdt = DT[dtype][1]
    wide = 1 + 15 * (torch.rand(h, generator=_gen(dev, seed), device=dev) < 0.02)
    x, f = (_rand(dev, seed + 1, rows, h, scale=scale) * wide).to(tdt), _rand(dev, seed + 2, rows, h, dtype=tdt, scale=scale)
    y, n, sf, sy = _join_forward(dev, dtype, x, f, p, offset)
    want = ref.join_forward(x, f, p, tdt)
    ref.check(y, want["y"], "y")
    if p["pre_gain"] is not None:
        ref.check(n, want["n"], "n")
    for t, s in ((f, sf), (y, sy)):
        codes, scales = ref.encode(t)
        got = ref.split(s, rows, h)
        assert torch.equal(got[0].cpu(), codes) and torch.equal(got[1].cpu(), scales)
    dy, dn = _rand(dev, seed + 3, rows, h, dtype=tdt), _rand(dev, seed + 4, rows, h, dtype=tdt) if p["pre_gain"] is not None else None
    again = p["pre_gain"] is not None
    got = _join_backward(dev, dtype, dy, dn, sy, sf, p, rows, h, again=again, offset=offset)
    want = ref.join_backward(dy, dn, ref.stored(sy, rows, h), ref.stored(sf, rows, h), p, tdt, again=again)
    assert set(got) == set(want)
    for k in want:
        ref.check(got[k], want[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "columns", "values"])
@pytest.mark.parametrize("rows,h", [(1, 1), (3, 8), (5, 37), (130, 256), (7, 1000), (600, 520)])
def test_join(gpu_device, dtype, rms, post, gate, rows, h):
    _join_case(gpu_device, dtype, rows, h, _params(gpu_device, DT[dtype][1], h, rows, rms, post, gate))


WIDE = [(2, 512), (3, 513), (600, 2048), (5, 4096), (3, 4104), (4, 5120), (3, 8192), (2, 8193), (3, 10240), (2, 12288), (3, 16384), (2, 16383)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [(False, False, "none"), (True, False, "none"), (False, True, "columns"), (True, True, "columns"), (True, True, "values"), (False, True, "values")], ids=str)
@pytest.mark.parametrize("rows,h", WIDE)
def test_join_of_wide_rows(gpu_device, dtype, kind, rows, h):
    _join_case(gpu_device, dtype, rows, h, _params(gpu_device, DT[dtype][1], h, rows, *kind))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [64, 96, 520])
def test_join_addresses_off_16_bytes(gpu_device, dtype, h):
    _join_case(gpu_device, dtype, 21, h, _params(gpu_device, DT[dtype][1], h, 21, False, True, "values"), offset=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
def test_join_without_what_may_be_left_out(gpu_device, dtype, rms):
    """No norm in front of the next block; no norms at all; no shifts; no dy; y and f from tensors; no checkpoints; sums added to what is there."""
    dev, tdt, rows, h = gpu_device, DT[dtype][1], 70, 200
    x, f, dy, dn = (_rand(dev, 40 + k, rows, h, dtype=tdt) for k in range(4))
    for post in (False, True):
        for gate in ("none", "columns", "values"):
            p = _params(dev, tdt, h, rows, rms, post, gate, shifts=False)
            bare = dict(p, pre_gain=None, pre_shift=None)
            y, _, _, _ = _join_forward(dev, dtype, x, f, bare, save=False)
            ref.check(y, ref.join_forward(x, f, bare, tdt)["y"], "y")
            got = _join_backward(dev, dtype, dy, None, None, f, bare, rows, h, saved=False, again=False)
            want = ref.join_backward(dy, None, None, f, bare, tdt)
            for k in want:
                ref.check(got[k], want[k], k)
            got = _join_backward(dev, dtype, None, dn, x, f, p, rows, h, saved=False, again=False, start=2.5)
            want = ref.join_backward(None, dn, x, f, p, tdt)
            for k in want:
                more = 2.5 if k in NAMES and got[k].dim() == 1 else 0.0
                ref.check(got[k], want[k] + more if more else want[k], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,h", [(40, 264), (700, 2048), (9, 8200), (33, 517)])
def test_join_from_checkpoints_and_from_what_they_hold(gpu_device, dtype, rows, h):
    """y and f from checkpoints, from tensors of the same values, one of each."""
    dev, (code, tdt) = gpu_device, DT[dtype]
    p = _params(dev, tdt, h, rows, False, True, "columns")
    dy, dn = _rand(dev, 56, rows, h, dtype=tdt), _rand(dev, 57, rows, h, dtype=tdt)
    saved = [_saved(_rand(dev, 58 + k, rows, h, dtype=tdt)) for k in range(2)]
    held = [torch.empty(rows, h, dtype=tdt, device=dev) for _ in range(2)]
    po.po_op_restore8(code, saved, held)
    want = ref.join_backward(dy, dn, *held, p, tdt)
    results = []
    for ys in (0, 1):
        for fs in (0, 1):
            dx, df = torch.empty_like(dy), torch.empty_like(dy)
            sums = torch.zeros(5, h, device=dev)
            ws = torch.empty(po.po_op_norm_join_backward_workspace(rows, h), dtype=torch.uint8, device=dev)
            po.po_op_norm_join_backward(code, _norm_kind(p), dy, dn, (held, saved)[ys][0], ys, (held, saved)[fs][1], fs, p["post_gain"], p["post_shift"], p["gate"], 0,
                                        p["skip"], p["branch"], p["pre_gain"], p["pre_shift"], dx, df, sums[4], sums[0], sums[1], sums[2], sums[3], None, ws, rows, h,
                                        p["eps"])
            results.append((dx, df, sums))
            for k, t in dict(dx=dx, df=df, dpost_gain=sums[0], dpost_shift=sums[1], dpre_gain=sums[2], dpre_shift=sums[3], dgate=sums[4]).items():
                ref.check(t, want[k], f"{k}, y saved {ys}, f saved {fs}")
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[3]))  # the same arithmetic on the same numbers


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_join_in_place(gpu_device, dtype):
    dev, (code, tdt), rows, h = gpu_device, DT[dtype], 33, 264
    p = _params(dev, tdt, h, rows, False, True, "columns")
    x, f, dy, dn = (_rand(dev, 50 + k, rows, h, dtype=tdt) for k in range(4))
    y, n, sf, sy = _join_forward(dev, dtype, x, f, p)
    want = _join_backward(dev, dtype, dy, dn, sy, sf, p, rows, h)
    x2, f2 = x.clone(), f.clone()
    po.po_op_norm_join_forward(code, _norm_kind(p), x2, f2, p["post_gain"], p["post_shift"], p["gate"], 0, p["skip"], p["branch"], p["pre_gain"], p["pre_shift"],
                               x2, f2, None, None, rows, h, p["eps"])
    assert torch.equal(x2, y) and torch.equal(f2, n)
    sums = torch.zeros(5, h, device=dev)
    ws = torch.empty(po.po_op_norm_join_backward_workspace(rows, h), dtype=torch.uint8, device=dev)
    po.po_op_norm_join_backward(code, _norm_kind(p), dy, dn, sy, 1, sf, 1, p["post_gain"], p["post_shift"], p["gate"], 0, p["skip"], p["branch"], p["pre_gain"],
                                p["pre_shift"], dy, dn, sums[0], sums[1], sums[2], sums[3], sums[4], None, ws, rows, h, p["eps"])
    assert torch.equal(dy, want["dx"]) and torch.equal(dn, want["df"])


@pytest.mark.parametrize("h", [40, 1000, 12288])
def test_join_workspace_kept_from_more_rows(gpu_device, h):
    dev, tdt = gpu_device, torch.bfloat16
    ws = torch.full((po.po_op_norm_join_backward_workspace(700, h) + EDGE,), 255, dtype=torch.uint8, device=dev)
    for rows in (700, 513, 512, 100, 1):
        size = po.po_op_norm_join_backward_workspace(rows, h)
        p = _params(dev, tdt, h, rows, False, True, "columns")
        y, f, dy, dn = (_rand(dev, 60 + k, rows, h, dtype=tdt) for k in range(4))
        ws[size:] = 255
        got = _join_backward(dev, "bf16", dy, dn, y, f, p, rows, h, saved=False, workspace=ws)
        want = ref.join_backward(dy, dn, y, f, p, tdt, again=True)
        for k in want:
            ref.check(got[k], want[k], k)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("where", ["x", "f", "dy", "dn"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_join_values_that_are_not_finite_stay_in_their_row(gpu_device, rms, post, where, value):
    dev, rows, h, bad = gpu_device, 40, 300, 17
    p = _params(dev, torch.float32, h, rows, rms, post, "values")
    x, f, dy, dn = (_rand(dev, 70 + k, rows, h) for k in range(4))

    def run():
        y, n, sf, sy = _join_forward(dev, "f32", x, f, p)
        return dict(y=y, n1=n, **_join_backward(dev, "f32", dy, dn, sy, sf, p, rows, h))

    clean = run()
    dict(x=x, f=f, dy=dy, dn=dn)[where][bad, 5] = value
    got = run()
    keep = torch.arange(rows, device=dev) != bad
    for k in clean:
        if clean[k].dim() == 2:
            assert torch.equal(got[k][keep], clean[k][keep]), k
    assert not got["dx"][bad].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gate", ["none", "columns"])
@pytest.mark.parametrize("h", [1, 37, 40, 300, 8200])
def test_join_checkpoints_of_rows_that_are_not_finite_end_in_zeros(gpu_device, dtype, rms, gate, h):
    """Rows whose norm is nowhere finite: what lies behind the last column is po_op_save8's zeros, in f's checkpoint and in y's."""
    dev, (code, tdt), rows = gpu_device, DT[dtype], 6
    p = dict(_params(dev, tdt, h, rows, rms, True, gate), eps=0.0)
    x, f = _rand(dev, 75, rows, h, dtype=tdt), _rand(dev, 76, rows, h, dtype=tdt)
    f[1, h // 2], f[2, h - 1], f[3, 0] = math.nan, math.inf, -math.inf
    f[4] = 0.0  # a variance of zero, and no eps
    y, n, sf, sy = _join_forward(dev, dtype, x, f, p)
    assert y[4].isnan().all() and n[4].isnan().all()
    for t, s in ((f, sf), (y, sy)):
        codes, scales = ref.encode(t)
        got = [v.cpu() for v in ref.split(s, rows, h)]
        nan = (codes & 127) == 127
        assert torch.equal((got[0] & 127) == 127, nan) and torch.equal(got[0][~nan], codes[~nan]) and torch.equal(got[1], scales)


@pytest.mark.parametrize("rms", [False, True])
def test_join_of_rows_that_hold_one_value(gpu_device, rms):
    """Variances of zero (LayerNorm of constant rows, rows of zeros), and small and large rows."""
    dev, h = gpu_device, 96
    x = torch.zeros(6, h, device=dev)
    x[1], x[2], x[3], x[4] = 3.0, -1e-3, 1e15 * _rand(dev, 80, h), 1e-15 * _rand(dev, 81, h)
    f = x.flip(0).contiguous()
    dy, dn = _rand(dev, 82, 6, h), _rand(dev, 83, 6, h)
    p = dict(_params(dev, torch.float32, h, 6, rms, True, "none"), skip=1.0, branch=0.0)
    got = _join_backward(dev, "f32", dy, dn, x, f, p, 6, h, saved=False)
    want = ref.join_backward(dy, dn, x, f, p, torch.float32, again=True)
    for k in want:
        ref.check(got[k], want[k], k)
    y, n, _, _ = _join_forward(dev, "f32", x, f, p)
    assert torch.equal(y, x) and n.isfinite().all()


# ---- weight gradients ---------------------------------------------------------------------------------------------
def _weight_grad(dtype, saved, dy, dw, accumulate, k, rows=None, n=None, workspace=None):
    code = DT[dtype][0]
    rows, n = rows or dy.shape[0], n or dy.shape[1]
    size = po.po_op_weight_grad_saved8_workspace(code, rows, k, n)
    if workspace is None and size:
        workspace = torch.full((size + EDGE,), 255, dtype=torch.uint8, device=dy.device)
    po.po_op_weight_grad_saved8(code, saved, dy, dy.stride(0) if dy.shape[0] > 1 else n, dw, dw.stride(0) if k > 1 else n, accumulate, workspace, rows, k, n)
    if size:
        assert bool((workspace[size:] == 255).all())


WEIGHTS = [(1, 1, 1), (1, 40, 24), (7, 33, 5), (63, 64, 64), (64, 64, 72), (65, 100, 130), (200, 128, 128), (129, 256, 1024), (1000, 96, 771), (257, 300, 264),
           (2000, 40, 56), (3000, 640, 256), (300, 2048, 2048), (130, 2056, 1544), (513, 1000, 4104),
           (1, 2100, 3800), (64, 2048, 4096), (127, 2056, 3784), (129, 2100, 3801), (192, 2305, 3592), (700, 2100, 3800),
           # many splits, few, results that are no whole vectors; large tiles aligned and not
           (16384, 64, 64), (5000, 65, 77), (1500, 33, 35), (9000, 640, 256), (1733, 2048, 2048), (700, 2050, 2051), (4000, 1030, 1032),
           # wide tiles with splits
           (2391, 136, 6368), (3414, 7120, 528), (12171, 496, 2320)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n", WEIGHTS)
def test_weight_grad(gpu_device, dtype, rows, k, n):
    dev, tdt = gpu_device, DT[dtype][1]
    saved = _saved(_rand(dev, 90, rows, k, dtype=tdt))
    dy = _rand(dev, 91, rows, n, dtype=tdt)
    x = ref.stored(saved, rows, k)
    dw = Guarded(dev, torch.float32, k, n)
    _weight_grad(dtype, saved, dy, dw.t, 0, k)
    ref.check(dw.t, ref.weight_grad(x, dy), "dw")
    assert dw.intact()
    before = _rand(dev, 92, k, n)
    dw.t.copy_(before)
    _weight_grad(dtype, saved, dy, dw.t, 1, k)
    ref.check(dw.t, ref.weight_grad(x, dy, before), "dw added to")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n", WEIGHTS)
def test_weight_grad_of_whole_numbers_is_exact(gpu_device, dtype, rows, k, n):
    """Sums that fp32 holds: any term lost, counted twice or out of place shows."""
    dev, tdt = gpu_device, DT[dtype][1]
    g = _gen(dev, 93)
    x = torch.randint(-8, 9, (rows, k), generator=g, device=dev).to(tdt)
    dy = torch.randint(-100, 101, (rows, n), generator=g, device=dev).to(tdt)
    saved = _saved(x)
    dw = torch.full((k, n), math.nan, device=dev)
    _weight_grad(dtype, saved, dy, dw, 0, k)
    want = x.double().T @ dy.double()
    assert torch.equal(dw.double(), want)
    _weight_grad(dtype, saved, dy, dw, 1, k)
    assert torch.equal(dw.double(), 2 * want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n,off", [(100, 64, 48, 0), (300, 200, 136, 0), (300, 200, 136, 1), (520, 2048, 1088, 0), (260, 2048, 1088, 3),
                                            (150, 2100, 3800, 0), (150, 2100, 3800, 2)])
def test_weight_grad_of_columns_of_wider_tensors(gpu_device, dtype, rows, k, n, off):
    """dy and dw with row strides, off 16 bytes too; what lies beside is neither read into the result (it is NaN) nor written."""
    dev, tdt = gpu_device, DT[dtype][1]
    wide = torch.full((rows + 2, n + 24), math.nan, dtype=tdt, device=dev)
    dy = wide[1:rows + 1, 8 + off:8 + off + n]
    dy.copy_(_rand(dev, 94, rows, n))
    saved = _saved(_rand(dev, 95, rows, k, dtype=tdt))
    field = torch.full((k + 2, n + 24), MARK, device=dev)
    dw = field[1:k + 1, 4 + off:4 + off + n]
    _weight_grad(dtype, saved, dy, dw, 0, k)
    ref.check(dw, ref.weight_grad(ref.stored(saved, rows, k), dy), "dw")
    dw.fill_(MARK)
    assert bool((field == MARK).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n,off", [(16384, 64, 64, 0), (16384, 64, 64, 1), (5000, 65, 77, 1), (700, 100, 120, 0), (700, 100, 120, 3), (3000, 136, 2048, 1),
                                          (2391, 136, 6368, 0), (3414, 7120, 528, 0)])
def test_weight_grad_of_columns_of_wider_tensors_in_splits(gpu_device, dtype, rows, k, n, off):
    """Sums over splits of dy and dw with row strides: more than eight of them, fewer, of small, of middle (fp32) and of wide tiles; whole numbers, exactly, made
    and added to; what lies beside dy is NaN, what lies beside dw is left alone."""
    dev, tdt = gpu_device, DT[dtype][1]
    g = _gen(dev, 140)
    x = torch.randint(-8, 9, (rows, k), generator=g, device=dev).to(tdt)
    values = torch.randint(-100, 101, (rows, n), generator=g, device=dev).to(tdt)
    wide = torch.full((rows + 2, n + 24), math.nan, dtype=tdt, device=dev)
    dy = wide[1:rows + 1, 8 + off:8 + off + n]
    dy.copy_(values)
    saved = _saved(x)
    want = x.double().T @ values.double()
    field = torch.full((k + 2, n + 24), MARK, device=dev)
    dw = field[1:k + 1, 4 + off:4 + off + n]
    dw.fill_(math.nan)
    _weight_grad(dtype, saved, dy, dw, 0, k)
    assert torch.equal(dw.double(), want)
    _weight_grad(dtype, saved, dy, dw, 1, k)
    assert torch.equal(dw.double(), 2 * want)
    dw.fill_(MARK)
    assert bool((field == MARK).all())


@pytest.mark.parametrize("rows,k,n", [(1, 40, 24), (2, 2048, 2048), (1, 96, 33)])
@pytest.mark.parametrize("exponent", [-100, -105, -109, -118, -126])
def test_weight_grad_of_small_gradients(gpu_device, rows, k, n, exponent):
    """fp32 dy whose lower bf16 terms are under the normal numbers, and X large enough for a lost one to show: every bit of it down to 2^-110, below that all but
    what is under 2^-133."""
    dev = gpu_device
    bits = torch.randint(0, 1 << 23, (rows, n), generator=_gen(dev, 141), device=dev, dtype=torch.int32)
    dy = (bits | ((exponent + 127) << 23)).view(torch.float32)
    dy[:, ::2] *= -1
    saved = _saved(_rand(dev, 142, rows, k) * 2.0 ** 60)
    x = ref.stored(saved, rows, k)
    dw = torch.empty(k, n, device=dev)
    _weight_grad("f32", saved, dy, dw, 0, k)
    want = ref.weight_grad(x, dy)
    if exponent < -110:
        want = ref.Near(want.v, want.e + x.abs().sum(0)[:, None] * 2.0 ** -133)
    ref.check(dw, want, "dw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_grad_workspace_kept_from_more_rows(gpu_device, dtype):
    dev, tdt, k, n = gpu_device, DT[dtype][1], 192, 80
    code = DT[dtype][0]
    ws = torch.full((po.po_op_weight_grad_saved8_workspace(code, 5000, k, n) + EDGE,), 255, dtype=torch.uint8, device=dev)
    for rows in (5000, 3000, 700, 130, 3):
        ws[po.po_op_weight_grad_saved8_workspace(code, rows, k, n):] = 255
        saved, dy = _saved(_rand(dev, 96, rows, k, dtype=tdt)), _rand(dev, 97, rows, n, dtype=tdt)
        dw = torch.empty(k, n, device=dev)
        _weight_grad(dtype, saved, dy, dw, 0, k, workspace=ws)
        ref.check(dw, ref.weight_grad(ref.stored(saved, rows, k), dy), f"dw of {rows} rows")


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3.3e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,n", [(100, 48, 64), (300, 2048, 1152), (90, 2100, 3800), (1500, 33, 133), (700, 2050, 2051)])
def test_weight_grad_special_values(gpu_device, dtype, rows, k, n, value):
    """One value that is not finite, or near the largest, in dy: its column alone, with the infinity that the formula has; in X: its row alone."""
    dev, tdt = gpu_device, DT[dtype][1]
    x, dy = _rand(dev, 98, rows, k).abs().add(0.5).to(tdt), _rand(dev, 99, rows, n, dtype=tdt)
    clean, got = torch.empty(k, n, device=dev), torch.empty(k, n, device=dev)
    _weight_grad(dtype, _saved(x), dy, clean, 0, k)
    dy2 = dy.clone()
    dy2[rows // 2, 5] = value
    _weight_grad(dtype, _saved(x), dy2, got, 0, k)
    keep = torch.arange(n, device=dev) != 5
    assert torch.equal(got[:, keep], clean[:, keep])
    if abs(value) == math.inf:
        assert bool((got[:, 5] == value).all())
    elif value != value:
        assert bool(got[:, 5].isnan().all())
    else:
        big = float(torch.tensor(value).to(tdt))
        held = ref.stored(_saved(x), rows, k)[rows // 2]
        fits = held * big < 3.4e38
        torch.testing.assert_close(got[fits, 5].double(), (held * big)[fits], rtol=1e-6, atol=0)
        assert bool((got[held * big > 3.5e38, 5] == math.inf).all())
    if abs(value) == math.inf or value != value:
        x2 = x.clone()
        x2[rows // 2, 7] = value
        _weight_grad(dtype, _saved(x2), dy, got, 0, k)
        assert bool(got[7].isnan().all())
        keep = torch.ones(k, dtype=torch.bool, device=dev)
        keep[7] = False  # the others of its block keep their own scale only where the value was not its largest
        keep[:32] = False
        assert torch.equal(got[keep], clean[keep])


def test_weight_grad_offsets_past_32_bits(gpu_device):
    """dy of 2^31 values and more; rows that hold something at both ends only."""
    dev, rows, k, n = gpu_device, 70000, 40, 32768
    x = torch.zeros(rows, k, dtype=torch.bfloat16, device=dev)
    dy = torch.zeros(rows, n, dtype=torch.bfloat16, device=dev)
    g = _gen(dev, 130)
    some = torch.cat([torch.arange(3), torch.arange(rows - 5, rows)]).to(dev)
    x[some] = torch.randint(-8, 9, (8, k), generator=g, device=dev).to(torch.bfloat16)
    dy[some] = torch.randint(-100, 101, (8, n), generator=g, device=dev).to(torch.bfloat16)
    dw = torch.empty(k, n, device=dev)
    _weight_grad("bf16", _saved(x), dy, dw, 0, k)
    assert torch.equal(dw.double(), x[some].double().T @ dy[some].double())


def test_join_offsets_past_32_bits(gpu_device):
    """Rows at the end of tensors of more than 2^31 values, forward and backward, against a call on those rows alone."""
    dev, rows, h, last = gpu_device, 270000, 8192, 7
    p = _params(dev, torch.bfloat16, h, rows, True, True, "columns")
    x = torch.full((rows, h), 0.5, dtype=torch.bfloat16, device=dev)
    f, y = torch.full_like(x, 0.25), torch.empty_like(x)
    x[-last:], f[-last:] = _rand(dev, 131, last, h).to(x.dtype), _rand(dev, 132, last, h).to(x.dtype)
    forward = lambda x, f, y, n: po.po_op_norm_join_forward(po.PO_BF16, po.PO_NORM_RMS, x, f, p["post_gain"], None, p["gate"], 0, p["skip"], p["branch"], p["pre_gain"],
                                                           None, y, n, None, None, x.shape[0], h, p["eps"])
    fx, ff = x[-last:].clone(), f[-last:].clone()
    fy, fn = torch.empty_like(fx), torch.empty_like(fx)
    forward(fx, ff, fy, fn)
    forward(x, f, y, f)
    assert torch.equal(y[-last:], fy) and torch.equal(f[-last:], fn)
    assert torch.equal(y[0], y[rows // 2]) and torch.equal(f[0], f[rows - last - 1])

    def backward(dy, dn, y, f):
        sums = torch.zeros(3, h, device=dev)
        ws = torch.empty(po.po_op_norm_join_backward_workspace(y.shape[0], h), dtype=torch.uint8, device=dev)
        po.po_op_norm_join_backward(po.PO_BF16, po.PO_NORM_RMS, dy, dn, y, 0, f, 0, p["post_gain"], None, p["gate"], 0, p["skip"], p["branch"], p["pre_gain"], None,
                                    dy, dn, sums[0], sums[1], None, sums[2], None, None, ws, y.shape[0], h, p["eps"])
        return sums

    dy, dn = torch.zeros_like(x), x  # (x is not needed again: the gradient of n, zero but at the end)
    dn.zero_()
    dy[-last:], dn[-last:] = _rand(dev, 133, last, h).to(x.dtype), _rand(dev, 134, last, h).to(x.dtype)
    gy, gn = dy[-last:].clone(), dn[-last:].clone()
    want = ref.join_backward(gy, gn, fy, ff, p | dict(pre_shift=None, post_shift=None), torch.bfloat16)
    backward(gy, gn, fy, ff)
    f[-last:] = ff
    sums = backward(dy, dn, y, f)
    assert torch.equal(dy[-last:], gy) and torch.equal(dn[-last:], gn)
    assert not dy[:-last].any() and not dn[:-last].any()
    for got, name in zip(sums, ("dgate", "dpost_gain", "dpre_gain")):  # the other rows add zeros
        ref.check(got, want[name], name)


# ---- together -----------------------------------------------------------------------------------------------------
def _layer(dev, dtype, rows, h, f, state=None):
    """A feed-forward block between two norms, forward and backward from checkpoints: the buffers, and a function that runs all of it."""
    code, tdt = DT[dtype]
    new = lambda *s, t=tdt: torch.zeros(*s, dtype=t, device=dev)
    room = lambda c: torch.zeros(po.po_op_saved8_bytes(rows, c), dtype=torch.uint8, device=dev)
    p = _params(dev, tdt, h, rows, True, True, "columns")
    w1, w2 = _rand(dev, 101, h, 2 * f, dtype=tdt, scale=h ** -0.5), _rand(dev, 102, f, h, dtype=tdt, scale=f ** -0.5)
    b = dict(p=p, w1=w1, w2=w2, x=_rand(dev, 103, rows, h, dtype=tdt), n0=_rand(dev, 104, rows, h, dtype=tdt), dy=_rand(dev, 105, rows, h, dtype=tdt),
             dn=_rand(dev, 106, rows, h, dtype=tdt), u=new(rows, 2 * f), a=new(rows, f), out=new(rows, h), y=new(rows, h), n=new(rows, h), n0_8=room(h), u8=room(2 * f),
             a8=room(f), f8=room(h), y8=room(h), dx=new(rows, h), df=new(rows, h), da=new(rows, f), du=new(rows, 2 * f), dn0=new(rows, h),
             sums=new(3, h, t=torch.float32), dw1=new(h, 2 * f, t=torch.float32), dw2=new(f, h, t=torch.float32))
    size = lambda k, n: po.po_op_weight_grad_saved8_workspace(code, rows, k, n)
    ws = [torch.empty(max(s, 16), dtype=torch.uint8, device=dev) for s in (po.po_op_norm_join_backward_workspace(rows, h), size(h, 2 * f), size(f, h))]

    def run():
        po.po_op_save8(code, [b["n0"]], [b["n0_8"]])
        po.po_op_gemm(code, 0, 0, rows, 2 * f, h, b["n0"], h, w1, 2 * f, out=b["u"])
        po.po_op_activation_forward(code, po.PO_ACT_SILU, 1, b["u"], b["a"], b["u8"], rows, f)
        po.po_op_save8(code, [b["a"]], [b["a8"]])
        po.po_op_gemm(code, 0, 0, rows, h, f, b["a"], f, w2, h, out=b["out"])
        po.po_op_norm_join_forward(code, po.PO_NORM_RMS, b["x"], b["out"], p["post_gain"], None, p["gate"], 0, p["skip"], p["branch"], p["pre_gain"], None, b["y"],
                                   b["n"], b["f8"], b["y8"], rows, h, p["eps"])
        b["sums"].zero_()
        po.po_op_norm_join_backward(code, po.PO_NORM_RMS, b["dy"], b["dn"], b["y8"], 1, b["f8"], 1, p["post_gain"], None, p["gate"], 0, p["skip"], p["branch"],
                                    p["pre_gain"], None, b["dx"], b["df"], b["sums"][0], b["sums"][1], None, b["sums"][2], None, None, ws[0], rows, h, p["eps"])
        po.po_op_weight_grad_saved8(code, b["a8"], b["df"], h, b["dw2"], h, 0, ws[2], rows, f, h)
        po.po_op_gemm(code, 0, 1, rows, f, h, b["df"], h, w2, h, out=b["da"])
        po.po_op_activation_backward(code, po.PO_ACT_SILU, 1, b["u8"], 1, b["da"], b["du"], None, rows, f)
        po.po_op_weight_grad_saved8(code, b["n0_8"], b["du"], 2 * f, b["dw1"], 2 * f, 0, ws[1], rows, h, 2 * f)
        po.po_op_gemm(code, 0, 1, rows, h, 2 * f, b["du"], 2 * f, w1, 2 * f, out=b["dn0"])

    return b, run


OUTPUTS = ("u", "a", "out", "y", "n", "dx", "df", "da", "du", "dn0", "sums", "dw1", "dw2")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,h,f", [(70, 64, 96), (300, 256, 512)])
def test_a_block_from_checkpoints(gpu_device, dtype, rows, h, f):
    """Every step against 64 bits of its own inputs as the step before left them."""
    code, tdt = DT[dtype]
    b, run = _layer(gpu_device, dtype, rows, h, f)
    run()
    p = b["p"]
    ref.check(b["a"], ref.activation_forward(b["u"], True, True, tdt), "a")
    want = ref.join_forward(b["x"], b["out"], p, tdt)
    ref.check(b["y"], want["y"], "y")
    ref.check(b["n"], want["n"], "n")
    want = ref.join_backward(b["dy"], b["dn"], ref.stored(b["y8"], rows, h), ref.stored(b["f8"], rows, h), p, tdt)
    for k, got in dict(dx=b["dx"], df=b["df"], dgate=b["sums"][0], dpost_gain=b["sums"][1], dpre_gain=b["sums"][2]).items():
        ref.check(got, want[k], k)
    ref.check(b["dw2"], ref.weight_grad(ref.stored(b["a8"], rows, f), b["df"]), "dw2")
    ref.check(b["du"], ref.activation_backward(ref.stored(b["u8"], rows, 2 * f), b["da"], True, True, tdt)["du"], "du")
    ref.check(b["dw1"], ref.weight_grad(ref.stored(b["n0_8"], rows, h), b["du"]), "dw1")
    for name, t in (("n0_8", "n0"), ("a8", "a"), ("u8", "u"), ("f8", "out"), ("y8", "y")):
        codes, scales = ref.encode(b[t])
        got = ref.split(b[name], *b[t].shape)
        assert torch.equal(got[0].cpu(), codes) and torch.equal(got[1].cpu(), scales), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_captured_and_replayed(gpu_device, dtype):
    """Replays with new inputs, eager work between them, each against the eager result."""
    dev = gpu_device
    b, run = _layer(dev, dtype, 300, 256, 512)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (1, 2, 3):
        for k in ("x", "n0", "dy", "dn"):
            b[k].copy_(_rand(dev, 200 + seed, *b[k].shape))
        for k in OUTPUTS:
            b[k].fill_(math.nan)
        b["sums"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: b[k].clone() for k in OUTPUTS}
        run()
        for k in OUTPUTS:
            assert torch.equal(got[k], b[k]), k


def test_two_blocks_on_two_streams(gpu_device):
    """Each with its own buffers, at once, many times: the same bits as alone."""
    dev = gpu_device
    blocks = [_layer(dev, dtype, 300, 256, 512) for dtype in ("bf16", "f32")]
    alone = []
    for b, run in blocks:
        run()
        torch.cuda.synchronize()
        alone.append({k: b[k].clone() for k in OUTPUTS})
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(10):
        for s, (_, run) in zip(streams, blocks):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (b, _), want in zip(blocks, alone):
        for k in OUTPUTS:
            assert torch.equal(b[k], want[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_are_those_of_differences(gpu_device, dtype):
    """sum(dy y + dn n) along random directions: central differences in 64 bits of the definition against the kernels' gradients, y and f in full."""
    dev, (code, tdt), rows, h = gpu_device, DT[dtype], 40, 200
    p = _params(dev, tdt, h, rows, False, True, "columns")
    x, f, dy, dn = (_rand(dev, 110 + k, rows, h, dtype=tdt) for k in range(4))
    names = ("post_gain", "post_shift", "pre_gain", "pre_shift", "gate")

    def loss(move, step):
        q = dict(p, **{k: p[k].double() + step * move[k] for k in names})
        out = ref.join_forward(x.double() + step * move["x"], f.double() + step * move["f"], q, torch.float32)
        return float((out["y"].v * dy.double()).sum() + (out["n"].v * dn.double()).sum())

    y = ref.join_forward(x, f, p, torch.float32)["y"].v.to(tdt)
    got = _join_backward(dev, dtype, dy, dn, y, f, p, rows, h, saved=False)
    want = ref.join_backward(dy, dn, y, f, p, tdt, again=True)
    full = ref.join_backward(dy, dn, ref.join_forward(x, f, p, torch.float32)["y"].v, f, p, tdt, again=True)  # y as the definition has it
    for name, grad in dict(x="dx", f="df", post_gain="dpost_gain", post_shift="dpost_shift", pre_gain="dpre_gain", pre_shift="dpre_shift", gate="dgate").items():
        move = {k: torch.zeros_like(t, dtype=torch.float64) for k, t in dict(p, x=x, f=f).items() if torch.is_tensor(t)}
        move[name] = _rand(dev, 120, *move[name].shape).double()
        step = 1e-5
        slope = (loss(move, step) - loss(move, -step)) / (2 * step)
        # the kernels' own bound, and what y's rounding to the type moves the gradient by
        tol = (want[grad].e + (want[grad].v - full[grad].v).abs()) * move[name].abs()
        assert abs(float((got[grad].double() * move[name]).sum()) - slope) <= float(tol.sum()) + 1e-6 * (abs(slope) + 1)
