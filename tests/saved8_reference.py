"""8-bit checkpoints and the operators around them in plain form, 64 bits, with a bound on how far fp32 may be off.

The bounds are a running error analysis: Near carries a value in 64 bits and how far a result computed in fp32 by the same formula can be from it.
u = 2^-24 is the largest relative error of one rounding to fp32; an operation adds one, and passes its operands' errors on by its derivative.  A
sum of N terms in any order is off by at most depth u times the sum of their magnitudes, depth the longest chain of additions that a term goes
through: in a row's sums up to 31 in a lane (32 values, the first of which is added to a zero), six over the wave, three over eight waves (the other eight of sixteen
places hold zeros), or 15, six and four over sixteen, so that 40 covers them.  Hardware exp2, rcp and rsq are good to 1 ulp
(2 u).  A result rounded to bf16 is off by half a step more, 2^-8 of it at most relative to the power of two below: torch.finfo(t).eps / 2."""
import math

import torch

U = 2.0 ** -24
ROW_DEPTH = 40
BLOCK = 32


# ---- the form -----------------------------------------------------------------------------------------------------
def padded(cols):
    return -(-cols // BLOCK) * BLOCK


def _grid():
    """The 127 magnitudes of e4m3, by code."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append((f / 8) * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return torch.tensor(out, dtype=torch.float64)


GRID = _grid()


def encode(x):
    """(codes, scale bytes) of x [rows, cols] on the CPU; codes by search in the table of magnitudes."""
    rows, cols = x.shape
    b = torch.zeros(rows, padded(cols), dtype=torch.float64)
    b[:, :cols] = x.double().cpu()
    b = b.view(rows, -1, BLOCK)
    finite = b.isfinite()
    most = torch.tensor(1.875, dtype=torch.float64) * 2.0 ** 127
    b = torch.where(finite, b.clamp(-most, most), b)
    amax = torch.where(finite, x_abs := b.abs(), torch.zeros_like(b)).amax(-1)
    e = torch.full(amax.shape, -117, dtype=torch.int64)
    for i, v in enumerate(amax.flatten().tolist()):
        k = -117
        if v > 448 * 2.0 ** -117:
            k = max(-117, math.frexp(v)[1] - 10)
            while v > 448 * 2.0 ** k:
                k += 1
        e.view(-1)[i] = k
    y = torch.where(finite, x_abs, torch.zeros_like(b)) * torch.exp2(-e.double())[..., None]
    hi = torch.searchsorted(GRID, y.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = GRID[hi] - y, y - GRID[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = torch.where(torch.signbit(b), code + 128, code)
    code = torch.where(finite, code, torch.full_like(code, 127))
    return code.flatten(1).to(torch.uint8), (e + 127).to(torch.uint8)


def decode(codes, scales, cols):
    """[rows, cols] in 64 bits; codes 127 and 255 are NaN."""
    c = codes.cpu().long()
    v = torch.where((c & 127) == 127, torch.full((), math.nan, dtype=torch.float64), GRID[(c & 127).clamp(max=126)])
    v = torch.where(c > 127, -v, v).view(codes.shape[0], -1, BLOCK)
    return (v * torch.exp2(scales.cpu().double() - 127)[..., None]).flatten(1)[:, :cols]


def split(buffer, rows, cols):
    n = rows * padded(cols)
    return buffer[:n].view(rows, -1), buffer[n:n + n // BLOCK].view(rows, -1)


def stored(buffer, rows, cols):
    """What a checkpoint holds, in 64 bits on the buffer's device."""
    return decode(*split(buffer, rows, cols), cols).to(buffer.device)


# ---- values with bounds -------------------------------------------------------------------------------------------
class Near:
    def __init__(self, v, e=0.0):
        self.v = v.double()
        self.e = e if torch.is_tensor(e) else torch.full_like(self.v, e)

    def _of(o):
        return o if isinstance(o, Near) else Near(torch.as_tensor(o, dtype=torch.float64))

    def __add__(self, o):
        o = Near._of(o)
        v = self.v + o.v.to(self.v.device)
        e = self.e + o.e.to(v.device)
        return Near(v, e + U * (v.abs() + e))

    def __neg__(self):
        return Near(-self.v, self.e)

    def __sub__(self, o):
        return self + -Near._of(o)

    def __mul__(self, o):
        o = Near._of(o)
        ov, oe = o.v.to(self.v.device), o.e.to(self.v.device)
        v, e = self.v * ov, self.v.abs() * oe + ov.abs() * self.e + self.e * oe
        return Near(v, e + U * (v.abs() + e) + 2.0 ** -149)

    def mean(self):
        """Over a row."""
        return Near(self.v.mean(-1, keepdim=True), self.e.mean(-1, keepdim=True) + (ROW_DEPTH + 2) * U * (self.v.abs() + self.e).mean(-1, keepdim=True))

    def root(self):
        """One over the square root: the slope is half the cube; the error is taken at the smallest argument there can be."""
        least = (self.v - self.e).clamp(min=1e-300)
        return Near(self.v ** -0.5, 0.5 * self.e * least ** -1.5 + 2 * U * self.v ** -0.5)

    def columns(self, depth):
        """The sum of every column."""
        return Near(self.v.sum(0), self.e.sum(0) + depth * U * (self.v.abs() + self.e).sum(0))

    def rounded(self, dtype):
        half = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0
        return Near(self.v, self.e + half * (self.v.abs() + self.e) + 2.0 ** -133)


def single(v):
    """A scale or eps as the entry points take it: a float."""
    return float(torch.tensor(v, dtype=torch.float32))


def normed(v, rms, eps):
    """(N(v), one over the root)."""
    eps = single(eps)
    if not rms:
        v = v - v.mean()
    r = ((v * v).mean() + eps).root()
    return v * r, r


def back(a, hat, r, rms):
    inner = a - hat * (a * hat).mean()
    if not rms:
        inner = inner - a.mean()
    return inner * r


def join_forward(x, f, p, dtype):
    """p: dict of rms, eps, skip, branch, gate, post_gain, post_shift, pre_gain, pre_shift (tensors or None)."""
    x, f = Near(x), Near(f)
    z = f
    if p["post_gain"] is not None:
        z = normed(f, p["rms"], p["eps"])[0] * p["post_gain"].double()
        if p["post_shift"] is not None:
            z = z + p["post_shift"].double()
    if p["gate"] is not None:
        z = z * p["gate"].double()
    y = x * single(p["skip"]) + z * single(p["branch"])
    out = {"y": y.rounded(dtype)}
    if p["pre_gain"] is not None:
        n = normed(y, p["rms"], p["eps"])[0] * p["pre_gain"].double()
        if p["pre_shift"] is not None:
            n = n + p["pre_shift"].double()
        out["n"] = n.rounded(dtype)
    return out


def join_backward(dy, dn, y, f, p, dtype, again=False):
    rms, eps, rows = p["rms"], p["eps"], f.shape[0] if f is not None else (dy if dy is not None else dn).shape[0]
    depth = rows / 256 + 40  # a block's rows one after another (256 blocks at least where there are as many rows), then the blocks'
    zero = torch.zeros_like(dy if dy is not None else dn)
    t, out = Near(dy if dy is not None else zero), {}
    if dn is not None:
        hat, r = normed(Near(y), rms, eps)
        d = Near(dn)
        out["dpre_gain"] = (d * hat).columns(depth)
        if p["pre_shift"] is not None:
            out["dpre_shift"] = d.columns(depth)
        t = t + back(d * p["pre_gain"].double(), hat, r, rms)
        if again:
            n = hat * p["pre_gain"].double()
            out["n"] = (n + p["pre_shift"].double() if p["pre_shift"] is not None else n).rounded(dtype)
    out["dx"] = (t * single(p["skip"])).rounded(dtype)
    w = t * single(p["branch"])
    fn = Near(f) if f is not None else None
    if p["post_gain"] is not None:
        fhat, fr = normed(fn, rms, eps)
    dz = w
    if p["gate"] is not None:
        z = fn
        if p["post_gain"] is not None:
            z = fhat * p["post_gain"].double()
            if p["post_shift"] is not None:
                z = z + p["post_shift"].double()
        dg = w * z
        out["dgate"] = dg.rounded(dtype) if p["gate"].dim() == 2 else dg.columns(depth)
        dz = w * p["gate"].double()
    if p["post_gain"] is not None:
        out["dpost_gain"] = (dz * fhat).columns(depth)
        if p["post_shift"] is not None:
            out["dpost_shift"] = dz.columns(depth)
        dz = back(dz * p["post_gain"].double(), fhat, fr, rms)
    out["df"] = dz.rounded(dtype)
    return out


# ---- activations --------------------------------------------------------------------------------------------------
def _curve(a, silu):
    """act(a), its slope, and bounds of both: the exponent's argument is off by 5 u of itself (a cubic in a), exp2 makes log(2) times that a relative error of the
    gate and of its complement, and exp2, 1 + e, rcp and the product add 8 u.  Under 2^-118 the gate counts as zero."""
    a = a.double()
    c = math.sqrt(2 / math.pi)
    z = a if silu else 2 * c * (a + 0.044715 * a ** 3)
    gate, rest = torch.sigmoid(z), torch.sigmoid(-z)
    slope_z = torch.ones_like(a) if silu else 2 * c * (1 + 3 * 0.044715 * a * a)
    off = (5 * z.abs().clamp(max=300) + 8) * U
    bend = a * rest * slope_z
    v, slope = a * gate, gate * (1 + bend)
    return v, slope, v.abs() * off + a.abs() * 2.0 ** -118, gate * (1 + bend.abs()) * 2 * (off + 4 * U) + 2.0 ** -100 * (1 + bend.abs())


def activation_forward(u, silu, gated, dtype):
    f = u.shape[1] // 2 if gated else u.shape[1]
    v, _, e, _ = _curve(u[:, :f], silu)
    out = Near(v, e)
    return (out * u[:, f:].double() if gated else out).rounded(dtype)


def activation_backward(u, d, silu, gated, dtype):
    f = u.shape[1] // 2 if gated else u.shape[1]
    v, slope, ev, es = _curve(u[:, :f], silu)
    v, slope, d = Near(v, ev), Near(slope, es), Near(d)
    if gated:
        b = Near(u[:, f:])
        parts = [(d * slope) * b, d * v]
        du = Near(torch.cat([q.v for q in parts], 1), torch.cat([q.e for q in parts], 1))
        return {"du": du.rounded(dtype), "out": (v * b).rounded(dtype)}
    return {"du": (d * slope).rounded(dtype), "out": v.rounded(dtype)}


# ---- weight gradient ----------------------------------------------------------------------------------------------
def weight_grad(x, dy, before=None):
    """Exact products; a sum of `rows` terms (three for each row where dy is fp32) in any order: each term goes through at most as many additions."""
    x, d = x.double(), dy.double()
    terms = x.shape[0] * (3 if dy.dtype == torch.float32 else 1) + 70
    v, mag = x.T @ d, x.abs().T @ d.abs()
    if before is not None:
        v, mag = v + before.double(), mag + before.double().abs()
    return Near(v, terms * U * mag + 2.0 ** -120)


def check(got, want, what):
    bad = ~((got.double() - want.v).abs() <= want.e)
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])} for {float(want.v[i])} +- {float(want.e[i])}")
