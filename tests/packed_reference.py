"""Attention, norm and rotation of packed sequences in 64 bits, from their definitions, with how far a kernel may be off.

Bounds.  u is half a step of the stored type (bf16 2^-8, fp32 2^-24), e = 2^-24.  A score is a sum of dh products in fp32, off by
at most dh e times the sum of their absolute values, A at most; with the exponent's own roundings a probability is off by a relative
eps_p = e ((dh + 8) A + 16 + 4 max |lse|).  Products over n terms add (n + 8) e.  P and dS are rounded to the stored type before the second product.
Values below 2^-126 become 0 in fp32: each of the up to 2^14 terms of a sum here, factors of up to 2^10 on it, is off by no more than that, 2^-102 in all."""
import math

import torch

E = 2.0 ** -24
TINY = 2.0 ** -102


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def attention(qkv, d_o, lengths, h, a, akv, o=None, absent=None):
    """o, lse, dqkv in 64 bits and their bounds, of qkv [rows, ..] (any float type; bounds for its type) and d_o; rows of no sequence
    are NaN.  absent [rows]: keys whose scores are -inf whatever qkv says; rows that see no other key must be left out by the caller, with the
    gradients of the keys that they see."""
    dt, dev, rows, dh = qkv.dtype, qkv.device, qkv.shape[0], h // a
    u, hkv, group, scale = half_step(dt), akv * dh, a // akv, 1 / math.sqrt(dh)
    new = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=dev)
    r = dict(o=new(rows, h), lse=new(a, rows), dqkv=new(rows, h + 2 * hkv))
    t = {k: torch.zeros_like(v) for k, v in r.items()}
    at = 0
    for n in lengths:
        s, at = slice(at, at + n), at + n
        if n == 0:
            continue
        x, d = qkv[s].double(), d_o[s].double()
        heads = lambda y, k: y.reshape(n, k, dh).transpose(0, 1)
        q = heads(x[:, :h], a)
        k, v = (heads(y, akv).repeat_interleave(group, 0) for y in x[:, h:].split(hkv, 1))
        d = heads(d, a)
        hidden = torch.ones(n, n, dtype=torch.bool, device=dev).triu(1)
        if absent is not None:
            hidden |= absent[s] & ~(hidden | absent[s]).all(1, keepdim=True)
        sc = (q @ k.mT * scale).masked_fill(hidden, -math.inf)
        lse = torch.logsumexp(sc, -1)
        p = torch.exp(sc - lse[..., None])
        o = p @ v
        dp = d @ v.mT
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        A = max(1.0, float((q.abs() @ k.abs().mT * scale).max()))
        eps_p = E * ((dh + 8) * A + 16 + 4 * float(lse.abs().max()))
        sums = (n + 8) * E
        t_o = (u + eps_p + sums) * (p @ v.abs()) + u * o.abs() + TINY
        # delta is formed from the stored o
        t_delta = (d.abs() * (t_o + (dh + 8) * E * o.abs())).sum(-1, keepdim=True)
        t_ds = (u + eps_p) * ds.abs() + p * (t_delta + (dh + 8) * E * (d.abs() @ v.abs().mT) + 4 * E * (dp.abs() + delta.abs()))
        flat = lambda y: y.transpose(0, 1).reshape(n, -1)
        shared = lambda y: y.reshape(akv, group, n, dh).sum(1)
        dq, dk, dv = ds @ k * scale, shared(ds.mT @ q) * scale, shared(p.mT @ d)
        gs = sums + group * E
        t_dq = (t_ds + sums * ds.abs()) @ k.abs() * scale
        t_dk = shared((t_ds + gs * ds.abs()).mT @ q.abs()) * scale
        t_dv = shared(((u + eps_p + gs) * p).mT @ d.abs())
        r["o"][s], r["lse"][:, s] = flat(o), lse
        t["o"][s], t["lse"][:, s] = flat(t_o), eps_p + sums + 8 * E * lse.abs()
        r["dqkv"][s] = torch.cat([flat(dq), flat(dk), flat(dv)], 1)
        t["dqkv"][s] = torch.cat([flat(t_dq), flat(t_dk), flat(t_dv)], 1) + u * r["dqkv"][s].abs() + TINY
    return r, t


def turn(x, angle, neighbours, back=False):
    """x [rows, heads, dh] with its first pairs turned by angle [rows, pairs]."""
    n = angle.shape[1]
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None] * (-1 if back else 1)
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    y = x.clone()
    if neighbours:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a * c - b * s, a * s + b * c
    else:
        y[..., :n], y[..., n:2 * n] = a * c - b * s, a * s + b * c
    return y


def rotary(qkv, gain_q, gain_k, positions, inv_freq, axis_pairs, neighbours, h, a, akv, eps, d_out=None):
    """out, dqkv and the gains' gradients in 64 bits, and their bounds.  Every element of the result is a sum of at most two products of values that
    took a dozen roundings: 32 e of the sum of their absolute values is more than they can be off.  (A gradient through the norm is a difference: of its
    terms' absolute values.)  Angles reduced to a turn in fp32 are off by 2^-25 turns and the cosine by as much in radians: 8 e.  A gain's gradient is
    a sum of rows * heads terms."""
    dt, dev, dh = qkv.dtype, qkv.device, h // a
    u, hkv, held = half_step(dt), akv * dh, positions[0] >= 0
    axis = [i for i, n in enumerate(axis_pairs) for _ in range(n)]
    angle = positions[:, held].double().T[:, axis] * inv_freq.double()
    x = qkv[held].double()[:, :h + hkv].reshape(-1, a + akv, dh)
    gain = 1.0
    xn, r = x, torch.ones_like(x[..., :1])
    if gain_q is not None:
        gain = torch.cat([gain_q.double().expand(a, dh), gain_k.double().expand(akv, dh)])
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        xn = x * r
    absolute = lambda y: turn_abs(y, angle, neighbours)
    sums = E * (dh + 40)
    new = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=dev)
    res, tol = dict(out=new(*qkv.shape)), dict(out=torch.zeros(qkv.shape, dtype=torch.float64, device=dev))
    y = turn(xn * gain, angle, neighbours)
    v = qkv[held][:, h + hkv:].double()
    res["out"][held] = torch.cat([y.flatten(1), v], 1)
    tol["out"][held] = torch.cat([(u * y.abs() + sums * absolute((xn * gain).abs())).flatten(1), 0 * v], 1)
    if d_out is None:
        return res, tol
    d = d_out[held].double()
    g0 = d[:, :h + hkv].reshape(-1, a + akv, dh)
    g, g_abs = turn(g0, angle, neighbours, back=True), absolute(g0.abs())
    if gain_q is not None:
        t, t_abs = g * xn, g_abs * xn.abs()
        n_terms = x.shape[0] * a
        res["dgain_q"], res["dgain_k"] = t[:, :a].sum((0, 1)), t[:, a:].sum((0, 1))
        tol["dgain_q"], tol["dgain_k"] = ((sums + n_terms * E) * t_abs[:, i].sum((0, 1)) for i in (slice(0, a), slice(a, None)))
        w, w_abs = g * gain, g_abs * (gain if gain_q is None else gain.abs())
        dx = r * (w - xn * (w * xn).mean(-1, keepdim=True))
        t_dx = 3 * sums * r * (w_abs + xn.abs() * (w_abs * xn.abs()).mean(-1, keepdim=True))
    else:
        dx, t_dx = g, sums * g_abs
    res["dqkv"], tol["dqkv"] = new(*qkv.shape), torch.zeros(qkv.shape, dtype=torch.float64, device=dev)
    dv = d[:, h + hkv:]
    res["dqkv"][held] = torch.cat([dx.flatten(1), dv], 1)
    tol["dqkv"][held] = torch.cat([(t_dx + u * dx.abs()).flatten(1), 0 * dv], 1)
    return res, tol


def turn_abs(x, angle, neighbours):
    """The sums of absolute values that `turn` of x (not negative) adds."""
    n = angle.shape[1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    y = x.clone()
    for k in (0, 1):
        if neighbours:
            y[..., k:2 * n:2] = a + b
        else:
            y[..., k * n:(k + 1) * n] = a + b
    return y


def maps(lengths, rows):
    """starts, sequence, positions as lists, lengths cut as the library cuts them."""
    starts, seq, pos = [0], [-1] * rows, [-1] * rows
    for j, n in enumerate(lengths):
        end = min(rows, starts[-1] + max(0, n))
        for r in range(starts[-1], end):
            seq[r], pos[r] = j, r - starts[-1]
        starts.append(end)
    return starts, seq, pos
