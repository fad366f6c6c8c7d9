"""fp64 oracle of the norm of a site, the tail of a residual block and the 8-bit checkpoints.

Rows are sites; a field list is ((l, multiplicity), ...) in channel order.  Independent of the library: entry by
entry in numpy.
"""
import numpy as np

BLOCK = 32


def entries(fields):
    """(first channel, first field, fields, components) of every entry."""
    c = f = 0
    for l, m in fields:
        yield c, f, m, 2 * l + 1
        c += m * (2 * l + 1)
        f += m


def gate_fields(fields):
    g = sum(m for l, m in fields if l > 0)
    return tuple(fields) + (((0, g),) if g else ())


def spread(fields, p):
    """A value per field as one per channel."""
    if p is None:
        return 1.0
    return np.concatenate([np.repeat(np.asarray(p, np.float64)[f:f + m], d) for _, f, m, d in entries(fields)])


def by_field(fields, v):
    """Sums over the components of every field of a vector of channels."""
    return np.concatenate([v[c:c + m * d].reshape(m, d).sum(1) for c, _, m, d in entries(fields)])


def norm_hat(fields, x, eps):
    """xhat [n, C] and 1 / sqrt(v + eps) [n, C]."""
    x = np.asarray(x, np.float64)
    hat, r = np.empty_like(x), np.empty_like(x)
    for c, _, m, d in entries(fields):
        f = x[:, c:c + m * d]
        if d == 1:
            f = f - f.mean(1, keepdims=True)
        rr = 1 / np.sqrt((f * f).sum(1, keepdims=True) / m + eps)
        hat[:, c:c + m * d] = f * rr
        r[:, c:c + m * d] = rr
    return hat, r


def norm_forward(fields, x, gain=None, eps=1e-5):
    return norm_hat(fields, x, eps)[0] * spread(fields, gain)


def norm_backward(fields, x, dy, gain=None, eps=1e-5):
    """(dx, dgain)."""
    hat, r = norm_hat(fields, x, eps)
    dy = np.asarray(dy, np.float64)
    t = dy * spread(fields, gain)
    dx = np.empty_like(t)
    for c, _, m, d in entries(fields):
        s = slice(c, c + m * d)
        v = t[:, s] - hat[:, s] * ((t[:, s] * hat[:, s]).sum(1, keepdims=True) / m)
        if d == 1:
            v = v - t[:, s].mean(1, keepdims=True)
        dx[:, s] = r[:, s] * v
    return dx, by_field(fields, (dy * hat).sum(0))


def gate_factor(fields, u):
    """What the gated nonlinearity multiplies every regular channel of u (gates behind them) with."""
    C = sum(m * (2 * l + 1) for l, m in fields)
    out, g = np.empty((len(u), C)), C
    for c, _, m, d in entries(fields):
        if d == 1:
            out[:, c:c + m] = u[:, c:c + m] > 0
        else:
            out[:, c:c + m * d] = np.repeat(1 / (1 + np.exp(-u[:, g:g + m])), d, 1)
            g += m
    return out


def residual_forward(fields, y, h, scale=None, gain_post=None, eps=1e-5):
    """h_out before it is rounded."""
    u = norm_forward(gate_fields(fields), y, gain_post, eps)
    f = gate_factor(fields, u)
    return np.asarray(h, np.float64) + spread(fields, scale) * f * u[:, :f.shape[1]]


def residual_backward(fields, y, h_out, dh, dx=None, scale=None, gain_post=None, gain_next=None, eps=1e-5):
    """(dy, dh_in, dscale, dgain_post, dgain_next)."""
    full = gate_fields(fields)
    dh, dnext = np.asarray(dh, np.float64), None
    if dx is not None:
        back, dnext = norm_backward(fields, h_out, dx, gain_next, eps)
        dh = dh + back
    u = norm_forward(full, y, gain_post, eps)
    f = gate_factor(fields, u)
    C = f.shape[1]
    dg = dh * spread(fields, scale)
    du, g = np.zeros_like(u), C
    du[:, :C] = np.where(f == 0, 0, dg * f)   # a closed relu is a selection (sigmoids are above 0)
    for c, _, m, d in entries(fields):
        if d > 1:
            s = 1 / (1 + np.exp(-u[:, g:g + m]))
            du[:, g:g + m] = (dg[:, c:c + m * d] * u[:, c:c + m * d]).reshape(-1, m, d).sum(2) * s * (1 - s)
            g += m
    dy, dpost = norm_backward(full, y, du, gain_post, eps)
    return dy, dh, by_field(fields, (dh * f * u[:, :C]).sum(0)), dpost, dnext


def pack(fields, x):
    """(q int8 [n, C], exps uint8 [n, blocks]) of values exact in fp64."""
    x = np.asarray(x, np.float64)
    qs, es = [], []
    for c, _, m, d in entries(fields):
        for at in range(0, m * d, BLOCK):
            f = x[:, c + at:c + min(at + BLOCK, m * d)]
            bad = ~np.isfinite(f).all(1)
            f = np.where(bad[:, None], 0.0, f)
            amax = np.abs(f).max(1)
            mant, e = np.frexp(amax)                       # amax = mant 2^e, 1/2 <= mant < 1
            k = np.where(amax > 0, e - 7 + (mant > 127 / 128), -126)
            k = np.clip(k, -126, 121)                      # at 122 the largest values would be 64 2^122 = 2^128
            qs.append(np.clip(np.rint(np.ldexp(f, -k[:, None])), -127, 127).astype(np.int8))
            es.append(np.where(bad, 255, k + 127).astype(np.uint8))
    return np.concatenate(qs, 1), np.stack(es, 1)


def unpack(fields, q, exps):
    out, b = np.empty(q.shape), 0
    for c, _, m, d in entries(fields):
        for at in range(0, m * d, BLOCK):
            s = slice(c + at, c + min(at + BLOCK, m * d))
            k = exps[:, b].astype(np.int64) - 127
            out[:, s] = np.where(exps[:, b:b + 1] == 255, np.nan, np.ldexp(q[:, s].astype(np.float64), k[:, None]))
            b += 1
    return out
