"""The norm of a site and the tail of a residual block on the GPU against the fp64 oracle: every field-list shape,
both types, rows and checkpoints, forward and gradients.

Tolerances count roundings (u = 2^-24). No sum over an entry is deeper than 32 additions, so a mean is off by 34 u of
the entry's largest magnitude A, and with r = 1 / sqrt(v + eps), e = 40 u (1 + A r) bounds the error of xhat by
e (1 + |xhat|) and the relative error of r by e. Errors of a formula's inputs are carried through it term by term; a
result in bf16 adds half a step, 2^-8 of itself. Inputs are standard normal, so nothing is near the types' ends.
"""
import numpy as np
import pytest

from oracle import site as os_
from workloads.gen import round_bf16

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2111_07383_amd")

DEV = "cuda:0"
EPS = 1e-5
U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16]

# field lists: widths off and on multiples of 8 and 32, entries narrower than 8, one scalar, no scalars, every order,
# the most entries and channels, rows of 1 to 1024
FIELDS = {
    "one": ((0, 1),),
    "tiny": ((0, 2), (1, 2)),
    "gate1": ((1, 1),),
    "f104": ((0, 16), (1, 16), (2, 8)),
    "f208": ((0, 32), (1, 32), (2, 16)),
    "ragged": ((0, 13), (1, 11), (2, 5)),
    "order4": ((4, 3), (0, 9), (3, 2), (0, 1)),
    "seven": ((0, 8), (1, 3), (0, 40), (2, 2), (1, 9), (3, 1), (4, 1)),
    "f36": ((0, 4), (1, 4), (2, 4)),
    "w52": ((0, 8), (1, 8), (2, 4)),                 # 52 + 12 gates: 64
    "w61": ((0, 33), (0, 28)),
    "w128": ((0, 40), (1, 10), (2, 8)),              # 110 + 18 gates: 128
    "w256": ((0, 128), (1, 24), (2, 4)),             # 220 + 28
    "w400": ((0, 100), (1, 50), (2, 30)),            # 400 + 80
    "w510": ((1, 127),),                             # 381 + 127
    "w900": ((0, 500), (1, 100), (2, 10)),           # 850 + 110
    "w1024": ((0, 496), (1, 100), (2, 16), (0, 32)),  # 908 + 116: all of the 1024, 129 chunks of 8
    # an entry under 8 channels in rows of more lanes and more chunks a lane
    "narrow16": ((0, 60), (1, 5), (2, 1)),
    "narrow32": ((0, 130), (1, 5), (2, 1), (0, 3)),
    "narrow64": ((0, 3), (0, 300), (1, 20), (2, 1)),
    "narrow128": ((0, 600), (1, 7), (2, 1), (0, 150)),
    "narrow192": ((0, 3), (0, 770), (1, 60), (2, 1)),  # 958 + 61: 130 chunks of 8
}
NORM_ONLY = {"eight": ((0, 3), (1, 2)) * 4, "all1024": ((0, 1024),), "vec1023": ((1, 341),),
             "odd1023": ((0, 129),) * 7 + ((0, 120),)}
ROWS = [1, 3, 37]


def channels(f):
    return sum(m * (2 * l + 1) for l, m in f)


def count(f):
    return sum(m for _, m in f)


def values(rng, n, C, dtype, shift=0.0):
    x = (rng.standard_normal((n, C)) + shift).astype(np.float32)
    return round_bf16(x) if dtype == torch.bfloat16 else x


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy()


def params(rng, f):
    return (1 + 0.3 * rng.standard_normal(count(f))).astype(np.float32)


def half_step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def spread_max(f, x):
    """The largest magnitude of the entry of every channel."""
    out = np.empty(x.shape)
    for c, _, m, d in os_.entries(f):
        out[:, c:c + m * d] = np.abs(x[:, c:c + m * d]).max(1, keepdims=True)
    return out


def spread_mean(f, v):
    """Sum over an entry's channels over its fields, by channel."""
    out = np.empty(v.shape)
    for c, _, m, d in os_.entries(f):
        out[:, c:c + m * d] = v[:, c:c + m * d].sum(1, keepdims=True) / m
    return out


def norm_err(f, x):
    """(xhat, r, bound of xhat's error, relative bound of r's)."""
    hat, r = os_.norm_hat(f, x, EPS)
    e = 40 * U * (1 + spread_max(f, x) * r)
    return hat, r, e * (1 + np.abs(hat)), e


def norm_back_err(f, x, t, dt):
    """Bound of the error of r (t - mean t - xhat mean(t xhat)) where t is off by dt."""
    hat, r, dhat, er = norm_err(f, x)
    at, ah = np.abs(t), np.abs(hat)
    a, b = spread_mean(f, at), spread_mean(f, at * ah)
    size = at + a + ah * b
    off = dt + spread_mean(f, dt) + ah * spread_mean(f, dt * ah + at * dhat) + dhat * b
    return r * (off + (er + 40 * U) * size)


def close(got, want, tol, what):
    got = host(got) if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - want) / tol)))


def row_sums(f, products, dproducts):
    """Bound of the error of a parameter's gradient: sums over rows and components in any order."""
    n = products.shape[0] * 9 + 64
    return os_.by_field(f, (dproducts + n * U * np.abs(products)).sum(0)) + 1e-30


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("name", list(FIELDS) + list(NORM_ONLY))
def test_norm(name, n, dtype):
    f = {**FIELDS, **NORM_ONLY}[name]
    C, rng = channels(f), np.random.default_rng(n)
    x, dy, dres = (values(rng, n, C, dtype, s) for s in (0.4, 0, 0))
    gain = params(rng, f)
    g = os_.spread(f, gain)
    hat, r, dhat, er = norm_err(f, x.astype(np.float64))
    want = hat * g
    y, kept = P.site_norm_forward(f, dev(x, dtype), dev(gain), EPS, checkpoint=True)
    close(y, want, half_step(dtype) * np.abs(want) + 1.01 * np.abs(g) * dhat + 1e-37, "y")
    q, e = os_.pack(f, x)
    assert np.array_equal(kept.q.cpu().numpy(), q) and np.array_equal(kept.exps.cpu().numpy(), e)
    assert torch.equal(P.site_norm_forward(f, dev(x, dtype), dev(gain), EPS), y)

    t = dy * g
    wdx, wdg = os_.norm_backward(f, x, dy, gain, EPS)
    wdx = wdx + dres
    tol = norm_back_err(f, x.astype(np.float64), t, U * np.abs(t)) + 2 * U * (np.abs(wdx) + np.abs(dres))
    dx, dgain = P.site_norm_backward(f, dev(x, dtype), dev(dy, dtype), dev(gain), EPS, dres=dev(dres, dtype))
    close(dx, wdx, tol + half_step(dtype) * np.abs(wdx) + 1e-37, "dx")
    close(dgain, wdg, row_sums(f, dy * hat, np.abs(dy) * dhat), "dgain")
    dx0, none = P.site_norm_backward(f, dev(x, dtype), dev(dy, dtype), eps=EPS)
    w0 = os_.norm_backward(f, x, dy, None, EPS)[0]
    close(dx0, w0, norm_back_err(f, x.astype(np.float64), dy.astype(np.float64), 0 * dy) + (half_step(dtype) + U) * np.abs(w0) + 1e-37, "dx without gain")
    assert none is None

    # from the checkpoint: the same formulas at the values that it stands for
    v = os_.unpack(f, q, e)
    hat, r, dhat, er = norm_err(f, v)
    close(P.site_norm_forward(f, kept, dev(gain), EPS, dtype=dtype), hat * g,
          half_step(dtype) * np.abs(hat * g) + 1.01 * np.abs(g) * dhat + 1e-37, "y of the checkpoint")
    dx, dgain = P.site_norm_backward(f, kept, dev(dy, dtype), dev(gain), EPS)
    wdx, wdg = os_.norm_backward(f, v, dy, gain, EPS)
    close(dx, wdx, norm_back_err(f, v, t, U * np.abs(t)) + (half_step(dtype) + U) * np.abs(wdx) + 1e-37, "dx of the checkpoint")
    close(dgain, wdg, row_sums(f, dy * hat, np.abs(dy) * dhat), "dgain of the checkpoint")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("name", list(FIELDS))
def test_residual_forward(name, n, dtype):
    f = FIELDS[name]
    full = os_.gate_fields(f)
    C, S, rng = channels(f), channels(full), np.random.default_rng(n + 1)
    y, h = values(rng, n, S, dtype, 0.4), values(rng, n, C, dtype, 0.2)
    sc, gp, gn = params(rng, f), params(rng, full), params(rng, f)
    ho, x, yk, hk = P.residual_forward(f, dev(y, dtype), dev(h, dtype), dev(sc), dev(gp), dev(gn), EPS, checkpoint=True)

    hat, _, dhat, _ = norm_err(full, y.astype(np.float64))
    g = os_.spread(full, gp)
    u, du = hat * g, 1.01 * np.abs(g) * dhat + U * np.abs(hat * g)
    fac = os_.gate_factor(f, u)
    dfac, gi = np.zeros((n, C)), C
    for c, _, m, d in os_.entries(f):
        if d > 1:   # sigmoid' <= 1/4, and the exponential and the division to 2^-20
            dfac[:, c:c + m * d] = np.repeat(du[:, gi:gi + m] / 4 + 2.0 ** -20, d, 1)
            gi += m
    s = np.abs(os_.spread(f, sc))
    want = os_.residual_forward(f, y, h, sc, gp, EPS)
    tol = s * (du[:, :C] + np.abs(u[:, :C]) * dfac + 4 * U * np.abs(u[:, :C])) + 2 * U * (np.abs(want) + np.abs(h))
    close(ho, want, 1.01 * tol + half_step(dtype) * np.abs(want), "h")

    hv = host(ho)    # the next norm and the checkpoint are those of the rows that were returned
    hat, _, dhat, _ = norm_err(f, hv)
    g = os_.spread(f, gn)
    close(x, hat * g, half_step(dtype) * np.abs(hat * g) + 1.01 * np.abs(g) * dhat + 1e-37, "x")
    for kept, fl, v in ((yk, full, y), (hk, f, hv)):
        q, e = os_.pack(fl, v)
        assert kept.fields == fl
        assert np.array_equal(kept.q.cpu().numpy(), q) and np.array_equal(kept.exps.cpu().numpy(), e)

    # without options, and into h's own buffer
    h0, none, *rest = P.residual_forward(f, dev(y, dtype), dev(h, dtype), dev(sc), dev(gp), eps=EPS, next_norm=False)
    assert torch.equal(h0, ho) and none is None and rest == [None, None]
    hin = dev(h, dtype)
    h1, x1, *_ = P.residual_forward(f, dev(y, dtype), hin, dev(sc), dev(gp), dev(gn), EPS, out=hin)
    assert h1 is hin and torch.equal(h1, ho) and torch.equal(x1, x)
    plain, *_ = P.residual_forward(f, dev(y, dtype), dev(h, dtype), eps=EPS)
    ones, *_ = P.residual_forward(f, dev(y, dtype), dev(h, dtype), torch.ones(count(f), device=DEV),
                                  torch.ones(count(full), device=DEV), torch.ones(count(f), device=DEV), EPS)
    assert torch.equal(plain, ones)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("name", list(FIELDS))
def test_residual_backward(name, n, packed, dtype):
    f = FIELDS[name]
    full = os_.gate_fields(f)
    C, S, rng = channels(f), channels(full), np.random.default_rng(n + 2)
    y, h = values(rng, n, S, dtype, 0.4), values(rng, n, C, dtype, 0.2)
    dh, dx = values(rng, n, C, dtype), values(rng, n, C, dtype)
    sc, gp, gn = params(rng, f), params(rng, full), params(rng, f)
    yt, ht = dev(y, dtype), dev(h, dtype)
    if packed:
        yt, ht = P.pack(full, yt), P.pack(f, ht)
        y, h = os_.unpack(full, *os_.pack(full, y)), os_.unpack(f, *os_.pack(f, h))
    y, h = y.astype(np.float64), h.astype(np.float64)
    hat, _, dhat, _ = norm_err(full, y)
    g = os_.spread(full, gp)
    u, eu = hat * g, 1.01 * np.abs(g) * dhat + U * np.abs(hat * g)
    scalar = np.concatenate([np.full(m * d, d == 1) for _, _, m, d in os_.entries(f)])
    border = (np.abs(u[:, :C]) <= eu[:, :C]) & scalar   # relu' may be either there
    got = P.residual_backward(f, yt, ht, dev(dh, dtype), dev(dx, dtype), dev(sc), dev(gp), dev(gn), EPS)
    want = os_.residual_backward(f, y, h, dh, dx, sc, gp, gn, EPS)

    hhat, _, dhhat, _ = norm_err(f, h)
    tn = dx * os_.spread(f, gn)
    edh = norm_back_err(f, h, tn, U * np.abs(tn)) + 2 * U * (np.abs(want[1]) + np.abs(dh))
    close(got[1], want[1], 1.01 * edh + half_step(dtype) * np.abs(want[1]) + 1e-37, "dh")
    fac = os_.gate_factor(f, u)
    efac, ew, gi = np.zeros((n, C)), np.zeros((n, S)), C
    s = os_.spread(f, sc)
    dg = want[1] * s
    edg = 1.01 * np.abs(s) * edh + U * np.abs(dg)
    uc, euc = u[:, :C], eu[:, :C]
    du = np.zeros((n, S))
    du[:, :C] = dg * fac
    for c, _, m, d in os_.entries(f):
        if d == 1:
            continue
        k = slice(c, c + m * d)
        sig = 1 / (1 + np.exp(-u[:, gi:gi + m]))
        esig = eu[:, gi:gi + m] / 4 + 2.0 ** -20
        efac[:, k] = np.repeat(esig, d, 1)
        dot = (dg[:, k] * uc[:, k]).reshape(n, m, d).sum(2)
        edot = (edg[:, k] * np.abs(uc[:, k]) + np.abs(dg[:, k]) * euc[:, k] + 10 * U * np.abs(dg[:, k] * uc[:, k])).reshape(n, m, d).sum(2)
        du[:, gi:gi + m] = dot * sig * (1 - sig)
        ew[:, gi:gi + m] = edot / 4 + np.abs(dot) * 1.01 * esig + 4 * U * np.abs(dot)
        gi += m
    ew[:, :C] = edg * fac + np.abs(dg) * (efac + border) + 2 * U * np.abs(du[:, :C])
    t = du * g
    tol = norm_back_err(full, y, t, 1.01 * np.abs(g) * ew + U * np.abs(t))
    close(got[0], want[0], 1.02 * tol + (half_step(dtype) + U) * np.abs(want[0]) + 1e-37, "dy")
    prod = want[1] * fac * uc
    eprod = edh * np.abs(fac * uc) + np.abs(want[1]) * (efac * np.abs(uc) + fac * euc) + 4 * U * np.abs(prod)
    close(got[2], want[2], 1.02 * row_sums(f, prod, eprod), "dscale")
    close(got[3], want[3], 1.02 * row_sums(full, du * hat, ew * np.abs(hat) + np.abs(du) * dhat), "dgain_post")
    close(got[4], want[4], 1.02 * row_sums(f, dx * hhat, np.abs(dx) * dhhat), "dgain_next")

    # without a next norm
    got = P.residual_backward(f, yt, None, dev(dh, dtype), None, dev(sc), dev(gp), None, EPS)
    assert torch.equal(got[1], dev(dh, dtype)) and got[4] is None
    want = os_.residual_backward(f, y, None, dh, None, sc, gp, None, EPS)
    close(got[2], want[2], row_sums(f, dh * fac * uc, np.abs(dh) * (efac * np.abs(uc) + fac * euc) + 4 * U * np.abs(dh * fac * uc)), "dscale alone")


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows(dtype):
    """More rows than workgroups, every row against the same row alone; sums over all of them."""
    f = FIELDS["f104"]
    full, n = os_.gate_fields(f), 70001
    rng = np.random.default_rng(9)
    y, h = dev(values(rng, n, 128, dtype), dtype), dev(values(rng, n, 104, dtype), dtype)
    dh, dx = dev(values(rng, n, 104, dtype), dtype), dev(values(rng, n, 104, dtype), dtype)
    sc, gp, gn = (dev(params(rng, k)) for k in (f, full, f))
    ho, x, yk, hk = P.residual_forward(f, y, h, sc, gp, gn, EPS, checkpoint=True)
    back = P.residual_backward(f, yk, hk, dh, dx, sc, gp, gn, EPS)
    at = [0, 1, 63, 64, 4096, 8191, 8192, 65535, 65536, n - 2, n - 1]
    for a in at:
        s = slice(a, a + 1)
        one = P.residual_forward(f, y[s].clone(), h[s].clone(), sc, gp, gn, EPS, checkpoint=True)
        assert torch.equal(one[0], ho[s]) and torch.equal(one[1], x[s])
        assert torch.equal(one[2].q, yk.q[s]) and torch.equal(one[3].exps, hk.exps[s])
        b1 = P.residual_backward(f, one[2], one[3], dh[s].clone(), dx[s].clone(), sc, gp, gn, EPS)
        assert torch.equal(b1[0], back[0][s]) and torch.equal(b1[1], back[1][s])
    again = P.residual_backward(f, yk, hk, dh, dx, sc, gp, gn, EPS)
    for a, b in zip(back, again):
        assert torch.equal(a, b)
    # the parameters' gradients, against those of parts of the rows: 8 parts, each sum at most 70001 * 5 terms of size
    # ~1 in random order of fp32 partials; both are within 1e-4 of the sum of magnitudes / sqrt(rows)
    parts = [P.residual_backward(f, P.Packed(full, yk.q[i::8].contiguous(), yk.exps[i::8].contiguous()),
                                 P.Packed(f, hk.q[i::8].contiguous(), hk.exps[i::8].contiguous()),
                                 dh[i::8].contiguous(), dx[i::8].contiguous(), sc, gp, gn, EPS) for i in range(8)]
    for k in (2, 3, 4):
        whole = sum(p[k].double() for p in parts)
        assert float((back[k].double() - whole).abs().max()) <= 1e-4 * n ** 0.5 * 5
    nx, ndg = P.site_norm_backward(f, h, dx, gn, EPS, dres=dh)
    ref = os_.norm_backward(f, host(h), host(dx), host(gn), EPS)
    assert float(np.abs(host(ndg) - ref[1]).max()) <= 1e-4 * n ** 0.5 * 5
    close(nx[-3:], (ref[0] + host(dh))[-3:], (half_step(dtype) + 1e-5) * (np.abs(ref[0]) + np.abs(host(dh)) + 1)[-3:], "last rows")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["ragged", "f104", "w400", "gate1", "tiny", "order4", "f36", "narrow64", "w900", "narrow192"])
def test_views_off_alignment(name, dtype):
    """Buffers that start at any element give the same bits, and nothing outside them is written."""
    f = FIELDS[name]
    full, n = os_.gate_fields(f), 19
    C, S, rng = channels(f), channels(full), np.random.default_rng(10)

    def shifted(t, k=1):
        b = torch.full((t.numel() + 16,), 7, dtype=t.dtype, device=DEV)
        v = b[k:k + t.numel()].view(t.shape)
        v.copy_(t)
        return v, b, k

    y, h, dh, dx = (dev(values(rng, n, c, dtype), dtype) for c in (S, C, C, C))
    sc, gp, gn = (dev(params(rng, k)) for k in (f, full, f))
    ref = P.residual_forward(f, y, h, sc, gp, gn, EPS, checkpoint=True)
    out, buf, k = shifted(torch.zeros_like(h), 3)
    got = P.residual_forward(f, shifted(y)[0], shifted(h)[0], shifted(sc)[0], shifted(gp)[0], shifted(gn)[0], EPS,
                             checkpoint=True, out=out)
    for a, b in zip(ref[:2], got[:2]):
        assert torch.equal(a, b)
    assert torch.equal(ref[2].q, got[2].q) and torch.equal(ref[3].q, got[3].q)
    assert bool((buf[:k] == 7).all()) and bool((buf[k + n * C:] == 7).all())
    yk, hk = ref[2], ref[3]
    ys = P.Packed(full, shifted(yk.q, 3)[0], shifted(yk.exps, 1)[0])
    hs = P.Packed(f, shifted(hk.q, 5)[0], shifted(hk.exps, 1)[0])
    a = P.residual_backward(f, yk, hk, dh, dx, sc, gp, gn, EPS)
    b = P.residual_backward(f, ys, hs, shifted(dh)[0], shifted(dx, 5)[0], sc, gp, gn, EPS)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    out, buf, k = shifted(torch.zeros_like(h), 5)
    a = P.site_norm_backward(f, h, dx, gn, EPS, dres=dh)
    b = P.site_norm_backward(f, shifted(h)[0], shifted(dx)[0], gn, EPS, dres=shifted(dh, 3)[0], out=out)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool((buf[:k] == 7).all()) and bool((buf[k + n * C:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["ragged", "gate1", "order4", "f36", "narrow64", "narrow192"])
def test_in_place(name, dtype):
    f, n = FIELDS[name], 300
    full = os_.gate_fields(f)
    C, S, rng = channels(f), channels(full), np.random.default_rng(11)
    x, dy, dres = (dev(values(rng, n, C, dtype), dtype) for _ in range(3))
    gain = dev(params(rng, f))
    y = P.site_norm_forward(f, x, gain, EPS)
    b = x.clone()
    assert torch.equal(P.site_norm_forward(f, b, gain, EPS, out=b), y)
    ref, _ = P.site_norm_backward(f, x, dy, gain, EPS, dres=dres)
    for which in ("dy", "dres"):
        d, r = dy.clone(), dres.clone()
        got, _ = P.site_norm_backward(f, x, d, gain, EPS, dres=r, out=d if which == "dy" else r)
        assert torch.equal(got, ref)


@pytest.mark.parametrize("dtype", DTYPES)
def test_non_finite_and_zero_rows(dtype):
    """A NaN or an infinity stays in its entry of its row (and a gate's in what it gates); rows of zeros are zeros."""
    f, n = FIELDS["f104"], 40
    full = os_.gate_fields(f)
    rng = np.random.default_rng(12)
    y, h = values(rng, n, 128, dtype), values(rng, n, 104, dtype)
    clean = P.residual_forward(f, dev(y, dtype), dev(h, dtype), eps=EPS, checkpoint=True)
    y2, h2 = y.copy(), h.copy()
    y2[5, 3] = np.nan       # a scalar: the 16 scalars
    y2[6, 20] = np.inf      # a vector component: inf / inf there, 0 for the entry's others
    y2[7, 104 + 2] = -np.inf    # a gate: every gated field
    h2[8, 70] = np.nan      # the stream: that channel, and the order-2 fields of the next norm
    y2[9], h2[9] = 0, 0
    ho, x, yk, hk = P.residual_forward(f, dev(y2, dtype), dev(h2, dtype), eps=EPS, checkpoint=True)
    nan_h, nan_x = np.isnan(host(ho)), np.isnan(host(x))
    want = np.zeros((n, 104), bool)
    want[5, :16] = want[7, 16:] = True
    want[6, 20] = want[8, 70] = True
    assert np.array_equal(nan_h, want)
    want[6, 16:64] = want[8, 64:] = True
    assert np.array_equal(nan_x, want)
    assert torch.equal(ho[9], torch.zeros_like(ho[9])) and torch.equal(x[9], torch.zeros_like(x[9]))
    rows = [i for i in range(n) if i not in (5, 6, 7, 8, 9)]
    assert torch.equal(ho[rows], clean[0][rows]) and torch.equal(x[rows], clean[1][rows])
    assert bool((yk.exps == 255).any()) and int((yk.exps == 255).sum()) == 3
    dh, dx = dev(values(rng, n, 104, dtype), dtype), dev(values(rng, n, 104, dtype), dtype)
    a = P.residual_backward(f, clean[2], clean[3], dh, dx, eps=EPS)
    b = P.residual_backward(f, yk, hk, dh, dx, eps=EPS)
    assert torch.equal(a[0][rows], b[0][rows]) and torch.equal(a[1][rows], b[1][rows])
    assert bool(torch.isnan(b[0][5, :16]).all()) and bool(torch.isfinite(b[0][9]).all())
    assert bool(torch.isnan(b[1][8, 64:]).all()) and bool(torch.isfinite(b[1][8, :64]).all())
    # a gradient of infinity
    dh[4, 0] = float("inf")
    c = P.residual_backward(f, clean[2], clean[3], dh, dx, eps=EPS)
    assert torch.equal(c[0][rows[5:]], a[0][rows[5:]])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["seven", "order4", "tiny", "f36", "ragged", "narrow64", "narrow192", "w900"])
def test_non_finite_stays_in_its_entry(name, dtype):
    """Chunks read channels of neighbouring entries: with a NaN in one entry of every row, the others keep their bits."""
    f, n = FIELDS[name], 11
    C, rng = channels(f), np.random.default_rng(13)
    x, d = values(rng, n, C, dtype), values(rng, n, C, dtype)
    gain = dev(params(rng, f))
    ref = P.site_norm_forward(f, dev(x, dtype), gain, EPS, checkpoint=True)
    back = P.site_norm_backward(f, dev(x, dtype), dev(d, dtype), gain, EPS)
    packed = P.site_norm_backward(f, ref[1], dev(d, dtype), gain, EPS)
    ch = f0 = 0
    for l, m in f:
        w = m * (2 * l + 1)
        for at, v in ((ch, np.nan), (ch + w - 1, np.inf)):
            bad = x.copy()
            bad[:, at] = v
            got = P.site_norm_forward(f, dev(bad, dtype), gain, EPS, checkpoint=True)
            keep = [c for c in range(C) if not ch <= c < ch + w]
            assert bool(torch.isnan(got[0][:, at]).all())
            assert torch.equal(got[0][:, keep], ref[0][:, keep]) and torch.equal(got[1].q[:, keep], ref[1].q[:, keep])
            fields = [i for i in range(sum(m for _, m in f)) if not f0 <= i < f0 + m]
            for u, v in ((P.site_norm_backward(f, dev(bad, dtype), dev(d, dtype), gain, EPS), back),
                         (P.site_norm_backward(f, got[1], dev(d, dtype), gain, EPS), packed)):
                assert torch.equal(u[0][:, keep], v[0][:, keep]) and torch.equal(u[1][fields], v[1][fields])
                assert bool(torch.isnan(u[0][:, at]).all())
        ch, f0 = ch + w, f0 + m


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["order4", "tiny", "f36", "ragged", "narrow64", "narrow192", "w900"])
def test_non_finite_tail_stays_in_its_entry(name, dtype):
    """The same of the tail: a NaN in one entry of the stream, of the convolution output or of a gradient."""
    f, n = FIELDS[name], 11
    full = os_.gate_fields(f)
    C, S, rng = channels(f), channels(full), np.random.default_rng(14)
    y, h, dh, dx = (values(rng, n, c, dtype) for c in (S, C, C, C))
    run = lambda y, h, dh: (P.residual_forward(f, dev(y, dtype), dev(h, dtype), eps=EPS)[:2] +  # noqa: E731
                            P.residual_backward(f, dev(y, dtype), dev(h, dtype), dev(dh, dtype), dev(dx, dtype), eps=EPS)[:2])
    ref = run(y, h, dh)
    gates = list(range(C, S))
    ch = 0
    for l, m in f:
        w = m * (2 * l + 1)
        keep = [c for c in range(C) if not ch <= c < ch + w]
        for which in range(3):
            bad = [y.copy(), h.copy(), dh.copy()]
            bad[which][:, ch + w - 1] = np.nan
            got = run(*bad)
            for g, r in zip(got[:2] if which < 2 else (), ref[:2]):
                assert torch.equal(g[:, keep], r[:, keep]) and bool(torch.isnan(g[:, ch + w - 1]).all())
            for g, r in zip(got[2:], ref[2:]):
                k = keep if l else keep + (gates if g.shape[1] == S else [])  # a field's gate sees its field
                assert torch.equal(g[:, k], r[:, k])
        ch += w


def test_empty():
    f = FIELDS["f104"]
    full = os_.gate_fields(f)
    e = lambda c: torch.empty((0, c), device=DEV)  # noqa: E731
    sc, gp, gn = (torch.full((count(k),), 3.0, device=DEV) for k in (f, full, f))
    ho, x, yk, hk = P.residual_forward(f, e(128), e(104), sc, gp, gn, checkpoint=True)
    assert ho.shape == x.shape == (0, 104) and yk.q.shape == (0, 128)
    dy, dh, *grads = P.residual_backward(f, yk, hk, e(104), e(104), sc, gp, gn)
    assert dy.shape == (0, 128) and all(bool((g == 0).all()) for g in grads)
    dx, dgain = P.site_norm_backward(f, e(104), e(104), gn)
    assert dx.shape == (0, 104) and bool((dgain == 0).all())


def test_streams_and_graph():
    """Calls on a given stream, and captured: replays give the eager result with other work between them."""
    f, n = FIELDS["f104"], 3001
    full, dtype = os_.gate_fields(f), torch.bfloat16
    rng = np.random.default_rng(13)
    y, h, dh, dx = (dev(values(rng, n, c, dtype), dtype) for c in (128, 104, 104, 104))
    sc, gp, gn = (dev(params(rng, k)) for k in (f, full, f))

    def step(stream=None):
        ho, x, yk, hk = P.residual_forward(f, y, h, sc, gp, gn, EPS, checkpoint=True, stream=stream)
        back = P.residual_backward(f, yk, hk, dh, dx, sc, gp, gn, EPS, stream=stream)
        nb = P.site_norm_backward(f, hk, dx, gn, EPS, dres=dh, stream=stream)
        return (ho, x, P.unpack(yk, stream=stream), P.unpack(P.pack(f, h, stream=stream), stream=stream), *back, *nb)

    ref = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    graph2 = torch.cuda.CUDAGraph()     # a second graph of the same calls has scratch of its own
    with torch.cuda.graph(graph2):
        out2 = step()
    for _ in range(4):
        for o in (*out, *out2):
            o.fill_(0)
        graph.replay()
        graph2.replay()
        eager = step()
        torch.cuda.synchronize()
        for a, b, c in zip(eager, out, out2):
            assert torch.equal(a, b) and torch.equal(a, c)
    y.add_(0.5)                          # new values in the captured buffers
    graph.replay()
    for a, b in zip(step(), out):
        assert torch.equal(a, b)


def test_binding_refusals():
    f = ((0, 2), (1, 2))
    full = P.gate_fields(f)
    x = torch.zeros((4, 8), device=DEV)
    y = torch.zeros((4, 10), device=DEV)
    ok = torch.ones(4, device=DEV)
    for bad in (x.cpu(), x[:, ::2], x.t().contiguous(), x[0], torch.zeros((4, 9), device=DEV)):
        with pytest.raises(ValueError):
            P.site_norm_forward(f, bad)
    with pytest.raises(TypeError):
        P.site_norm_forward(f, x.half())
    with pytest.raises(TypeError):
        P.pack(f, x.double())
    with pytest.raises(TypeError):
        P.site_norm_forward(f, x, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P.site_norm_forward(f, x, torch.ones(3, device=DEV))
    with pytest.raises(TypeError):
        P.site_norm_forward(f, x, ok.double())
    with pytest.raises(ValueError):
        P.site_norm_forward(f, P.pack(f, x), checkpoint=True)
    with pytest.raises(ValueError):
        P.site_norm_forward(((0, 8),), P.pack(f, x))
    with pytest.raises(ValueError):
        P.residual_forward(f, x, x)                      # no gate channels
    with pytest.raises(TypeError):
        P.residual_forward(f, y.bfloat16(), x)
    with pytest.raises(ValueError):
        P.residual_forward(f, y, x, gain_next=ok, next_norm=False)
    with pytest.raises(ValueError):
        P.residual_forward(f, y[:3], x)
    with pytest.raises(ValueError):
        P.residual_backward(f, y, None, x, x)
    with pytest.raises(ValueError):
        P.residual_backward(f, y, x, x, None, gain_next=ok)
    with pytest.raises(ValueError):
        P.residual_backward(f, P.pack(f, x), x, x, x)    # a checkpoint of other fields
    with pytest.raises(ValueError):
        P.site_norm_backward(f, x.repeat(99, 1), x.repeat(99, 1), ok, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        P.unpack(P.Packed(full, P.pack(f, x).q, P.pack(f, x).exps))


def test_offsets_past_32_bits():
    """More than 2^32 bytes and 2^31 elements in one matrix: the last rows are those of a small call, and the rows in
    front of them are not touched by it."""
    f, tail = FIELDS["f208"], 5
    full = os_.gate_fields(f)
    n = (1 << 31) // 208 + 1000
    rng = np.random.default_rng(21)
    part = dev(values(rng, tail, 208, torch.bfloat16), torch.bfloat16)
    yp = dev(values(rng, tail, 256, torch.bfloat16), torch.bfloat16)
    assert n * 208 > 1 << 31 and n * 208 * 2 > 1 << 32
    h = torch.zeros((n, 208), dtype=torch.bfloat16, device=DEV)
    y = torch.zeros((n, 256), dtype=torch.bfloat16, device=DEV)
    h[-tail:], y[-tail:] = part, yp
    small = P.residual_forward(f, yp, part, eps=EPS, checkpoint=True)
    ho, x, yk, hk = P.residual_forward(f, y, h, eps=EPS, checkpoint=True, out=h)
    assert torch.equal(ho[-tail:], small[0]) and torch.equal(x[-tail:], small[1])
    assert torch.equal(yk.q[-tail:], small[2].q) and torch.equal(hk.exps[-tail:], small[3].exps)
    assert not bool(x[:-tail].any()) and not bool(yk.q[:-tail].any())
    del x, y
    dh = torch.zeros((n, 208), dtype=torch.bfloat16, device=DEV)
    dh[-tail:] = part
    one = torch.ones(count(f), device=DEV)
    sb = P.residual_backward(f, small[2], small[3], part, part, one, None, one, EPS)
    dy, dhi, ds, _, dn = P.residual_backward(f, yk, hk, dh, dh, one, None, one, EPS)
    assert torch.equal(dy[-tail:], sb[0]) and torch.equal(dhi[-tail:], sb[1]) and not bool(dy[:-tail].any())
    # 5 rows of up to 5 components: sums of at most 25 products in two orders, off by 24 u of their magnitudes (about 5)
    assert torch.allclose(ds, sb[2], rtol=1e-5, atol=1e-5) and torch.allclose(dn, sb[4], rtol=1e-5, atol=1e-5)
    del dy, dhi, dh
    assert torch.equal(P.unpack(hk)[-tail:], P.unpack(small[3]))
    assert torch.equal(P.site_norm_forward(f, hk, eps=EPS)[-tail:], P.site_norm_forward(f, small[3], eps=EPS))
