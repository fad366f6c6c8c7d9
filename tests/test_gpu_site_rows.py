"""Rows of every layout in grids that loop: a workgroup takes its turns one after the other in the same registers and the
same LDS, so every row of a large call is compared with the same row in a call of one turn."""
import ctypes

import numpy as np
import pytest

from oracle import site as os_
from test_gpu_site import FIELDS, channels, dev, host, params, values

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2111_07383_amd")
from paper_2111_07383_amd import _abi, binding  # noqa: E402

DEV = "cuda:0"
EPS = 1e-5
BASE = 3     # rows that repeat: one turn of one workgroup in every layout, and odd, so that every lane meets all of them


def lanes(f):
    """Lanes of a row: chunks of 8 channels of an entry, on 64 lanes more than one a lane."""
    n = sum(-(-m * d // 8) for _, _, m, d in os_.entries(f))
    return next(v for v in (8, 16, 32, 64, 10 ** 9) if n <= v or v == 64)


def many(f):
    """Rows for at least two turns of every kernel: no compute unit holds more than 8 workgroups of 256 lanes."""
    return 2 * 8 * 256 * (256 // lanes(f)) + 5


def data(name, dtype):
    f = FIELDS[name]
    full = os_.gate_fields(f)
    rng = np.random.default_rng(31)
    rows = [dev(values(rng, BASE, channels(k), dtype, s), dtype) for k, s in ((full, 0.4), (f, 0.2), (f, 0), (f, 0))]
    return f, full, many(full), rows, [dev(params(rng, k)) for k in (f, full, f)]


def repeated(t, n):
    return t.repeat(-(-n // BASE), 1)[:n].contiguous()


def same_rows(got, small):
    n = len(got)
    assert torch.equal(got, repeated(small, n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", list(FIELDS))
def test_rows_of_all_turns(name, dtype):
    f, full, n, small, (sc, gp, gn) = data(name, dtype)
    y, h, dh, dx = (repeated(t, n) for t in small)
    ho, x, yk, hk = P.residual_forward(f, y, h, sc, gp, gn, EPS, checkpoint=True)
    so, sx, syk, shk = P.residual_forward(f, small[0], small[1], sc, gp, gn, EPS, checkpoint=True)
    for a, b in ((ho, so), (x, sx), (yk.q, syk.q), (yk.exps, syk.exps), (hk.q, shk.q), (hk.exps, shk.exps)):
        same_rows(a, b)
    for big, one in (((y, ho), (small[0], so)), ((yk, hk), (syk, shk))):
        a = P.residual_backward(f, *big, dh, dx, sc, gp, gn, EPS)
        b = P.residual_backward(f, *one, small[2], small[3], sc, gp, gn, EPS)
        same_rows(a[0], b[0])
        same_rows(a[1], b[1])
    for big, one in ((h, small[1]), (hk, shk)):
        same_rows(P.site_norm_forward(f, big, gn, EPS, dtype=dtype), P.site_norm_forward(f, one, gn, EPS, dtype=dtype))
        same_rows(P.site_norm_backward(f, big, dx, gn, EPS, dres=dh)[0],
                  P.site_norm_backward(f, one, small[3], gn, EPS, dres=small[2])[0])
    same_rows(P.unpack(hk, dtype), P.unpack(shk, dtype))
    same_rows(P.pack(f, h).q, P.pack(f, small[1]).q)


def magnitudes(f, y, h, dh, dx, sc, gp, gn):
    """Sums over the components of every field of the magnitudes of the products that a row adds to dscale, dgain_post,
    dgain_next and to the gain of the norm of h alone, in fp64."""
    full, C = os_.gate_fields(f), channels(f)
    uhat = os_.norm_hat(full, y, EPS)[0]
    u = uhat * os_.spread(full, gp)
    fac = os_.gate_factor(f, u)
    hhat = os_.norm_hat(f, h, EPS)[0]
    e = os_.residual_backward(f, y, h, dh, dx, sc, gp, gn, EPS)[1]
    dg = e * os_.spread(f, sc)
    du, g = np.zeros_like(u), C
    du[:, :C] = dg * fac
    for c, _, m, d in os_.entries(f):
        if d > 1:
            s = 1 / (1 + np.exp(-u[:, g:g + m]))
            du[:, g:g + m] = (dg[:, c:c + m * d] * u[:, c:c + m * d]).reshape(-1, m, d).sum(2) * s * (1 - s)
            g += m
    sums = lambda fl, v: np.stack([os_.by_field(fl, r) for r in np.abs(v)])  # noqa: E731
    return sums(f, e * fac * u[:, :C]), sums(full, du * uhat), sums(f, dx * hhat)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", list(FIELDS))
def test_parameter_sums_of_all_turns(name, dtype):
    """The parameters' gradients of a large call against the sum in fp64 of those of its rows, each alone (which
    test_gpu_site.py holds to the oracle).

    Both calls make the same products.  The large one adds at most 17 of them on a lane in fp32 (a grid holds at least
    256 workgroups of 4 rows, and there are 4096 of those and five rows more; grids of more rows a workgroup or more
    workgroups take fewer turns), rounds a parameter's factor and a workgroup's sum once each, and the result: 20 u of the
    sum of their magnitudes, which are the oracle's.  A row alone rounds its product's factor and its result: 3 u."""
    f, full, n, small, (sc, gp, gn) = data(name, dtype)
    y, h, dh, dx = (repeated(t, n) for t in small)
    times = np.bincount(np.arange(n) % BASE).astype(np.float64)
    got = P.residual_backward(f, y, h, dh, dx, sc, gp, gn, EPS)[2:]
    got += (P.site_norm_backward(f, h, dx, gn, EPS)[1],)
    row = lambda t, i: t[i:i + 1].contiguous()  # noqa: E731
    alone = []
    for i in range(BASE):
        r = [row(t, i) for t in small]
        alone.append(P.residual_backward(f, *r, sc, gp, gn, EPS)[2:] + (P.site_norm_backward(f, r[1], r[3], gn, EPS)[1],))
    a = [host(t) for t in small] + [host(t) for t in (sc, gp, gn)]
    size = magnitudes(f, *a)
    size += (size[2],)
    for k in range(4):
        want = sum(times[i] * host(alone[i][k]) for i in range(BASE))
        most = 24 * 2.0 ** -24 * (times[:, None] * size[k]).sum(0)
        assert (np.abs(host(got[k]) - want) <= 1.01 * most + 1e-30).all(), (k, float(np.max(np.abs(host(got[k]) - want) / (most + 1e-30))))
    # from checkpoints, and again: the same bits
    kept = P.pack(full, y), P.pack(f, h)
    first = P.residual_backward(f, *kept, dh, dx, sc, gp, gn, EPS)[2:]
    for u, v in zip(first, P.residual_backward(f, *kept, dh, dx, sc, gp, gn, EPS)[2:]):
        assert torch.equal(u, v)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", ["tiny", "f104", "ragged", "f36", "narrow64", "w510", "w900", "narrow192"])
def test_gradient_of_the_stream_in_place(name, dtype, packed):
    """ssconv_residual_backward with dh_in in dh's buffer and in dx's: the bits of a call with one of its own."""
    f, full, n, small, ps = data(name, dtype)
    n = 1203
    y, h, dh, dx = (repeated(t, n) for t in small)
    sc, gp, gn = ps
    if packed:
        y, h = P.pack(full, y), P.pack(f, h)
    want = P.residual_backward(f, y, h, dh, dx, sc, gp, gn, EPS)
    at = lambda x: ctypes.byref(_abi.Rows(x.q.data_ptr(), x.exps.data_ptr()) if packed else _abi.Rows(x.data_ptr(), None))  # noqa: E731
    fields = binding.make_fields(f)
    size = _abi.lib().ssconv_residual_workspace_size(ctypes.byref(fields), n)
    for into_dx in (False, True):
        d, x = dh.clone(), dx.clone()
        into = x if into_dx else d
        dy, ds, dp, dn = (torch.empty_like(t) for t in (want[0], sc, gp, gn))
        ws = torch.empty(size, dtype=torch.uint8, device=DEV)
        _abi.check(_abi.lib().ssconv_residual_backward(
            ctypes.byref(fields), at(y), at(h), d.data_ptr(), x.data_ptr(), _abi.F32 if dtype == torch.float32 else _abi.BF16, n,
            EPS, gp.data_ptr(), sc.data_ptr(), gn.data_ptr(), dy.data_ptr(), into.data_ptr(), dp.data_ptr(), ds.data_ptr(),
            dn.data_ptr(), ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream), "ssconv_residual_backward")
        for u, v in zip((dy, into, ds, dp, dn), want):
            assert torch.equal(u, v)
        assert torch.equal(d if into_dx else x, dh if into_dx else dx)
