"""Rows of every layout in grids that loop: a workgroup takes its turns one after the other in the same registers and the
same LDS, so every row of a large call is compared with the same row in a call of one turn."""
import numpy as np
import pytest

from oracle import site as os_
from test_gpu_site import FIELDS, channels, count, dev, params, values

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2111_07383_amd")

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
