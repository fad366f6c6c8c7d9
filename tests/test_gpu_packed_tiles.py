"""Coefficient gradients from checkpoints on the fp32 route of three bf16 parts, in 3x3x3 and 5x5x5."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2111_07383_amd")

DEV = "cuda:0"
F104 = ((0, 16), (1, 16), (2, 8))


def random_sites(rng, n, grid):
    c = np.stack([np.zeros(n, np.int64)] + [rng.integers(0, grid, n) for _ in range(3)], 1)
    return np.unique(c, axis=0).astype(np.int32)


def layer(rng, f, ks, n, grid):
    full = P.gate_fields(f)
    rb = P.Rulebook(torch.from_numpy(random_sites(rng, n, grid)).to(DEV), grid, ks, 1, True)
    desc = P.basis_desc(f, full, ks, tuple(float(i) for i in range(ks // 2 + 1)))
    basis = torch.from_numpy(P.basis_build(desc)).to(DEV)
    C, S = P.n_channels(f), P.n_channels(full)
    W = torch.zeros((ks ** 3, S, C), device=DEV)
    x, g = (torch.from_numpy(rng.standard_normal((rb.n_in, c)).astype(np.float32)).to(DEV) for c in (C, S))
    return rb, desc, basis, W, x, g


def test_many_offsets_keep_their_slices():
    """One round of work units is two slices of each of 125 lists, whose rows then no longer meet in an L2 (1.3 times
    ssconv_backward's time): there the call takes the units, and so the order of the sums, of ssconv_backward."""
    rb, desc, basis, W, x, g = layer(np.random.default_rng(1), F104, 5, 30000, 40)
    assert 10 ** 6 < rb.n_pairs < 1.5 * 10 ** 6
    p = P.pack(F104, x)
    got = P.backward_packed(p, g, rb, W, desc, basis, need_feats=False)[1]
    assert torch.equal(got, P.backward(P.unpack(p, torch.float32), g, rb, W, desc, basis, need_feats=False)[1])
    rb.close()
