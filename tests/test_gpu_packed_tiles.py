"""Coefficient gradients from checkpoints on the fp32 route of three bf16 parts, in 3x3x3 and 5x5x5."""
import numpy as np
import pytest

from cases import rel_err
from oracle import conv as oc
from oracle import rulebook as orb
from oracle import site as os_
from workloads.configs import LayerSpec

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


@pytest.fixture
def variant():
    """Sets the kernel override, and takes it back."""
    yield lambda v: P.debug_set(3, v)
    P.debug_set(3, 0)


# fields, kernel size, sites drawn, grid, override: 0 where the rule itself is to take the three parts, 13 where a case is
# smaller than it asks for
CASES = {
    "f104_k3_rule": (F104, 3, 60000, 24, 0),
    "f104_k3": (F104, 3, 900, 10, 13),
    "f104_k5": (F104, 5, 500, 9, 13),
    "ragged_k3": (((0, 13), (1, 11), (2, 5)), 3, 700, 10, 13),
    "f36_k3": (((0, 4), (1, 4), (2, 4)), 3, 300, 8, 13),
    "f208_k3": (((0, 32), (1, 32), (2, 16)), 3, 400, 8, 13),
    "one_site": (((0, 4), (1, 1)), 3, 1, 4, 13),
}


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_three_parts(name, norm, variant):
    """Against the fp64 oracle and against ssconv_backward of the same rows, and in one workspace between calls whose
    gradients (3e38, infinity) do not split: what those leave there the next one does not see."""
    f, ks, n, grid, force = CASES[name]
    rng = np.random.default_rng(n)
    rb, desc, basis, W, x, g = layer(rng, f, ks, n, grid)
    C, S = P.n_channels(f), P.n_channels(P.gate_fields(f))
    gain = torch.from_numpy((1 + 0.2 * rng.standard_normal(sum(m for _, m in f))).astype(np.float32)).to(DEV)
    kw = dict(norm=True, gain=gain) if norm else {}
    variant(7)
    other = P.backward_packed_workspace_size(rb, torch.float32, C, S)
    variant(13)
    size = P.backward_packed_workspace_size(rb, torch.float32, C, S)
    variant(force)
    assert P.backward_packed_workspace_size(rb, torch.float32, C, S) == size != other   # the route that is meant
    p = P.pack(f, x)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    call = lambda g: P.backward_packed(p, g, rb, W, desc, basis, need_feats=False, workspace=ws, **kw)[1]  # noqa: E731
    got = call(g)
    for bad in (3e38, float("inf")):
        b = g.clone()
        b[-1, 3] = bad
        assert not torch.equal(call(b), got)
        assert torch.equal(call(g), got)
    rows = P.site_norm_forward(f, p, gain, dtype=torch.float32) if norm else P.unpack(p, torch.float32)
    plain = P.backward(rows, g, rb, W, desc, basis, need_feats=False)[1]

    coords = random_sites(np.random.default_rng(n), n, grid)
    spec = LayerSpec(ks, 1, True, f, P.gate_fields(f), shells=tuple(float(i) for i in range(ks // 2 + 1)), gated=True)
    lay, R = oc.Layer(spec), orb.rulebook(coords, coords, ks, 1)
    v = os_.unpack(f, *os_.pack(f, x.double().cpu().numpy()))
    if norm:
        v = os_.norm_forward(f, v, gain.double().cpu().numpy())
    gh, shape = g.double().cpu().numpy(), (ks ** 3, S, C)
    want = oc.synth_adjoint(spec, lay.basis, oc.grad_kappa(v, gh, R, shape))
    assert rel_err(got.cpu().numpy(), want) < 1e-4 and rel_err(plain.cpu().numpy(), want) < 1e-4
    # both sums of at most `most` products in fp32, in whatever order, each off by at most that many 2^-24 of the sum of
    # their magnitudes (1.01: second order, and the basis in fp32); 8 for the products of parts that are left out, under
    # 2^-24 of the whole product, and for the rows' own roundings
    most = 2 * max(len(r) for r in R) + max(b[0].size for b in lay.basis.values()) + 8
    size = oc.grad_kappa(np.abs(v), np.abs(gh), R, shape)
    bound = 2.02 * most * 2.0 ** -24 * oc.synth_adjoint(spec, {k: np.abs(b) for k, b in lay.basis.items()}, size)
    assert (np.abs((got - plain).double().cpu().numpy()) <= bound).all()
    rb.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [False, True])
def test_streams_and_graphs(norm, dtype, variant):
    """Both gradients on a given stream and captured twice: every replay has the bits of the eager call, with other work and
    another call whose gradient does not split between them, and follows new values in the captured buffers."""
    variant(13)
    rng = np.random.default_rng(5)
    rb, desc, basis, W, x, g = layer(rng, F104, 3, 900, 10)
    x, g = x.to(dtype), g.to(dtype)
    W = (torch.from_numpy(rng.standard_normal(tuple(W.shape)).astype(np.float32)).to(DEV) / 60).to(dtype)
    p = P.pack(F104, x)
    call = lambda g, stream=None: P.backward_packed(p, g, rb, W, desc, basis, norm=norm, eps=1e-5, stream=stream)  # noqa: E731
    ref = call(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(g, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call(g))
    bad = g.clone()
    bad[3, 5] = 3e38
    for step in range(4):
        for o in outs:
            for t in o:
                t.fill_(7)
        for graph in graphs:
            graph.replay()
        call(bad)
        want = call(g)
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o, want))
        g.mul_(-0.5 if step else 1)
        p.q.add_(1)
    rb.close()
