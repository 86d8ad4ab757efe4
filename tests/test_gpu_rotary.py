"""GPU parity of hs_rotary and hs_tree_rotary against the float64 checker.

Tolerance.  In float32: the angle's rest is at most half a turn and rounded to 24 bits (pi 2^-24 of a radian), sine and cosine
are within 4 units in the last place, and the factor, the two products and the sum each round once: an output (a c - b s) is
within 16 * 2^-24 * mscale * (|a| + |b|).  bfloat16 outputs are rounded once more, by 2^-8 of their size at most."""
import numpy as np
import pytest

from oracle import rotary, tree_positions

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_13254_amd as h
    return h


def _bound(x, want, h, interleaved, mscale, dtype):
    a, b = (np.s_[..., 0:2 * h:2], np.s_[..., 1:2 * h:2]) if interleaved else (np.s_[..., :h], np.s_[..., h:2 * h])
    tol = np.zeros_like(want)
    tol[a] = tol[b] = 16 * 2.0 ** -24 * mscale * (np.abs(x[a]) + np.abs(x[b])) + 1e-30
    return tol + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0)


def _check(got, x, pos, f, interleaved, mscale):
    x = x.double().cpu().numpy()
    want = rotary(x, pos, f, interleaved, mscale)
    err = np.abs(got.double().cpu().numpy() - want)
    tol = _bound(x, want, len(f), interleaved, mscale, got.dtype)
    assert (err <= tol).all(), (err - tol).max()


def _positions(rs, n):
    p = rs.randint(0, 200, n)
    p[::3] = rs.randint(0, 1 << 20, len(p[::3]))
    p[-1] = (1 << 24) - 1
    return p


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,Hq,Hkv,D,rot", [(1, 32, 8, 128, 128), (61, 32, 8, 128, 64), (7, 5, 3, 64, 64), (3, 1, 1, 40, 22), (2, 4, 0, 96, 96), (9, 2, 1, 2, 2),
                                            (2051, 3, 1, 128, 32), (2049, 2, 2, 18, 10), (5, 1, 1, 1024, 1024), (4, 8, 1, 80, 80)])
def test_rotary(hs, N, Hq, Hkv, D, rot, dtype, interleaved):
    rs, g = np.random.RandomState(N + D), torch.Generator(device=DEV).manual_seed(N)
    q = torch.randn((N, Hq, D), generator=g, device=DEV).to(dtype)
    k = torch.randn((N, Hkv, D), generator=g, device=DEV).to(dtype) if Hkv else None
    pos = _positions(rs, N)
    f, m = hs.hs_rotary_frequencies(rot, 500000.0, scaling="none" if rot == 2 else "yarn", factor=4.0, context=8192.0, low=1.0, high=32.0, device=DEV)
    before = q.clone()
    qo, ko = hs.hs_rotary(q, k, torch.from_numpy(pos).to(DEV), f, interleaved=interleaved, mscale=m)
    assert torch.equal(q, before)
    _check(qo, q, pos, f.cpu().numpy(), interleaved, m)
    if k is not None:
        _check(ko, k, pos, f.cpu().numpy(), interleaved, m)
    assert torch.equal(qo[..., rot:], q[..., rot:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_slices_of_a_projection_in_place(hs, dtype, pad):
    """q and k are slices of one projection, turned where they are (pad = 3: rows that begin at no multiple of 16 bytes)."""
    N, Hq, Hkv, D = 33, 4, 2, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    flat = torch.randn((N, (Hq + 2 * Hkv) * D + pad), generator=g, device=DEV).to(dtype)
    q, k = flat[:, :Hq * D].unflatten(1, (Hq, D)), flat[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    q0, k0, rest = q.clone(), k.clone(), flat[:, (Hq + Hkv) * D:].clone()
    pos = torch.arange(N, device=DEV) * 37
    f, _ = hs.hs_rotary_frequencies(48, device=DEV)
    want = hs.hs_rotary(q, k, pos, f)
    hs.hs_rotary(q, k, pos, f, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(flat[:, (Hq + Hkv) * D:], rest)
    _check(q, q0, pos.cpu().numpy(), f.cpu().numpy(), False, 1.0)
    _check(k, k0, pos.cpu().numpy(), f.cpu().numpy(), False, 1.0)


def _parents(rs, n, back):
    return [-1] + [int(rs.randint(max(0, i - back), i)) for i in range(1, n)]


@pytest.mark.parametrize("sizes,back", [([1], 5), ([61], 5), ([0, 9, 0, 0, 130, 1, 0], 3), ([2] * 70 + [0] * 60 + [17], 2), ([700], 1), ([1500, 2], 1), ([1100], 400), ([64, 65, 63], 1)])
@pytest.mark.parametrize("D,rot", [(128, 128), (20, 6)])
def test_tree_rotary(hs, sizes, back, D, rot):
    """Depths by the tree's own arrays: chains, stars, trees beyond the staged 1024 rows, empty sequences."""
    rs, g = np.random.RandomState(len(sizes)), torch.Generator(device=DEV).manual_seed(1)
    parent = np.concatenate([_parents(rs, n, back) if n else [] for n in sizes]).astype(np.int32)
    no = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    lens = rs.randint(0, 100000, len(sizes)).astype(np.int64)
    N = int(no[-1])
    q, k = (torch.randn((N, h, D), generator=g, device=DEV) for h in (3, 1))
    f, _ = hs.hs_rotary_frequencies(rot, device=DEV)
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    qo, ko = hs.hs_tree_rotary(q, k, dev(parent), dev(no), dev(lens), f)
    pos = tree_positions(parent, no, lens)
    _check(qo, q, pos, f.cpu().numpy(), False, 1.0)
    assert torch.equal(qo, hs.hs_rotary(q, k, dev(pos), f)[0]) and torch.equal(ko, hs.hs_rotary(q, k, dev(pos), f)[1])


@pytest.mark.parametrize("D,interleaved", [(128, False), (64, True), (20, False)])
def test_rows_behind_the_last_sequence(hs, D, interleaved):
    """A fixed budget of rows of which the trees use fewer (a captured step, say): the rows behind are left as they were."""
    sizes, N = [5, 0, 9, 0], 40
    rs, g = np.random.RandomState(3), torch.Generator(device=DEV).manual_seed(1)
    parent = torch.zeros(N, dtype=torch.int32, device=DEV)
    parent[:14] = torch.tensor(_parents(rs, 5, 3) + _parents(rs, 9, 3), dtype=torch.int32)
    no = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).to(DEV)
    lens = torch.tensor([7, 100, 30, 5], device=DEV)
    f, _ = hs.hs_rotary_frequencies(min(D, 18), device=DEV)
    q, k = (torch.randn((N, h, D), generator=g, device=DEV) for h in (3, 1))
    out = (torch.full_like(q, 5.0), torch.full_like(k, 5.0))
    hs.hs_tree_rotary(q, k, parent, no, lens, f, interleaved=interleaved, q_out=out[0], k_out=out[1])
    for x, y in zip((q, k), out):
        want, _ = hs.hs_tree_rotary(x[:14], None, parent[:14].contiguous(), no, lens, f, interleaved=interleaved)
        assert torch.equal(y[:14], want) and (y[14:] == 5.0).all()


def test_the_most_rows(hs):
    """As many rows as the count holds, in place, a pair each: 26 GB."""
    N, ends = (1 << 31) - 1, [0, 1, 255, 1 << 23, (1 << 31) - 258, (1 << 31) - 257, (1 << 31) - 256, (1 << 31) - 3, (1 << 31) - 2]
    q = torch.ones((N, 1, 2), dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(N, device=DEV)
    f = torch.tensor([0.25], dtype=torch.float64, device=DEV)
    hs.hs_rotary(q, None, pos, f, q_out=q)
    rows = torch.tensor(ends, device=DEV)
    _check(q[rows], torch.ones((len(ends), 1, 2), dtype=torch.bfloat16), np.asarray(ends), f.cpu().numpy(), False, 1.0)


def test_gradient_is_the_opposite_rotation(hs):
    """d/dx <w, rotary(x)> against central differences of the call itself (float32, steps of a power of two: the outputs' rounding
    of 2^-24 of numbers of order one over a step of 2^-6 leaves 2^-17 a term, of which two contribute)."""
    g = torch.Generator(device=DEV).manual_seed(3)
    x, w = (torch.randn((4, 2, 16), generator=g, device=DEV) for _ in range(2))
    pos = torch.tensor([0, 3, 77, 100000], device=DEV)
    f, _ = hs.hs_rotary_frequencies(12, device=DEV)
    grad = hs.hs_rotary(w, None, pos, -f)[0].double().cpu()
    step = 2.0 ** -6
    for d in range(16):
        e = torch.zeros_like(x)
        e[..., d] = step
        up, down = (hs.hs_rotary(x + s * e, None, pos, f)[0].double() for s in (1, -1))
        diff = (((up - down) / (2 * step)) * w.double()).sum(-1).cpu()
        assert (diff - grad[..., d]).abs().max() < 4 * 8 * 2.0 ** -17


def test_streams_graphs_and_refusals(hs):
    g = torch.Generator(device=DEV).manual_seed(4)
    q, k = (torch.randn((50, h, 128), generator=g, device=DEV).bfloat16() for h in (8, 2))
    pos, (f, _) = torch.arange(50, device=DEV), hs.hs_rotary_frequencies(128, device=DEV)
    want = hs.hs_rotary(q, k, pos, f)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = hs.hs_rotary(q, k, pos, f, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = [torch.empty_like(q), torch.empty_like(k)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hs_rotary(q, k, pos, f, q_out=out[0], k_out=out[1])
    for shift in (0, 9, 1000):
        pos.copy_(torch.arange(50, device=DEV) + shift)
        want = hs.hs_rotary(q, k, pos, f)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    for bad in [dict(positions=pos[:49]), dict(positions=pos.int()), dict(k=k[:49]), dict(k=k.float()), dict(q=q.half()), dict(q=q.cpu()), dict(inv_freq=f.float()),
                dict(q=q.transpose(1, 2)), dict(q_out=out[0][:49]), dict(k=None, k_out=out[1])]:
        with pytest.raises(ValueError):
            hs.hs_rotary(**{**dict(q=q, k=k, positions=pos, inv_freq=f), **bad})
    with pytest.raises(ValueError):
        hs.hs_rotary(q[..., :64], None, pos, f)          # heads that are not dense
    with pytest.raises(hs.HsError):
        hs.hs_rotary(q[..., :64].contiguous(), None, pos, f)   # more pairs than a head has
