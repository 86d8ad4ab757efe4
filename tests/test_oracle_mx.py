"""The checkers of rotary positions and of the quantised cache, against hand-worked values and brute force (CPU), the host-side
table of scaled rotations, and the refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest

from oracle import mx_cache as mx
from oracle.rotary import rotary, tree_positions


# ------------------------------------------------------------------------------------------------ rotary
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_turns_pairs(interleaved):
    rs = np.random.RandomState(0)
    x = rs.standard_normal((5, 3, 16))
    f = 1.0 / 7.0 ** np.arange(6)
    y = rotary(x, np.arange(5) * 11, f, interleaved)
    assert np.array_equal(y[..., 12:], x[..., 12:]) and np.array_equal(y[0], x[0])
    a, b = (slice(0, 12, 2), slice(1, 12, 2)) if interleaved else (slice(0, 6), slice(6, 12))
    assert np.allclose(y[..., a] ** 2 + y[..., b] ** 2, x[..., a] ** 2 + x[..., b] ** 2)
    # a quarter turn sends (a, b) to (-b, a)
    q = rotary(x, np.full(5, 1), np.full(6, math.pi / 2), interleaved, mscale=2.0)
    assert np.allclose(q[..., a], -2 * x[..., b]) and np.allclose(q[..., b], 2 * x[..., a])
    # scores depend on the distance alone
    p, r = np.array([3, 9, 40, 0, 7]), 1000
    u, v = rotary(x, p, f, interleaved)[..., :12], rotary(x[::-1], p + 5, f, interleaved)[..., :12]
    u2, v2 = rotary(x, p + r, f, interleaved)[..., :12], rotary(x[::-1], p + 5 + r, f, interleaved)[..., :12]
    assert np.allclose((u * v).sum(-1), (u2 * v2).sum(-1))


def test_rotary_gradient_is_the_opposite_rotation():
    rs = np.random.RandomState(1)
    x, w, pos, f = rs.standard_normal((3, 2, 8)), rs.standard_normal((3, 2, 8)), np.array([2, 5, 1]), np.array([0.7, 0.1, 1.3])
    grad = rotary(w, pos, -f, False, 1.5)
    step = 1e-6
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = step
        d = ((rotary(x + e, pos, f, False, 1.5) - rotary(x - e, pos, f, False, 1.5)) * w).sum() / (2 * step)
        assert abs(d - grad[i]) < 1e-8


def test_tree_positions_by_hand():
    parent = [-1, 0, 0, 1, 3, -1, 0]
    assert list(tree_positions(parent, [0, 5, 5, 7], [10, 99, 0])) == [10, 11, 11, 12, 13, 0, 1]


@pytest.fixture(scope="module")
def hs():
    import paper_2505_13254_amd as h
    h.lib()
    return h


def test_frequencies(hs):
    f, m = hs.hs_rotary_frequencies(8, 10000.0)
    assert np.allclose(f.numpy(), [1.0, 0.1, 0.01, 0.001], rtol=1e-15) and m == 1.0
    f, m = hs.hs_rotary_frequencies(8, 10000.0, scaling="linear", factor=4.0)
    assert np.allclose(f.numpy(), np.array([1.0, 0.1, 0.01, 0.001]) / 4, rtol=1e-15) and m == 1.0
    f, m = hs.hs_rotary_frequencies(8, 10000.0, scaling="base", factor=8.0)
    assert np.allclose(f.numpy(), (10000.0 * 8.0 ** (8 / 6)) ** (-np.arange(4) / 4), rtol=1e-14) and m == 1.0
    # the slowest pair of the stretched base turns exactly `factor` times slower
    assert abs(f[3].item() * 8.0 / 0.001 - 1) < 1e-13
    # waves of 2 pi, 20 pi, 200 pi, 2000 pi tokens in a context of 200 pi: 100, 10, 1 and 0.1 turns
    f, m = hs.hs_rotary_frequencies(8, 10000.0, scaling="wavelength", factor=8.0, context=200 * math.pi, low=1.0, high=19.0)
    assert np.allclose(f.numpy(), [1.0, 0.1 * (0.5 + 0.5 / 8), 0.01 / 8, 0.001 / 8], rtol=1e-12) and m == 1.0
    # a ramp from pair floor(c(100)) = 0 to ceil(c(0.1)) = 3 (c of a pair's own number of turns is the pair)
    f, m = hs.hs_rotary_frequencies(8, 10000.0, scaling="yarn", factor=4.0, context=200 * math.pi, low=0.10001, high=99.99)
    keep = 1 - np.arange(4) / 3
    assert np.allclose(f.numpy(), np.array([1.0, 0.1, 0.01, 0.001]) * (keep + (1 - keep) / 4), rtol=1e-12)
    assert abs(m - (0.1 * math.log(4.0) + 1)) < 1e-7
    for bad in [dict(rot_dim=7), dict(rot_dim=0), dict(base=1.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5), dict(scaling="wavelength", context=0.0),
                dict(scaling="yarn", context=100.0, low=3.0, high=2.0), dict(scaling="base", rot_dim=2, factor=2.0)]:
        with pytest.raises(hs.HsError):
            hs.hs_rotary_frequencies(**{"rot_dim": 8, **bad})
    with pytest.raises(ValueError):
        hs.hs_rotary_frequencies(8, scaling="other")


# ------------------------------------------------------------------------------------------------ the quantised cache
def _row(first, n=32):
    x = np.zeros(n)
    x[:len(first)] = first
    return x


def test_codes_by_hand():
    c, s = mx.quantise(_row([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, 0.2501, -0.1]), "e2m1")
    assert s.tolist() == [127] and c[:11].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 14, 1, 8]   # ties go to the even code
    assert mx.quantise(_row([6.001]), "e2m1")[1].tolist() == [128] and mx.quantise(_row([3.0]), "e2m1")[1].tolist() == [126]
    c, s = mx.quantise(_row([448.0, 1.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, -448.0]), "e4m3")
    assert s.tolist() == [127] and c[:7].tolist() == [126, 56, 56, 58, 0, 2, 254]
    assert mx.quantise(_row([448.001]), "e4m3")[1].tolist() == [128]
    assert mx.quantise(_row([]), "e4m3")[1].tolist() == [27] and mx.quantise(_row([1e-300]), "e4m3")[0].max() == 0
    for bad in (np.nan, np.inf, -np.inf):
        c, s = mx.quantise(_row([1.0, bad]), "e4m3")
        assert s.tolist() == [255] and not c.any() and np.isnan(mx.values(c, s, "e4m3")).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_every_value_is_kept_and_others_go_to_the_nearest(fmt):
    mags = mx._magnitudes(fmt)
    for e in (-90, -3, 0, 40):
        for i in range(0, len(mags), 31):
            row = _row(np.concatenate([[mags[-1]], mags[i:i + 31]])[:32]) * 2.0 ** e
            assert np.array_equal(mx.values(*mx.quantise(row, fmt), fmt), row)
    rs = np.random.RandomState(3)
    x = rs.standard_normal((64, 64)) * np.exp(3 * rs.standard_normal((64, 1)))
    c, s = mx.quantise(x, fmt)
    v = mx.values(c, s, fmt)
    every = np.concatenate([mags, -mags])
    for i in range(64):
        for b in range(2):
            scale = 2.0 ** (int(s[i, b]) - 127)
            amax = np.abs(x[i, 32 * b:32 * b + 32]).max()
            assert amax <= mags[-1] * scale and amax > mags[-1] * scale / 2
            for j in range(32 * b, 32 * b + 32):
                assert abs(v[i, j] - x[i, j]) == np.abs(every * scale - x[i, j]).min()


# ------------------------------------------------------------------------------------------------ refusals, on the host
def test_refusals_need_no_gpu(hs):
    lib = hs.lib()
    d = 256                                              # an aligned address that nothing looks at

    def rotary_call(q=d, qs=512, k=d, ks=512, pos=d, N=4, Hq=4, Hkv=4, D=128, dt=1, f=d, rot=128, pairs=0, m=1.0, qo=d, qos=512, ko=d, kos=512):
        return lib.hs_rotary(q, qs, k, ks, pos, N, Hq, Hkv, D, dt, f, rot, pairs, m, qo, qos, ko, kos, None)

    assert rotary_call(N=0) == 0
    for want, bad in [(2, dict(rot=127)), (2, dict(rot=130)), (2, dict(rot=0)), (2, dict(N=-1)), (2, dict(Hq=0)), (2, dict(Hkv=-1)), (2, dict(qs=511)),
                      (2, dict(kos=100)), (2, dict(dt=2)), (2, dict(pairs=2)), (2, dict(qs=1024)), (1, dict(q=None)), (1, dict(ko=None)), (1, dict(pos=None)),
                      (1, dict(f=None)), (3, dict(D=2048, rot=64, qs=1 << 14, ks=1 << 14, qos=1 << 14, kos=1 << 14)), (3, dict(q=257, qo=d))]:
        assert rotary_call(**bad) == want, bad

    def tree_call(parent=d, no=d, lens=d, B=2, N=4):
        return lib.hs_tree_rotary(d, 512, d, 512, parent, no, lens, B, N, 4, 4, 128, 1, d, 128, 0, 1.0, d, 512, d, 512, None)

    assert tree_call(N=0, B=0) == 0 and tree_call(B=-1) == 2
    assert [tree_call(parent=None), tree_call(no=None), tree_call(lens=None), tree_call(B=0)] == [1] * 4

    def append(k=d, ks=1024, v=d, vs=1024, no=d, NN=5, kc=d, sc=d, fmt=0, table=d, blocks=4, pages=9, lens=d, new=4096, B=2, Hkv=8, D=128, dt=1):
        return lib.hs_kv_append_mx(k, ks, v, vs, no, NN, kc, sc, kc, sc, fmt, table, blocks, pages, lens, new, B, Hkv, D, dt, None)

    assert append(B=0, NN=0) == 0 and append(NN=0, new=None) == 0
    for want, bad in [(2, dict(NN=-1)), (2, dict(B=0)), (2, dict(B=-1)), (2, dict(fmt=2)), (2, dict(dt=5)), (2, dict(Hkv=0)), (2, dict(blocks=-1)), (2, dict(pages=-1)),
                      (3, dict(D=80, ks=4096, vs=4096)), (2, dict(ks=1000)), (2, dict(new=d)), (2, dict(new=d + 8)), (3, dict(ks=1028)), (3, dict(k=d + 8)), (3, dict(kc=d + 8)),
                      (3, dict(sc=d + 2)), (1, dict(k=None)), (1, dict(v=None)), (1, dict(no=None)), (1, dict(kc=None)), (1, dict(table=None)), (1, dict(lens=None)),
                      (3, dict(NN=2 ** 31 - 1, Hkv=4096, ks=1 << 20, vs=1 << 20))]:
        assert append(**bad) == want, bad

    def commit(path=d, length=d, depth=6, B=2):
        return lib.hs_kv_commit_mx(d, 1024, d, 1024, d, path, length, depth, d, d, d, d, 0, d, 4, 9, d, 4096, B, 8, 128, 1, None)

    assert [commit(path=None), commit(length=None), commit(depth=0), commit(B=-1), commit(B=2 ** 20, depth=2 ** 12), commit(B=0)] == [1, 1, 2, 2, 3, 0]

    def read(kc=d, fmt=0, table=d, first=None, off=d, total=10, ko=d, vo=d, B=2, Hkv=8, D=128, dt=1):
        return lib.hs_kv_read_mx(kc, d, d, d, fmt, table, 4, 9, first, off, total, ko, vo, B, Hkv, D, dt, None)

    assert read(total=0) == 0 and read(B=0, total=0) == 0
    for want, bad in [(2, dict(total=-1)), (2, dict(B=0)), (2, dict(fmt=-1)), (2, dict(dt=3)), (3, dict(D=48)), (1, dict(kc=None)), (1, dict(table=None)), (1, dict(off=None)),
                      (1, dict(ko=None)), (3, dict(vo=d + 8)), (3, dict(total=1 << 40))]:
        assert read(**bad) == want, bad

    i32, i64 = ctypes.c_int32, ctypes.c_int64

    def attend(no=(0, 3, 10), lens=(100, 70), blocks=4, pages=9, Hq=32, Hkv=8, D=128, dt=1, scale=0.1, fmt=0, q=d, qs=4096, kt=d, ks=1024, table=d, ws=d, ws_bytes=1 << 30,
               o=d, parent=d, dno=d, dlens=d):
        a = (i32 * len(no))(*no) if no else None
        b = (i64 * max(1, len(lens)))(*lens) if lens is not None else None
        return lib.hs_tree_attention_mx(q, qs, d, d, d, d, fmt, kt, ks, kt, ks, parent, dno, a, table, blocks, pages, dlens, b, len(no) - 1 if no else 1, Hq, Hkv, D, dt, scale, o,
                                        None, ws, ws_bytes, None)

    assert attend(no=(0, 0, 0)) == 0 and attend(no=(0,), lens=()) == 0
    for want, bad in [(2, dict(Hq=30)), (2, dict(Hkv=0)), (3, dict(D=96)), (3, dict(dt=0)), (2, dict(dt=7)), (2, dict(fmt=3)), (3, dict(scale=0.0)), (3, dict(scale=-1.0)),
                      (3, dict(scale=float("nan"))), (3, dict(scale=float("inf"))), (2, dict(no=(1, 3, 10))), (2, dict(no=(0, 5, 3))), (3, dict(no=(0, 3, 1028))), (2, dict(lens=(-1, 5))),
                      (2, dict(lens=(100, 257))), (3, dict(lens=(100, 1 << 40), blocks=2 ** 31 - 1)), (2, dict(pages=0)), (1, dict(q=None)), (1, dict(kt=None)), (1, dict(o=None)),
                      (1, dict(parent=None)), (1, dict(dno=None)), (1, dict(dlens=None)), (1, dict(table=None)), (1, dict(lens=None)), (2, dict(qs=100)), (2, dict(ks=1000)),
                      (3, dict(qs=4100)), (3, dict(q=d + 8))]:
        assert attend(**bad) == want, bad
    long = dict(lens=(4096, 70), blocks=64, pages=64)  # (a call that splits its keys: one that does not needs no workspace)
    assert lib.hs_tree_attention_mx_workspace((i32 * 3)(0, 3, 10), (i64 * 2)(4096, 70), 2, 32, 8, 128) > 100
    for bad in (dict(ws=None), dict(ws=d + 16), dict(ws_bytes=100)):
        assert attend(**long, **bad) == 4, bad


def test_rows_of_no_sequence_are_refused(hs):
    """q with rows, but no sequence that they belong to: nothing would be written to the output."""
    import torch
    pool = hs.new_mx_cache(1, 2, 64, 0, "cpu")
    i32, rows = dict(dtype=torch.int32), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    none = torch.zeros(0, dtype=torch.int64)
    with pytest.raises(ValueError, match="the last one NN"):
        hs.hs_tree_attention_mx(rows, pool, rows, rows, torch.zeros(3, **i32), torch.zeros(1, **i32), torch.zeros(1, **i32), torch.zeros((0, 1), **i32), none, none, 0.1)


def test_workspace_query_is_host_arithmetic(hs):
    import torch
    def need(rows, lens, *a):
        ws = hs.hs_tree_attention_mx_workspace(torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32), torch.tensor(lens, dtype=torch.int64), *a, "cpu")
        return 0 if ws is None else ws.numel()
    assert need([1], [2048], 32, 8, 128) > 0
    assert need([5], [0], 32, 8, 128) == 0 and need([0], [5000], 32, 8, 128) == 0
    assert need([1], [2048], 30, 8, 128) == 0 and need([2000], [2048], 32, 8, 128) == 0     # refused calls
    for rows in (1, 61, 1024):
        for lens in (64, 5000, 10 ** 6):
            assert need([rows] * 20, [lens] * 20, 64, 8, 128) <= 2 ** 18 * 132 * 4 + 2 ** 16


def test_workspace_query_checks_its_arrays(hs):
    import torch
    no, lens = torch.tensor([0, 1, 2], dtype=torch.int32), torch.tensor([5, 6], dtype=torch.int64)
    for bad in ((no[:2], lens), (no, lens[:1]), (no[:0], lens[:0])):
        with pytest.raises(ValueError):
            hs.hs_tree_attention_mx_workspace(*bad, 8, 2, 128, "cpu")


def test_plans_of_many_sequences(hs):
    """The query's cost does not grow with the list of cuts it weighs beyond 64 sequences, and its records stay within their bound."""
    import time

    import torch
    rs = np.random.RandomState(1)
    for n, most in ((65, 300), (5000, 60), (3000, 1)):
        rows, lens = rs.randint(0, most + 1, n), rs.randint(0, 9000, n)
        lens[n // 2] = 10 ** 6
        no, pl = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32), torch.tensor(lens, dtype=torch.int64)
        hs.lib()
        t = time.perf_counter()
        bytes_ = hs.lib().hs_tree_attention_mx_workspace(no.data_ptr(), pl.data_ptr(), n, 64, 8, 128)
        assert time.perf_counter() - t < 0.05
        assert bytes_ % (4 * 132) == 0 and bytes_ // (4 * 132) <= 1 << 18


def test_calls_beyond_a_launch_are_refused(hs):
    """Host arithmetic alone refuses them: nothing is launched, no pointer is looked at."""
    lib, d = hs.lib(), 0x100000
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    n = 1 << 21                                       # sequences of one row, 32 KV heads: 2^26 work items
    no, lens = (i32 * (n + 1))(*range(n + 1)), (i64 * n)()
    args = [d, 4096, d, d, d, d, 0, d, 4096, d, 4096, d, d, no, d, 4, 9, d, lens, n, 32, 32, 128, 1, 0.1, d, None, d, 1 << 40, None]
    assert lib.hs_tree_attention_mx(*args) == 3
    args[19:22] = [n, 16, 16]                         # (2^25 rows of a head, 2^25 work items)
    assert lib.hs_tree_attention_mx(*args) == 3
    assert lib.hs_tree_rotary(d, 4096, None, 0, d, d, d, 1, (1 << 23) + 1, 4, 0, 128, 1, d, 128, 0, 1.0, d, 4096, None, 0, None) == 3
