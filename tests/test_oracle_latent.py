"""The checkers of block tables, slots and attention over latents, against hand-worked values and closed forms (CPU), and the refusals that need no GPU."""
import numpy as np
import pytest

from oracle import latent_attention as la
from oracle import page_tables as pt


def test_block_tables_by_hand():
    table = np.array([[7, 8, 9, -1], [3, -1, -1, -1], [5, 6, -1, -1]])
    # sequence 0 keeps one page of three, 1 asks for two, 2 for one more than the table has
    t, held, stack, refused = pt.block_tables([10, 33, 65], 16, table, [3, 1, 2], [0, 1])
    assert held == [1, 3, 2] and refused == [0, 0, 2] and stack == [0, 1]
    assert t.tolist() == [[7, 8, 9, -1], [3, 9, 8, -1], [5, 6, -1, -1]]
    # nothing is served from the first that does not fit on, though a later one would fit
    t, held, stack, refused = pt.block_tables([16, 48, 48], 16, table, [1, 1, 2], [4])
    assert held == [1, 1, 2] and refused == [0, 1, 1] and stack == [4]
    # everything goes back
    t, held, stack, refused = pt.block_tables([0, -3, 0], 16, table, [3, 1, 2], [])
    assert held == [0, 0, 0] and stack == [7, 8, 9, 3, 5, 6] and np.array_equal(t, table)


def test_slots_by_hand():
    table = np.array([[4, 2], [0, 9]])
    slots, new = pt.slot_map([0, 4, 6], 8, [14, 15], table, 16, 5)
    assert slots.tolist() == [78, 79, 32, 33, 15, -1, -1, -1] and new.tolist() == [18, 17]   # page 9 is none
    slots, new = pt.slot_map([0, 4, 6], 6, [14, 15], table, 16, 5, held=[1, 2])
    assert slots.tolist() == [78, 79, -1, -1, 15, -1] and new.tolist() == [16, 17]
    slots, new = pt.slot_map([0, 4, 6], 6, [14, 3], table, 16, 5, accept_path=[[2, 3, -1], [-1, -1, -1]], accept_len=[2, 0])
    assert slots.tolist() == [78, -1, 79, 32, 3, -1] and new.tolist() == [17, 4]


def test_latent_attention_is_attention_with_shared_heads():
    from oracle.tree_attention import tree_attention
    rs = np.random.RandomState(0)
    NN, Hq, R, Dr, L = 5, 3, 8, 4, 6
    q, qr = rs.standard_normal((NN, Hq, R)), rs.standard_normal((NN, Hq, Dr))
    pre, ct, rt = rs.standard_normal((L, R + Dr)), rs.standard_normal((NN, R)), rs.standard_normal((NN, Dr))
    parent = np.array([-1, 0, 0, 1, 3], np.int32)
    o, lse = la.tree(q, qr, [pre], ct, rt, parent, [0, NN], 0.3)
    # one KV head of R + Dr columns whose values are the latents and zeros behind them
    keys, tree = pre.copy(), np.concatenate([ct, rt], 1)
    val, vtree = pre.copy(), tree.copy()
    val[:, R:] = 0.0
    vtree[:, R:] = 0.0
    f = lambda x: np.ascontiguousarray(x, dtype=np.float32)  # noqa: E731
    want, wlse = tree_attention(f(np.concatenate([q, qr], 2)), f(keys[:, None]), f(val[:, None]), f(tree[:, None]), f(vtree[:, None]), parent, [0, NN], [0, L], 0.3)
    assert np.abs(want[..., :R] - o).max() < 1e-5 and np.abs(wlse - lse).max() < 1e-5


def test_prompt_attention_closed_forms():
    rs = np.random.RandomState(1)
    v = rs.standard_normal((7, 2, 3))
    z = lambda *s: np.zeros(s)  # noqa: E731
    # equal scores: a row's result is the mean of what it sees; rows without keys are zero
    o, lse = la.prompt(z(5, 2, 4), z(5, 2, 2), rs.standard_normal((7, 2, 4)), rs.standard_normal((7, 2)), v, [0, 2, 5], [0, 5, 7], 1.0)
    for row, keys in ((0, range(0, 4)), (1, range(0, 5)), (3, [5]), (4, [5, 6])):
        assert np.allclose(o[row], v[list(keys)].mean(0)) and np.allclose(lse[row], np.log(len(keys)))
    assert not o[2].any() and np.isneginf(lse[2]).all()
    # absorbed and expanded are the same attention: k = c Wk, v = c Wv
    c, r, Wk, Wv = rs.standard_normal((6, 5)), rs.standard_normal((6, 2)), rs.standard_normal((2, 5, 4)), rs.standard_normal((2, 5, 3))
    q, qr = rs.standard_normal((6, 2, 4)), rs.standard_normal((6, 2, 2))
    o, lse = la.prompt(q, qr, np.einsum("tc,hcd->thd", c, Wk), r, np.einsum("tc,hcd->thd", c, Wv), [0, 6], [0, 6], 0.5)
    chain = np.arange(-1, 5)
    lat, wlse = la.tree(np.einsum("nhd,hcd->nhc", q, Wk), qr, [z(0, 7)], c, r, chain, [0, 6], 0.5)
    assert np.allclose(np.einsum("nhc,hcd->nhd", lat, Wv), o) and np.allclose(lse, wlse)


# ------------------------------------------------------------------------------------------------ refusals, on the host
@pytest.fixture(scope="module")
def hs():
    import paper_2505_13254_amd as h
    h.lib()
    return h


def test_refusals_need_no_gpu(hs):
    lib = hs.lib()
    d = 1 << 12                                              # an aligned address that nothing looks at

    def tables(want=d, page=64, table=d, blocks=4, held=d, new=2 * d, free=d, pages=9, count=d, new_count=2 * d, refused=None, B=3):
        return lib.hs_block_tables(want, page, table, blocks, held, new, free, pages, count, new_count, refused, B, None)

    assert tables(B=0) == 0
    for want, bad in [(2, dict(B=-1)), (2, dict(page=0)), (2, dict(blocks=-1)), (2, dict(pages=-1)), (1, dict(want=None)), (1, dict(table=None)), (1, dict(held=None)),
                      (1, dict(new=None)), (1, dict(free=None)), (1, dict(count=None)), (1, dict(new_count=None)), (2, dict(new=d)), (2, dict(new=d + 8)),
                      (2, dict(new_count=d)), (3, dict(B=1 << 15, blocks=1 << 15, new=1 << 20)), (3, dict(pages=1 << 30))]:
        assert tables(**bad) == want, bad

    def slots(no=d, NN=5, path=None, length=None, depth=0, table=d, blocks=4, page=64, pages=9, held=None, lens=d, out=d, new=2 * d, B=2):
        return lib.hs_slot_map(no, NN, path, length, depth, table, blocks, page, pages, held, lens, out, new, B, None)

    assert slots(B=0, NN=0) == 0
    for want, bad in [(2, dict(NN=-1)), (2, dict(B=-1)), (2, dict(B=0)), (2, dict(page=0)), (2, dict(blocks=-1)), (2, dict(pages=-1)), (2, dict(path=d)), (2, dict(length=d)),
                      (2, dict(path=d, length=d)), (1, dict(no=None)), (1, dict(lens=None)), (1, dict(out=None)), (1, dict(table=None)), (2, dict(new=d)), (2, dict(new=d + 8))]:
        assert slots(**bad) == want, bad

    def rows(c=d, cs=576, r=d, rs=576, sl=d, N=4, pool=d, n=640, R=512, Dr=64, dt=1, store=True):
        return lib.hs_latent_store(c, cs, r, rs, sl, N, pool, n, R, Dr, dt, None) if store else lib.hs_latent_read(pool, n, sl, N, c, cs, r, rs, R, Dr, dt, None)

    for store in (True, False):
        assert rows(N=0, store=store) == 0
        for want, bad in [(2, dict(N=-1)), (2, dict(n=-1)), (2, dict(R=0)), (2, dict(Dr=-1)), (2, dict(dt=2)), (3, dict(R=509)), (3, dict(Dr=60)), (3, dict(R=1 << 21, cs=1 << 21)),
                          (1, dict(c=None)), (1, dict(r=None)), (1, dict(sl=None)), (1, dict(pool=None)), (3, dict(c=d + 8)), (3, dict(r=d + 2)), (3, dict(pool=d + 4)),
                          (3, dict(cs=580)), (3, dict(rs=66)), (2, dict(cs=-8)), (3, dict(cs=1 << 40)), (3, dict(n=1 << 40)), (3, dict(N=2 ** 31 - 1))]:
            assert rows(**bad, store=store) == want, bad
        assert rows(R=510, dt=0, store=store) == 3
    assert rows(cs=504, store=False) == 2 and rows(rs=0, store=False) == 2


def _tree_call(hs, sizes=(3, 2), lens=(70, 64), q=1 << 12, qs=(16 * 512, 512), qr=1 << 12, qrs=(16 * 64, 64), pool=1 << 12, ct=1 << 12, cs=512, rt=1 << 12, rs=64,
               parent=1 << 12, no=1 << 12, hno=True, table=1 << 12, blocks=4, pages=9, pl=1 << 12, hpl=True, B=None, Hq=16, R=512, Dr=64, dt=1, scale=0.1, o=1 << 12,
               os=(16 * 512, 512), lse=None, ws=None, nws=0):
    n = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    l = np.array(lens, np.int64)
    return hs.lib().hs_tree_attention_latent(q, *qs, qr, *qrs, pool, ct, cs, rt, rs, parent, no, n.ctypes.data if hno else None, table, blocks, pages, pl,
                                             l.ctypes.data if hpl else None, len(sizes) if B is None else B, Hq, R, Dr, dt, scale, o, *os, lse, ws, nws, None)


def test_tree_attention_refusals_need_no_gpu(hs):
    assert _tree_call(hs, B=0) == 0 and _tree_call(hs, sizes=(0, 0)) == 0
    for want, bad in [(2, dict(B=-1)), (2, dict(Hq=0)), (2, dict(R=0)), (2, dict(Dr=-1)), (2, dict(blocks=-1)), (2, dict(pages=-1)), (2, dict(dt=2)), (2, dict(scale=0.0)),
                      (2, dict(scale=float("nan"))), (2, dict(scale=float("inf"))), (3, dict(R=1032)), (3, dict(Dr=1032)), (1, dict(hno=False)), (1, dict(hpl=False)),
                      (2, dict(sizes=(3, -1))), (3, dict(sizes=(1025, 1))), (2, dict(lens=(-1, 5))), (2, dict(lens=(257, 5))), (3, dict(lens=(1 << 24, (1 << 24) + 1), blocks=1 << 20)),
                      (2, dict(pages=0)), (1, dict(q=None)), (1, dict(qr=None)), (1, dict(pool=None)), (1, dict(ct=None)), (1, dict(rt=None)), (1, dict(parent=None)),
                      (1, dict(no=None)), (1, dict(table=None)), (1, dict(pl=None)), (1, dict(o=None)), (2, dict(qs=(-1, 512))), (2, dict(qrs=(64, -64))), (2, dict(cs=-1)),
                      (2, dict(os=(16 * 512 - 1, 512))), (2, dict(os=(16 * 512, 511))), (2, dict(os=(512, 512))), (2, dict(os=(0, 512))), (3, dict(sizes=(1000, 1000), Hq=16384))]:
        assert _tree_call(hs, **bad) == want, bad


def _prompt_call(hs, rows=(3, 2), keys=(70, 2), q=1 << 12, qs=(16 * 128, 128), qr=1 << 12, qrs=(16 * 64, 64), k=1 << 12, ks=(16 * 256, 256), kr=1 << 12, krs=64, v=1 << 12,
                 vs=(16 * 256, 256), qo=1 << 12, ko=1 << 12, hqo=True, hko=True, first=0, B=None, H=16, Dn=128, Dr=64, Dv=128, dt=1, scale=0.1, o=1 << 12, os=(16 * 128, 128),
                 lse=None, ws=None, nws=0):
    n = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32) + first
    t = np.concatenate([[0], np.cumsum(keys)]).astype(np.int64)
    return hs.lib().hs_prompt_attention_latent(q, *qs, qr, *qrs, k, *ks, kr, krs, v, *vs, qo, ko, n.ctypes.data if hqo else None, t.ctypes.data if hko else None,
                                               len(rows) if B is None else B, H, Dn, Dr, Dv, dt, scale, o, *os, lse, ws, nws, None)


def test_prompt_attention_refusals_need_no_gpu(hs):
    assert _prompt_call(hs, B=0) == 0 and _prompt_call(hs, rows=(0, 0)) == 0
    for want, bad in [(2, dict(B=-1)), (2, dict(H=0)), (2, dict(Dn=0)), (2, dict(Dr=-1)), (2, dict(Dv=0)), (2, dict(dt=2)), (2, dict(scale=-1.0)), (3, dict(Dn=1032)), (3, dict(Dr=1032)),
                      (3, dict(Dv=1032)), (1, dict(hqo=False)), (1, dict(hko=False)), (2, dict(first=1)), (2, dict(rows=(3, -1))), (2, dict(keys=(70, -1))),
                      (3, dict(keys=((1 << 24) + 1, 5))), (1, dict(q=None)), (1, dict(qr=None)), (1, dict(k=None)), (1, dict(kr=None)), (1, dict(v=None)), (1, dict(qo=None)),
                      (1, dict(ko=None)), (1, dict(o=None)), (2, dict(qs=(-1, 128))), (2, dict(ks=(128, -1))), (2, dict(vs=(-1, 128))), (2, dict(krs=-64)), (2, dict(qrs=(-1, 64))),
                      (2, dict(os=(16 * 128 - 1, 128))), (2, dict(os=(16 * 128, 100))), (3, dict(rows=(1 << 20, 1), keys=(1 << 20, 1)))]:
        assert _prompt_call(hs, **bad) == want, bad


def test_a_step_without_sequences_still_needs_its_counts(hs):
    d = 1 << 12                                              # an address that no device has: the call leaves it alone
    call = lambda count, new: hs.lib().hs_block_tables(None, 64, None, 4, None, None, None, 0, count, new, None, 0, None)  # noqa: E731
    assert call(d, 2 * d) == 0
    assert call(None, d) == 1 and call(d, None) == 1 and call(d, d) == 2 and call(d, d + 2) == 2
