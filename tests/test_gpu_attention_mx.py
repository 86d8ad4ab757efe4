"""GPU parity of hs_tree_attention_mx against the float64 checker on the values that the cache reads back, alone and in a decoding
loop with the cache's writers, rotary positions and the accept walk.

Tolerance, with u = 2^-8 (bfloat16) and what the kernel rounds: keys and values are exact in bfloat16 and Q is used as it is, so a
score is off by float32 accumulation alone, delta = (D + 8) 2^-24 scale max_j sum_d |q_d k_jd|; a weight is rounded to bfloat16
(u) while the denominator sums the unrounded ones; the output is rounded once (u); sums of up to a few 10^4 terms and the
exponentials: 5e-5.  |error| <= u |o| + ((1 + u) exp(2 delta) - 1 + 5e-5) A, A the exact weights on |V|."""
import math

import numpy as np
import pytest

from oracle import mx_cache, rotary, tree_attention, tree_positions
from oracle.tree_attention import ancestor_mask

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
U = 2.0 ** -8


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_13254_amd as h
    return h


def dev(a, kind=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if kind is None else t.to(kind)).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


def parents(rs, n, back):
    return [-1] + [int(rs.randint(max(0, i - back), i)) for i in range(1, n)]


class Step:
    """Inputs of one call on a filled cache."""

    def __init__(self, hs, rows, lens, Hq, Hkv, D, fmt=0, back=9, seed=0, blocks=None, gain=1.0):
        rs, g = np.random.RandomState(seed), torch.Generator(device=DEV).manual_seed(seed)
        B, NN = len(rows), sum(rows)
        self.rows, self.lens, self.scale, self.D = rows, np.asarray(lens, np.int64), D ** -0.5, D
        self.no = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.parent = np.concatenate([parents(rs, n, back) if n else [] for n in rows] + [[]]).astype(np.int32)
        need = blocks or max(1, max(-(-l // 64) for l in lens))
        pages = B * need + 1
        self.table = (1 + rs.permutation(pages - 1)).reshape(B, need).astype(np.int32)
        self.cache = hs.new_mx_cache(pages, Hkv, D, fmt, DEV)
        for n in ("k", "v"):                               # what nobody stored is NaN
            self.cache[n + "_codes"].view(torch.uint8).fill_(255)
            self.cache[n + "_scales"].fill_(255)
        r = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
        k, v = r(int(sum(lens)), Hkv, D) * gain, r(int(sum(lens)), Hkv, D)
        po = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        self.po = po
        hs.hs_kv_append_mx(k, v, dev(po.astype(np.int32)), self.cache, dev(self.table), torch.zeros(B, dtype=torch.int64, device=DEV))
        self.q, self.kt, self.vt = r(NN, Hq, D).bfloat16(), (r(NN, Hkv, D) * gain).bfloat16(), r(NN, Hkv, D).bfloat16()
        self.hs = hs

    def args(self):
        return dict(q=self.q, cache=self.cache, k_tree=self.kt, v_tree=self.vt, parent=dev(self.parent), node_offsets=dev(self.no),
                    host_node_offsets=torch.from_numpy(self.no), block_table=dev(self.table), prefix_lens=dev(self.lens),
                    host_prefix_lens=torch.from_numpy(self.lens), scale=self.scale)

    def prefix(self):
        return tuple(f64(x) for x in self.hs.hs_kv_read_mx(self.cache, dev(self.table), dev(self.po), int(self.po[-1]), dtype=torch.float32))

    def check(self, o, lse):
        kp, vp = self.prefix()
        q, kt, vt = f64(self.q), f64(self.kt), f64(self.vt)
        want, want_lse = tree_attention(q, kp, vp, kt, vt, self.parent, self.no, self.po, self.scale)
        A, _ = tree_attention(q, kp, np.abs(vp), kt, np.abs(vt), self.parent, self.no, self.po, self.scale)
        G = q.shape[1] // kt.shape[1]
        delta = np.zeros(want_lse.shape)
        for s in range(len(self.rows)):
            n0, n1, p0, p1 = self.no[s], self.no[s + 1], self.po[s], self.po[s + 1]
            if n1 == n0:
                continue
            anc = ancestor_mask(self.parent[n0:n1])
            for h in range(q.shape[1]):
                aq = np.abs(q[n0:n1, h])
                d = np.where(anc, aq @ np.abs(kt[n0:n1, h // G]).T, 0.0).max(axis=1)
                if p1 > p0:
                    d = np.maximum(d, (aq @ np.abs(kp[p0:p1, h // G]).T).max(axis=1))
                delta[n0:n1, h] = (self.D + 8) * 2.0 ** -24 * self.scale * d
        tol = U * np.abs(want) + ((1 + U) * np.exp(2 * delta) - 1 + 5e-5)[..., None] * A + 1e-7
        err = np.abs(f64(o) - want)
        assert (err <= tol).all(), (float((err - tol).max()), np.unravel_index((err - tol).argmax(), err.shape))
        if lse is not None:
            assert (np.abs(f64(lse) - want_lse) <= 2 * delta + 2e-5 + 2.0 ** -22 * np.abs(want_lse)).all()

    def run(self, **kw):
        o, lse = self.hs.hs_tree_attention_mx(**{**self.args(), "want_lse": True, **kw})
        torch.cuda.synchronize()
        return o, lse


SHAPES = [
    # rows, lens, Hq, Hkv, back
    ([1], [0], 8, 8, 1),                                        # a root alone
    ([1], [1], 4, 1, 1),
    ([1], [2048], 32, 8, 1),                                    # a token
    ([1] * 5, [31, 32, 33, 64, 65], 8, 2, 1),                   # lengths around a block and a page
    ([1] * 70, [(37 * i) % 300 for i in range(70)], 8, 8, 1),   # more sequences than a wave has lanes
    ([61], [2048], 32, 8, 9),                                   # the 8B shape
    ([61], [0], 32, 8, 9),                                      # a tree alone
    ([33], [63], 6, 3, 2),                                      # an odd number of KV heads
    ([97], [1000], 64, 8, 9),                                   # 776 rows to a KV head
    ([129], [777], 5, 5, 4),                                    # no sharing of heads
    ([9, 0, 40, 1, 0], [130, 500, 0, 7, 0], 32, 8, 9),          # ragged, with empty sequences
    ([300], [100], 4, 4, 3),                                    # trees beyond 256 rows
    ([300], [65], 4, 2, 1),                                     # a chain: causal attention
    ([1024], [130], 2, 1, 1),                                   # the longest chain
    ([1024], [10], 2, 2, 700),
    ([12, 129, 31], [5000, 321, 1500], 8, 2, 9),                # cuts of several splits beside whole sequences
    ([2], [9001], 7, 1, 1),                                     # seven heads to a KV head
]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("rows,lens,Hq,Hkv,back", SHAPES)
def test_matches_the_checker(hs, rows, lens, Hq, Hkv, back, D, fmt):
    st = Step(hs, rows, lens, Hq, Hkv, D, fmt, back, seed=len(rows) + D)
    o, lse = st.run()
    st.check(o, lse)
    again = st.run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])     # the same bits


FULL = [  # calls that fill the chip: work items of two to eight row blocks, whose waves share their keys
    ([5, 9, 16] * 20, [64, 200, 700] * 20, 32, 8, 9),                       # one and two blocks
    ([17, 33, 33, 20] * 8, [400, 1, 64, 700] * 8, 32, 8, 9),                # three and five
    ([12, 20, 33, 65, 97, 129] * 2, [700, 130, 64, 1, 300, 555] * 2, 64, 8, 9),  # up to 33, trees beyond 64 and 128 rows
    ([64] * 24, [600, 64, 63, 0, 128, 191] * 4, 32, 8, 1),                  # eight, chains
    ([20, 0, 41] * 24, [(29 * i) % 400 for i in range(72)], 24, 3, 9),      # more sequences than a wave has lanes
    ([1] * 69 + [3], [(30 * i) % 200 for i in range(69)] + [9000], 8, 1, 1),
]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("rows,lens,Hq,Hkv,back", FULL)
def test_full_chips(hs, rows, lens, Hq, Hkv, back, D, fmt):
    test_matches_the_checker(hs, rows, lens, Hq, Hkv, back, D, fmt)


@pytest.mark.parametrize("fmt", [0, 1])
def test_scores_of_any_size_on_a_full_chip(hs, fmt):
    for rows, lens in (([64] * 16, [300] * 16), ([20] * 32, [130, 64] * 16), ([9] * 48, [200] * 48)):
        st = Step(hs, rows, lens, 32, 8, 128, fmt, gain=30.0, seed=3)
        st.check(*st.run())


def test_splits_of_shared_groups(hs):
    """Long prefixes behind wide groups: items of eight blocks whose keys are cut, and the records' merge."""
    st = Step(hs, [97, 61, 130], [2600, 2500, 2100], 64, 8, 128, 1, seed=4)
    st.check(*st.run())
    assert hs.hs_tree_attention_mx_workspace(torch.from_numpy(st.no), torch.from_numpy(st.lens), 64, 8, 128, DEV).numel() > 0


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("n,L", [(33, 4500), (20, 4500), (9, 9000), (1, 17000)])
def test_long_items(hs, n, L, fmt):
    """Work items of more pages than a look-up of 64 covers: 32 sequences of the same rows and pages give the same bits, which are right."""
    st, many = Step(hs, [n], [L], 32, 8, 128, fmt, seed=n), 32
    host = [torch.arange(many + 1, dtype=torch.int32) * n, torch.full((many,), L, dtype=torch.int64)]
    o, lse = st.run(q=st.q.repeat(many, 1, 1), k_tree=st.kt.repeat(many, 1, 1), v_tree=st.vt.repeat(many, 1, 1), parent=dev(np.tile(st.parent, many)),
                    node_offsets=host[0].to(DEV), host_node_offsets=host[0], block_table=dev(st.table).repeat(many, 1), prefix_lens=host[1].to(DEV), host_prefix_lens=host[1])
    st.check(o[:n], lse[:n])
    assert torch.equal(o, o[:n].repeat(many, 1, 1)) and torch.equal(lse, lse[:n].repeat(many, 1))


def test_the_same_rows_in_other_company(hs):
    """A sequence's result alone and in a batch that takes its rows in other groups and splits: within both tolerances of the checker."""
    st = Step(hs, [33] * 20, [700] * 20, 32, 8, 128, 0, seed=6)
    st.check(*st.run())
    one = dict(q=st.q[:33], k_tree=st.kt[:33], v_tree=st.vt[:33], parent=dev(st.parent[:33]), node_offsets=dev(st.no[:2]), host_node_offsets=torch.from_numpy(st.no[:2]),
               block_table=dev(st.table[:1]), prefix_lens=dev(st.lens[:1]), host_prefix_lens=torch.from_numpy(st.lens[:1]))
    o, lse = st.run(**one)
    full, full_lse = st.run()
    # both are within the checker's tolerance of the same value: |error| <= u |o| + (u + 5e-5 + ...) A with A <= max |V|
    top = max(float(st.vt.abs().max()), float(np.abs(st.prefix()[1]).max()))
    assert (np.abs(f64(o) - f64(full)[:33]) <= 4 * U * (1 + U) * top + 4e-4).all()
    assert np.abs(f64(lse) - f64(full_lse)[:33]).max() < 1e-3


def test_odd_tree_values_on_a_full_chip(hs):
    """NaN and infinity in a tree row's value reach the rows below it, in groups whose waves share the tile, and leave the others' bits."""
    for rows, lens in (([60] * 24, [130] * 24), ([70] * 12, [64] * 12)):
        st = Step(hs, rows, lens, 32, 8, 128, 0, back=4, seed=9)
        n = rows[0]
        tree = np.concatenate([[-1, 0, 0, 1], np.where(np.arange(n - 4) % 2, 3, 2)])
        st.parent[:] = np.tile(tree, len(rows))
        o, _ = st.run()
        below = np.zeros(len(rows) * n, bool)
        below[5 * n + 2] = True
        below[5 * n + 4:6 * n] = np.arange(n - 4) % 2 == 0
        for bad in (float("nan"), float("inf")):
            st.vt[5 * n + 2] = bad
            o2, _ = st.run()
            assert not o2[dev(below)].isfinite().any() and torch.equal(o2[dev(~below)], o[dev(~below)])


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("gain", [30.0, 2.0 ** -20])
def test_scores_of_any_size(hs, gain, fmt):
    """Scores of several hundred (single keys take all the weight, the maximum moves many times) and of next to nothing."""
    for rows, lens in (([37], [1500]), ([1, 1], [700, 40])):
        st = Step(hs, rows, lens, 8, 2, 128, fmt, gain=gain, seed=3)
        st.check(*st.run())


def test_rising_scores(hs):
    """Every key's score is above the ones before it, by octaves and by less than one, and the last key is the largest or the least."""
    for step in (0.01, 0.7, 40.0, -40.0):
        st = Step(hs, [3], [900], 4, 1, 64, 0, seed=5)
        k = torch.zeros((900, 1, 64), device=DEV)
        k[:, 0, 0] = torch.arange(900, device=DEV) * step
        hs.hs_kv_append_mx(k, k.flip(0).contiguous(), dev(np.asarray([0, 900], np.int32)), st.cache, dev(st.table), torch.zeros(1, dtype=torch.int64, device=DEV))
        st.q[..., 0] = 1.0
        st.check(*st.run())


# Groups of four and of eight row blocks whose keys are cut into several splits, in either format (tests/test_attention_mx_plan.py)
CUT = ([28, 64, 20, 40, 40, 20, 40, 40, 20], [3366, 3908, 4233, 4111, 2127, 2849, 3401, 3979, 4476])


@pytest.mark.parametrize("fmt", [0, 1])
def test_cut_groups_of_either_shared_kind(hs, fmt):
    st = Step(hs, *CUT, 32, 8, 128, fmt, seed=4)
    st.check(*st.run())


# Calls of one kind of work item each (tests/test_attention_mx_plan.py holds them to it): (kind, rows of the trees)
KINDS = [(0, [5] * 48), (1, [16] * 24), (2, [20] * 32), (2, [32] * 24), (3, [40] * 24), (3, [64] * 24)]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("L", [100, 230])
@pytest.mark.parametrize("kind,rows", KINDS)
def test_scores_that_jump_behind_the_first_keys(hs, kind, rows, L, fmt):
    """Scores of 0 for the tree and the first 32 keys, then far above them in the full pages and again in the page that ends inside a
    tile, by less and by more octaves than a float32 sum holds, with small and large values."""
    st = Step(hs, rows, [L] * len(rows), 32, 8, 128, fmt, seed=5)
    N = sum(st.lens)
    st.kt.zero_()
    st.q[..., 0] = 1.0
    v = torch.randn((N, 8, 128), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV)
    token = torch.arange(N, device=DEV) % L
    for full, rest in ((60, 60), (120, 120), (200, 200), (60, 200), (120, 260), (200, 60), (-60, 200)):
        for gain in (1.0, 1000.0):
            octaves = torch.where(token < 32, 0, torch.where(token < L // 64 * 64, full, rest))
            k = torch.zeros((N, 8, 128), device=DEV)
            k[..., 0] = (octaves * (math.log(2.0) / st.scale))[:, None]
            hs.hs_kv_append_mx(k, v * gain, dev(st.po.astype(np.int32)), st.cache, dev(st.table), torch.zeros(len(rows), dtype=torch.int64, device=DEV))
            st.check(*st.run())


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kind,rows", KINDS + [("cut", None)])
def test_large_values(hs, kind, rows, fmt):
    """Values that float32 holds, whose sums weighted against the first keys' maximum it does not: far above it in the scores, or so
    large that a few of them overflow.  The weighted mean is always in range."""
    rows, lens = CUT if kind == "cut" else (rows, [230] * len(rows))
    st = Step(hs, rows, lens, 32, 8, 128, fmt, seed=5)
    N = sum(st.lens)
    g = torch.Generator(device=DEV).manual_seed(6)
    q, kt, vt = st.q.clone(), st.kt.clone(), st.vt.clone()
    token = torch.cat([torch.arange(int(n), device=DEV) for n in lens])
    for jump, size in ((0, 1e37), (60, 1e25), (70, 1e37), (-40, 1e37)):
        st.q, st.kt, st.vt = q.clone(), torch.zeros_like(kt) if jump else kt, (vt.float() * size).bfloat16()
        k = torch.randn((N, 8, 128), generator=g, device=DEV)
        if jump:                                         # scores of 0, and of `jump` octaves behind the first 40 keys
            st.q[..., 0] = 1.0
            k.zero_()
            k[..., 0] = (torch.where(token < 40, 0, jump) * (math.log(2.0) / st.scale))[:, None]
        v = torch.randn((N, 8, 128), generator=g, device=DEV)
        v = v.clamp(-4, 4) + 2.0                         # (mostly of one sign)
        hs.hs_kv_append_mx(k, v * size, dev(st.po.astype(np.int32)), st.cache, dev(st.table), torch.zeros(len(rows), dtype=torch.int64, device=DEV))
        st.check(*st.run())


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("kind,rows", [KINDS[0], KINDS[1], KINDS[2], KINDS[5], ("cut", None)])
def test_a_nan_block_takes_its_columns(hs, kind, rows, fmt):
    """A NaN block among the values takes its 32 columns of its KV head's rows; the other columns keep their bits, also where sums overflow."""
    rows, lens = CUT if kind == "cut" else (rows, [230] * len(rows))
    st = Step(hs, rows, lens, 32, 8, 128, fmt, seed=5)
    N = sum(st.lens)
    vt, v = st.vt.clone(), torch.randn((N, 8, 128), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV) + 3.0
    for size in (1.0, 1e37):
        st.vt = (vt.float() * size).bfloat16()
        hs.hs_kv_append_mx(v, v * size, dev(st.po.astype(np.int32)), st.cache, dev(st.table), torch.zeros(len(rows), dtype=torch.int64, device=DEV))
        o, lse = st.run()
        assert o.isfinite().all()
        page, slot = st.table[0, 1], 70 - 64
        kept = int(st.cache["v_scales"][page, 5, slot, 2])
        st.cache["v_scales"][page, 5, slot, 2] = 255
        o2, lse2 = st.run()
        st.cache["v_scales"][page, 5, slot, 2] = kept
        hit = torch.zeros_like(o, dtype=torch.bool)
        hit[:rows[0], 20:24, 64:96] = True
        assert o2[hit].isnan().all() and torch.equal(o2[~hit], o[~hit]) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind,rows", [KINDS[0], KINDS[1], KINDS[2], KINDS[5], ("cut", None)])
def test_an_infinite_tree_value_takes_its_column(hs, kind, rows):
    """An infinity in one column of a tree row's value takes that column of the rows below it; all others keep their bits, also where sums overflow."""
    rows, lens = CUT if kind == "cut" else (rows, [230] * len(rows))
    st = Step(hs, rows, lens, 32, 8, 128, 0, seed=5)
    N, n = sum(st.lens), rows[0]
    st.parent[:n] = [-1, 0, 0] + [1 + (i & 1) for i in range(n - 3)]
    vt, v = st.vt.clone(), torch.randn((N, 8, 128), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV) + 3.0
    below = torch.zeros(len(st.parent), dtype=torch.bool, device=DEV)
    below[[2] + [i for i in range(3, n) if st.parent[i] == 2]] = True
    for size in (1.0, 1e37):
        st.vt = (vt.float() * size).bfloat16()
        hs.hs_kv_append_mx(v, v * size, dev(st.po.astype(np.int32)), st.cache, dev(st.table), torch.zeros(len(rows), dtype=torch.int64, device=DEV))
        o, lse = st.run()
        st.vt[2, 3, 77] = float("inf")
        o2, lse2 = st.run()
        hit = torch.zeros_like(o, dtype=torch.bool)
        hit[:, 12:16, 77] = below[:, None]
        assert o.isfinite().all() and not o2[hit].isfinite().any() and torch.equal(o2[~hit], o[~hit]) and torch.equal(lse, lse2)


def test_strided_rows_and_outputs(hs):
    """q, k and v of the tree as slices of one projection; outputs into given tensors, no lse."""
    st = Step(hs, [20, 5], [300, 64], 8, 2, 128, 0, seed=7)
    fused = torch.cat([st.q, st.kt, st.vt], 1)
    o, _ = st.run(q=fused[:, :8], k_tree=fused[:, 8:10], v_tree=fused[:, 10:])
    assert torch.equal(o, st.run()[0])
    out = torch.empty_like(st.q)
    got, lse = st.run(out=out, want_lse=False)
    assert got is out and lse is None and torch.equal(out, o)


def test_nan_tokens_and_what_lies_behind_the_end(hs):
    """A token with a NaN block makes the rows that see it NaN and no others; a row off whose path a NaN tree row lies does not see it."""
    st = Step(hs, [4, 4], [100, 100], 4, 2, 64, 0, back=4, seed=9)
    st.parent[:] = [-1, 0, 0, 1, -1, 0, 0, 1]
    o, lse = st.run()
    st.check(o, lse)                                             # (everything behind the ends is NaN)
    page, slot = st.table[0, 1], 70 - 64
    st.cache["k_scales"][page, 1, slot, 0] = 255
    o2, _ = st.run()
    assert o2[:4, 2:].isnan().all() and torch.equal(o2[:4, :2], o[:4, :2]) and torch.equal(o2[4:], o[4:])


def test_a_nan_tree_row_reaches_its_descendants_only(hs):
    st = Step(hs, [40], [100], 4, 2, 128, 0, back=4, seed=9)
    st.parent[:] = np.concatenate([[-1, 0, 0, 1], np.where(np.arange(36) % 2, 3, 2)])
    o, _ = st.run()
    st.kt[2] = float("nan")
    o2, _ = st.run()
    below = np.zeros(40, bool)
    below[2] = True
    below[4:] = np.arange(36) % 2 == 0
    assert o2[dev(below)].isnan().all() and torch.equal(o2[dev(~below)], o[dev(~below)])
    st = Step(hs, [40], [100], 4, 2, 128, 0, back=4, seed=9)
    st.parent[:] = np.concatenate([[-1, 0, 0, 1], np.where(np.arange(36) % 2, 3, 2)])
    for bad in (float("nan"), float("inf")):
        st.vt[2] = bad                                           # values of masked rows count as little as their keys
        o3, _ = st.run()
        assert not o3[dev(below)].isfinite().any() and torch.equal(o3[dev(~below)], o[dev(~below)])


def test_pages_that_are_shared_and_foreign_entries_behind_the_end(hs):
    """Two sequences share their first page; entries behind a sequence's last page name no page at all."""
    st = Step(hs, [3, 5], [64, 100], 8, 2, 128, 1, seed=11, blocks=4)
    st.table[1, 0] = st.table[0, 0]
    st.table[0, 1:] = -5
    st.table[1, 2:] = 1 << 30
    st.check(*st.run())


def test_pools_beyond_32_bit_offsets(hs):
    pages, Hkv, D = 70000, 8, 128
    st = Step(hs, [3], [100], 8, Hkv, D, 0, seed=13)
    far = hs.new_mx_cache(pages, Hkv, D, 0, DEV)
    for n in far:
        far[n][pages - 2] = st.cache[n][int(st.table[0, 0])].view(far[n].dtype)
        far[n][pages - 1] = st.cache[n][int(st.table[0, 1])].view(far[n].dtype)
    o, _ = st.run()
    o2, _ = st.run(cache=far, block_table=dev(np.asarray([[pages - 2, pages - 1]], np.int32)))
    assert torch.equal(o, o2)


def test_graphs_that_share_a_workspace_and_streams(hs):
    a, b = Step(hs, [9], [3000], 8, 2, 128, 0, seed=1), Step(hs, [1, 1], [5000, 77], 8, 2, 128, 1, seed=2)
    want = [a.run(), b.run()]
    ws = torch.empty(max(hs.hs_tree_attention_mx_workspace(torch.from_numpy(s.no), torch.from_numpy(s.lens), 8, 2, 128, DEV).numel() for s in (a, b)),
                     dtype=torch.uint8, device=DEV)
    outs, graphs = [], []
    for st in (a, b):
        args, out, lse = st.args(), torch.empty_like(st.q), torch.empty(st.q.shape[:2], device=DEV)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            hs.hs_tree_attention_mx(**args, out=out, lse=lse, ws=ws)
        outs.append((out, lse, args))
        graphs.append(graph)
    for _ in range(4):
        for x in (0, 1, 1, 0):
            outs[x][0].zero_()
            graphs[x].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[x][0], want[x][0]) and torch.equal(outs[x][1], want[x][1])
            a.run()
    side = torch.cuda.Stream()
    args = a.args()
    torch.cuda.synchronize()
    got = hs.hs_tree_attention_mx(**args, want_lse=True, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0][0])


@pytest.mark.parametrize("rows,lens", [([3], [700]), ([2, 1, 0] * 23 + [40], [90, 300, 5] * 23 + [5000]),
                                       ([1] * 254 + [9, 0, 17] + [2] * 300, [200] * 255 + [9000, 9000] + [70] * 300)])
def test_captured_calls_keep_their_lengths(hs, rows, lens):
    """A captured call attends to the lengths and rows of its capture, however many sequences it has, after the device arrays have changed;
    batches beyond 64 and beyond 255 sequences, cut sequences among them."""
    st = Step(hs, rows, lens, 8, 2, 128, 0, seed=2)
    want = st.run()
    st.check(*want)
    args, out, lse = st.args(), torch.empty_like(st.q), torch.empty(st.q.shape[:2], device=DEV)
    ws = hs.hs_tree_attention_mx_workspace(args["host_node_offsets"], args["host_prefix_lens"], 8, 2, 128, DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hs.hs_tree_attention_mx(**args, out=out, lse=lse, ws=ws)
    for change in (lambda: args["prefix_lens"].add_(64), lambda: args["node_offsets"].zero_(), lambda: args["prefix_lens"].zero_()):
        change()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_refusals(hs):
    st = Step(hs, [3, 2], [100, 70], 8, 2, 128, 0, seed=1)
    good = st.args()
    bf = torch.bfloat16
    for bad in [dict(q=st.q[:4]), dict(k_tree=st.kt[:4]), dict(v_tree=st.vt[:, :1]), dict(q=st.q[..., :64].contiguous()), dict(q=st.q.half()), dict(q=st.q.cpu()),
                dict(k_tree=st.kt.float()), dict(parent=good["parent"][:4]), dict(parent=good["parent"].long()), dict(node_offsets=good["node_offsets"][:2]),
                dict(prefix_lens=good["prefix_lens"].int()), dict(host_prefix_lens=torch.tensor([100])), dict(host_node_offsets=torch.tensor([0, 3, 6], dtype=torch.int32)),
                dict(block_table=good["block_table"][:1]), dict(out=torch.empty((5, 8, 64), dtype=bf, device=DEV)), dict(out=torch.empty((5, 8, 128), device=DEV)),
                dict(lse=torch.empty((5, 7), device=DEV)), dict(lse=torch.empty((5, 8), dtype=bf, device=DEV)), dict(ws=torch.empty(1 << 20, device=DEV)),
                dict(ws=torch.empty(1 << 20, dtype=torch.uint8)), dict(cache=dict(st.cache, v_scales=st.cache["v_scales"][:2]))]:
        with pytest.raises(ValueError):
            hs.hs_tree_attention_mx(**{**good, **bad})
    for bad in [dict(scale=0.0), dict(scale=float("nan")), dict(host_prefix_lens=torch.tensor([100, 129])), dict(host_prefix_lens=torch.tensor([-1, 1])),
                dict(q=st.q.float(), k_tree=st.kt.float(), v_tree=st.vt.float())]:
        with pytest.raises(hs.HsError):
            hs.hs_tree_attention_mx(**{**good, **bad})


def test_host_arrays_are_converted(hs):
    """Host copies of another integer type, or on the GPU, are copied, as the other attention calls do; with and without a workspace."""
    st = Step(hs, [3, 2], [3000, 70], 8, 2, 128, 0, seed=1)
    good = st.args()
    want, _ = st.run()
    ws = hs.hs_tree_attention_mx_workspace(good["host_node_offsets"], good["host_prefix_lens"], 8, 2, 128, DEV)
    for other in (dict(host_node_offsets=good["node_offsets"]), dict(host_prefix_lens=good["prefix_lens"]),
                  dict(host_node_offsets=good["host_node_offsets"].long(), host_prefix_lens=good["host_prefix_lens"].int())):
        for w in (None, ws):
            assert torch.equal(hs.hs_tree_attention_mx(**{**good, **other}, ws=w)[0], want)


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_decoding_loop(hs, fmt):
    """Prompts are rotated and stored, then several steps of two sequences: rotary of the tree's rows, attention, the greedy walk, the
    accepted path joins the cache.  Every step's outputs, lengths and stored values are followed in float64."""
    rs, g = np.random.RandomState(21), torch.Generator(device=DEV).manual_seed(21)
    B, Hq, Hkv, D, V, depth = 2, 8, 2, 64, 97, 5
    f, m = hs.hs_rotary_frequencies(32, 10000.0, scaling="linear", factor=2.0, device=DEV)
    prompt = [70, 3]
    blocks = 4
    cache, table = hs.new_mx_cache(B * blocks, Hkv, D, fmt, DEV), np.asarray([[5, 0, 7, 2], [1, 6, 3, 4]], np.int32)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).bfloat16()  # noqa: E731
    lens, gtable = torch.zeros(B, dtype=torch.int64, device=DEV), dev(table)
    pno = dev(np.asarray([0, 70, 73], np.int32))
    k, v = r(73, Hkv, D), r(73, Hkv, D)
    pos = dev(np.concatenate([np.arange(n) for n in prompt]))
    q, kr = hs.hs_rotary(r(73, Hq, D), k, pos, f, mscale=m)
    new = torch.empty_like(lens)
    hs.hs_kv_append_mx(kr, v, pno, cache, gtable, lens, new_lens=new)
    name = "e4m3" if fmt == 0 else "e2m1"

    def stored(x):
        return mx_cache.values(*mx_cache.quantise(f64(x), name), name)
    kept = [[stored(kr[a:b]), stored(v[a:b])] for a, b in ((0, 70), (70, 73))]
    lens, new = new, lens
    for step in range(3):
        rows = [int(rs.randint(2, 40)), int(rs.randint(2, 40))]
        par = np.concatenate([parents(rs, n, 3) for n in rows]).astype(np.int32)
        no = np.asarray([0, rows[0], sum(rows)], np.int32)
        N = sum(rows)
        hl = lens.cpu()
        q0, k0, vt = r(N, Hq, D), r(N, Hkv, D), r(N, Hkv, D)
        q, kt = hs.hs_tree_rotary(q0, k0, dev(par), dev(no), lens, f, mscale=m)
        wq = rotary(f64(q0), tree_positions(par, no, hl), f.cpu().numpy(), False, m)
        assert (np.abs(f64(q) - wq) <= 2.0 ** -8 * np.abs(wq) + 1e-5).all()
        o, lse = hs.hs_tree_attention_mx(q, cache, kt, vt, dev(par), dev(no), torch.from_numpy(no), gtable, lens, hl, D ** -0.5, want_lse=True)
        kp, vp = (np.concatenate([kept[s][x] for s in range(B)]) for x in (0, 1))
        po = np.concatenate([[0], np.cumsum([len(kept[s][0]) for s in range(B)])])
        assert po[-1] == int(hl.sum())
        want, want_lse = tree_attention(f64(q), kp, vp, f64(kt), f64(vt), par, no, po, D ** -0.5)
        A, _ = tree_attention(f64(q), kp, np.abs(vp), f64(kt), np.abs(f64(vt)), par, no, po, D ** -0.5)
        assert (np.abs(f64(o) - want) <= U * np.abs(want) + (U + 1e-4) * A).all() and np.abs(f64(lse) - want_lse).max() < 1e-4
        token = torch.from_numpy(rs.randint(0, V, N).astype(np.int32)).to(DEV)
        logits = torch.randn((N, V), generator=g, device=DEV)
        for n in range(N):                                # most nodes' argmax is a child's token
            s = int(n >= rows[0])
            kids = [j for j in range(n + 1, int(no[s + 1])) if par[j] == n - int(no[s])]
            if kids and rs.uniform() < 0.8:
                logits[n, int(token[kids[0]])] = 50.0
        acc = hs.hs_verify_accept(logits, None, token, dev(par), dev(no), 0, 1.0, None, depth)
        hs.hs_kv_commit_mx(kt, vt, dev(no), acc["accept_path"], acc["accept_len"], cache, gtable, lens, new_lens=new)
        for s in range(B):
            path = [int(no[s])] + [int(no[s]) + int(x) for x in acc["accept_path"][s, :int(acc["accept_len"][s])]]
            for x, t in ((0, kt), (1, vt)):
                kept[s][x] = np.concatenate([kept[s][x], stored(t[path])])
        assert new.tolist() == [len(kept[s][0]) for s in range(B)]
        lens, new = new, lens
    off = np.concatenate([[0], np.cumsum(lens.tolist())]).astype(np.int64)
    got = hs.hs_kv_read_mx(cache, gtable, dev(off), int(off[-1]))
    for x in (0, 1):
        assert np.array_equal(f64(got[x]), np.concatenate([kept[s][x] for s in range(B)]))
