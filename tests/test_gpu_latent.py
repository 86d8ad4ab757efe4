"""GPU parity of the cache of latents and of the attention over it: rows bit for bit, attention against 64 bits within derived bounds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from latent_util import DEV, Prompt, Tree, compare, dev, offsets  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_13254_amd as h
    return h


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("N,R,Dr,dtype", [(1, 512, 64, BF), (300, 512, 64, BF), (77, 24, 8, BF), (5, 16, 0, F32), (1000, 100, 4, F32), (4097, 512, 64, F32)])
def test_rows_go_to_their_slots_and_come_back(hs, N, R, Dr, dtype):
    rs = np.random.RandomState(N)
    pages = -(-N // 64) + 2
    slots = rs.permutation(pages * 64)[:N].astype(np.int64)
    for x in range(0, N, 7):
        slots[x] = (-1, pages * 64, 2 ** 40, -2 ** 40)[x % 4]     # no slot
    wide = torch.randn((N, R + Dr + 16), device=DEV).to(dtype)
    c, r = wide[:, :R], wide[:, R:R + Dr]                          # rows with a stride
    pool = torch.full((pages, 64, R + Dr), 7.0, dtype=dtype, device=DEV)
    want = pool.clone().view(-1, R + Dr)
    ok = (slots >= 0) & (slots < pages * 64)
    want[dev(slots[ok])] = torch.cat([c, r], 1)[dev(np.nonzero(ok)[0])]
    hs.hs_latent_store(c, r, dev(slots), pool)
    assert torch.equal(pool.view(-1, R + Dr), want)
    out = torch.full((N, R + Dr), 3.0, dtype=dtype, device=DEV)
    hs.hs_latent_read(pool, dev(slots), R, out=(out[:, :R], out[:, R:]))
    keep = dev(ok)[:, None]
    assert torch.equal(out, torch.where(keep, wide[:, :R + Dr], torch.full_like(out, 3.0)))
    got = hs.hs_latent_read(pool, dev(slots[ok][::-1].copy()), R)   # tensors of its own
    assert torch.equal(torch.cat(got, 1), wide[:, :R + Dr][dev(np.nonzero(ok)[0][::-1].copy())])


def test_rows_beyond_32_bits(hs):
    """Slots whose bytes lie behind 2^32 and whose elements behind 2^31."""
    pages = 60000
    pool = torch.empty((pages, 64, 576), dtype=BF, device=DEV)
    slots = dev(np.array([pages * 64 - 1, 0, 2 ** 31 // 576 + 3, 2 ** 32 // 1152 + 1], np.int64))
    pool.view(-1, 576)[slots] = 0.0
    x = torch.randn((4, 576), device=DEV).to(BF)
    hs.hs_latent_store(x[:, :512], x[:, 512:], slots, pool)
    assert torch.equal(pool.view(-1, 576)[slots], x)
    c, r = hs.hs_latent_read(pool, slots, 512)
    assert torch.equal(torch.cat([c, r], 1), x)


# ------------------------------------------------------------------------------------------------ absorbed
CHAIN = [np.arange(-1, 99, dtype=np.int32)]
TREES = [  # rows, tokens
    ([1], [0]), ([1], [1]), ([1], [63]), ([1], [64]), ([1], [65]), ([1], [2048]), ([2], [31]), ([61], [2047]), ([5, 0, 33, 1], [100, 50, 0, 700]), ([129], [130]),
    ([7, 8, 9], [64, 128, 192]), ([1] * 70, list(range(0, 700, 10))), ([33], [0])]


@pytest.mark.parametrize("Hq", [16, 1, 3, 20, 64, 128])
@pytest.mark.parametrize("sizes,lens", TREES)
def test_tree_attention(hs, sizes, lens, Hq):
    Tree(sizes, lens, Hq, seed=Hq + sum(lens)).check(hs)


@pytest.mark.parametrize("sizes,lens,Hq,R,Dr,dtype", [([61], [200], 8, 512, 64, F32), ([5, 0, 33, 1], [100, 50, 0, 700], 3, 96, 32, F32), ([9, 2], [65, 1], 5, 100, 20, BF),
                                                      ([3], [64], 2, 1024, 128, BF), ([4], [70], 4, 33, 7, F32), ([6], [130], 16, 256, 64, BF), ([6], [130], 16, 512, 0, BF),
                                                      ([1, 1], [0, 2048], 16, 512, 64, F32)])
def test_tree_attention_other_shapes(hs, sizes, lens, Hq, R, Dr, dtype):
    Tree(sizes, lens, Hq, R, Dr, dtype, seed=R).check(hs)


@pytest.mark.parametrize("n,Hq", [(300, 2), (1024, 1), (1000, 16)])
def test_large_trees_and_chains(hs, n, Hq):
    Tree([n], [70], Hq, seed=n).check(hs)
    Tree([n], [0], Hq, seed=n, trees=[np.arange(-1, n - 1, dtype=np.int32)]).check(hs)
    star = np.zeros(n, np.int32)
    star[0] = -1
    Tree([n], [1], Hq, seed=n, trees=[star]).check(hs)


def _full_chip(Hq, seed=0, B=140):
    """More items than a launch of small groups is made for: groups of up to 128 rows, with every number of row blocks."""
    rs = np.random.RandomState(seed)
    lens = [0, 1, 63, 64, 65, 127, 128, 129, 191, 700, 1500] + [int(v) for v in rs.randint(0, 400, B - 11)]
    return Tree([int(v) for v in rs.randint(1, 4, B)], lens, Hq, seed=seed)


@pytest.mark.parametrize("Hq", [16, 40, 64, 100, 128])
def test_full_chips(hs, Hq):
    _full_chip(Hq, seed=Hq).check(hs)


@pytest.mark.parametrize("Hq", [16, 64, 128])
def test_full_chips_scores_that_grow(hs, Hq):
    t = _full_chip(Hq, seed=1)
    t.q[:] = 0.0
    t.q[:, :, 5] = 8.0
    t.q[:, 1::2, 5] = -8.0
    for s, (p, l) in enumerate(zip(t.prefix, t.lens)):
        p[:, 5] = (torch.arange(l, device=DEV) * (2.0 if s % 2 else -1.5)).to(BF)
        for b in range(-(-l // 64)):
            part = p[64 * b:64 * b + 64]
            t.pool[int(t.table_host[s, b]), :part.shape[0]] = part
    t.check(hs)


@pytest.mark.parametrize("Hq", [16, 64, 128])
def test_full_chips_nan(hs, Hq):
    from latent_util import ancestors
    t = _full_chip(Hq, seed=2)
    want = t.want()
    first = np.concatenate([[0], np.cumsum(t.sizes)])
    clean = torch.ones(t.NN, dtype=torch.bool, device=DEV)
    for s in range(0, t.B, 7):                                            # the last tree row of every seventh sequence
        row = int(first[s + 1]) - 1
        t.c_tree[row, 11] = float("nan") if s % 2 else float("inf")
        clean[int(first[s]):int(first[s + 1])] = dev(~ancestors(t.parents[s])[:, t.sizes[s] - 1])
    t.pool[int(t.table_host[9, 3]), 17, 570] = float("nan")               # a stored token of the tenth
    clean[int(first[9]):int(first[10])] = False
    o, lse = t.call(hs)
    compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
    assert (~torch.isfinite(o[~clean])).flatten(1).any(1).all()


@pytest.mark.parametrize("B,Hq,long", [(300, 16, 20000), (700, 3, 9000), (257, 128, 3000)])
def test_many_sequences_and_a_long_one(hs, B, Hq, long):
    rs = np.random.RandomState(B)
    lens = [int(v) for v in rs.randint(0, 200, B)]
    lens[B // 2] = long
    sizes = [int(v) for v in rs.randint(0, 3, B)]
    sizes[B // 2] = 2
    t = Tree(sizes, lens, Hq, seed=B)
    t.check(hs)
    ws = hs.hs_tree_attention_latent_workspace(t.host_no, t.host_pl, Hq, 512, 64, DEV)
    if ws is not None:                                                    # records of the sequences that are cut, not of all
        assert ws.numel() < 2064 * 2 * Hq * 400
        with pytest.raises(hs.HsError):
            t.call(hs, ws=ws[:ws.numel() - 256])
        with pytest.raises(ValueError):
            t.call(hs, ws=ws.cpu())


def test_a_long_sequence_among_more_than_fill_the_chip(hs):
    rs = np.random.RandomState(5)
    lens = [int(v) for v in rs.randint(0, 130, 1500)]
    lens[700] = 60000
    Tree([1] * 1500, lens, 16, seed=5).check(hs)
    keys = [int(v) for v in rs.randint(1, 70, 1500)]
    keys[3] = 30000
    Prompt([1] * 1500, keys, 2, seed=6).check(hs)


def test_long_caches(hs):
    Tree([1, 3, 1], [70000, 33333, 16384], 16, seed=3).check(hs)
    Tree([2], [40001], 128, seed=4).check(hs)


@pytest.mark.parametrize("Hq", [16, 128])
@pytest.mark.parametrize("way", ["up", "down", "late"])
def test_scores_that_grow(hs, Hq, way):
    """Maxima that move by hundreds from page to page, or all at once at the end."""
    t = Tree([3], [513], Hq, seed=8)
    t.q[:] = 0.0
    t.q[:, :, 5] = 8.0
    t.q[:, 1::2, 5] = -8.0
    size = {"up": torch.linspace(0, 900, 513), "down": torch.linspace(900, 0, 513), "late": torch.cat([torch.zeros(512), torch.full((1,), 2000.0)])}[way]
    t.prefix[0][:, 5] = size.to(DEV).to(BF)
    for b in range(9):
        part = t.prefix[0][64 * b:64 * b + 64]
        t.pool[int(t.table_host[0, b]), :part.shape[0]] = part
    t.check(hs)


def test_values_of_large_magnitude(hs):
    t = Tree([5], [200], 16, seed=9)
    for x in (t.pool, t.c_tree, t.r_tree):
        x.mul_(2.0 ** 85)
    t.prefix = [p * 2.0 ** 85 for p in t.prefix]
    t.scale *= 2.0 ** -85
    t.check(hs)


def test_strides_and_transposed_heads(hs):
    """Queries and results head by head, as products over heads leave and take them; tree rows out of a fused projection."""
    t = Tree([61, 3], [300, 70], 16, seed=10)
    want = t.want()
    turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    t.q, t.q_rope = turned(t.q), turned(t.q_rope)
    fused = torch.cat([torch.zeros_like(t.r_tree), t.c_tree, t.r_tree], 1)
    t.c_tree, t.r_tree = fused[:, 64:576], fused[:, 576:]
    o = torch.empty((16, t.NN, 512), dtype=BF, device=DEV).transpose(0, 1)
    got = t.call(hs, out=o)
    assert got[0] is o
    compare(got, want)
    wide = torch.zeros((t.NN, 16, 600), dtype=BF, device=DEV)
    compare(t.call(hs, out=wide[..., 8:520]), want)
    assert not wide[..., :8].any() and not wide[..., 520:].any()
    odd = torch.zeros((t.NN, 16, 513), dtype=BF, device=DEV)              # rows that begin at odd addresses
    compare(t.call(hs, out=odd[..., 1:]), want)
    shifted = torch.empty(t.q.numel() + 1, dtype=BF, device=DEV)[1:].view(t.NN, 16, 512)
    shifted.copy_(t.q)
    t.q = shifted
    compare(t.call(hs), want)


@pytest.mark.parametrize("Hq", [16, 64])
def test_nan_reaches_the_rows_that_see_it_alone(hs, Hq):
    t = Tree([40, 5], [100, 70], Hq, seed=11)
    want = t.want()
    for row, at, value in ((7, 3, float("nan")), (20, 511, float("inf")), (33, 100, float("-inf")), (12, None, float("nan"))):
        keep = t.c_tree.clone(), t.r_tree.clone()
        if at is None:
            t.r_tree[row, 9] = value
        else:
            t.c_tree[row, at] = value
        o, lse = t.call(hs)
        from latent_util import ancestors
        sees = dev(ancestors(t.parents[0])[:, row])
        clean = torch.ones(45, dtype=torch.bool, device=DEV)
        clean[:40] = ~sees
        compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
        assert (~torch.isfinite(o[~clean])).flatten(1).any(1).all() or at is None and torch.isnan(lse[~clean]).all()
        t.c_tree, t.r_tree = keep
    t.pool[int(t.table_host[1, 0]), 3, 17] = float("nan")                 # a stored token of the second sequence
    o, lse = t.call(hs)
    compare((o[:40], lse[:40]), tuple(w[:40] for w in want))
    assert torch.isnan(o[40:]).any(-1).all()


def test_rows_behind_the_last_sequence_and_bad_entries(hs):
    t = Tree([4, 3], [100, 64], 16, seed=12)
    want = t.want()
    big = torch.full((9, 16, 512), 5.0, dtype=BF, device=DEV)
    compare(t.call(hs, out=big[:7]), want)
    assert (big[7:] == 5.0).all()
    t.table[1, 0] = -3                                                    # an entry that is no page: values are not defined, the other sequence's are
    o, lse = t.call(hs)
    compare((o[:4], lse[:4]), tuple(w[:4] for w in want))


def test_same_bits_other_streams_and_a_captured_call(hs):
    t = Tree([61, 1, 30], [700, 2000, 3], 16, seed=13)
    want = t.want()
    a = t.check(hs)
    b = t.call(hs)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c = t.call(hs, stream=side)
    side.synchronize()
    assert torch.equal(a[0], c[0])
    ws = hs.hs_tree_attention_latent_workspace(t.host_no, t.host_pl, 16, 512, 64, DEV)
    o, lse = torch.empty_like(a[0]), torch.empty_like(a[1])
    t.call(hs, out=o, lse=lse, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.call(hs, out=o, lse=lse, ws=ws)
    for x in range(3):
        o.fill_(9.0)
        lse.fill_(9.0)
        t.q.mul_(1.0 if x < 2 else 2.0)
        graph.replay()
        torch.cuda.synchronize()
        d = t.call(hs)
        assert torch.equal(o, d[0]) and torch.equal(lse, d[1])
    assert want is not None


def test_a_cache_beyond_32_bits(hs):
    """Pages at the end of a pool of 5 GB."""
    t = Tree([5], [130], 16, seed=14)
    want = t.want()
    pages = 70000
    big = torch.empty((pages, 64, 576), dtype=BF, device=DEV)
    for b in range(3):
        big[pages - 1 - 20000 * b] = t.pool[int(t.table_host[0, b])]
        t.table[0, b] = pages - 1 - 20000 * b
    t.pool = big
    compare(t.call(hs), want)


def test_tree_refusals(hs):
    t = Tree([4], [100], 16, seed=15)
    for name, bad in (("q", t.q[..., :511]), ("q", t.q.float()), ("q_rope", t.q_rope[:3]), ("pool", t.pool[..., :575]), ("pool", t.pool[:, :32]), ("c_tree", t.c_tree[:3]),
                      ("r_tree", t.r_tree.cpu()), ("parent", t.parent[:3]), ("no", t.no[:1]), ("pl", t.pl.int()), ("table", t.table[0]), ("table", t.table.long())):
        keep = getattr(t, name)
        setattr(t, name, bad)
        with pytest.raises(ValueError):
            t.call(hs)
        setattr(t, name, keep)
    with pytest.raises(ValueError):
        t.call(hs, out=torch.empty((4, 16, 511), dtype=BF, device=DEV))
    with pytest.raises(ValueError):
        t.call(hs, out=torch.empty((4, 16, 512), dtype=F32, device=DEV))
    with pytest.raises(hs.HsError):
        t.call(hs, out=torch.empty((1, 16, 512), dtype=BF, device=DEV).expand(4, 16, 512))
    t.host_pl = t.host_pl + 64 * 64
    with pytest.raises(hs.HsError):
        t.call(hs)


# ------------------------------------------------------------------------------------------------ expanded
PROMPTS = [  # rows, keys
    ([1], [1]), ([1], [700]), ([64], [64]), ([65], [65]), ([63], [127]), ([256], [256]), ([257], [300]), ([300], [2000]), ([5, 0, 33, 1], [100, 50, 33, 700]),
    ([130, 1, 700, 64], [163, 9000, 733, 64]), ([7, 4], [3, 0]), ([100], [40]), ([1] * 70, list(range(1, 701, 10)))]


@pytest.mark.parametrize("H", [16, 1, 5])
@pytest.mark.parametrize("rows,keys", PROMPTS)
def test_prompt_attention(hs, rows, keys, H):
    Prompt(rows, keys, H, seed=H + sum(keys)).check(hs)


@pytest.mark.parametrize("rows,keys,H,Dn,Dr,Dv,dtype", [([61], [200], 4, 128, 64, 128, F32), ([5, 0, 33], [100, 50, 33], 3, 96, 32, 64, F32), ([9, 2], [65, 1], 5, 100, 20, 36, BF),
                                                        ([70], [70], 2, 128, 0, 128, BF), ([30], [90], 2, 64, 64, 256, BF), ([40], [41], 3, 128, 64, 64, BF)])
def test_prompt_attention_other_shapes(hs, rows, keys, H, Dn, Dr, Dv, dtype):
    Prompt(rows, keys, H, Dn, Dr, Dv, dtype, seed=Dn).check(hs)


@pytest.mark.parametrize("B,H,long", [(600, 4, 9000), (70, 8, 20000)])
def test_many_prompts_and_a_long_one(hs, B, H, long):
    rs = np.random.RandomState(B)
    rows = [int(v) for v in rs.randint(0, 20, B)]
    keys = [n + int(v) for n, v in zip(rows, rs.randint(0, 100, B))]
    rows[B // 2], keys[B // 2] = 40, long
    p = Prompt(rows, keys, H, seed=B)
    p.check(hs)
    ws = hs.hs_prompt_attention_latent_workspace(p.host_qo, p.host_ko, H, 128, DEV)
    if ws is not None:
        assert ws.numel() < 528 * H * 40 * 400
        with pytest.raises(hs.HsError):
            p.call(hs, ws=ws[:ws.numel() - 256])



WIDE = [([257] * 9, [300] * 9, 64), ([700, 1, 257, 40, 0, 33], [900, 500, 257, 20, 100, 33], 96), ([300, 900], [20000, 5000], 24), ([513], [3001], 96)]


@pytest.mark.parametrize("rows,keys,H", WIDE)
def test_prompts_that_fill_the_chip(hs, rows, keys, H):
    """Eight waves with rows of their own, where the calls of few heads have four."""
    Prompt(rows, keys, H, seed=H).check(hs)


def test_prompts_that_fill_the_chip_with_nan(hs):
    p = Prompt([300, 260], [513, 260], 128, seed=13)
    want = p.want()
    p.v[500, :, 3], p.k[700, :, 5] = float("nan"), float("nan")
    o, lse = p.call(hs)
    clean = torch.ones(560, dtype=torch.bool, device=DEV)
    clean[500 - 213:300] = False
    clean[300 + 700 - 513:] = False
    compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
    assert torch.isnan(o[~clean]).any(-1).all()


def test_prompts_that_fill_the_chip_with_scores_that_grow(hs):
    p = Prompt([300], [513], 256, seed=14)
    p.q[:] = 0.0
    p.q[:, :, 5] = 8.0
    p.k[:, :, 5] = torch.linspace(0, 900, 513).to(DEV).to(BF)[:, None]
    p.check(hs)


def test_long_prompts(hs):
    Prompt([2500], [2500], 8, seed=3).check(hs)
    Prompt([300, 900], [20000, 5000], 2, seed=4).check(hs)


@pytest.mark.parametrize("way", ["up", "down", "late"])
def test_prompt_scores_that_grow(hs, way):
    p = Prompt([300], [513], 4, seed=8)
    p.q[:] = 0.0
    p.q[:, :, 5] = 8.0
    p.q[:, 1::2, 5] = -8.0
    size = {"up": torch.linspace(0, 900, 513), "down": torch.linspace(900, 0, 513), "late": torch.cat([torch.zeros(512), torch.full((1,), 2000.0)])}[way]
    p.k[:, :, 5] = size.to(DEV).to(BF)[:, None]
    p.check(hs)


def test_prompt_strides(hs):
    p = Prompt([70, 30], [100, 30], 6, seed=10)
    want = p.want()
    turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    p.q, p.q_rope, p.k = turned(p.q), turned(p.q_rope), turned(p.k)
    o = torch.empty((6, p.N, 128), dtype=BF, device=DEV).transpose(0, 1)
    compare(p.call(hs, out=o), want)
    both = torch.cat([p.q, p.q_rope], 2)                                  # the query as one row a head
    p.q, p.q_rope = both[..., :128], both[..., 128:]
    wide = torch.zeros((p.N, 6, 144), dtype=BF, device=DEV)
    compare(p.call(hs, out=wide[..., 8:136]), want)
    assert not wide[..., :8].any() and not wide[..., 136:].any()
    shifted = torch.empty(p.T * 65, dtype=BF, device=DEV).view(p.T, 65)[:, 1:]
    shifted.copy_(p.k_rope)
    p.k_rope = shifted
    compare(p.call(hs), want)


def test_prompt_nan_reaches_the_rows_that_see_it_alone(hs):
    for at, value in ((90, float("nan")), (130, float("inf")), (199, float("-inf")), (64, float("nan"))):
        for name in ("k", "v", "k_rope"):
            p = Prompt([150, 20], [200, 30], 3, seed=11)
            want = p.want()
            getattr(p, name)[at, ..., 2] = value
            o, lse = p.call(hs)
            clean = torch.ones(170, dtype=torch.bool, device=DEV)
            clean[max(0, at - 50):150] = False
            compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
            if name == "v":
                assert (~torch.isfinite(o[~clean])).any(-1).all()
            elif value != value:
                assert torch.isnan(o[~clean]).all()


def test_prompt_rows_behind_and_between(hs):
    """Keys behind a sequence's last are another's: with NaN in them, nothing of them is seen; output rows behind the last are left."""
    p = Prompt([10, 40], [33, 90], 4, seed=12)
    want = p.want()
    p.k[33:], p.v[33:], p.k_rope[33:] = float("nan"), float("nan"), float("nan")
    big = torch.full((60, 4, 128), 5.0, dtype=BF, device=DEV)
    o, lse = p.call(hs, out=big[:50])
    compare((o[:10], lse[:10]), tuple(w[:10] for w in want))
    assert torch.isnan(o[10:]).all() and (big[50:] == 5.0).all()


def test_prompt_same_bits_other_streams_and_a_captured_call(hs):
    p = Prompt([130, 1, 300], [400, 2000, 300], 8, seed=13)
    a = p.check(hs)
    b = p.call(hs)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c = p.call(hs, stream=side)
    side.synchronize()
    assert torch.equal(a[0], c[0])
    ws = hs.hs_prompt_attention_latent_workspace(p.host_qo, p.host_ko, 8, 128, DEV)
    o, lse = torch.empty_like(a[0]), torch.empty_like(a[1])
    p.call(hs, out=o, lse=lse, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(hs, out=o, lse=lse, ws=ws)
    for x in range(3):
        o.fill_(9.0)
        lse.fill_(9.0)
        p.q.mul_(1.0 if x < 2 else 2.0)
        graph.replay()
        torch.cuda.synchronize()
        d = p.call(hs)
        assert torch.equal(o, d[0]) and torch.equal(lse, d[1])


def test_prompt_refusals(hs):
    p = Prompt([4], [100], 4, seed=15)
    for name, bad in (("q", p.q[..., :127]), ("q", p.q.float()), ("q_rope", p.q_rope[:3]), ("k", p.k[:, :3]), ("k_rope", p.k_rope[:5]), ("v", p.v[:5]), ("qo", p.qo.long()),
                      ("ko", p.ko.int()), ("ko", p.ko[:1]), ("host_qo", p.host_qo + 1), ("host_ko", p.host_ko + 1)):
        keep = getattr(p, name)
        setattr(p, name, bad)
        with pytest.raises((ValueError, hs.HsError)):
            p.call(hs)
        setattr(p, name, keep)
    with pytest.raises(ValueError):
        p.call(hs, out=torch.empty((4, 4, 127), dtype=BF, device=DEV))


# ------------------------------------------------------------------------------------------------ together
def test_a_request_from_prompt_to_accepted_drafts(hs):
    """Two requests: pages, the prompt in two chunks (stored, read back, expanded attention), then steps of a draft tree (pages reserved, absorbed
    attention, the accepted path committed by its slots, the rest given back), against attention over plain copies of what was stored."""
    rs = np.random.RandomState(0)
    g = torch.Generator(device=DEV).manual_seed(0)
    B, H, R, Dr, D, scale = 2, 4, 512, 64, 128, 192 ** -0.5
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF)  # noqa: E731
    Wk, Wv = (rnd(H, R, D).float() * R ** -0.5 for _ in range(2))
    t = hs.new_page_tables(B, 8, 14)
    pool = hs.new_latent_cache(14, R, Dr)
    pool.fill_(float("nan"))
    lens = torch.zeros(B, dtype=torch.int64, device=DEV)
    kept = [torch.zeros((0, R + Dr), dtype=BF, device=DEV) for _ in range(B)]
    for chunk in ([70, 9], [50, 130]):
        rows, off = np.array(chunk), offsets(chunk, np.int32)
        n = int(off[-1])
        held, count = hs.hs_block_tables(lens + dev(rows), t["block_table"], t["held"], t["free_pages"], t["free_count"])
        t["held"], t["free_count"] = held, count
        new = torch.empty_like(lens)
        slots = hs.hs_slot_map(dev(off), n, lens, t["block_table"], 14, held=held, new_lens=new)
        x = rnd(n, R + Dr)
        hs.hs_latent_store(x[:, :R], x[:, R:], slots, pool)
        kept = [torch.cat([k, x[off[s]:off[s + 1]]]) for s, k in enumerate(kept)]
        total = offsets([len(k) for k in kept])
        where = hs.hs_slot_map(dev(total.astype(np.int32)), int(total[-1]), torch.zeros_like(lens), t["block_table"], 14, held=held)
        c, r = hs.hs_latent_read(pool, where, R)
        assert torch.equal(torch.cat([c, r], 1), torch.cat(kept))
        assert new.tolist() == [len(k) for k in kept]
        p = Prompt(chunk, [len(k) for k in kept], H, seed=1)
        p.k = torch.stack([c.float() @ Wk[h] for h in range(H)], 1).to(BF)
        p.v = torch.stack([c.float() @ Wv[h] for h in range(H)], 1).to(BF)
        p.k_rope = r
        p.check(hs)
        lens = new
    for step in range(3):
        sizes = [int(v) for v in rs.randint(1, 40, B)]
        tr = Tree(sizes, [len(k) for k in kept], H, seed=step)
        tr.prefix, tr.pool, tr.table, tr.pl = kept, pool, t["block_table"], lens
        held, count = hs.hs_block_tables(lens + dev(np.array(sizes)), t["block_table"], t["held"], t["free_pages"], t["free_count"])
        tr.check(hs)
        path, length = np.full((B, 5), -1, np.int32), np.zeros(B, np.int32)
        for s in range(B):
            at = 0
            while length[s] < 5 and (tr.parents[s] == at).any():
                at = int(np.nonzero(tr.parents[s] == at)[0][0])
                path[s, length[s]] = at
                length[s] += 1
        new = torch.empty_like(lens)
        slots = hs.hs_slot_map(tr.no, tr.NN, lens, t["block_table"], 14, held=held, accept_path=dev(path), accept_len=dev(length), new_lens=new)
        hs.hs_latent_store(tr.c_tree, tr.r_tree, slots, pool)
        t["held"], t["free_count"] = hs.hs_block_tables(new, t["block_table"], held, t["free_pages"], count)
        first = [0, sizes[0]]
        for s in range(B):
            rows = [first[s]] + [first[s] + int(v) for v in path[s, :length[s]]]
            kept[s] = torch.cat([kept[s], torch.cat([tr.c_tree, tr.r_tree], 1)[rows]])
        lens = new
        assert lens.tolist() == [len(k) for k in kept]
        assert t["held"].tolist() == [-(-len(k) // 64) for k in kept] and int(t["free_count"]) == 14 - sum(t["held"].tolist())


# ------------------------------------------------------------------------------------------------ scores of -infinity
# By the definition such a score is a weight of zero, 0 x infinity is NaN, and a row that sees no other score is 0 / 0: NaN, with a logarithm of -infinity.  A row
# that sees no key is 0.
OTHER = [(96, 32, F32), (100, 20, BF), (512, 64, F32), (512, 0, BF)]


@pytest.mark.parametrize("R,Dr,dtype", OTHER)
@pytest.mark.parametrize("L,n", [(5, 1), (70, 1), (200, 1), (300, 1), (0, 3), (5, 3), (300, 3)])
def test_other_shapes_a_latent_that_scores_minus_infinity(hs, L, n, R, Dr, dtype):
    """The tree's last row holds an infinity against which its own query points; no other row sees it."""
    t = Tree([n, 2], [L, 70], 3, R, Dr, dtype, seed=L + R, trees=[np.array([-1, 0, 0], np.int32)[:n], np.array([-1, 0], np.int32)])
    want = t.want()
    row, clean = n - 1, [x for x in range(n + 2) if x != n - 1]
    t.q[row, :, 0] = 1.0
    t.c_tree[row, 0] = float("-inf")
    o, lse = t.call(hs)
    compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
    assert torch.isnan(o[row, :, 0]).all()
    rest = torch.cat([t.prefix[0], torch.cat([t.c_tree, t.r_tree], 1)[:min(row, 1)]])  # what the row sees besides: the prefix and the root
    compare((o[row:row + 1, :, 1:], lse[row:row + 1]), Rest(t, row, rest).want(slice(1, None)))


class Rest:
    """One tree row's attention over given tokens alone."""

    def __init__(self, t, row, tokens):
        self.t, self.q, self.tokens = t, torch.cat([t.q[row], t.q_rope[row]], 1).double(), tokens.double()

    def want(self, columns=slice(None)):
        from latent_util import fill
        H, R = self.t.Hq, self.t.R
        o, lse = torch.zeros((H, R), dtype=torch.float64, device=DEV), torch.zeros(H, dtype=torch.float64, device=DEV)
        bo, bl = torch.zeros_like(o), torch.zeros_like(lse)
        fill(self.q, self.tokens, self.tokens[:, :R], torch.zeros((H, len(self.tokens)), dtype=torch.bool, device=DEV), self.t.scale, self.t.dtype, o, lse, bo, bl)
        return o[None, :, columns], lse[None], bo[None, :, columns], bl[None]


@pytest.mark.parametrize("R,Dr,dtype", OTHER + [(512, 64, BF)])
def test_tree_rows_that_see_scores_of_minus_infinity_alone(hs, R, Dr, dtype):
    """A root without a prefix, and a root whose whole prefix scores -infinity too."""
    t = Tree([2, 1], [0, 150], 3, R, Dr, dtype, seed=R)
    want = t.want()
    t.q[0, :, 0], t.q[2, :, 0] = 1.0, 1.0
    t.c_tree[0, 0] = t.c_tree[2, 0] = float("-inf")
    for b in range(3):
        t.pool[int(t.table_host[1, b]), :, 0] = float("-inf")
    o, lse = t.call(hs)
    for row in (0, 2):
        assert torch.isnan(o[row]).all()
        assert not torch.isfinite(lse[row]).any() and not (lse[row] > 0).any()
    assert want is not None


@pytest.mark.parametrize("R,Dr,dtype", [(96, 32, F32), (100, 20, BF), (512, 64, F32), (512, 64, BF)])
def test_a_stored_rotary_part_of_minus_infinity_is_a_weight_of_zero(hs, R, Dr, dtype):
    t = Tree([2, 1], [130, 70], 3, R, Dr, dtype, seed=R + 1)
    t.q_rope[:2, :, 1] = 1.0
    t.pool[int(t.table_host[0, 1]), 9, R + 1] = float("-inf")             # token 73 of the first sequence
    whole = t.prefix[0]
    t.prefix[0] = torch.cat([whole[:73], whole[74:]])
    t.lens[0] = 129
    want = t.want()
    compare(t.call(hs), want)


@pytest.mark.parametrize("R,Dr,dtype", OTHER)
def test_other_shapes_nan_reaches_the_rows_that_see_it_alone(hs, R, Dr, dtype):
    from latent_util import ancestors
    t = Tree([70, 5], [100, 70], 2, R, Dr, dtype, seed=R + 2)
    want = t.want()
    for row, at, value in ((7, 3, float("nan")), (66, R - 1, float("inf")), (30, 2, float("-inf"))):
        keep = t.c_tree.clone()
        t.c_tree[row, at] = value
        o, lse = t.call(hs)
        clean = torch.ones(75, dtype=torch.bool, device=DEV)
        clean[:70] = ~dev(ancestors(t.parents[0])[:, row])
        compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
        assert (~torch.isfinite(o[~clean])).flatten(2).any(2).all()
        t.c_tree = keep
    t.pool[int(t.table_host[1, 0]), 3, 5] = float("nan")
    o, lse = t.call(hs)
    compare((o[:70], lse[:70]), tuple(w[:70] for w in want))
    assert torch.isnan(o[70:]).all()


PROMPT_OTHER = [(96, 32, 64, F32), (100, 20, 36, BF), (128, 64, 128, F32)]


def _keys_of_minus_infinity(hs, Dn, Dr, Dv, dtype, rows, keys, H, cut):
    """The first sequence's keys all score -infinity, as does the first key of the second and a later one; the third has rows in front of its keys."""
    p = Prompt(rows, keys, H, Dn, Dr, Dv, dtype, seed=Dn + sum(rows))
    if cut:
        assert hs.hs_prompt_attention_latent_workspace(p.host_qo, p.host_ko, H, Dv, DEV) is not None
    qo, ko = p.host_qo.tolist(), p.host_ko.tolist()
    p.q[:, :, 1] = 1.0
    later = (ko[1] + ko[2]) // 2                                          # seen by some rows of the second sequence, or all
    p.k[:, :, 1] = 0.0
    want = p.want()
    p.k[:ko[1], :, 1] = float("-inf")
    p.k[ko[1], :, 1] = p.k[later, :, 1] = float("-inf")
    o, lse = p.call(hs)
    none = torch.tensor([keys[0] - rows[0] + i + 1 <= 0 for i in range(rows[0])], device=DEV)
    first, lone = slice(0, qo[1]), keys[1] - rows[1] == 0
    assert (o[first][none] == 0).all() and torch.isnan(o[first][~none]).all() and torch.isneginf(lse[first]).all()
    if lone:                                                              # the row that sees the first key alone
        assert torch.isnan(o[qo[1]]).all() and torch.isneginf(lse[qo[1]]).all()
    compare((o[qo[2]:], lse[qo[2]:]), tuple(w[qo[2]:] for w in want))
    # the others, as if those keys were not there: their weights are zero
    a, b, k0, k1 = qo[1], qo[2], ko[1], ko[2]
    hide = torch.arange(k1 - k0, device=DEV)[None] > (torch.arange(b - a, device=DEV) + (k1 - k0) - (b - a))[:, None]
    hide[:, 0] = hide[:, later - k0] = True
    from latent_util import fill
    p.k[:, :, 1] = 0.0
    skip = 1 if lone else 0
    for h in range(H):
        part = [torch.zeros(b - a, Dv, dtype=torch.float64, device=DEV), torch.zeros(b - a, dtype=torch.float64, device=DEV)]
        more = [torch.zeros_like(x) for x in part]
        fill(torch.cat([p.q[a:b, h], p.q_rope[a:b, h]], 1).double(), torch.cat([p.k[k0:k1, h], p.k_rope[k0:k1]], 1).double(), p.v[k0:k1, h].double(), hide, p.scale, dtype,
             part[0], part[1], more[0], more[1])
        compare((o[a + skip:b, h], lse[a + skip:b, h]), (part[0][skip:], part[1][skip:], more[0][skip:], more[1][skip:]))


@pytest.mark.parametrize("Dn,Dr,Dv,dtype", PROMPT_OTHER)
@pytest.mark.parametrize("rows,keys", [([3, 9, 4], [3, 9, 2]), ([70, 150, 30], [40, 150, 20]), ([5, 3, 1], [300, 200, 1])])
def test_prompts_of_other_shapes_keys_that_score_minus_infinity(hs, rows, keys, Dn, Dr, Dv, dtype):
    _keys_of_minus_infinity(hs, Dn, Dr, Dv, dtype, rows, keys, 3, False)


@pytest.mark.parametrize("Dn,Dr,Dv,dtype", PROMPT_OTHER)
def test_prompts_of_other_shapes_nan_reaches_the_rows_that_see_it_alone(hs, Dn, Dr, Dv, dtype):
    for at, value in ((90, float("nan")), (130, float("inf")), (199, float("-inf"))):
        p = Prompt([150, 20], [200, 30], 2, Dn, Dr, Dv, dtype, seed=at)
        want = p.want()
        p.v[at, :, 2] = value
        o, lse = p.call(hs)
        clean = torch.ones(170, dtype=torch.bool, device=DEV)
        clean[at - 50:150] = False
        compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
        assert (~torch.isfinite(o[~clean, :, 2])).all()


@pytest.mark.parametrize("rows,keys,H,cut", [([3, 9, 4], [3, 9, 2], 3, False), ([70, 150, 30], [40, 150, 20], 16, False), ([257, 300, 90], [300, 300, 50], 3, False),
                                             ([5, 3, 1], [3000, 2500, 1], 3, True), ([700, 650, 300], [640, 2000, 40], 1, True), ([300, 257, 3], [400, 257, 2], 128, False)])
def test_prompt_keys_that_score_minus_infinity(hs, rows, keys, H, cut):
    _keys_of_minus_infinity(hs, 128, 64, 128, BF, rows, keys, H, cut)


@pytest.mark.parametrize("rows,keys", [(64, 64), (300, 300), (200, 210), (700, 700)])
@pytest.mark.parametrize("H", [3, 64])
def test_a_lone_prompt_nan_among_its_first_keys(hs, rows, keys, H):
    """One sequence, whose first tile is masked: what is found in its values has to reach the rows that see it, and only those."""
    for at, column, value in ((0, 3, float("nan")), (5, 127, float("inf")), (40, 0, float("-inf")), (63, 64, float("nan"))):
        p = Prompt([rows], [keys], H, seed=at)
        want = p.want()
        p.v[at, :, column] = value
        for _ in range(3):
            o, lse = p.call(hs)
            clean = torch.ones(rows, dtype=torch.bool, device=DEV)
            clean[max(0, at - (keys - rows)):] = False
            compare((o[clean], lse[clean]), tuple(w[clean] for w in want))
            assert (~torch.isfinite(o[~clean])).any(-1).all()


def test_a_lone_prompt_of_more_rows_than_keys_that_is_cut(hs):
    p = Prompt([700], [640], 1, seed=5)
    assert hs.hs_prompt_attention_latent_workspace(p.host_qo, p.host_ko, 1, 128, DEV) is not None
    p.check(hs)
    p.k[:, :, 1] = float("-inf")
    p.q[:, :, 1] = 1.0
    o, lse = p.call(hs)
    assert (o[:60] == 0).all() and torch.isnan(o[60:]).all() and torch.isneginf(lse).all()


# ------------------------------------------------------------------------------------------------ scores of any magnitude
@pytest.mark.parametrize("power", [20, 30, 33, 40, 60, 100])
@pytest.mark.parametrize("Hq,sizes,lens", [(16, [1, 1], [0, 64]), (3, [40, 2], [0, 200]), (128, [3, 2], [70, 513])])
def test_scores_of_any_magnitude(hs, Hq, sizes, lens, power):
    """Scores far above 2^24 are one-hot: every row's own token has the largest, by a factor, and is the result."""
    NN = sum(sizes)
    t = Tree(sizes, lens, Hq, seed=power)
    t.pool[..., 512:], t.q[:], t.q_rope[:], t.r_tree[:] = 0.0, 0.0, 0.0, 0.0
    t.q_rope[:, :, 7] = 2.0 ** (power // 2) * 1.3
    depth = torch.zeros(NN)
    at = 0
    for n, parent in zip(sizes, t.parents):
        for i in range(1, n):
            depth[at + i] = depth[at + int(parent[i])] + 1
        at += n
    t.r_tree[:, 7] = ((1.0 + depth).to(DEV) * 2.0 ** (power - power // 2) * 1.7).to(BF)
    o, lse = t.call(hs)
    assert torch.equal(o, t.c_tree[:, None].expand(-1, Hq, -1))
    x = (t.q_rope.double()[:, :, 7] * t.r_tree.double()[:, None, 7]) * t.scale
    assert ((lse.double() - x).abs() <= 8 * 2.0 ** -24 * x).all()
    t.q_rope.neg_()                                       # all scores far below zero: the least of them, the root's, or the prefix's zeros
    o, lse = t.call(hs)
    at = 0
    for s, (n, L) in enumerate(zip(sizes, lens)):
        if L == 0:
            assert torch.equal(o[at:at + n], t.c_tree[at:at + 1, None].expand(n, Hq, -1))
        else:
            mean = t.prefix[s][:, :512].double().mean(0)
            size = t.prefix[s][:, :512].double().abs().mean(0)
            assert ((o[at:at + n].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + (2.0 ** -8 + 2.0 ** -17) * size).all()
            assert ((lse[at:at + n] - float(np.log(L))).abs() <= 1e-5).all()
        at += n


@pytest.mark.parametrize("power", [20, 30, 33, 40, 60, 100])
@pytest.mark.parametrize("rows,keys,H", [([1, 64], [1, 64], 3), ([100, 300], [130, 300], 16), ([5, 3], [3000, 2000], 2), ([300, 257], [300, 300], 128)])
def test_prompt_scores_of_any_magnitude(hs, rows, keys, H, power):
    """The last key that a row sees has the largest score by 1/64 of it at least: the result is its value."""
    p = Prompt(rows, keys, H, seed=power)
    p.q[:], p.q_rope[:], p.k[:], p.k_rope[:] = 0.0, 0.0, 0.0, 0.0
    p.q[:, :, 9] = 2.0 ** (power // 2) * 1.3
    ko, qo = p.host_ko.tolist(), p.host_qo.tolist()
    own = torch.cat([torch.arange(n) + ko[s + 1] - n for s, n in enumerate(rows)]).to(DEV)
    for s in range(2):                                    # rising in steps that bfloat16 holds: 64 of them to an octave
        i = torch.arange(keys[s], device=DEV).double()
        p.k[ko[s]:ko[s + 1], :, 9] = (2.0 ** (power - power // 2 - (keys[s] >> 6) + torch.floor(i / 64)) * (1.0 + (i % 64) / 64)).to(BF)[:, None]
    o, lse = p.call(hs)
    assert torch.equal(o, p.v[own])
    x = p.q.double()[:, :, 9] * p.k.double()[own, :, 9] * p.scale
    assert ((lse.double() - x).abs() <= 8 * 2.0 ** -24 * x).all()


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("R,Dr,dtype", [(512, 64, BF), (96, 32, F32)])
@pytest.mark.parametrize("L", [0, 70])
def test_scores_next_to_the_largest_float(hs, L, R, Dr, dtype, sign):
    """Products of 1.9 * 2^127, with a scale of 1: a row that sees nothing else is its own token, and one that sees a prefix of zero scores the prefix's mean or its own token."""
    t = Tree([1, 1], [L, L], 3, R, Dr, dtype, seed=L)
    t.pool[..., R:], t.q[:], t.q_rope[:], t.r_tree[:] = 0.0, 0.0, 0.0, 0.0
    t.q_rope[:, :, 7], t.r_tree[:, 7], t.scale = 2.0 ** 64, sign * 1.8984375 * 2.0 ** 63, 0.25
    o, lse = t.call(hs)
    t.scale = 1.0
    for got, scale in ((o, 0.25), (t.call(hs)[0], 1.0)):
        if L == 0 or sign > 0:
            assert torch.equal(got, t.c_tree[:, None].expand(-1, 3, -1)), scale
        else:
            for s in range(2):
                x = t.prefix[s][:, :R].double()
                assert ((got[s].double() - x.mean(0)).abs() <= 2.0 ** -8 * x.mean(0).abs() + 2.0 ** -7 * x.abs().mean(0)).all(), scale
    x = sign * 1.8984375 * 2.0 ** 125 if L == 0 or sign > 0 else float(np.log(L))
    assert ((lse.double() - x).abs() <= 8 * 2.0 ** -24 * abs(x)).all()


def test_prompt_scores_next_to_the_largest_float(hs):
    p = Prompt([3, 1], [3, 1], 3, seed=1)
    p.q[:], p.q_rope[:], p.k[:], p.k_rope[:] = 0.0, 0.0, 0.0, 0.0
    p.q[:, :, 9], p.k[:, :, 9], p.scale = 2.0 ** 64, -1.8984375 * 2.0 ** 63, 1.0
    o, _ = p.call(hs)
    assert torch.equal(o[[0, 3]], p.v[[0, 3]]) and torch.isfinite(o).all()
