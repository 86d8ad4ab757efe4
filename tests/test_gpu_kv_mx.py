"""GPU parity of the quantised cache's writers and reader: codes, scales and values are equal to the checker's, bit for bit, and what
a call does not name stays as it was."""
import numpy as np
import pytest

from oracle import mx_cache as mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
FMT = {"e4m3": 0, "e2m1": 1}


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_13254_amd as h
    return h


def dev(a, kind=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if kind is None else t.to(kind)).to(DEV)


class Cache:
    """A cache on the GPU and the checker's copy of it, filled with recognisable bytes."""

    def __init__(self, hs, pages, Hkv, D, fmt, seed=0):
        rs = np.random.RandomState(seed)
        self.fmt, self.pages = fmt, pages
        self.gpu = hs.new_mx_cache(pages, Hkv, D, FMT[fmt], DEV)
        self.ref = {}
        for n in ("k", "v"):
            codes = rs.randint(0, 16 if fmt == "e2m1" else 120, (pages, Hkv, 64, D)).astype(np.uint8)
            scales = rs.randint(110, 140, (pages, Hkv, 64, D // 32)).astype(np.uint8)
            self.ref[n + "_codes"], self.ref[n + "_scales"] = codes, scales
            stored = codes if fmt == "e4m3" else codes[..., 0::2] | (codes[..., 1::2] << 4)
            self.gpu[n + "_codes"].view(torch.uint8).copy_(dev(stored))
            self.gpu[n + "_scales"].copy_(dev(scales))

    def equal(self):
        torch.cuda.synchronize()
        for n in ("k", "v"):
            got = self.gpu[n + "_codes"].view(torch.uint8).cpu().numpy()
            if self.fmt == "e2m1":
                got = np.stack([got & 15, got >> 4], -1).reshape(self.ref[n + "_codes"].shape)
            assert np.array_equal(got, self.ref[n + "_codes"]), n
            assert np.array_equal(self.gpu[n + "_scales"].cpu().numpy(), self.ref[n + "_scales"]), n


def _rows(seed, shape, dtype, special=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(shape, generator=g, device=DEV) * torch.exp2(torch.randint(-20, 20, shape[:2] + (1,), generator=g, device=DEV).float())
    if special and shape[0] > 3:
        f = x.view(-1, 32)
        f[0] = 0.0
        f[1, 5], f[2, 31], f[3, 0] = float("nan"), float("inf"), float("-inf")
        f[4] = torch.arange(32, device=DEV).float() * 0.25 - 4.0          # ties of both formats
        f[5] = -0.0
        f[6] = 2.0 ** -126
        f[7] = 3.3e38 * torch.sign(f[7])
        f[8, 1:] = 2.0 ** -14 * f[8, 1:].sign()
        f[8, 0] = 448.0
    return x.to(dtype)


def _table(rs, B, blocks, pages):
    return rs.permutation(pages)[:B * blocks].reshape(B, blocks).astype(np.int32)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,Hkv,sizes,lens,blocks", [(128, 8, [9, 0, 70, 1], [60, 5, 0, 127], 3), (64, 3, [1], [0], 1), (32, 1, [130], [1], 3), (96, 2, [5, 6], [63, 64], 2),
                                                     (256, 1, [3, 3, 3], [190, 191, 500], 3), (64, 2, [0, 0], [7, 9], 1), (128, 1, [1] * 150, list(range(150)), 3)])
def test_append_and_read(hs, D, Hkv, sizes, lens, blocks, dtype, fmt):
    """Rows behind what is stored; sequences that are full, overflow, or are empty; more sequences than a wave has lanes."""
    rs, B, NN = np.random.RandomState(D), len(sizes), sum(sizes)
    pages = B * blocks + 2
    c, table = Cache(hs, pages, Hkv, D, fmt), _table(rs, B, blocks, pages)
    no, lens = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), np.asarray(lens, np.int64)
    k, v = _rows(1, (NN, Hkv, D), dtype), _rows(2, (NN, Hkv, D), dtype)
    new, glens = torch.full((B,), -7, dtype=torch.int64, device=DEV), dev(lens)
    hs.hs_kv_append_mx(k, v, dev(no), c.gpu, dev(table), glens, new_lens=new)
    rows = [list(range(no[s], no[s + 1])) for s in range(B)]
    for n, x in (("k", k), ("v", v)):
        want = mx.store(x.double().cpu().numpy(), rows, lens, table, pages, c.ref[n + "_codes"], c.ref[n + "_scales"], fmt)
    c.equal()
    assert new.tolist() == want.tolist() and glens.tolist() == lens.tolist()
    # what was stored, read back
    took = want - lens
    off = np.concatenate([[0], np.cumsum(took)]).astype(np.int64)
    for kind in (torch.bfloat16, torch.float32):
        got = hs.hs_kv_read_mx(c.gpu, dev(table), dev(off), int(off[-1]), first=dev(lens), dtype=kind)
        for n, x in zip(("k", "v"), got):
            for s in range(B):
                ref = mx.fetch(c.ref[n + "_codes"], c.ref[n + "_scales"], table, s, range(lens[s], want[s]), fmt)
                with np.errstate(over="ignore"):           # (3.3e38 rounds to 2^128, which neither type has: infinity)
                    ref = ref.astype(np.float32)
                assert np.array_equal(x[off[s]:off[s + 1]].float().cpu().numpy(), ref, equal_nan=True)


@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, "e4m3"), (torch.float32, "e2m1")])
@pytest.mark.parametrize("D,Hkv,sizes,lens,blocks", [(32, 1, [5000, 0, 1, 3500, 800], [60, 5, 0, 3, 127], 80), (64, 3, [2049, 2, 1500], [1, 63, 0], 33),
                                                     (128, 8, [3000, 0, 2, 1200], [61, 64, 190, 0], 48), (96, 5, [1300, 7, 900], [0, 1, 2], 21)])
def test_append_and_read_many_rows(hs, D, Hkv, sizes, lens, blocks, dtype, fmt):
    """Several rows to a workgroup, of sequences that begin and end inside it."""
    test_append_and_read(hs, D, Hkv, sizes, lens, blocks, dtype, fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,Hkv", [(128, 8), (64, 3)])
def test_commit(hs, D, Hkv, dtype, fmt):
    sizes, lens = [9, 0, 33, 1, 17, 20], [60, 5, 0, 127, 125, 128]     # (the fifth overflows, the last is full)
    paths = [[1, 4, 8], [], [0, 5, 30, 32, 31, 2], [], [3, 7, 9, 16], [4]]
    rs, B, blocks, depth = np.random.RandomState(3), 6, 2, 6
    pages = 14
    c, table = Cache(hs, pages, Hkv, D, fmt), _table(rs, B, blocks, pages)
    no = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    path = np.full((B, depth), -1, np.int32)
    for s, p in enumerate(paths):
        path[s, :len(p)] = p
    length = np.asarray([len(p) for p in paths], np.int32)
    k, v = _rows(3, (80, Hkv, D), dtype), _rows(4, (80, Hkv, D), dtype)
    new = torch.zeros(B, dtype=torch.int64, device=DEV)
    hs.hs_kv_commit_mx(k, v, dev(no), dev(path), dev(length), c.gpu, dev(table), dev(np.asarray(lens, np.int64)), new_lens=new)
    rows = [[no[s]] + [no[s] + r for r in p] if sizes[s] else [] for s, p in enumerate(paths)]
    for n, x in (("k", k), ("v", v)):
        want = mx.store(x.double().cpu().numpy(), rows, lens, table, pages, c.ref[n + "_codes"], c.ref[n + "_scales"], fmt)
    c.equal()
    assert new.tolist() == want.tolist()


def test_every_stored_byte_reads_back(hs):
    """All codes under all scales that a cache holds, as float32: exact."""
    for fmt, count in (("e4m3", 256), ("e2m1", 16)):
        scales = np.r_[27:247, 255]
        pages = len(scales) * max(1, count // 32) // 64 + 1
        c = Cache(hs, pages, 1, 32, fmt)
        codes = np.tile(np.arange(count, dtype=np.uint8), -(-pages * 64 * 32 // count))[:pages * 64 * 32].reshape(pages, 1, 64, 32)
        sc = np.repeat(scales, max(1, count // 32))
        sc = np.concatenate([sc, np.full(pages * 64 - len(sc), 127)]).reshape(pages, 1, 64, 1).astype(np.uint8)
        stored = codes if fmt == "e4m3" else codes[..., 0::2] | (codes[..., 1::2] << 4)
        for n in ("k", "v"):
            c.gpu[n + "_codes"].view(torch.uint8).copy_(dev(stored))
            c.gpu[n + "_scales"].copy_(dev(sc))
        table = np.arange(pages, dtype=np.int32)[None]
        for kind in (torch.float32, torch.bfloat16):
            k, v = hs.hs_kv_read_mx(c.gpu, dev(table), dev(np.asarray([0, pages * 64], np.int64)), pages * 64, dtype=kind)
            want = mx.values(codes, sc, fmt).transpose(0, 2, 1, 3).reshape(-1, 1, 32)
            assert np.array_equal(k.double().cpu().numpy(), want, equal_nan=True) and np.array_equal(v.double().cpu().numpy(), want, equal_nan=True)


def test_strided_rows_shared_lengths_and_no_new_lens(hs):
    """k and v are slices of a fused projection, the second layer stores behind the same lengths."""
    N, Hkv, D = 21, 2, 64
    flat = _rows(7, (N, 4 * Hkv, D), torch.bfloat16)
    k, v = flat[:, Hkv:2 * Hkv], flat[:, 3 * Hkv:]
    table, lens, no = dev(np.asarray([[2, 0]], np.int32)), dev(np.asarray([50], np.int64)), dev(np.asarray([0, N], np.int32))
    for seed in (0, 1):
        a, b = Cache(hs, 3, Hkv, D, "e4m3", seed), Cache(hs, 3, Hkv, D, "e4m3", seed)
        hs.hs_kv_append_mx(k, v, no, a.gpu, table, lens)
        hs.hs_kv_append_mx(k.contiguous(), v.contiguous(), no, b.gpu, table, lens)
        torch.cuda.synchronize()
        assert all(torch.equal(a.gpu[n].view(torch.uint8), b.gpu[n].view(torch.uint8)) for n in a.gpu) and lens.item() == 50


def test_rows_without_a_page_are_dropped(hs):
    """Block-table entries outside the pool: their rows go nowhere, reads of them leave the output alone."""
    c = Cache(hs, 3, 1, 64, "e4m3")
    table = np.asarray([[1, -1], [3, 2], [1 << 30, 0]], np.int32)
    no, lens = np.asarray([0, 3, 6, 9], np.int32), np.asarray([62, 62, 62], np.int64)
    k, v = _rows(1, (9, 1, 64), torch.float32, False), _rows(2, (9, 1, 64), torch.float32, False)
    new = torch.zeros(3, dtype=torch.int64, device=DEV)
    hs.hs_kv_append_mx(k, v, dev(no), c.gpu, dev(table), dev(lens), new_lens=new)
    for n, x in (("k", k), ("v", v)):
        mx.store(x.double().cpu().numpy(), [range(0, 3), range(3, 6), range(6, 9)], lens, table, 3, c.ref[n + "_codes"], c.ref[n + "_scales"], "e4m3")
    c.equal()
    assert new.tolist() == [65, 65, 65]
    out = (torch.full((9, 1, 64), 5.0, device=DEV), torch.full((9, 1, 64), 5.0, device=DEV))
    hs.hs_kv_read_mx(c.gpu, dev(table), dev(no.astype(np.int64)), 9, first=dev(lens), out=out)
    kept = [(out[0][r] == 5.0).all().item() for r in range(9)]
    assert kept == [False, False, True, True, True, False, True, True, False]
    far = (torch.full((2, 1, 64), 5.0, device=DEV), torch.full((2, 1, 64), 5.0, device=DEV))
    hs.hs_kv_read_mx(c.gpu, dev(table[1:2]), dev(np.asarray([0, 2], np.int64)), 2, first=dev(np.asarray([127], np.int64)), out=far)
    assert not (far[0][0] == 5.0).all() and (far[0][1] == 5.0).all()


def test_pools_beyond_32_bit_offsets(hs):
    """The last pages of a pool of 4.6 GB a tensor."""
    pages, Hkv, D = 70000, 8, 128
    cache = hs.new_mx_cache(pages, Hkv, D, 0, DEV)
    table, no, lens = dev(np.asarray([[pages - 1, pages - 2]], np.int32)), dev(np.asarray([0, 9], np.int32)), dev(np.asarray([60], np.int64))
    k, v = _rows(1, (9, Hkv, D), torch.bfloat16, False), _rows(2, (9, Hkv, D), torch.bfloat16, False)
    hs.hs_kv_append_mx(k, v, no, cache, table, lens)
    got = hs.hs_kv_read_mx(cache, table, dev(np.asarray([0, 9], np.int64)), 9, first=lens)
    for x, y in zip((k, v), got):
        codes, scales = mx.quantise(x.double().cpu().numpy(), "e4m3")
        assert np.array_equal(y.double().cpu().numpy(), mx.values(codes, scales, "e4m3"))


def test_graphs_streams_and_refusals(hs):
    c = Cache(hs, 4, 2, 64, "e2m1")
    table, no = dev(np.asarray([[3, 1]], np.int32)), dev(np.asarray([0, 4], np.int32))
    lens, new = dev(np.asarray([10], np.int64)), torch.zeros(1, dtype=torch.int64, device=DEV)
    k, v = _rows(1, (4, 2, 64), torch.bfloat16), _rows(2, (4, 2, 64), torch.bfloat16)
    out, off = (torch.zeros((4, 2, 64), device=DEV), torch.zeros((4, 2, 64), device=DEV)), dev(np.asarray([0, 4], np.int64))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hs.hs_kv_append_mx(k, v, no, c.gpu, table, lens, new_lens=new, stream=side)
    hs.hs_kv_read_mx(c.gpu, table, off, 4, first=lens, out=out, stream=side)
    side.synchronize()
    want = [x.clone() for x in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hs_kv_append_mx(k, v, no, c.gpu, table, lens, new_lens=new)
        hs.hs_kv_read_mx(c.gpu, table, off, 4, first=lens, out=out)
        lens.copy_(new)                                   # the next replay stores behind it
    for n in range(5):
        out[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0].nan_to_num(), want[0].nan_to_num()) and torch.equal(out[1].nan_to_num(), want[1].nan_to_num()) and lens.item() == 14 + 4 * n
    lens.fill_(10)
    good = dict(k=k, v=v, node_offsets=no, cache=c.gpu, block_table=table, cache_lens=lens)
    for bad in [dict(k=k[:, :1]), dict(v=v[:3]), dict(k=k.half()), dict(v=v.float()), dict(k=k.cpu()), dict(node_offsets=no.long()), dict(block_table=table[0]),
                dict(block_table=table.long()), dict(cache_lens=lens.int()), dict(cache_lens=lens.repeat(2)), dict(cache=dict(c.gpu, k_scales=c.gpu["k_scales"][:3])),
                dict(cache=dict(c.gpu, v_codes=c.gpu["v_codes"].view(torch.float8_e4m3fn))), dict(k=k.transpose(1, 2)), dict(new_lens=new.int())]:
        with pytest.raises(ValueError):
            hs.hs_kv_append_mx(**{**good, **bad})
    with pytest.raises(hs.HsError):
        hs.hs_kv_append_mx(**good, new_lens=lens)
    for bad in [dict(total=3), dict(first=lens.int()), dict(out=(out[0], out[1][:3])), dict(out_offsets=no)]:
        with pytest.raises(ValueError):
            hs.hs_kv_read_mx(**{**dict(cache=c.gpu, block_table=table, out_offsets=off, total=4, first=lens, out=out), **bad})
    with pytest.raises(ValueError):
        hs.hs_kv_commit_mx(k, v, no, dev(np.asarray([1], np.int32)), dev(np.asarray([1], np.int32)), c.gpu, table, lens)
    with pytest.raises(ValueError):
        hs.new_mx_cache(2, 1, 48)
