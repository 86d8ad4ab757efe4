"""Calls on another stream than the current one, which make their outputs and workspaces themselves while the current stream writes to memory that
it has just dropped and to tensors that it makes afterwards: none of it is theirs."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_13254_amd as h
    return h


def calls(hs):
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    rows, L, Hq, Hkv, D = 61, 6000, 32, 8, 128
    parent = i32([-1] + [i // 3 for i in range(rows - 1)])
    no, pl = torch.tensor([0, rows], dtype=torch.int32), torch.tensor([L])
    q, kt, vt = r(rows, Hq, D).bfloat16(), r(rows, Hkv, D).bfloat16(), r(rows, Hkv, D).bfloat16()
    k, v = r(L, Hkv, D).bfloat16(), r(L, Hkv, D).bfloat16()
    blocks = -(-L // 64)
    cache, table = hs.new_mx_cache(blocks, Hkv, D, device=DEV), torch.arange(blocks, dtype=torch.int32, device=DEV)[None]
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    hs.hs_kv_append_mx(k, v, i32([0, L]), cache, table, zero)
    po, dpl, dno = torch.tensor([0, L]), pl.to(DEV), no.to(DEV)
    dpo = po.to(DEV)
    f, _ = hs.hs_rotary_frequencies(D, device=DEV)
    logits, draft, token, u = r(rows, 5000), r(rows, 5000), i32(list(range(rows))), torch.rand(rows + 1, generator=g, device=DEV)
    yield lambda s: hs.hs_tree_attention_mx(q, cache, kt, vt, parent, dno, no, table, dpl, pl, 0.1, want_lse=True, stream=s)
    yield lambda s: hs.hs_tree_attention(q, k, v, kt, vt, parent, dno, dpo, no, po, 0.1, want_lse=True, stream=s)
    yield lambda s: hs.hs_kv_read_mx(cache, table, dpo, L, stream=s)
    yield lambda s: hs.hs_tree_rotary(q, kt, parent, dno, dpl, f, stream=s)
    yield lambda s: tuple(hs.hs_draft_entropy_topk(logits, 8, stream=s).values())
    lim = [i32([5]), torch.full((1,), -30.0, device=DEV), i32([40])]
    logc = -draft[:, 0].abs()
    yield lambda s: tuple(hs.hs_tree_prune(parent, logc, dno, *lim, stream=s).values())
    yield lambda s: tuple(hs.hs_verify_accept(logits, draft, token, parent, dno, 1, 1.0, u, 6, stream=s).values())


def test_what_calls_make_on_another_stream(hs):
    side, cycles = torch.cuda.Stream(), 20_000_000
    sizes = [1 << n for n in range(9, 26)] * 3
    for call in list(calls(hs)):
        want = [t.clone() for t in call(None)]
        torch.cuda.synchronize()
        before = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes]
        torch.cuda._sleep(cycles)
        for t in before:
            t.fill_(0xff)                                # (queued behind the sleep)
        del before, t
        with torch.cuda.stream(side):
            torch.cuda._sleep(cycles)
        got = call(side)
        after = [torch.empty(n, dtype=torch.uint8, device=DEV).fill_(0xff) for n in sizes]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert all(bool((t == 0xff).all()) for t in after)
