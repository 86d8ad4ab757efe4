"""Tensors that a binding call makes for itself (outputs, workspaces) belong to the stream that the call runs on, whatever stream is the
current one: torch's allocator hands a dropped tensor's memory to the next one of the SAME stream at once.  On the CPU: the allocations are
watched, the native calls are stubs."""
import contextlib

import pytest
import torch

from paper_2505_13254_amd import binding


class OnGpu(torch.Tensor):
    is_cuda = True  # (host memory that passes for the GPU's; nothing runs on it)


def gpu(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(OnGpu, torch.zeros(shape, dtype=dtype))


@pytest.fixture
def watch(monkeypatch):
    """(stream object, list of the streams that were current when a tensor was made)"""
    made, current = [], [None]

    class Side:
        cuda_stream = 7

    class Calls:
        def __getattr__(self, name):
            return lambda *a: 0

    @contextlib.contextmanager
    def stream(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    def watched(make):
        def f(*a, **kw):
            made.append(current[0])
            return make(*a, **kw)
        return f

    monkeypatch.setattr(binding, "_calls", Calls())
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda p, **kw: ("external", p))
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, watched(getattr(torch, name)))
    yield Side(), made


I32, I64, BF = torch.int32, torch.int64, torch.bfloat16


def calls():
    no, pl = torch.tensor([0, 3, 5], dtype=I32), torch.tensor([9000, 70])
    q, kt = gpu(5, 8, 128, dtype=BF), gpu(5, 2, 128, dtype=BF)
    pool = {"k_codes": gpu(4, 2, 64, 128, dtype=torch.float8_e4m3fn), "v_codes": gpu(4, 2, 64, 128, dtype=torch.float8_e4m3fn),
            "k_scales": gpu(4, 2, 64, 4, dtype=torch.uint8), "v_scales": gpu(4, 2, 64, 4, dtype=torch.uint8)}
    tree, table, off = gpu(5, dtype=I32), gpu(2, 200, dtype=I32), torch.tensor([0, 9000, 9070])
    cache = gpu(9070, 2, 128, dtype=BF)
    yield "hs_tree_attention_mx", lambda s: binding.hs_tree_attention_mx(q, pool, kt, kt, tree, gpu(3, dtype=I32), no, table, gpu(2, dtype=I64), pl, 0.1, want_lse=True, stream=s)
    yield "hs_tree_attention", lambda s: binding.hs_tree_attention(q, cache, cache, kt, kt, tree, gpu(3, dtype=I32), off, no, off, 0.1, want_lse=True, stream=s)
    yield "hs_tree_attention_paged", lambda s: binding.hs_tree_attention_paged(q, gpu(4, 64, 2, 128, dtype=BF), gpu(4, 64, 2, 128, dtype=BF), kt, kt, tree, gpu(3, dtype=I32), no,
                                                                               table, gpu(2, dtype=I64), pl, 0.1, want_lse=True, stream=s)
    yield "hs_kv_read_mx", lambda s: binding.hs_kv_read_mx(pool, table, off, 9070, stream=s)
    yield "hs_rotary", lambda s: binding.hs_rotary(q, kt, gpu(5, dtype=I64), gpu(64, dtype=torch.float64), stream=s)
    yield "hs_tree_rotary", lambda s: binding.hs_tree_rotary(q, kt, tree, gpu(3, dtype=I32), gpu(2, dtype=I64), gpu(64, dtype=torch.float64), stream=s)
    yield "hs_draft_entropy_topk", lambda s: binding.hs_draft_entropy_topk(gpu(2, 50000), 8, stream=s)
    yield "hs_tree_prune", lambda s: binding.hs_tree_prune(tree, gpu(5), gpu(3, dtype=I32), gpu(2, dtype=I32), gpu(2), gpu(2, dtype=I32), stream=s)
    yield "hs_adaptive_control", lambda s: binding.hs_adaptive_control(tree, gpu(5), gpu(5), gpu(3, dtype=I32), None, [1.0], [0.5], 2, 5, 60, stream=s)
    yield "hs_verify_accept", lambda s: binding.hs_verify_accept(gpu(5, 1000), gpu(5, 1000), tree, tree, gpu(3, dtype=I32), 1, 1.0, gpu(7), 4, stream=s)


@pytest.mark.parametrize("name", [n for n, _ in calls()])
def test_what_a_call_makes_belongs_to_its_stream(watch, name):
    side, made = watch
    call = dict(calls())[name]
    del made[:]
    call(side)
    assert made and all(s == ("external", 7) for s in made), made
    del made[:]
    call(None)                                       # the current stream's own: nothing is switched
    assert made and all(s is None for s in made)


def test_a_report_belongs_to_its_stream(watch, monkeypatch):
    side, made = watch

    class Lib:
        def hs_tree_validate(self, *a):
            return 0
    monkeypatch.setattr(binding, "lib", Lib)
    tree, no = gpu(5, dtype=I32), gpu(3, dtype=I32)
    del made[:]
    binding.hs_tree_validate(tree, None, no, stream=side)
    assert made == [("external", 7)]
