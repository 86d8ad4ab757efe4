"""The operators of a verification step over a paged cache of latents, as cases that can be timed and compared.

A case is a dict of plain values.  Kinds:

  "tables"  block tables grow by the pages that new rows need, the rows' slots in the pool are looked up, and the
            pages go back (a request's rows are not committed, or the request ends)
  "append"  the slots of prompt rows and the rows into the pool; with `back` they are read back at once (what a
            prefill that attends to cached tokens does)
  "commit"  the slots of a draft tree's accepted path and the rows into the pool
  "attn"    absorbed latent attention of tree rows over the paged latents and the tree's own rows; single tokens
            are trees of one row
  "prompt"  expanded latent attention: the rows of a prompt chunk over cached and own tokens, causal, each head
            with keys and values of its own besides the keys' shared rotary part

The pool: pages of 64 tokens, [n_pages, 64, 576]; a token is a latent of 512 elements and 64 rotary ones.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
PAGE = 64
R, DR, DN, DV = 512, 64, 128, 128  # latent, rotary part, a head's own key part, a head's values
SCALE = (DN + DR) ** -0.5


def listed():
    tables = dict(kind="tables", mix=0, scarce=False)
    attn = dict(kind="attn", mix=0)
    prompt = dict(kind="prompt", mix=0)
    return [
        # a batched verification step: 16 requests reserve pages for their trees' rows, and give back what they did not use
        dict(tables, name="tables_step", B=16, L_lo=100, L_hi=1500, n_lo=9, n_hi=129),
        # 512 requests come with their prompts and go again
        dict(tables, name="tables_admit", B=512, L_lo=0, L_hi=0, n_lo=64, n_hi=16384),
        # 16 sequences commit the paths that their trees' walks accepted
        dict(kind="commit", name="commit_batch", B=16, L_lo=100, L_hi=1500, n_lo=9, n_hi=129, depth=10, mix=0),
        # chunks of four long prompts join what is cached, and are read back
        dict(kind="append", name="append_read", B=4, L_lo=0, L_hi=900, n_lo=2000, n_hi=16384, back=True, mix=0),
        # one new token of 16 heads on 2048 cached ones: latency
        dict(attn, name="decode_one", B=1, Hq=16, L_lo=2048, L_hi=2048, M_lo=1, M_hi=1),
        # 64 sequences decode a token each, 16 heads (a share of a model's), ragged lengths: a stream of the cache
        dict(attn, name="decode_batch", B=64, Hq=16, L_lo=512, L_hi=16384, M_lo=1, M_hi=1),
        # 32 sequences with all of 128 heads: as many operations as a stream of bytes allows
        dict(attn, name="decode_heads", B=32, Hq=128, L_lo=512, L_hi=16384, M_lo=1, M_hi=1),
        # batched verification, ragged trees and lengths
        dict(attn, name="tree_batch", B=16, Hq=16, L_lo=512, L_hi=16384, M_lo=9, M_hi=129),
        # trees of 97 rows of 64 heads on 8192 tokens, four sequences: matrix work
        dict(attn, name="tree_heads", B=4, Hq=64, L_lo=8192, L_hi=8192, M_lo=97, M_hi=97),
        # the last part of one prompt
        dict(prompt, name="prompt_rest", B=1, H=16, n_lo=300, n_hi=300, L_lo=1700, L_hi=1700),
        # chunks of six prompts behind what is cached already
        dict(prompt, name="prompt_chunks", B=6, H=16, n_lo=130, n_hi=1700, L_lo=33, L_hi=9000),
        # a prompt of 8192 tokens, 32 heads
        dict(prompt, name="prompt_long", B=1, H=32, n_lo=8192, n_hi=8192, L_lo=0, L_hi=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["tables", "admit", "append", "commit", "decode", "decode", "tree", "tree", "batch", "prompt", "prompt", "chunks"])
    mix = rng.randrange(1 << 20)
    if what == "tables":
        return dict(kind="tables", B=_log(rng, 1, 2048), L_lo=rng.randint(0, 90), L_hi=_log(rng, 100, 8000), n_lo=1, n_hi=rng.randint(1, 129),
                    scarce=rng.random() < 0.3, mix=mix)
    if what == "admit":
        return dict(kind="tables", B=_log(rng, 1, 512), L_lo=0, L_hi=0, n_lo=_log(rng, 1, 500), n_hi=_log(rng, 600, 12000), scarce=rng.random() < 0.3, mix=mix)
    if what == "append":
        return dict(kind="append", B=rng.randint(1, 8), L_lo=0, L_hi=_log(rng, 1, 2000), n_lo=(n := _log(rng, 1, 2500)), n_hi=n + rng.randint(0, 900),
                    back=rng.random() < 0.5, mix=mix)
    if what == "commit":
        return dict(kind="commit", B=_log(rng, 1, 64), L_lo=rng.randint(0, 90), L_hi=_log(rng, 100, 2000), n_lo=rng.randint(1, 9), n_hi=rng.randint(10, 129),
                    depth=rng.randint(2, 12), mix=mix)
    if what in ("decode", "tree", "batch"):
        attn = dict(kind="attn", Hq=rng.choice([8, 16, 16, 20, 32, 64, 128]), mix=mix)
        if what == "decode":
            B = _log(rng, 1, 48)
            return dict(attn, B=B, L_lo=_log(rng, 1, 300), L_hi=_log(rng, 400, 16000 if B < 16 else 6000), M_lo=1, M_hi=1)
        if what == "tree":
            return dict(attn, B=1, L_lo=(n := _log(rng, 1, 9000)), L_hi=n, M_lo=(m := rng.randint(2, 129)), M_hi=m)
        return dict(attn, Hq=rng.choice([8, 16, 20, 32]), B=rng.randint(2, 12), L_lo=_log(rng, 20, 500), L_hi=_log(rng, 600, 8000), M_lo=rng.randint(1, 20), M_hi=rng.randint(21, 140))
    H = rng.choice([8, 16, 16, 20, 32])
    if what == "prompt":
        return dict(kind="prompt", H=H, B=1, n_lo=(n := _log(rng, 1, 5000)), n_hi=n, L_lo=(m := rng.choice([0, _log(rng, 1, 3000)])), L_hi=m, mix=mix)
    return dict(kind="prompt", H=H, B=rng.randint(2, 6), n_lo=_log(rng, 1, 200), n_hi=_log(rng, 200, 1500), L_lo=rng.randint(0, 90), L_hi=_log(rng, 100, 6000), mix=mix)


# ------------------------------------------------------------------------------------------------- what a case holds
def _spread(c, lo, hi, salt):
    """One number of the range for each sequence; the first and the last are its ends."""
    r = np.random.RandomState(1000 * salt + c["mix"] % 100003)
    v = np.round(np.exp(r.uniform(np.log(lo + 1), np.log(hi + 1), c["B"])) - 1).astype(np.int64).clip(lo, hi)
    v[0], v[-1] = lo, hi
    return v


def _lens(c):
    return _spread(c, c["L_lo"], c["L_hi"], 1)


def _rows(c):
    return _spread(c, c.get("M_lo", c.get("n_lo")), c.get("M_hi", c.get("n_hi")), 2)


def _pages(tokens):
    return -(-np.asarray(tokens, dtype=np.int64) // PAGE)


def _trees(c, rows):
    """Parents and depths (local) of each sequence's rows: a new row hangs off one of the 12 before it."""
    r = np.random.RandomState(c["mix"] % 100003 + 7)
    parents, depths = [], []
    for n in rows:
        p = np.array([-1] + [int(r.randint(max(0, i - 12), i)) for i in range(1, n)], dtype=np.int32)
        d = np.zeros(n, dtype=np.int64)
        for i in range(1, n):
            d[i] = d[p[i]] + 1
        parents.append(p)
        depths.append(d)
    return parents, depths


def _accepted(c, rows):
    """Accepted paths [B, depth] (local rows, -1 behind the end) and their lengths: a walk down from the root."""
    parents, _ = _trees(c, rows)
    r = np.random.RandomState(c["mix"] % 100003 + 11)
    path, length = np.full((c["B"], c["depth"]), -1, np.int32), np.zeros(c["B"], np.int32)
    for s, p in enumerate(parents):
        at = 0
        while length[s] < c["depth"] and r.uniform() < 0.8:
            kids = np.nonzero(p == at)[0]
            if not len(kids):
                break
            at = int(kids[r.randint(len(kids))])
            path[s, length[s]] = at
            length[s] += 1
    return path, length


def work(c):
    rows, lens = _rows(c), _lens(c)
    if c["kind"] == "tables":  # three calls: lengths and counts of each request, the entries that change hands, the slots
        moved = float((_pages(lens + rows) - _pages(lens)).sum())
        return {"bytes": 3 * 24.0 * c["B"] + 2 * 8.0 * moved + 8.0 * float(rows.sum()), "flops": 0.0}
    if c["kind"] == "append":
        return {"bytes": float(rows.sum()) * ((2 * 2 * (R + DR)) * (2 if c["back"] else 1) + 8), "flops": 0.0}
    if c["kind"] == "commit":
        return {"bytes": float((1 + _accepted(c, rows)[1]).sum()) * 2 * 2 * (R + DR) + 8.0 * float(rows.sum()), "flops": 0.0}
    L, n = lens.astype(float), rows.astype(float)
    if c["kind"] == "attn":
        paths = sum(float((d + 1).sum()) for d in _trees(c, rows)[1])
        b = L.sum() * 2 * (R + DR) + n.sum() * (2.0 * (R + DR) * (1 + c["Hq"]) + 2.0 * R * c["Hq"] + 4.0 * c["Hq"])
        return {"bytes": float(b), "flops": 2.0 * (2 * R + DR) * c["Hq"] * (float((L * n).sum()) + paths)}
    pairs = float((n * L + n * (n + 1) / 2).sum())
    b = 2.0 * c["H"] * (n.sum() * (DN + DR + DV) + (L + n).sum() * (DN + DV)) + 2.0 * DR * (L + n).sum() + 4.0 * c["H"] * n.sum()
    return {"bytes": float(b), "flops": 2.0 * (DN + DR + DV) * c["H"] * pairs}


def _offsets(v, kind=np.int64):
    return np.concatenate([[0], np.cumsum(v)]).astype(kind)


def _latents(g, n):
    """Normalised latents with a few strong columns, and rotary parts."""
    x = torch.randn((n, R + DR), generator=g, device=DEV)
    x[:, : R : R // 4] *= 4.0
    return x.to(torch.bfloat16)


def _pool(g, lens, spare):
    """A shuffled pool's block table (-1 behind a sequence's last page) for these lengths and rows, and the number of its pages."""
    blocks = np.maximum(1, _pages(lens + spare))
    used = torch.from_numpy(np.arange(blocks.max())[None] < blocks[:, None]).to(DEV)
    need = int(blocks.sum())
    table = torch.full(used.shape, -1, dtype=torch.int32, device=DEV)
    table[used] = torch.randperm(need + 3, generator=g, device=DEV)[:need].to(torch.int32)
    return table, need + 3


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    rows, lens, bf = _rows(c), _lens(c), torch.bfloat16
    n = int(rows.sum())
    st = dict(c, n=n)
    if c["kind"] == "prompt":
        T, H = int((rows + lens).sum()), c["H"]
        kv = torch.randn((T, H, DN + DV), generator=g, device=DEV).to(bf)  # one product's result: keys and values side by side
        host = torch.from_numpy(_offsets(rows, np.int32)), torch.from_numpy(_offsets(rows + lens))
        st.update(q=torch.randn((n, H, DN), generator=g, device=DEV).to(bf), q_rope=torch.randn((n, H, DR), generator=g, device=DEV).to(bf),
                  k=kv[..., :DN], v=kv[..., DN:], k_rope=torch.randn((T, DR), generator=g, device=DEV).to(bf), host_q_offsets=host[0],
                  host_kv_offsets=host[1], q_offsets=host[0].to(DEV), kv_offsets=host[1].to(DEV), most=int(rows.max()), most_keys=int((rows + lens).max()),
                  o=torch.empty((n, H, DV), dtype=bf, device=DEV), lse=torch.empty((n, H), device=DEV), ws=[])
        return st
    st.update(lens=dev(lens), node_offsets=dev(_offsets(rows, np.int32)))
    if c["kind"] == "tables":
        held = _pages(lens)
        need = int(_pages(lens + rows).sum())
        n_pages = int(held.sum()) + max(1, (need - int(held.sum())) // 2) if c["scarce"] else need + 5
        ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((c["B"], int(_pages(lens + rows).max())), -1, dtype=torch.int32, device=DEV)
        used = torch.arange(table.shape[1], device=DEV)[None] < dev(held)[:, None]
        table[used] = ids[: int(held.sum())]
        free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        left = n_pages - int(held.sum())
        free[:left] = ids[int(held.sum()):]
        i32 = dict(dtype=torch.int32, device=DEV)
        st.update(table=table, n_pages=n_pages, want=dev(lens + rows), held=[dev(held.astype(np.int32)), torch.zeros(c["B"], **i32)], free_pages=free,
                  free_count=[torch.full((1,), left, **i32), torch.zeros(1, **i32)], refused=torch.zeros(c["B"], **i32), refused_back=torch.zeros(c["B"], **i32),
                  slots=torch.zeros(n, dtype=torch.int64, device=DEV), new_lens=torch.zeros(c["B"], dtype=torch.int64, device=DEV))
        return st
    table, pages = _pool(g, lens, rows if c["kind"] != "attn" else np.zeros_like(rows))
    st.update(table=table, n_pages=pages)
    if c["kind"] in ("append", "commit"):
        x = _latents(g, n)
        st.update(pool=torch.zeros((pages, PAGE, R + DR), dtype=bf, device=DEV), c=x[:, :R], r=x[:, R:], slots=torch.zeros(n, dtype=torch.int64, device=DEV),
                  new_lens=torch.zeros(c["B"], dtype=torch.int64, device=DEV), back=c.get("back", False))
        if c["kind"] == "commit":
            path, length = _accepted(c, rows)
            st.update(path=dev(path), length=dev(length))
        elif c["back"]:
            st.update(c_out=torch.empty((n, R), dtype=bf, device=DEV), r_out=torch.empty((n, DR), dtype=bf, device=DEV))
        return st
    parents, _ = _trees(c, rows)
    most = int(rows.max())
    see = np.zeros((c["B"], most, most), dtype=bool)  # which tree rows a row attends to
    for s, p in enumerate(parents):
        for i in range(len(p)):
            if i:
                see[s, i] = see[s, p[i]]
            see[s, i, i] = True
    host = torch.from_numpy(_offsets(rows, np.int32)), torch.from_numpy(lens.copy())
    tree = _latents(g, n)
    st.update(pool=_latents(g, pages * PAGE).reshape(pages, PAGE, R + DR), q=torch.randn((n, c["Hq"], R), generator=g, device=DEV).to(bf),
              q_rope=torch.randn((n, c["Hq"], DR), generator=g, device=DEV).to(bf), c_tree=tree[:, :R], r_tree=tree[:, R:], parent=dev(np.concatenate(parents)),
              see=dev(see), host_node_offsets=host[0], host_lens=host[1], most=most, o=torch.empty((n, c["Hq"], R), dtype=bf, device=DEV),
              lse=torch.empty((n, c["Hq"]), device=DEV), ws=[])
    return st


# ------------------------------------------------------------------------------------------------- the plain forms
def _update_plain(st, want, held, free_count, new_held, new_free_count, refused):
    """Pages behind the wanted ones go back on the stack of free pages, missing ones come off it, first requests first."""
    table, stack = st["table"], st["free_pages"]
    col = torch.arange(table.shape[1], device=DEV)[None]
    need = (want.clamp(min=0) + PAGE - 1) // PAGE
    beyond = need > table.shape[1]
    need = torch.where(beyond, held.long(), need)
    back, ask = (held - need).clamp(min=0), (need - held).clamp(min=0)
    total = free_count[0] + back.sum()
    upto = ask.cumsum(0)
    served = (upto <= total) | (ask == 0)
    given = torch.where(served, ask, 0).sum()
    at = free_count[0] + (back.cumsum(0) - back)[:, None] + col - need[:, None]
    going = (col >= need[:, None]) & (col < held[:, None])
    whole = torch.cat([stack, stack[:1]])  # (a place for what does not go back)
    whole.scatter_(0, torch.where(going, at, stack.numel()).reshape(-1), table.reshape(-1))
    coming = (col >= held[:, None]) & (col < need[:, None]) & served[:, None]
    order = (upto - ask)[:, None] + col - held[:, None]
    table.copy_(torch.where(coming, whole[(total - 1 - order).clamp(0, stack.numel())], table))
    place = torch.arange(stack.numel(), device=DEV)
    stack.copy_(torch.where((place >= free_count[0]) & (place < total - given), whole[:-1], stack))
    new_held.copy_(torch.where(served, need, held))
    new_free_count.copy_((total - given)[None])
    refused.copy_(torch.where(beyond, 2, torch.where(served, 0, 1)))


def _slots_plain(st, held, path=None, length=None):
    n, table = st["n"], st["table"]
    row = torch.arange(n, device=DEV)
    off = st["node_offsets"].long()
    seq = torch.searchsorted(off[1:].contiguous(), row, right=True)
    local = row - off[seq]
    room = held.long() * PAGE
    if path is None:
        at, count = local, off.diff()
    else:
        hit = (path[seq] == local[:, None]) & (torch.arange(path.shape[1], device=DEV)[None] < length[seq][:, None])
        at = torch.where(local == 0, 0, torch.where(hit.any(1), hit.int().argmax(1) + 1, -1))
        count = 1 + length.long()
    token = st["lens"][seq] + at
    fits = (at >= 0) & (token < room[seq])
    page = table[seq, (token.clamp(min=0) // PAGE).clamp(max=table.shape[1] - 1)].long()
    st["slots"].copy_(torch.where(fits, page * PAGE + token % PAGE, -1))
    st["new_lens"].copy_(torch.maximum(st["lens"], torch.minimum(st["lens"] + count, room)))


def _tables_plain(st):
    held, count = st["held"], st["free_count"]
    _update_plain(st, st["want"], held[0], count[0], held[1], count[1], st["refused"])
    _slots_plain(st, held[1])
    _update_plain(st, st["lens"], held[1], count[1], held[0], count[0], st["refused_back"])
    return _tables_result(st)


def _tables_result(st):
    return [st["table"], st["held"], st["free_pages"], st["free_count"], st["refused"], st["refused_back"], st["slots"], st["new_lens"]]


def _whole(st):
    return torch.full((st["B"],), st["table"].shape[1], dtype=torch.int32, device=DEV)


def _rows_plain(st):
    _slots_plain(st, _whole(st), st.get("path"), st.get("length"))
    flat = st["pool"].view(-1, R + DR)
    keep = (st["slots"] >= 0).nonzero()[:, 0]
    flat[st["slots"][keep]] = torch.cat([st["c"], st["r"]], 1)[keep]
    if st["back"]:
        x = flat[st["slots"]]
        st["c_out"].copy_(x[:, :R])
        st["r_out"].copy_(x[:, R:])
        return [st["c_out"], st["r_out"], st["new_lens"]]
    return [st["pool"], st["new_lens"]]


def _softmax_parts(x):
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)  # (rows behind a sequence's last see nothing)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    return x, total, (top + total.log()).squeeze(-1)


def _places(st, offsets):
    row = torch.arange(st["n"], device=DEV)
    off = offsets.long()
    seq = torch.searchsorted(off[1:].contiguous(), row, right=True)
    return seq, row - off[seq]


def _attention_plain(st):
    B, most, Hq = st["B"], st["most"], st["Hq"]
    seq, local = _places(st, st["node_offsets"])
    q = torch.zeros((B, most, Hq, R + DR), device=DEV)
    q[seq, local] = torch.cat([st["q"], st["q_rope"]], 2).float()
    stored = st["pool"][st["table"].long().clamp(min=0)].reshape(B, -1, R + DR).float()
    tree = torch.zeros((B, most, R + DR), device=DEV)
    tree[seq, local] = torch.cat([st["c_tree"], st["r_tree"]], 1).float()
    keys = torch.cat([stored, tree], 1)
    tokens = stored.shape[1]
    del stored
    seen = (torch.arange(tokens, device=DEV)[None] < st["lens"][:, None])[:, None, :].expand(B, most, tokens)
    seen = torch.cat([seen, st["see"]], 2)
    x = torch.matmul(q.reshape(B, most * Hq, R + DR), keys.transpose(1, 2).contiguous()) * SCALE
    x = x.reshape(B, most, Hq, -1).masked_fill_(~seen[:, :, None], -torch.inf)
    x, total, lse = _softmax_parts(x)
    o = torch.matmul(x.reshape(B, most * Hq, -1), keys[..., :R].contiguous()).reshape(B, most, Hq, R) / total
    st["o"].copy_(o[seq, local])
    st["lse"].copy_(lse[seq, local])
    return [st["o"], st["lse"]]


def _prompt_plain(st):
    B, most, keys, H = st["B"], st["most"], st["most_keys"], st["H"]
    seq, local = _places(st, st["q_offsets"])
    off = st["kv_offsets"]
    at = torch.arange(st["k"].shape[0], device=DEV)
    kseq = torch.searchsorted(off[1:].contiguous(), at, right=True)
    klocal = at - off[kseq]
    q = torch.zeros((B, H, most, DN + DR), device=DEV)
    q[seq, :, local] = torch.cat([st["q"], st["q_rope"]], 2).float()
    k = torch.zeros((B, H, DN + DR, keys), device=DEV)
    k[kseq, :, :, klocal] = torch.cat([st["k"], st["k_rope"][:, None].expand(-1, H, -1)], 2).float()
    x = torch.matmul(q, k) * SCALE
    del q, k
    count = st["q_offsets"].diff().long()
    last = (off.diff() - count)[:, None] + torch.arange(most, device=DEV)[None]  # the last key that a row sees
    x = x.masked_fill_((torch.arange(keys, device=DEV) > last[..., None])[:, None], -torch.inf)
    x, total, lse = _softmax_parts(x)
    v = torch.zeros((B, H, keys, DV), device=DEV)
    v[kseq, :, klocal] = st["v"].float()
    o = torch.matmul(x, v) / total
    st["o"].copy_(o[seq, :, local])
    st["lse"].copy_(lse[seq, :, local])
    return [st["o"], st["lse"]]


PLAIN = {"tables": _tables_plain, "append": _rows_plain, "commit": _rows_plain, "attn": _attention_plain, "prompt": _prompt_plain}


# ------------------------------------------------------------------------------------------------- the framework's calls
def _run_own(st):
    import paper_2505_13254_amd as hs
    kind = st["kind"]
    if kind == "tables":
        held, count = st["held"], st["free_count"]
        hs.hs_block_tables(st["want"], st["table"], held[0], st["free_pages"], count[0], new_held=held[1], new_free_count=count[1], refused=st["refused"])
        hs.hs_slot_map(st["node_offsets"], st["n"], st["lens"], st["table"], st["n_pages"], held=held[1], slots=st["slots"], new_lens=st["new_lens"])
        hs.hs_block_tables(st["lens"], st["table"], held[1], st["free_pages"], count[1], new_held=held[0], new_free_count=count[0], refused=st["refused_back"])
        return _tables_result(st)
    if kind in ("append", "commit"):
        hs.hs_slot_map(st["node_offsets"], st["n"], st["lens"], st["table"], st["n_pages"], accept_path=st.get("path"), accept_len=st.get("length"),
                       slots=st["slots"], new_lens=st["new_lens"])
        hs.hs_latent_store(st["c"], st["r"], st["slots"], st["pool"])
        if st["back"]:
            c, r = hs.hs_latent_read(st["pool"], st["slots"], R, out=(st["c_out"], st["r_out"]))
            return [c, r, st["new_lens"]]
        return [st["pool"], st["new_lens"]]
    if kind == "attn":
        if not st["ws"]:  # a program keeps its workspace
            st["ws"].append(hs.hs_tree_attention_latent_workspace(st["host_node_offsets"], st["host_lens"], st["Hq"], R, DR, st["q"].device))
        return list(hs.hs_tree_attention_latent(st["q"], st["q_rope"], st["pool"], st["c_tree"], st["r_tree"], st["parent"], st["node_offsets"],
                                                st["host_node_offsets"], st["table"], st["lens"], st["host_lens"], SCALE, out=st["o"], lse=st["lse"],
                                                ws=st["ws"][0]))
    if not st["ws"]:
        st["ws"].append(hs.hs_prompt_attention_latent_workspace(st["host_q_offsets"], st["host_kv_offsets"], st["H"], DV, st["q"].device))
    return list(hs.hs_prompt_attention_latent(st["q"], st["q_rope"], st["k"], st["k_rope"], st["v"], st["q_offsets"], st["kv_offsets"], st["host_q_offsets"],
                                              st["host_kv_offsets"], SCALE, out=st["o"], lse=st["lse"], ws=st["ws"][0]))


def run(st):
    if own:
        return _run_own(st)
    return PLAIN[st["kind"]](st)


# ------------------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    c = case
    if c["kind"] in ("tables", "commit") or (c["kind"] == "append" and not c["back"]):
        return None  # whole numbers and copies
    st = prepare(case, seed)
    if c["kind"] == "append":
        return [st["c"].double(), st["r"].double(), None]
    o, lse = torch.empty(st["o"].shape, dtype=torch.float64, device=DEV), torch.empty(st["lse"].shape, dtype=torch.float64, device=DEV)
    if c["kind"] == "attn":
        off, lens = st["host_node_offsets"].tolist(), st["host_lens"].tolist()
        for s in range(c["B"]):
            a, b, L = off[s], off[s + 1], lens[s]
            kept = st["pool"][st["table"][s, : -(-L // PAGE)].long()].reshape(-1, R + DR)[:L].double()
            lat = torch.cat([kept[:, :R], st["c_tree"][a:b].double()])
            rot = torch.cat([kept[:, R:], st["r_tree"][a:b].double()])
            x = torch.einsum("nhd,td->nht", st["q"][a:b].double(), lat) + torch.einsum("nhd,td->nht", st["q_rope"][a:b].double(), rot)
            hidden = torch.zeros((b - a, L + b - a), dtype=torch.bool, device=DEV)
            hidden[:, L:] = ~st["see"][s, : b - a, : b - a]
            x = (x * SCALE).masked_fill(hidden[:, None], -math.inf)
            lse[a:b] = torch.logsumexp(x, -1)
            o[a:b] = torch.softmax(x, -1) @ lat
        return [o, lse]
    qo, ko = st["host_q_offsets"].tolist(), st["host_kv_offsets"].tolist()
    for s in range(c["B"]):
        a, b, k0, k1 = qo[s], qo[s + 1], ko[s], ko[s + 1]
        hidden = torch.ones((b - a, k1 - k0), dtype=torch.bool, device=DEV).triu(k1 - k0 - (b - a) + 1)
        for h in range(c["H"]):
            x = st["q"][a:b, h].double() @ st["k"][k0:k1, h].double().t() + st["q_rope"][a:b, h].double() @ st["k_rope"][k0:k1].double().t()
            x = (x * SCALE).masked_fill_(hidden, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, -1)
            o[a:b, h] = torch.softmax(x, -1) @ st["v"][k0:k1, h].double()
    return [o, lse]
