"""The operators of a verification step over a quantised cache, as cases that can be timed and compared.

A case is a dict of plain values.  Kinds:

  "rotary"  rotary positions of q and k rows: of a prompt (positions given) or of tree rows (tokens in the
            cache + depth in the tree); both pairings, whole heads or their first part, scaled tables, rows of
            q and k that are slices of one fused projection
  "append"  the K/V rows of prompt chunks join a quantised cache; with `back` what was stored is read back at
            once (a prefill that attends to the values which decoding will see)
  "commit"  the accepted path of a draft tree joins it
  "read"    stored tokens are read back
  "attn"    tree attention of the kept rows over the quantised cache and the tree's own rows; single tokens
            are trees of one row

The cache: pages of 64 tokens, [n_pages, Hkv, 64, D], found through a block table.  Blocks of 32 neighbours of a
row share one power of two; the elements are 8-bit (e4m3) or 4-bit (e2m1) floating point.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
PAGE, BLOCK = 64, 32
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # e2m1


def listed():
    rot = dict(kind="rotary", dtype="bf16", D=128, rot=128, pairs="half", scaling="none", mix=0)
    kv = dict(dtype="bf16", Hkv=8, D=128, mix=0)
    attn = dict(kind="attn", Hq=32, Hkv=8, D=128, mix=0)
    return [
        # the rows of one 61-row draft tree behind 2048 tokens, 8B shape: a launch
        dict(rot, name="rotary_tree", B=1, Hq=32, Hkv=8, L_lo=2048, L_hi=2048, n_lo=61, n_hi=61, tree=True),
        # a prompt of 8192 tokens of the 8B shape, slices of the fused projection
        dict(rot, name="rotary_prompt", B=1, Hq=32, Hkv=8, L_lo=0, L_hi=0, n_lo=8192, n_hi=8192, tree=False, scaling="wavelength"),
        # float32, neighbours as pairs, the first half of each head, positions far out on a stretched table, ragged rows
        dict(rot, name="rotary_far_f32", dtype="f32", B=5, Hq=40, Hkv=40, rot=64, pairs="interleaved", scaling="yarn", L_lo=100000,
             L_hi=1000000, n_lo=101, n_hi=777, tree=False),
        # 16 sequences commit the paths that their trees' walks accepted
        dict(kv, kind="commit", name="commit_batch", fmt="e4m3", B=16, L_lo=100, L_hi=1500, n_lo=9, n_hi=129, depth=10),
        # a prompt of 8192 tokens goes into the cache
        dict(kv, kind="append", name="append_prompt", fmt="e4m3", B=1, L_lo=0, L_hi=0, n_lo=8192, n_hi=8192, back=False),
        # chunks of six prompts behind what is there already, in 4 bits, and back
        dict(kv, kind="append", name="append_read_chunks", fmt="e2m1", Hkv=40, B=6, L_lo=33, L_hi=900, n_lo=130, n_hi=700, back=True),
        # four long sequences are read back
        dict(kv, kind="read", name="read_long", fmt="e4m3", B=4, L_lo=2000, L_hi=16384),
        # one new token on 2048 cached ones
        dict(attn, name="decode_one", fmt="e4m3", B=1, L_lo=2048, L_hi=2048, M_lo=1, M_hi=1),
        # 64 sequences decode a token each, ragged lengths: a stream of the cache
        dict(attn, name="decode_batch", fmt="e4m3", B=64, L_lo=512, L_hi=16384, M_lo=1, M_hi=1),
        # the 8B shape's tree of 61 rows on 2048 tokens
        dict(attn, name="tree_8b", fmt="e4m3", B=1, L_lo=2048, L_hi=2048, M_lo=61, M_hi=61),
        # batched verification on the 8B shape, ragged trees and lengths
        dict(attn, name="tree_batch", fmt="e4m3", B=16, L_lo=512, L_hi=16384, M_lo=9, M_hi=129),
        # the 70B shape's tree of 97 rows on 8192 tokens, four sequences, in 4 bits: 776 rows share a KV head
        dict(attn, name="tree_70b", fmt="e2m1", Hq=64, B=4, L_lo=8192, L_hi=8192, M_lo=97, M_hi=97),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["rotary", "tree_rotary", "append", "commit", "read", "decode", "decode", "tree", "tree", "batch"])
    mix = rng.randrange(1 << 20)
    D = rng.choice([64, 128, 128])
    Hq, Hkv = rng.choice([(32, 8), (64, 8), (40, 40), (8, 8), (12, 4), (6, 3)])
    fmt = rng.choice(["e4m3", "e4m3", "e2m1"])
    if what in ("rotary", "tree_rotary"):
        tree = what == "tree_rotary"
        base = dict(kind="rotary", dtype=rng.choice(["bf16", "bf16", "f32"]), Hq=Hq, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, D // 4 * 3 + 2]),
                    pairs=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "wavelength", "yarn"]), tree=tree, mix=mix)
        if tree:
            return dict(base, B=rng.randint(1, 16), L_lo=rng.randint(0, 500), L_hi=_log(rng, 600, 900000), n_lo=rng.randint(1, 20), n_hi=rng.randint(20, 300))
        return dict(base, B=rng.randint(1, 4), L_lo=0, L_hi=_log(rng, 1, 900000), n_lo=(n := _log(rng, 1, 1500)), n_hi=n + rng.randint(0, 500))
    kv = dict(dtype=rng.choice(["bf16", "bf16", "f32"]), fmt=fmt, Hkv=Hkv, D=D, mix=mix)
    if what == "append":
        back = fmt == "e2m1" or rng.random() < 0.3
        return dict(kv, kind="append", B=rng.randint(1, 8), L_lo=0, L_hi=_log(rng, 1, 2000), n_lo=(n := _log(rng, 1, 800)), n_hi=n + rng.randint(0, 200), back=back)
    if what == "commit":
        return dict(kv, kind="commit", fmt="e4m3", B=_log(rng, 1, 64), L_lo=rng.randint(0, 90), L_hi=_log(rng, 100, 2000), n_lo=rng.randint(1, 9),
                    n_hi=rng.randint(10, 129), depth=rng.randint(2, 12))
    if what == "read":
        return dict(kv, kind="read", B=rng.randint(1, 6), L_lo=_log(rng, 1, 500), L_hi=_log(rng, 500, 6000))
    attn = dict(kind="attn", Hq=Hq, Hkv=Hkv, D=D, fmt=fmt, mix=mix)
    if what == "decode":
        B = _log(rng, 1, 48)
        return dict(attn, B=B, L_lo=_log(rng, 1, 300), L_hi=_log(rng, 400, 12000 if B < 12 else 4000), M_lo=1, M_hi=1)
    if what == "tree":
        return dict(attn, B=1, L_lo=(n := _log(rng, 60, 9000)), L_hi=n, M_lo=(m := rng.randint(2, 129)), M_hi=m)
    return dict(attn, B=rng.randint(2, 12), L_lo=_log(rng, 20, 500), L_hi=_log(rng, 600, 8000), M_lo=rng.randint(1, 20), M_hi=rng.randint(21, 140))


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


def _mx_bytes(c):
    return (1.0 if c["fmt"] == "e4m3" else 0.5) + 1.0 / BLOCK


def work(c):
    if c["kind"] == "rotary":
        size = 4 if c["dtype"] == "f32" else 2
        n = int(_rows(c).sum())
        return {"bytes": 2.0 * n * (c["Hq"] + c["Hkv"]) * c["D"] * size, "flops": 3.0 * n * (c["Hq"] + c["Hkv"]) * c["rot"]}
    size = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "append":
        e = 2.0 * float(_rows(c).sum()) * c["Hkv"] * c["D"]
        return {"bytes": e * (size + _mx_bytes(c)) + (e * size if c["back"] else 0.0), "flops": 4.0 * e}
    if c["kind"] == "commit":
        e = 2.0 * float((1 + _accepted(c, _rows(c))[1]).sum()) * c["Hkv"] * c["D"]
        return {"bytes": e * (size + _mx_bytes(c)), "flops": 4.0 * e}
    if c["kind"] == "read":
        e = 2.0 * float(_lens(c).sum()) * c["Hkv"] * c["D"]
        return {"bytes": e * (size + _mx_bytes(c)), "flops": e}
    L, rows = _lens(c).astype(float), _rows(c)
    paths = sum(float((d + 1).sum()) for d in _trees(c, rows)[1])
    b = 2 * L.sum() * c["Hkv"] * c["D"] * _mx_bytes(c) + rows.sum() * c["D"] * 2.0 * (2 * c["Hkv"] + 2 * c["Hq"]) + 4.0 * rows.sum() * c["Hq"]
    return {"bytes": float(b), "flops": 4.0 * c["Hq"] * c["D"] * (float((L * rows).sum()) + paths)}


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


def _offsets(v, kind=np.int64):
    return np.concatenate([[0], np.cumsum(v)]).astype(kind)


def _frequencies(c):
    """Radians per position of each pair and the factor on the result, from the definitions, in 64 bits."""
    rot, base, factor, context = c["rot"], 500000.0, 8.0, 8192.0
    j = np.arange(rot // 2, dtype=np.float64)
    f = base ** (-2.0 * j / rot)
    if c["scaling"] == "linear":
        return f / factor, 1.0
    if c["scaling"] == "ntk":
        return (base * factor ** (rot / (rot - 2.0))) ** (-2.0 * j / rot), 1.0
    if c["scaling"] == "wavelength":  # waves longer than the context are stretched, those under a quarter of it are not
        t = ((context / (2 * math.pi / f)) - 1.0) / (4.0 - 1.0)
        t = np.clip(t, 0.0, 1.0)
        return (1 - t) * f / factor + t * f, 1.0
    if c["scaling"] == "yarn":  # a ramp over the pairs, between 32 turns within the context and one
        edge = lambda turns: rot * math.log(context / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(edge(32.0)), 0), min(math.ceil(edge(1.0)), rot - 1)
        t = 1.0 - np.clip((j - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return (1 - t) * f / factor + t * f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _values(g, shape):
    """Keys and values as models have them: near to normal, a few strong columns, some rows of small size."""
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., :: shape[-1] // 4] *= 6.0
    return x * torch.exp2(torch.randint(-3, 2, (shape[0], 1, 1), generator=g, device=DEV).float())


def _table(g, lens, spare):
    """A block table over a shuffled pool, and the number of its pages.  (Entries behind a sequence's last page are 0.)"""
    blocks = np.array([max(1, -(-int(l + n) // PAGE)) for l, n in zip(lens, spare)])
    used = torch.from_numpy(np.arange(blocks.max())[None] < blocks[:, None]).to(DEV)
    need = int(blocks.sum())
    table = torch.zeros(used.shape, dtype=torch.int32, device=DEV)
    table[used] = torch.randperm(need + 3, generator=g, device=DEV)[:need].to(torch.int32)
    return table, need + 3


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    rows, lens = _rows(c) if c["kind"] != "read" else None, _lens(c)
    st = dict(c)
    if c["kind"] == "rotary":
        n, D, t = int(rows.sum()), c["D"], TYPES[c["dtype"]]
        fused = torch.randn((n, c["Hq"] + 2 * c["Hkv"], D), generator=g, device=DEV).to(t)
        f, m = _frequencies(c)
        seq = np.repeat(np.arange(c["B"]), rows)
        local = np.concatenate([np.arange(k) for k in rows])
        if c["tree"]:
            parents, depths = _trees(c, rows)
            st.update(parent=dev(np.concatenate(parents)), node_offsets=dev(_offsets(rows, np.int32)), prefix_lens=dev(lens))
            local = np.concatenate(depths)
        st.update(q=fused[:, :c["Hq"]], k=fused[:, c["Hq"]:c["Hq"] + c["Hkv"]], positions=dev(lens[seq] + local), inv_freq=dev(f), mscale=m,
                  q_out=torch.empty((n, c["Hq"], D), dtype=t, device=DEV), k_out=torch.empty((n, c["Hkv"], D), dtype=t, device=DEV))
        return st
    Hkv, D = c["Hkv"], c["D"]
    wide = D if c["fmt"] == "e4m3" else D // 2
    spare = rows if rows is not None else np.zeros_like(lens)
    table, pages = _table(g, lens, spare)
    code_type = torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.uint8
    cache = {}
    for name in ("k", "v"):
        if c["kind"] in ("append", "commit"):
            cache[name + "_codes"] = torch.zeros((pages, Hkv, PAGE, wide), dtype=torch.uint8, device=DEV).view(code_type)
            cache[name + "_scales"] = torch.full((pages, Hkv, PAGE, D // BLOCK), 127, dtype=torch.uint8, device=DEV)
        else:
            codes, scales = [], []
            for p in range(0, pages, 512):
                a, b = _quantise(_values(g, (min(512, pages - p), Hkv * PAGE, D)), c["fmt"])
                codes.append(a), scales.append(b)
            cache[name + "_codes"] = torch.cat([x.view(torch.uint8) for x in codes]).reshape(pages, Hkv, PAGE, wide).view(code_type)
            cache[name + "_scales"] = torch.cat(scales).reshape(pages, Hkv, PAGE, D // BLOCK)
    st.update(cache=cache, table=table, lens=dev(lens))
    if c["kind"] == "read":
        off = _offsets(lens)
        st.update(out_offsets=dev(off), total=int(off[-1]), seq=dev(np.repeat(np.arange(c["B"]), lens)), token=dev(np.concatenate([np.arange(k) for k in lens])))
        for name in ("k_out", "v_out"):
            st[name] = torch.empty((st["total"], Hkv, D), dtype=TYPES[c["dtype"]], device=DEV)
        return st
    n = int(rows.sum())
    st.update(node_offsets=dev(_offsets(rows, np.int32)), seq=dev(np.repeat(np.arange(c["B"]), rows)),
              local=dev(np.concatenate([np.arange(k) for k in rows])), new_lens=torch.zeros(c["B"], dtype=torch.int64, device=DEV))
    if c["kind"] in ("append", "commit"):
        t = TYPES[c["dtype"]]
        st.update(k=_values(g, (n, Hkv, D)).to(t), v=_values(g, (n, Hkv, D)).to(t))
        if c["kind"] == "commit":
            path, length = _accepted(c, rows)
            st.update(path=dev(path), length=dev(length))
        elif c["back"]:
            st.update(total=n, out_offsets=dev(_offsets(rows)))
            for name in ("k_out", "v_out"):
                st[name] = torch.empty((n, Hkv, D), dtype=t, device=DEV)
        return st
    parents, _ = _trees(c, rows)
    most = int(rows.max())
    see = np.zeros((c["B"], most, most), dtype=bool)  # which tree rows a row attends to
    for s, p in enumerate(parents):
        for i in range(len(p)):
            if i:
                see[s, i] = see[s, p[i]]
            see[s, i, i] = True
    bf = torch.bfloat16
    host = torch.from_numpy(_offsets(rows, np.int32)), torch.from_numpy(lens.copy())
    st.update(q=torch.randn((n, c["Hq"], D), generator=g, device=DEV).to(bf), k_tree=_values(g, (n, Hkv, D)).to(bf), v_tree=_values(g, (n, Hkv, D)).to(bf),
              parent=dev(np.concatenate(parents)), see=dev(see), host_node_offsets=host[0], host_lens=host[1], scale=D ** -0.5, most=most,
              o=torch.empty((n, c["Hq"], D), dtype=bf, device=DEV), lse=torch.empty((n, c["Hq"]), device=DEV), n=n, ws=[])
    return st


# ------------------------------------------------------------------------------------------------- the plain forms
def _quantise(x, fmt):
    """Codes and scale bytes of rows x [..., D] (32 bits)."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    amax = b.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875) if fmt == "e4m3" else e - 3 + (m > 0.75)
    e = torch.where(amax > 0, e, -100).clamp(min=-100)
    y = torch.ldexp(b, -e[..., None])
    fine = torch.isfinite(amax)
    y = torch.where(fine[..., None], y, 0.0).reshape(x.shape)
    scales = torch.where(fine, e + 127, 255).to(torch.uint8)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn), scales
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code.byte() + 8 * torch.signbit(y).byte()
    return code[..., 0::2] + 16 * code[..., 1::2], scales


def _decode(codes, scales):
    """What codes and scale bytes stand for, in 32 bits."""
    if codes.dtype == torch.uint8:
        nibbles = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).int()
        x = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)[nibbles]
    else:
        x = codes.float()
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    s = torch.where(scales == 255, torch.nan, torch.exp2(scales.float() - 127))
    return (b * s[..., None]).reshape(x.shape)


def _rotary_plain(st):
    turns = st["positions"].double()[:, None] * st["inv_freq"][None, :]
    cos, sin = (torch.cos(turns) * st["mscale"]).float()[:, None], (torch.sin(turns) * st["mscale"]).float()[:, None]
    return [_rotated(st, st["q"], cos, sin, st["q_out"]), _rotated(st, st["k"], cos, sin, st["k_out"])]


def _rotated(st, x, cos, sin, out):
    rot, h = st["rot"], st["rot"] // 2
    y = x.float()
    out.copy_(x)
    if st["pairs"] == "half":
        a, b = y[..., :h], y[..., h:rot]
        out[..., :h], out[..., h:rot] = (a * cos - b * sin).to(x.dtype), (b * cos + a * sin).to(x.dtype)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = (a * cos - b * sin).to(x.dtype), (b * cos + a * sin).to(x.dtype)
    return out


def _place(st, rows, seq, at):
    """Rows `rows` of k and v are stored as token `at` of their sequences."""
    page, slot = st["table"][seq, at // PAGE].long(), at % PAGE
    _place_one(st, st["k"][rows], "k", page, slot)
    _place_one(st, st["v"][rows], "v", page, slot)


def _place_one(st, x, name, page, slot):
    codes, scales = _quantise(x.float(), st["fmt"])
    st["cache"][name + "_codes"].view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
    st["cache"][name + "_scales"][page, :, slot] = scales


def _fetch(st, name, seq, at, out):
    page, slot = st["table"][seq, at // PAGE].long(), at % PAGE
    codes = st["cache"][name + "_codes"]
    picked = codes.view(torch.uint8)[page, :, slot].view(codes.dtype)
    out.copy_(_decode(picked, st["cache"][name + "_scales"][page, :, slot]))
    return out


def _append_plain(st):
    count = st["node_offsets"].diff().long()
    at = st["lens"][st["seq"]] + st["local"]
    _place(st, slice(None), st["seq"], at)
    st["new_lens"].copy_(st["lens"] + count)
    if st["back"]:
        return [_fetch(st, "k", st["seq"], at, st["k_out"]), _fetch(st, "v", st["seq"], at, st["v_out"]), st["new_lens"]]
    return [st["cache"], st["new_lens"]]


def _commit_plain(st):
    B, depth = st["path"].shape
    t = torch.arange(depth + 1, device=DEV)[None].minimum(st["length"].long()[:, None])  # (places behind the end repeat the last row)
    local = torch.where(t > 0, st["path"].long().gather(1, (t - 1).clamp(min=0)), 0)
    seq = torch.arange(B, device=DEV)[:, None].expand(B, depth + 1).reshape(-1)
    rows = (st["node_offsets"][:-1].long()[:, None] + local).reshape(-1)
    _place(st, rows, seq, (st["lens"][:, None] + t).reshape(-1))
    st["new_lens"].copy_(st["lens"] + 1 + st["length"])
    return [st["cache"], st["new_lens"]]


def _read_plain(st):
    return [_fetch(st, "k", st["seq"], st["token"], st["k_out"]), _fetch(st, "v", st["seq"], st["token"], st["v_out"])]


def _keys(st, name):
    """All keys (values) that a sequence's rows may see, in 32 bits: [B, Hkv, tokens of the table's pages + tree rows, D]."""
    B, blocks = st["table"].shape
    page = st["table"].long()
    x = _decode(st["cache"][name + "_codes"].view(torch.uint8)[page].view(st["cache"][name + "_codes"].dtype), st["cache"][name + "_scales"][page])
    x = x.transpose(1, 2).reshape(B, st["Hkv"], blocks * PAGE, st["D"])
    tree = torch.zeros((B, st["most"], st["Hkv"], st["D"]), device=DEV)
    tree[st["seq"], st["local"]] = st[name + "_tree"].float()
    return torch.cat([x, tree.transpose(1, 2)], 2)


def _attention_plain(st):
    B, most, Hq, Hkv, D = st["B"], st["most"], st["Hq"], st["Hkv"], st["D"]
    G = Hq // Hkv
    q = torch.zeros((B, most, Hq, D), device=DEV)
    q[st["seq"], st["local"]] = st["q"].float()
    q = q.reshape(B, most, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * most, D)
    keys = _keys(st, "k")
    tokens = keys.shape[2] - most
    seen = (torch.arange(tokens, device=DEV)[None] < st["lens"][:, None])[:, None, :].expand(B, most, tokens)
    seen = torch.cat([seen, st["see"]], 2)
    x = torch.matmul(q, keys.transpose(2, 3).contiguous()) * st["scale"]
    del keys
    x = x.reshape(B, Hkv, G, most, -1).masked_fill_(~seen[:, None, None], -torch.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)  # (rows behind a sequence's last see nothing)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(B, Hkv, G * most, -1), _keys(st, "v")).reshape(B, Hkv, G, most, D) / total
    lse = (top + total.log()).squeeze(-1)
    st["o"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, most, Hq, D)[st["seq"], st["local"]])
    st["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(B, most, Hq)[st["seq"], st["local"]])
    return [st["o"], st["lse"]]


PLAIN = {"rotary": _rotary_plain, "append": _append_plain, "commit": _commit_plain, "read": _read_plain, "attn": _attention_plain}


# ------------------------------------------------------------------------------------------------- the framework's calls
def _run_own(st):
    import paper_2505_13254_amd as hs
    kind = st["kind"]
    if kind == "rotary":
        how = dict(interleaved=st["pairs"] == "interleaved", mscale=st["mscale"], q_out=st["q_out"], k_out=st["k_out"])
        if st["tree"]:
            return list(hs.hs_tree_rotary(st["q"], st["k"], st["parent"], st["node_offsets"], st["prefix_lens"], st["inv_freq"], **how))
        return list(hs.hs_rotary(st["q"], st["k"], st["positions"], st["inv_freq"], **how))
    if kind == "append":
        hs.hs_kv_append_mx(st["k"], st["v"], st["node_offsets"], st["cache"], st["table"], st["lens"], new_lens=st["new_lens"])
        if st["back"]:
            k, v = hs.hs_kv_read_mx(st["cache"], st["table"], st["out_offsets"], st["total"], first=st["lens"], out=(st["k_out"], st["v_out"]))
            return [k, v, st["new_lens"]]
        return [st["cache"], st["new_lens"]]
    if kind == "commit":
        hs.hs_kv_commit_mx(st["k"], st["v"], st["node_offsets"], st["path"], st["length"], st["cache"], st["table"], st["lens"], new_lens=st["new_lens"])
        return [st["cache"], st["new_lens"]]
    if kind == "read":
        return list(hs.hs_kv_read_mx(st["cache"], st["table"], st["out_offsets"], st["total"], out=(st["k_out"], st["v_out"])))
    if not st["ws"]:  # a program keeps its workspace
        st["ws"].append(hs.hs_tree_attention_mx_workspace(st["host_node_offsets"], st["host_lens"], st["Hq"], st["Hkv"], st["D"], st["q"].device))
    return list(hs.hs_tree_attention_mx(st["q"], st["cache"], st["k_tree"], st["v_tree"], st["parent"], st["node_offsets"], st["host_node_offsets"],
                                        st["table"], st["lens"], st["host_lens"], st["scale"], out=st["o"], lse=st["lse"], ws=st["ws"][0]))


def run(st):
    if own:
        return _run_own(st)
    return PLAIN[st["kind"]](st)


# ------------------------------------------------------------------------------------------------- the definitions, in 64 bits
def _stored(x, fmt):
    """The elements (before the scale), the scale bytes and the values of rows x, by arithmetic on doubles."""
    x = x.double()
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    largest, least, bits = (448.0, -6, 3) if fmt == "e4m3" else (6.0, 0, 1)
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / largest))  # amax <= largest * 2^e; checked on both sides, as a logarithm is rounded
    e = e + (amax > largest * torch.exp2(e)).double()
    e = e - (amax <= largest * torch.exp2(e - 1)).double()
    e = torch.where(amax > 0, e, torch.full_like(e, -100.0)).clamp(min=-100.0)
    y = b / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** least))).clamp(min=least) - bits)
    element = torch.round(y / step) * step
    return element.reshape(x.shape), (e.squeeze(-1) + 127).to(torch.int64), (element * torch.exp2(e)).reshape(x.shape)


def _meaning(codes, scales):
    """The values of a cache, in 64 bits, from the bits."""
    u = codes.view(torch.uint8)
    if codes.dtype == torch.uint8:
        u = torch.stack([u % 16, u // 16], -1).reshape(*u.shape[:-1], -1).long()
        sign, ex, man, bias, bits = u // 8, (u // 2) % 4, u % 2, 1, 1
    else:
        u = u.long()
        sign, ex, man, bias, bits = u // 128, (u // 8) % 16, u % 8, 7, 3
    size = torch.where(ex > 0, (1 + man.double() / 2 ** bits) * torch.exp2(ex.double() - bias), man.double() / 2 ** bits * 2.0 ** (1 - bias))
    x = (1 - 2 * sign.double()) * size
    return (x.reshape(*x.shape[:-1], -1, BLOCK) * torch.exp2(scales.double() - 127)[..., None]).reshape(x.shape)


def exact(case, seed):
    st, c = prepare(case, seed), case
    if c["kind"] == "rotary":
        f, m = _frequencies(c)
        angle = st["positions"].double()[:, None, None] * torch.from_numpy(f).to(DEV)
        turn = torch.polar(torch.full_like(angle, m), angle)
        got = []
        for x in (st["q"], st["k"]):
            y, h = x.double().clone(), c["rot"] // 2
            at = (slice(0, h), slice(h, 2 * h)) if c["pairs"] == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
            z = torch.complex(y[..., at[0]].clone(), y[..., at[1]].clone()) * turn
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
            got.append(y)
        return got
    table, lens = st["table"].cpu().numpy(), st["lens"].cpu().numpy()
    if c["kind"] in ("append", "commit"):
        off = st["node_offsets"].cpu().numpy()
        where, rows, new = [], [], lens.copy()
        for s in range(c["B"]):
            if c["kind"] == "append":
                mine = list(range(off[s], off[s + 1]))
            else:
                mine = [off[s]] + [off[s] + int(r) for r in st["path"][s, : int(st["length"][s])].tolist()]
            new[s] += len(mine)
            rows += [int(r) for r in mine]
            where += [(int(table[s, (lens[s] + i) // PAGE]), int((lens[s] + i) % PAGE)) for i in range(len(mine))]
        rows, page, slot = (torch.tensor(v, device=DEV) for v in (rows, [w[0] for w in where], [w[1] for w in where]))
        made = {name: _stored(st[name][rows], c["fmt"]) for name in ("k", "v")}
        new = torch.from_numpy(new)
        if c["kind"] == "append" and c["back"]:
            return [made["k"][2], made["v"][2], new]
        cache = {}
        for name in ("k", "v"):
            codes = torch.zeros(st["cache"][name + "_codes"].shape, dtype=torch.float64, device=DEV)
            codes[page, :, slot] = made[name][0]
            cache[name + "_codes"], cache[name + "_scales"] = codes, None
        return [cache, new]
    if c["kind"] == "read":
        got = []
        for name in ("k", "v"):
            parts = []
            for s in range(c["B"]):
                pages = st["table"][s, : -(-int(lens[s]) // PAGE)].long()
                x = _meaning(st["cache"][name + "_codes"][pages], st["cache"][name + "_scales"][pages])
                parts.append(x.transpose(1, 2).reshape(-1, c["Hkv"], c["D"])[: int(lens[s])])
            got.append(torch.cat(parts))
        return got
    off, G = st["host_node_offsets"].tolist(), c["Hq"] // c["Hkv"]
    o, lse = torch.empty((st["n"], c["Hq"], c["D"]), dtype=torch.float64, device=DEV), torch.empty((st["n"], c["Hq"]), dtype=torch.float64, device=DEV)
    for s in range(c["B"]):
        a, b, L = off[s], off[s + 1], int(lens[s])
        pages = st["table"][s, : -(-L // PAGE)].long()
        kv = {}
        for name in ("k", "v"):
            x = _meaning(st["cache"][name + "_codes"][pages], st["cache"][name + "_scales"][pages])
            kv[name] = torch.cat([x.transpose(1, 2).reshape(-1, c["Hkv"], c["D"])[:L], st[name + "_tree"][a:b].double()])
        hidden = torch.zeros((b - a, L + b - a), dtype=torch.bool, device=DEV)
        hidden[:, L:] = ~st["see"][s, : b - a, : b - a]
        for h in range(c["Hq"]):
            x = (st["q"][a:b, h].double() @ kv["k"][:, h // G].t()) * st["scale"]
            x = x.masked_fill(hidden, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, 1)
            o[a:b, h] = torch.softmax(x, 1) @ kv["v"][:, h // G]
    return [o, lse]
