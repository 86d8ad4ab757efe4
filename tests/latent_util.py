"""Inputs, references in 64 bits and error bounds for the attention over latents.

Bounds.  u is half a step of the type (bf16 2^-8, float32 2^-24), e = 2^-24.  With X = scale * sum_d |q_d k_jd| (the largest over the keys that a row sees), n its keys
and A = sum_j w_j |v_j| by the exact weights:
  * a score is a float32 sum of d products: off by (d + 16) e X at most (the 16: the scale, the factor to octaves, the subtraction of the maximum, the
    exponential's argument), and the exponential instruction by 2^-22 of its result;
  * the weights' sum and the products' sums have n terms: n e of the sum of magnitudes each, and merging up to 64 partial sums 2^-18;
  * with bf16 a weight is rounded for the second product, u of it, and the result once, u of it.
So |error| <= u |o| + (u_weight + 2 (d + 16) e X + 2 n e + 2^-18) A, and of the logarithm (d + 16) e X + n e + 2^-18 + 4 e |lse|."""
import numpy as np
import torch

DEV = "cuda:0"
PAGE = 64


def dev(a, kind=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if kind is None else t.to(kind)).to(DEV)


def offsets(v, kind=np.int64):
    return np.concatenate([[0], np.cumsum(v)]).astype(kind)


def random_tree(rs, n, back=12):
    return np.array([-1] + [int(rs.randint(max(0, i - back), i)) for i in range(1, n)], dtype=np.int32)[:n]


def ancestors(parent):
    n = len(parent)
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if i:
            see[i] = see[parent[i]]
        see[i, i] = True
    return see


class Tree:
    """A call of hs_tree_attention_latent."""

    def __init__(self, sizes, lens, Hq, R=512, Dr=64, dtype=torch.bfloat16, seed=0, trees=None, spare_blocks=1, q_size=1.0):
        rs = np.random.RandomState(seed)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.sizes, self.lens, self.Hq, self.R, self.Dr, self.dtype = list(sizes), list(lens), Hq, R, Dr, dtype
        B, NN = len(sizes), int(sum(sizes))
        self.B, self.NN, self.scale = B, NN, (R // 4 + Dr) ** -0.5
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        blocks = [-(-l // PAGE) for l in lens]
        self.max_blocks = max(blocks) + spare_blocks
        need = sum(blocks)
        ids = rs.permutation(need + 3)
        self.pages = need + 3
        table = np.full((B, self.max_blocks), 2 ** 30, np.int32)   # entries behind the last page are no pages
        at = 0
        for s, b in enumerate(blocks):
            table[s, :b] = ids[at:at + b]
            at += b
        self.table_host = table
        self.pool = torch.full((self.pages, PAGE, R + Dr), float("nan"), dtype=dtype, device=DEV)  # what is not stored is NaN
        self.prefix = []
        for s, l in enumerate(lens):
            x = (rnd(l, R + Dr) * torch.exp2(torch.randint(-2, 2, (l, 1), generator=g, device=DEV).float())).to(dtype)
            self.prefix.append(x)
            for b in range(blocks[s]):
                part = x[b * PAGE:(b + 1) * PAGE]
                self.pool[int(table[s, b]), :part.shape[0]] = part
        self.parents = [random_tree(rs, n) for n in sizes] if trees is None else trees
        self.q = (rnd(NN, Hq, R) * q_size).to(dtype)
        self.q_rope = (rnd(NN, Hq, Dr) * q_size).to(dtype)
        self.c_tree, self.r_tree = rnd(NN, R).to(dtype), rnd(NN, Dr).to(dtype)
        self.host_no, self.host_pl = torch.from_numpy(offsets(sizes, np.int32)), torch.tensor(lens, dtype=torch.int64)
        self.parent = dev(np.concatenate(self.parents) if NN else np.zeros(0, np.int32))
        self.no, self.pl, self.table = self.host_no.to(DEV), self.host_pl.to(DEV), dev(table)

    def call(self, hs, **how):
        how.setdefault("want_lse", True)
        return hs.hs_tree_attention_latent(self.q, self.q_rope, self.pool, self.c_tree, self.r_tree, self.parent, self.no, self.host_no, self.table, self.pl,
                                           self.host_pl, self.scale, **how)

    def want(self):
        """(o, lse, bound of o, bound of lse) in 64 bits."""
        o = torch.zeros((self.NN, self.Hq, self.R), dtype=torch.float64, device=DEV)
        lse = torch.zeros((self.NN, self.Hq), dtype=torch.float64, device=DEV)
        bo, bl = torch.zeros_like(o), torch.zeros_like(lse)
        at = 0
        for s, n in enumerate(self.sizes):
            if n == 0:
                continue
            a, b = at, at + n
            at = b
            keys = torch.cat([self.prefix[s].double(), torch.cat([self.c_tree[a:b], self.r_tree[a:b]], 1).double()])
            q = torch.cat([self.q[a:b], self.q_rope[a:b]], 2).double().reshape(n * self.Hq, -1)
            hide = torch.zeros((n, self.lens[s] + n), dtype=torch.bool, device=DEV)
            hide[:, self.lens[s]:] = dev(~ancestors(self.parents[s]))
            self._fill(q, keys, keys[:, :self.R], hide.repeat_interleave(self.Hq, 0), o[a:b].view(n * self.Hq, -1), lse[a:b].view(-1), bo[a:b].view(n * self.Hq, -1),
                       bl[a:b].view(-1))
        return o, lse, bo, bl

    def _fill(self, q, k, v, hide, o, lse, bo, bl):
        fill(q, k, v, hide, self.scale, self.dtype, o, lse, bo, bl)

    def check(self, hs, **how):
        got = self.call(hs, **how)
        compare(got, self.want())
        return got


def fill(q, k, v, hide, scale, dtype, o, lse, bo, bl):
    u, e, d = torch.finfo(dtype).eps / 2, 2.0 ** -24, k.shape[1]
    uw = u if dtype == torch.bfloat16 else 0.0
    kt, ka = k.t().contiguous(), k.abs().t().contiguous()
    va = v.abs().contiguous()
    v = v.contiguous()
    for r in range(0, q.shape[0], 2048):
        h = hide[r:r + 2048]
        x = ((q[r:r + 2048] @ kt) * scale).masked_fill(h, -torch.inf)
        X = ((q[r:r + 2048].abs() @ ka) * scale).masked_fill(h, 0.0).amax(1) if k.shape[0] else torch.zeros(x.shape[0], dtype=torch.float64, device=DEV)
        some = ~h.all(1)
        n = (~h).sum(1).double()
        l = torch.logsumexp(x, 1)
        p = torch.where(some[:, None], torch.softmax(x, 1), 0.0) if k.shape[0] else x
        o[r:r + 2048] = p @ v
        lse[r:r + 2048] = l
        A = p @ va
        bo[r:r + 2048] = u * o[r:r + 2048].abs() + (uw + 2 * (d + 16) * e * X + 2 * n * e + 2.0 ** -18)[:, None] * A
        bl[r:r + 2048] = (d + 16) * e * X + n * e + 2.0 ** -18 + torch.where(some, 4 * e * l.abs(), 0.0)


def compare(got, want):
    o, lse = got
    wo, wl, bo, bl = want
    d = (o.double() - wo).abs()
    assert torch.isfinite(o).all(), "not finite: %s" % (~torch.isfinite(o)).nonzero()[:3].tolist()
    bad = ~(d <= bo)
    assert not bad.any(), "o: %d of %d beyond the bound, worst %.3g times, first at %s" % (bad.sum(), bad.numel(), (d / bo.clamp(min=1e-300)).max(), bad.nonzero()[0].tolist())
    if lse is not None:
        some = torch.isfinite(wl)
        assert torch.equal(lse[~some].double(), wl[~some])
        d = (lse.double() - wl).abs()[some]
        assert (d <= bl[some]).all(), "lse: worst %.3g times the bound" % (d / bl[some]).max()


class Prompt:
    """A call of hs_prompt_attention_latent."""

    def __init__(self, rows, keys, H, Dn=128, Dr=64, Dv=128, dtype=torch.bfloat16, seed=0, q_size=1.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.rows, self.keys, self.H, self.dtype, self.scale = list(rows), list(keys), H, dtype, (Dn + Dr) ** -0.5
        N, T = int(sum(rows)), int(sum(keys))
        self.N, self.T, self.Dv = N, T, Dv
        kv = rnd(T, H, Dn + Dv).to(dtype)
        self.k, self.v = kv[..., :Dn], kv[..., Dn:]
        self.q, self.q_rope, self.k_rope = (rnd(N, H, Dn) * q_size).to(dtype), (rnd(N, H, Dr) * q_size).to(dtype), rnd(T, Dr).to(dtype)
        self.host_qo, self.host_ko = torch.from_numpy(offsets(rows, np.int32)), torch.from_numpy(offsets(keys))
        self.qo, self.ko = self.host_qo.to(DEV), self.host_ko.to(DEV)

    def call(self, hs, **how):
        how.setdefault("want_lse", True)
        return hs.hs_prompt_attention_latent(self.q, self.q_rope, self.k, self.k_rope, self.v, self.qo, self.ko, self.host_qo, self.host_ko, self.scale, **how)

    def want(self):
        o = torch.zeros((self.N, self.H, self.Dv), dtype=torch.float64, device=DEV)
        lse = torch.full((self.N, self.H), -torch.inf, dtype=torch.float64, device=DEV)
        bo, bl = torch.zeros_like(o), torch.zeros_like(lse)
        qo, ko = self.host_qo.tolist(), self.host_ko.tolist()
        for s in range(len(self.rows)):
            a, b, k0, k1 = qo[s], qo[s + 1], ko[s], ko[s + 1]
            if b == a or k1 == k0:
                continue
            last = torch.arange(b - a, device=DEV) + (k1 - k0) - (b - a)
            hide = torch.arange(k1 - k0, device=DEV)[None] > last[:, None]
            for h in range(self.H):
                q = torch.cat([self.q[a:b, h], self.q_rope[a:b, h]], 1).double()
                k = torch.cat([self.k[k0:k1, h], self.k_rope[k0:k1]], 1).double()
                n = b - a
                part = [torch.zeros(n, self.Dv, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)]
                more = [torch.zeros_like(p) for p in part]
                fill(q, k, self.v[k0:k1, h].double(), hide, self.scale, self.dtype, part[0], part[1], more[0], more[1])
                o[a:b, h], lse[a:b, h], bo[a:b, h], bl[a:b, h] = part[0], part[1], more[0], more[1]
        return o, lse, bo, bl

    def check(self, hs, **how):
        got = self.call(hs, **how)
        compare(got, self.want())
        return got
