"""Attention over latents in 64 bits, from the definitions, one row and one head after the other."""
import numpy as np

from oracle.tree_attention import ancestor_mask


def _softmax(x):
    top = x.max()
    e = np.exp(x - top)
    return e / e.sum(), top + np.log(e.sum())


def tree(q, q_rope, prefix, c_tree, r_tree, parent, node_offsets, scale):
    """q [NN,Hq,R], q_rope [NN,Hq,Dr]; prefix: a list of [L, R + Dr] a sequence; c_tree [NN,R], r_tree [NN,Dr].  (o, lse)."""
    NN, Hq, R = q.shape
    o, lse = np.zeros((NN, Hq, R)), np.zeros((NN, Hq))
    for s in range(len(node_offsets) - 1):
        a, b = int(node_offsets[s]), int(node_offsets[s + 1])
        if a == b:
            continue
        see = ancestor_mask(np.asarray(parent[a:b]))
        for i in range(b - a):
            mine = np.nonzero(see[i])[0] + a
            lat = np.concatenate([prefix[s][:, :R], c_tree[mine]])
            rot = np.concatenate([prefix[s][:, R:], r_tree[mine]])
            for h in range(Hq):
                p, lse[a + i, h] = _softmax(scale * (lat @ q[a + i, h] + rot @ q_rope[a + i, h]))
                o[a + i, h] = p @ lat
    return o, lse


def prompt(q, q_rope, k, k_rope, v, q_offsets, kv_offsets, scale):
    """q [N,H,Dn], q_rope [N,H,Dr], k [T,H,Dn], k_rope [T,Dr], v [T,H,Dv].  (o, lse)."""
    N, H, _ = q.shape
    o, lse = np.zeros((N, H, v.shape[2])), np.full((N, H), -np.inf)
    for s in range(len(q_offsets) - 1):
        a, b, k0, k1 = int(q_offsets[s]), int(q_offsets[s + 1]), int(kv_offsets[s]), int(kv_offsets[s + 1])
        for i in range(b - a):
            end = k1 - (b - a) + i + 1
            if end <= k0:
                continue
            for h in range(H):
                p, lse[a + i, h] = _softmax(scale * (k[k0:end, h] @ q[a + i, h] + k_rope[k0:end] @ q_rope[a + i, h]))
                o[a + i, h] = p @ v[k0:end, h]
    return o, lse
