"""Rotary positions: pair j of a row at position p is turned by the angle p * inv_freq[j].

Float64; a pair is a complex number times mscale * exp(i t).  Test infrastructure only.
"""
import numpy as np


def rotary(x, positions, inv_freq, interleaved=False, mscale=1.0):
    """x [N, heads, D]; positions [N]; inv_freq [rot / 2].  Returns float64 [N, heads, D]."""
    y = np.array(x, dtype=np.float64)
    h = len(inv_freq)
    a, b = (np.s_[..., 0:2 * h:2], np.s_[..., 1:2 * h:2]) if interleaved else (np.s_[..., :h], np.s_[..., h:2 * h])
    t = np.asarray(positions, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    z = (y[a] + 1j * y[b]) * (mscale * np.exp(1j * t))
    y[a], y[b] = z.real, z.imag
    return y


def tree_positions(parent, node_offsets, prefix_lens):
    """Position of every tree row: the tokens in its sequence's cache plus its depth."""
    pos = np.zeros(int(node_offsets[-1]), np.int64)
    for s in range(len(node_offsets) - 1):
        for n in range(int(node_offsets[s]), int(node_offsets[s + 1])):
            depth, j = 0, n - int(node_offsets[s])
            while int(parent[int(node_offsets[s]) + j]) >= 0:
                j = int(parent[int(node_offsets[s]) + j])
                depth += 1
            pos[n] = int(prefix_lens[s]) + depth
    return pos
