"""How the calls on latents cut a batch, by the workspace that they ask for (no GPU needed)."""
import numpy as np
import pytest
import torch

from paper_2505_13254_amd.binding import lib


def tree_bytes(rows, lens, Hq):
    no = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
    pl = torch.from_numpy(np.asarray(lens, np.int64))
    return lib().hs_tree_attention_latent_workspace(no.data_ptr(), pl.data_ptr(), len(rows), Hq, 512, 64)


def prompt_bytes(rows, keys, H):
    qo = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
    ko = torch.from_numpy(np.concatenate([[0], np.cumsum(keys)]).astype(np.int64))
    return lib().hs_prompt_attention_latent_workspace(qo.data_ptr(), ko.data_ptr(), len(rows), H, 128)


@pytest.mark.parametrize("B", [10, 300, 1500, 5000])
def test_a_long_sequence_among_many_is_cut(B):
    lens = [100] * B
    lens[B // 2] = 300000                                   # 4688 pages; uncut, one workgroup would take milliseconds
    splits = tree_bytes([1] * B, lens, 16) / (2064 * 16)
    assert 30 <= splits <= 1024, splits                     # records of that sequence alone
    keys = [100] * B
    keys[B // 2] = 300000
    splits = prompt_bytes([1] * B, keys, 8) / (528 * 8)
    assert 16 <= splits <= 1024, splits


def test_what_one_workgroup_does_is_not_cut():
    assert tree_bytes([1], [64], 16) == 0 and tree_bytes([3, 2], [0, 0], 8) == 0
    assert prompt_bytes([60], [60], 16) == 0
    assert tree_bytes([1] * 4000, [500] * 4000, 16) == 0    # the sequences alone fill the chip


def test_workspaces_stay_bounded():
    rs = np.random.RandomState(0)
    for _ in range(200):
        B = int(rs.choice([1, 2, 7, 60, 700]))
        lens = np.exp(rs.uniform(0, 14, B)).astype(np.int64)
        Hq = int(rs.choice([1, 16, 128]))
        rows = rs.randint(0, 200, B) if B < 100 else rs.randint(0, 3, B)
        assert tree_bytes(rows, lens, Hq) <= 2064 * (1 << 22) + 256
        keys = lens + rows
        assert prompt_bytes(rows, keys, Hq) <= 528 * (1 << 24) + 256
