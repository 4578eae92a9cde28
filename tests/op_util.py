"""Inputs shared by the tests of the operators between the linear maps."""
import numpy as np
import torch

THETA = 10000.0


def inv_freq(rot, device="cpu"):
    return (THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(device)


def pages_for(lengths, page, rng, spare=2):
    """Page tables [len(lengths)][W] of distinct pages in random order, and the size of the pool."""
    need = [-(-n // page) for n in lengths]
    order = rng.permutation(sum(need) + spare).astype(np.int32)
    table, at = np.zeros((len(lengths), max(need + [1])), np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table), sum(need) + spare


def cu(counts):
    return torch.tensor(np.cumsum([0] + list(counts)), dtype=torch.int32)
