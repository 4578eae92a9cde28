"""Calls of the operators in flight at the same time, and the most sequences there may be."""
import numpy as np
import pytest
import torch

import paper_2609_17184_b200 as ls
from . import test_append_kv as ta
from . import test_prefix_attention as tp
from . import test_sample as ts

pytestmark = pytest.mark.gpu


def work(seed):
    """A call of each operator on inputs of its own: small ones and such as fill the device."""
    rng = np.random.default_rng(seed)
    B = (3, 90)[seed % 2]
    s = tp.make(700 + 64 * seed, [1] * B, [20 + b % 50 for b in range(B)], 8, 2, (64, 128)[seed % 2], 16, "bf16", seed=seed)
    _, g = ta.make([40, 1 + 1200 * (seed % 2)], [3, 0], 4, 2, 64, 16, "bf16", "bf16", 64, True, seed=seed)
    rows = (2, 200)[seed % 2]
    z = torch.from_numpy(rng.standard_normal((rows, 20000)).astype(np.float32)).cuda()
    u, k, p = torch.rand(rows, device="cuda"), torch.full((rows,), 600, dtype=torch.int32, device="cuda"), torch.full((rows,), 0.8, device="cuda")

    def run():
        q = ta.call(g)
        return [*tp.call(s), *ls.sample(z, u, top_k=k, top_p=p), q.clone(), g["kv"].clone()]
    return run


def test_calls_on_two_streams():
    """Each stream's calls leave what they leave alone, to the bit; the scratch of either is allocated by its calls."""
    for seeds in ((0, 1), (1, 3), (0, 2)):
        runs = [work(i) for i in seeds]
        alone = [[x.clone() for x in r()] for r in runs]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in runs]
        for st in streams:
            st.wait_stream(torch.cuda.current_stream())
        got = [[], []]
        for _ in range(6):
            for i, st in enumerate(streams):
                with torch.cuda.stream(st):
                    got[i].append(runs[i]())
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for many in got[i] for a, b in zip(many, alone[i]))


def test_graphs_replayed_at_the_same_time():
    runs = [work(i) for i in (1, 3)]
    alone = [[x.clone() for x in r()] for r in runs]
    graphs, outs = [], []
    for r in runs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(r())
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("P", [0, 100])
def test_as_many_sequences_as_there_may_be(P):
    B = 2048
    counts = [1 if b % 3 else 0 for b in range(B)]
    lens = [b % 7 for b in range(B)]
    s = tp.make(P, counts, lens, 2, 1, 64, 8, "fp16", pad=2, seed=P)
    T = sum(counts)
    got, lse = tp.call(s)
    tp.check(s, got, lse, rows=set(range(0, T, 97)) | {T - 1})
