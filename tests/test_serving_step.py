"""The operators as a serving program uses them: several samples of one prompt are decoded by a small model whose projections are the library's linear maps,
whose cache is filled by append_kv, whose attention is prefix_attention and whose tokens are drawn by sample - a step captured into a CUDA graph and replayed.
Checked against the model evaluated in 64 bits without a cache."""
import numpy as np
import pytest
import torch

import paper_2609_17184_b200 as ls
from .op_util import cu, inv_freq
from .test_sample import check as check_tokens

pytestmark = pytest.mark.gpu

V, H, NQ, NKV, D, PAGE, EPS = 512, 256, 4, 2, 64, 16, 1e-6


class Model:
    """x -> x + Wo attention(Wqkv x), logits = Wl x: queries and keys normed per head and rotated."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        w = lambda *s, k: (torch.randn(*s, generator=g) * k).to(torch.bfloat16)
        self.embed = torch.randn(V, H, generator=g)
        self.wqkv, self.wo, self.wl = w((NQ + 2 * NKV) * D, H, k=0.08), w(H, NQ * D, k=0.05), w(V, H, k=0.15)
        self.qn, self.kn = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
        self.f = inv_freq(D)

    def reference(self, tokens):
        """Logits of the last position in 64 bits, and how far the 16-bit cache may take them: queries, keys, values, weights and the output are rounded by half a
        step (2^-8) each, so a score by 2^-7 of the sum of its terms' sizes, a weight by twice that, the output by A (4 * 2^-8 * that sum + 3 * 2^-8)
        (A: the weighted sizes of the values), which the two maps behind it carry on; 2^-16 of the sizes for the maps' own fp32."""
        x = self.embed[tokens].double()
        n = len(tokens)
        y = (x @ self.wqkv.double().T).view(n, NQ + 2 * NKV, D)

        def head(z, gain):
            z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + EPS) * gain.double()
            angle = torch.arange(n, dtype=torch.float64)[:, None] * self.f
            c, s = angle.cos()[:, None], angle.sin()[:, None]
            a, b = z[..., :D // 2], z[..., D // 2:]
            return torch.cat([a * c - b * s, b * c + a * s], -1)

        q, k, v = head(y[:, :NQ], self.qn)[-1], head(y[:, NQ:NQ + NKV], self.kn), y[:, NQ + NKV:]
        k, v = k.repeat_interleave(NQ // NKV, 1), v.repeat_interleave(NQ // NKV, 1)
        score = torch.einsum("hd,nhd->hn", q, k) * D ** -0.5
        size = (torch.einsum("hd,nhd->hn", q.abs(), k.abs()) * D ** -0.5).amax(-1, keepdim=True)
        w = torch.softmax(score, -1)
        o, a = torch.einsum("hn,nhd->hd", w, v), torch.einsum("hn,nhd->hd", w, v.abs())
        err = (a * (4 * 2.0 ** -8 * size + 3 * 2.0 ** -8)).reshape(-1)
        out = x[-1] + o.reshape(-1) @ self.wo.double().T
        err = err @ self.wo.double().abs().T
        return out @ self.wl.double().T, (err + 2.0 ** -16 * out.abs()) @ self.wl.double().abs().T

    def cuda(self):
        for k, t in list(vars(self).items()):
            setattr(self, k, t.cuda())
        return self


class Cache:
    def __init__(self, prompt_len, samples, room):
        rng = np.random.default_rng(0)
        need = [-(-prompt_len // PAGE)] + [-(-room // PAGE)] * samples
        order = torch.from_numpy(rng.permutation(sum(need)).astype(np.int32)).cuda()
        self.kv = torch.full((sum(need), 2, NKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.prefix, self.table = order[:need[0]], order[need[0]:].view(samples, -1).contiguous()
        self.P = prompt_len

    @property
    def views(self):
        return self.kv[:, 0], self.kv[:, 1]


def test_samples_of_one_prompt_are_decoded_step_by_step():
    cpu, m = Model(1), Model(1).cuda()
    rng = np.random.default_rng(2)
    P, B, steps = 37, 5, 12
    prompt = rng.integers(0, V, P)
    cache = Cache(P, B, 40)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    # the prompt goes into the pages that all samples share
    qkv = ls.linear(m.wqkv, m.embed[torch.from_numpy(prompt).cuda()])
    ls.append_kv(qkv, *cache.views, cache.prefix[None], i32([0]), i32([0, P]), NQ, m.f, m.qn, m.kn, EPS)

    tokens, have, u = torch.zeros(B, dtype=torch.int64, device="cuda"), i32([0] * B), torch.zeros(B, device="cuda")
    rows, offset = cu([1] * B).cuda(), i32([P] * B)
    temperature, top_k, top_p = torch.tensor([0.0, 1.0, 0.7, 1.3, 1.0], device="cuda"), i32([0, 0, 40, 5, 0]), torch.tensor([1.0, 0.9, 1.0, 0.8, 1.0], device="cuda")

    def step():
        x = m.embed[tokens]
        q = ls.append_kv(ls.linear(m.wqkv, x), *cache.views, cache.table, have, rows, NQ, m.f, m.qn, m.kn, EPS, pos_offset=offset)
        have.add_(1)
        o, _ = ls.prefix_attention(q, *cache.views, cache.prefix, P, cache.table, have, rows)
        logits = ls.linear(m.wl, x + ls.linear(m.wo, o.view(B, -1).float()))
        return logits, ls.sample(logits, u, temperature, top_k, top_p)

    seqs = [list(prompt) + [int(t)] for t in rng.integers(0, V, B)]
    tokens.copy_(torch.tensor([s[-1] for s in seqs]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (once, uncaptured; its appends are made again)
        step()
    side.synchronize()
    have.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits, (drawn, probs) = step()
    have.zero_()
    for i in range(steps):
        u.copy_(torch.from_numpy(rng.random(B).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            want, tol = cpu.reference(seqs[b])
            assert ((logits[b].double().cpu() - want).abs() <= tol).all(), (i, b)
        check_tokens(logits, u.cpu().numpy(), (drawn, probs), temperature.cpu().numpy(), top_k.cpu().numpy(), top_p.cpu().numpy())
        for b, t in enumerate(drawn.tolist()):
            seqs[b].append(t)
        tokens.copy_(drawn)
    assert have.tolist() == [steps] * B


def test_drafts_of_several_tokens_agree_with_one_at_a_time():
    """Ragged drafts appended and attended to in one call: every row's logits are those of its own prefix."""
    cpu, m = Model(3), Model(3).cuda()
    rng = np.random.default_rng(4)
    P, counts = 50, [3, 1, 4, 0, 2]
    B, T = len(counts), sum(counts)
    prompt = rng.integers(0, V, P)
    cache = Cache(P, B, 24)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    ls.append_kv(ls.linear(m.wqkv, m.embed[torch.from_numpy(prompt).cuda()]), *cache.views, cache.prefix[None], i32([0]), i32([0, P]), NQ, m.f, m.qn, m.kn, EPS)
    old = [list(rng.integers(0, V, n)) for n in (0, 15, 14, 6, 1)]
    new = [list(rng.integers(0, V, n)) for n in counts]
    offset, zero = i32([P] * B), i32([0] * B)
    n_old = i32([len(s) for s in old])
    ids = torch.tensor(sum(old, []), device="cuda")
    ls.append_kv(ls.linear(m.wqkv, m.embed[ids]), *cache.views, cache.table, zero, cu([len(s) for s in old]).cuda(), NQ, m.f, m.qn, m.kn, EPS, pos_offset=offset)
    x = m.embed[torch.tensor(sum(new, []), device="cuda")]
    rows = cu(counts).cuda()
    q = ls.append_kv(ls.linear(m.wqkv, x), *cache.views, cache.table, n_old, rows, NQ, m.f, m.qn, m.kn, EPS, pos_offset=offset)
    o, _ = ls.prefix_attention(q, *cache.views, cache.prefix, P, cache.table, n_old + i32(counts), rows)
    logits = ls.linear(m.wl, x + ls.linear(m.wo, o.view(T, -1).float())).double().cpu()
    r = 0
    for b in range(B):
        for j in range(counts[b]):
            want, tol = cpu.reference(list(prompt) + old[b] + new[b][:j + 1])
            assert ((logits[r] - want).abs() <= tol).all(), (b, j)
            r += 1
