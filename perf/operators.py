"""The stand-alone operators of a serving step beside the linear maps, as measurable cases: what a program that drives its own
decode loop on the library calls between its projections.

Three operators:
  append   the QKV rows of new tokens: per-head RMS norm and rotary position of queries and keys, queries out, keys and values
           appended to a paged cache (`append_kv`)
  prefix   attention of a batch whose sequences share a long prefix (one system prompt, many samples of one prompt), the prefix
           read and multiplied once for all of them (`prefix_attention`)
  sample   one token per row of logits by temperature, top-k, top-p and min-p from given uniform numbers (`sample`)

Definitions.  Row j (of n) of sequence b has cached position cached[b] + j and rotary index pos_offset[b] + cached[b] + j; pairs (i, i + rot/2) of
a head turn by index * inv_freq[i].  In the attention it sees the whole prefix and the sequence's own positions below lens[b] - (n - 1 - j).
Sampling ranks tokens by logit (ties: lower index first); top-k keeps the first k; top-p then the shortest prefix of the ranking whose
share of what top-k kept reaches p; min-p then the tokens whose probability is at least min_p times the largest.  The token is the
first, by index, at which the running sum of the kept probabilities exceeds u times their sum; temperature 0 is the first largest logit.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
THETA = 10000.0
EPS = 1e-6


def listed():
    return [
        # one decoded token of one sequence of the 1.4B shape: the smallest call there is
        append("append_one", seqs=1, rows=(1, 1), cached=(512, 512), nq=16, nkv=16, d=128, page=64, dtype="bf16"),
        # a decode step of 64 sequences behind a shared prompt, straight from the fp32 output of a linear map, grouped heads
        append("append_decode_64", seqs=64, rows=(1, 1), cached=(0, 256), nq=32, nkv=8, d=128, page=16, dtype="fp32", cache="bf16", norm=True,
               offset=8192),
        # verification of ragged drafts, half of each head rotated, some padded rows at the end of the batch
        append("append_drafts", seqs=24, rows=(1, 7), cached=(0, 300), nq=6, nkv=6, d=64, page=32, dtype="fp16", norm=True, rot=32, pad=5),
        # prompts of three sequences in one call
        append("append_prompts", seqs=3, rows=(1900, 3400), cached=(0, 40), nq=32, nkv=8, d=128, page=32, dtype="bf16", norm=True),
        # one sequence behind a prompt: latency
        prefix("prefix_one", seqs=1, rows=(1, 1), prefix=512, lens=(33, 33), nq=16, nkv=16, d=128, page=64, dtype="bf16"),
        # a few sequences with short drafts, a prefix that ends inside a page
        prefix("prefix_drafts_8", seqs=8, rows=(1, 4), prefix=2001, lens=(100, 300), nq=32, nkv=8, d=64, page=16, dtype="fp16"),
        # a serving batch behind a long system prompt, grouped heads
        prefix("prefix_batch_64", seqs=64, rows=(1, 1), prefix=8192, lens=(128, 512), nq=32, nkv=8, d=128, page=32, dtype="bf16"),
        # many samples of one long prompt, every head with its own keys
        prefix("prefix_batch_256", seqs=256, rows=(1, 2), prefix=16384, lens=(2, 256), nq=16, nkv=16, d=128, page=64, dtype="bf16"),
        # one row at T = 1 with top-p 0.7
        sample("sample_one", rows=1, vocab=49152, dtype="fp32", mode="top_p"),
        # a small batch at T = 0.7 without filters
        sample("sample_plain_8", rows=8, vocab=49152, dtype="fp32", mode="plain"),
        # a serving batch, every row with settings of its own, some rows with tokens masked out
        sample("sample_mixed_64", rows=64, vocab=128256, dtype="fp32", mode="mixed", masked=True),
        # a large batch of 16-bit logits (many equal values) over an odd vocabulary
        sample("sample_top_k_256", rows=256, vocab=50001, dtype="bf16", mode="top_k"),
    ]


def append(name, seqs, rows, cached, nq, nkv, d, page, dtype, cache=None, norm=False, rot=0, offset=0, pad=0):
    c = dict(kind="append", seqs=seqs, rows_lo=rows[0], rows_hi=rows[1], cached_lo=cached[0], cached_hi=cached[1], nq=nq, nkv=nkv, d=d, page=page,
             dtype=dtype, cache=cache or dtype, norm=norm, rot=rot or d, offset=offset, pad=pad)
    return named(c, name)


def prefix(name, seqs, rows, prefix, lens, nq, nkv, d, page, dtype):
    c = dict(kind="prefix", seqs=seqs, rows_lo=rows[0], rows_hi=rows[1], prefix=prefix, lens_lo=lens[0], lens_hi=lens[1], nq=nq, nkv=nkv, d=d,
             page=page, dtype=dtype)
    return named(c, name)


def sample(name, rows, vocab, dtype, mode, masked=False):
    return named(dict(kind="sample", rows=rows, vocab=vocab, dtype=dtype, mode=mode, masked=masked), name)


def named(c, name):
    if name:
        c["name"] = name
    return c


def spread(rng, lo, hi):
    """An integer of [lo, hi], even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) - 0.5))))


HEADS = [(16, 16), (32, 8), (6, 6), (8, 2), (4, 1), (8, 1), (4, 4)]


def draw(rng):
    kind = rng.choice(["append", "prefix", "sample"])
    most = {}
    for c in listed():
        if c["kind"] == kind:
            w = work(c)
            for k in w:
                most[k] = max(most.get(k, 0), w[k])
    while True:
        nq, nkv = rng.choice(HEADS)
        d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
        if kind == "append":
            seqs, hi = spread(rng, 1, 256), spread(rng, 1, 4000)
            dtype = rng.choice(["fp32", "bf16", "fp16"])
            c = append(None, seqs, (rng.randint(1, hi), hi), (0, spread(rng, 1, 500)), nq, nkv, d, page, dtype,
                       cache=rng.choice(["bf16", "fp16"]) if dtype == "fp32" else dtype, norm=rng.random() < 0.5,
                       rot=rng.choice([d, d, d // 2, 16]), offset=rng.choice([0, spread(rng, 1, 1000000)]), pad=rng.choice([0, rng.randint(1, 9)]))
        elif kind == "prefix":
            hi, top = spread(rng, 1, 8), spread(rng, 8, 1500)
            c = prefix(None, spread(rng, 1, 256), (rng.randint(1, hi), hi), spread(rng, 1, 32000), (hi, top), nq, nkv, d, page,
                       rng.choice(["bf16", "fp16"]))
        else:
            c = sample(None, spread(rng, 1, 300), spread(rng, 500, 200000), rng.choice(["fp32", "bf16", "fp16"]),
                       rng.choice(["plain", "top_p", "top_k", "min_p", "mixed"]), rng.random() < 0.3)
        w = work(c)
        if all(w[k] <= most[k] for k in w):
            return c


# ---- what a program has in hand before the call --------------------------------------------------------------------------------


def counts(case, seed, lo, hi):
    """A number for every sequence: the case fixes which there are, the seed which sequence has which (together with its other numbers)."""
    rng, order = random.Random(lo), list(range(case["seqs"]))
    all_ = [rng.randint(case[lo], case[hi]) for _ in order]
    random.Random(seed).shuffle(order)
    return [all_[i] for i in order]


def middle(case, lo, hi):
    return case["seqs"] * (case[lo] + case[hi]) / 2


def paged(lengths, page, gen, spare=3):
    """Page tables of sequences of these lengths: pages in random order out of a pool with some to spare."""
    need = [(n + page - 1) // page for n in lengths]
    total = sum(need) + spare
    order = torch.randperm(total, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    width = max(max(need), 1)
    starts = torch.tensor(np.cumsum([0] + need[:-1]), device="cuda")[:, None] + torch.arange(width, device="cuda")[None, :]
    return order[starts.clamp(max=total - 1)].contiguous(), total


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    s = {"case": case}
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        z = normal(R, V, scale=2.0)
        # a trained model's readout: a bulk and a few candidates well above it
        best = torch.randint(0, V, (R, 32), generator=gen, device="cuda")
        z.scatter_add_(1, best, torch.rand(R, 32, generator=gen, device="cuda") * 10.0)
        if case["masked"]:
            gone = torch.rand(R, V, generator=gen, device="cuda") < 0.3
            gone[torch.arange(R, device="cuda") % 2 == 0] = False
            z = z.masked_fill(gone, -math.inf)
        s["logits"] = z.to(DTYPES[case["dtype"]])
        s["u"] = torch.rand(R, generator=gen, device="cuda")
        mode, dev = case["mode"], "cuda"
        t, k, p, m = torch.ones(R, device=dev), torch.zeros(R, dtype=torch.int32, device=dev), torch.ones(R, device=dev), torch.zeros(R, device=dev)
        if mode == "plain":
            t.fill_(0.7)
        elif mode == "top_p":
            p.fill_(0.7)
        elif mode == "top_k":
            t.fill_(0.8)
            k.fill_(50)
            m.fill_(0.05)
        elif mode == "min_p":
            m.fill_(0.02)
        else:  # rows of different requests: greedy, hot and cold ones, with and without each filter
            r = torch.arange(R, device=dev)
            t = 0.5 + 0.7 * torch.rand(R, generator=gen, device=dev)
            t[r % 8 == 3] = 0.0
            k[r % 3 == 1] = 1 + (r[r % 3 == 1] * 37 % 200).to(torch.int32)
            p = torch.where(r % 4 == 0, 1.0, 0.5 + 0.49 * torch.rand(R, generator=gen, device=dev))
            m = torch.where(r % 5 == 2, 0.1 * torch.rand(R, generator=gen, device=dev), 0.0)
        s.update(temperature=t, top_k=k, top_p=p, min_p=m)
        return s

    n = counts(case, seed, "rows_lo", "rows_hi")
    nq, nkv, d, page = case["nq"], case["nkv"], case["d"], case["page"]
    s["n"] = n
    s["cu_rows"] = torch.tensor(np.cumsum([0] + n), dtype=torch.int32, device="cuda")
    if case["kind"] == "append":
        old = counts(case, seed, "cached_lo", "cached_hi")
        s["page_table"], pages = paged([a + b for a, b in zip(old, n)], page, gen)
        s["cached"] = torch.tensor(old, dtype=torch.int32, device="cuda")
        s["pos_offset"] = torch.full((case["seqs"],), case["offset"], dtype=torch.int32, device="cuda") if case["offset"] else None
        T = sum(n) + case["pad"]
        s["qkv"] = normal(T, (nq + 2 * nkv) * d, dtype=DTYPES[case["dtype"]])
        s["q"] = normal(T, nq, d, dtype=DTYPES[case["cache"]])
        s["kv"] = normal(pages, 2, nkv, page, d, dtype=DTYPES[case["cache"]])
        s["inv_freq"] = THETA ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        s["q_norm"] = 1.0 + normal(d, scale=0.1) if case["norm"] else None
        s["k_norm"] = 1.0 + normal(d, scale=0.1) if case["norm"] else None
    else:
        lens = [max(a, b) for a, b in zip(n, counts(case, seed, "lens_lo", "lens_hi"))]
        table, pages = paged([case["prefix"]] + lens, page, gen)
        s["prefix_pages"] = table[0, :(case["prefix"] + page - 1) // page].clone()
        s["page_table"] = table[1:, :(max(lens) + page - 1) // page].clone()
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["lens_host"] = lens
        s["q"] = normal(sum(n), nq, d, dtype=DTYPES[case["dtype"]], scale=2.0)
        s["kv"] = normal(pages, 2, nkv, page, d, dtype=DTYPES[case["dtype"]])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------------


def run(state):
    if own:
        return run_own(state)
    return {"append": plain_append, "prefix": plain_prefix, "sample": plain_sample}[state["case"]["kind"]](state)


def run_own(s):
    import paper_2609_17184_b200 as ls

    c = s["case"]
    if c["kind"] == "append":
        q = ls.append_kv(s["qkv"], s["kv"][:, 0], s["kv"][:, 1], s["page_table"], s["cached"], s["cu_rows"], c["nq"], s["inv_freq"], q_norm=s["q_norm"],
                         k_norm=s["k_norm"], eps=EPS, pos_offset=s["pos_offset"], out=s["q"])
        return q, s["kv"]
    if c["kind"] == "prefix":
        return ls.prefix_attention(s["q"], s["kv"][:, 0], s["kv"][:, 1], s["prefix_pages"], c["prefix"], s["page_table"], s["lens"], s["cu_rows"])
    return ls.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


def plain_append(s):
    c = s["case"]
    nq, nkv, d, page, rot = c["nq"], c["nkv"], c["d"], c["page"], c["rot"]
    T = sum(s["n"])
    t = torch.arange(T, device="cuda")
    seq = (t[:, None] >= s["cu_rows"][None, 1:]).sum(1)
    pos = s["cached"][seq] + t - s["cu_rows"][seq]
    index = pos if s["pos_offset"] is None else pos + s["pos_offset"][seq]
    angle = index.double()[:, None] * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    x = s["qkv"][:T].float().view(T, nq + 2 * nkv, d)

    def turned(x, gain):
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        a, b, rest = x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)

    s["q"][:T] = turned(x[:, :nq], s["q_norm"]).to(s["q"].dtype)
    at, slot = s["page_table"][seq, pos // page].long(), pos % page
    s["kv"][at, 0, :, slot] = turned(x[:, nq:nq + nkv], s["k_norm"]).to(s["kv"].dtype)
    s["kv"][at, 1, :, slot] = x[:, nq + nkv:].to(s["kv"].dtype)
    return s["q"], s["kv"]


def plain_prefix(s):
    c = s["case"]
    nq, nkv, d, P, B = c["nq"], c["nkv"], c["d"], c["prefix"], c["seqs"]
    G, T, n, L = nq // nkv, sum(s["n"]), max(s["n"]), max(s["lens_host"])
    scale = 1.0 / math.sqrt(d)
    # the rows as [sequence][row], the missing ones repeat the last
    counts_ = s["cu_rows"][1:] - s["cu_rows"][:-1]
    j = torch.minimum(torch.arange(n, device="cuda")[None, :], counts_[:, None] - 1)
    row = (s["cu_rows"][:-1, None] + j).long()
    q = s["q"].float().view(T, nkv, G, d)
    kp, vp = (s["kv"][:, i][s["prefix_pages"].long()].transpose(0, 1).reshape(nkv, -1, d)[:, :P].float() for i in (0, 1))
    ks, vs = (s["kv"][:, i][s["page_table"].long()].transpose(1, 2).reshape(B, nkv, -1, d)[:, :, :L].float() for i in (0, 1))
    sp = torch.einsum("tkgd,kpd->tkgp", q, kp) * scale
    ss = torch.einsum("bnkgd,bkld->bnkgl", q[row], ks) * scale
    sees = (s["lens"] - counts_)[:, None] + j + 1
    hidden = torch.arange(L, device="cuda")[None, None, :] >= sees[:, :, None]
    ss = ss.masked_fill(hidden[:, :, None, None, :], -math.inf)
    m = torch.maximum(sp.amax(-1)[row], ss.amax(-1))
    mp = torch.empty(T, nkv, G, device="cuda")
    mp[row] = m
    ep, es = torch.exp(sp - mp[..., None]), torch.exp(ss - m[..., None])
    total = ep.sum(-1)[row] + es.sum(-1)
    out = torch.einsum("tkgp,kpd->tkgd", ep, vp)[row] + torch.einsum("bnkgl,bkld->bnkgd", es, vs)
    flat, lse = torch.empty(T, nkv, G, d, device="cuda"), torch.empty(T, nkv, G, device="cuda")
    flat[row] = out / total[..., None]
    lse[row] = m + torch.log(total)
    return flat.view(T, nq, d).to(s["q"].dtype), lse.view(T, nq)


def plain_sample(s):
    z = s["logits"]
    R, V = z.shape
    # in 64 bits: the token depends on which side of a border a running sum lies
    zd = z.double()
    greedy = (s["temperature"] <= 0)[:, None]
    t = torch.where(greedy, 1.0, s["temperature"][:, None].double())
    top = zd.amax(1, keepdim=True)
    w = torch.exp((zd - top) / t)
    ranked = torch.sort(z.float(), dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(ranked).scatter_(1, ranked, torch.arange(V, device=z.device).expand(R, V))
    k = torch.where(s["top_k"] > 0, s["top_k"].long(), V)[:, None]
    wr = w.gather(1, ranked)
    wr = wr.masked_fill(torch.arange(V, device=z.device)[None, :] >= k, 0.0)
    before = wr.cumsum(1) - wr
    p = s["top_p"][:, None].double()
    filtered = (p > 0) & (p < 1)
    n = torch.where(filtered, (before < p * wr.sum(1, keepdim=True)).sum(1, keepdim=True), V)
    kept = (rank < torch.minimum(n, k)) & (w >= s["min_p"][:, None].double())
    w = torch.where(kept, w, 0.0)
    run_ = w.cumsum(1)
    total = run_[:, -1:]
    token = torch.searchsorted(run_, s["u"][:, None].double() * total, right=True)
    first = ranked[:, :1]
    token = torch.where(greedy, first, token)
    prob = torch.where(greedy, 1.0, w.gather(1, token) / total)
    return token[:, 0].to(torch.int32), prob[:, 0].float()


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------


def work(case):
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * V * SIZES[case["dtype"]] + R * 28, "flops": 3 * R * V}
    nq, nkv, d, rows = case["nq"], case["nkv"], case["d"], middle(case, "rows_lo", "rows_hi")
    if case["kind"] == "append":
        width = (nq + 2 * nkv) * d
        return {"bytes": int(rows * width * (SIZES[case["dtype"]] + SIZES[case["cache"]])), "flops": int(rows * (nq + nkv) * d * (7 if case["norm"] else 3))}
    lens = middle(case, "lens_lo", "lens_hi")
    kv = 2 * nkv * d * SIZES[case["dtype"]]
    pairs = rows * case["prefix"] + lens * rows / case["seqs"]
    return {"bytes": int((case["prefix"] + lens) * kv + rows * nq * (2 * d * SIZES[case["dtype"]] + 4)), "flops": int(4 * pairs * nq * d)}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": exact_append, "prefix": exact_prefix, "sample": exact_sample}[case["kind"]](case, s)


def exact_append(c, s):
    nq, nkv, d, page, half = c["nq"], c["nkv"], c["d"], c["page"], c["rot"] // 2
    q, kv = s["q"].double(), s["kv"].double()
    x = s["qkv"].double().view(-1, nq + 2 * nkv, d)
    table, first = s["page_table"].cpu().numpy(), 0
    for b, n in enumerate(s["n"]):
        rows, start = x[first:first + n], int(s["cached"][b])
        angle = torch.arange(start + c["offset"], start + c["offset"] + n, device="cuda", dtype=torch.float64)[:, None] * s["inv_freq"][None]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
        parts = []
        for heads, gain in ((rows[:, :nq], s["q_norm"]), (rows[:, nq:nq + nkv], s["k_norm"])):
            y = heads
            if gain is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
            z = torch.complex(y[..., :half].contiguous(), y[..., half:2 * half].contiguous()) * turn
            parts.append(torch.cat([z.real, z.imag, y[..., 2 * half:]], -1))
        q[first:first + n] = parts[0]
        for i, y in ((0, parts[1]), (1, rows[:, nq + nkv:])):
            done = 0
            while done < n:  # page by page
                at = start + done
                take = min(n - done, page - at % page)
                kv[int(table[b, at // page]), i, :, at % page:at % page + take] = y[done:done + take].transpose(0, 1)
                done += take
        first += n
    return q, kv


def exact_prefix(c, s):
    nq, nkv, d, P, page = c["nq"], c["nkv"], c["d"], c["prefix"], c["page"]
    G, outs, lses, first = nq // nkv, [], [], 0

    def keys(pages, length, i):  # [head][position][d]
        return torch.cat([s["kv"][int(p), i] for p in pages[:(length + page - 1) // page].tolist()], 1)[:, :length].double()

    kp, vp = keys(s["prefix_pages"], P, 0), keys(s["prefix_pages"], P, 1)
    for b, n in enumerate(s["n"]):
        L = s["lens_host"][b]
        ks, vs = keys(s["page_table"][b], L, 0), keys(s["page_table"][b], L, 1)
        q = s["q"][first:first + n].double().view(n, nkv, G, d).permute(1, 2, 0, 3).reshape(nkv, G * n, d)
        score = torch.cat([q @ kp.transpose(1, 2), q @ ks.transpose(1, 2)], 2) * d ** -0.5
        see = torch.arange(L, device="cuda")[None, :] <= L - n + torch.arange(n, device="cuda")[:, None]
        see = torch.cat([torch.ones(n, P, dtype=torch.bool, device="cuda"), see], 1).repeat(G, 1)
        score = score.masked_fill(~see[None], -math.inf)
        lse = torch.logsumexp(score, 2)
        weight = torch.exp(score - lse[..., None])
        o = weight[:, :, :P] @ vp + weight[:, :, P:] @ vs
        outs.append(o.view(nkv, G, n, d).permute(2, 0, 1, 3).reshape(n, nq, d))
        lses.append(lse.view(nkv, G, n).permute(2, 0, 1).reshape(n, nq))
        first += n
    return torch.cat(outs), torch.cat(lses)


def exact_sample(c, s):
    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    t, k, p, m = (s[x].double().cpu().numpy() for x in ("temperature", "top_k", "top_p", "min_p"))
    tokens, probs = [], []
    for z, u_, t_, k_, p_, m_ in zip(logits, u, t, k, p, m):
        if t_ <= 0:
            tokens.append(int(np.argmax(z)))
            probs.append(1.0)
            continue
        w = np.exp((z - z.max()) / t_)
        order = np.lexsort((np.arange(len(z)), -z))
        if k_ > 0:
            order = order[:int(k_)]
        if 0 < p_ < 1:
            mass = np.cumsum(w[order])
            order = order[:int(np.searchsorted(mass, p_ * mass[-1], side="left")) + 1]
        chosen = np.sort(order[w[order] >= m_])
        mass = np.cumsum(w[chosen])
        i = min(int(np.searchsorted(mass, u_ * mass[-1], side="right")), len(chosen) - 1)
        tokens.append(int(chosen[i]))
        probs.append(w[chosen[i]] / mass[-1])
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64)
