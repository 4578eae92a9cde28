"""sample: a token per row by temperature, top-k, top-p and min-p from given uniform numbers."""
import math
import pathlib

import numpy as np
import pytest
import torch

import paper_2609_17184_b200 as ls

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def reference(z, u, t=1.0, k=0, p=1.0, m=0.0):
    """Token and probability of one row in 64 bits, and how near u came to the edge of the token's share (as a part of it)."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    if z.max() == -np.inf:
        return -1, 0.0, 1.0
    if not t > 0:
        return int(np.argmax(z)), 1.0, 1.0
    with np.errstate(invalid="ignore"):
        w = np.where((z == -np.inf) | ((z < np.inf) & (z.max() == np.inf)), 0.0, np.exp(np.where(z == z.max(), 0.0, z - z.max()) / t))
    order = np.argsort(-z, kind="stable")
    if k > 0:
        order = order[:k]
    if 0 < p < 1:
        mass = np.cumsum(w[order])
        order = order[:int(np.searchsorted(mass, p * mass[-1], side="left")) + 1]
    if m > 0:
        order = order[w[order] >= min(m, 1.0)]
    chosen = np.sort(order)
    mass = np.cumsum(w[chosen])
    at = float(u) * mass[-1]
    i = min(int(np.searchsorted(mass, at, side="right")), len(chosen) - 1)
    share = w[chosen[i]]
    return int(chosen[i]), share / mass[-1], min(at - (mass[i] - share), mass[i] - at) / share


def check(z, u, got, t=None, k=None, p=None, m=None):
    """The token of the definition.  A sum of V weights in 64 bits is off by at most V * 2^-53 of itself; where u comes nearer to an edge than 2^-30 of the
    largest weight's share either neighbour would do, and no input here comes that near.  Probabilities: fp32, half a step and 2^-30."""
    tok, prob = got[0].cpu().numpy(), got[1].cpu().numpy()
    zs = z.float().cpu().numpy()

    def of(x, r, default):
        return default if x is None else float(x[r])

    for r in range(len(zs)):
        want, pw, edge = reference(zs[r], float(u[r]), of(t, r, 1.0), int(of(k, r, 0)), of(p, r, 1.0), of(m, r, 0.0))
        assert tok[r] == want, (r, tok[r], want, edge)
        assert abs(prob[r] - pw) <= pw * (2.0 ** -24 + 2.0 ** -30) + 1e-30


def call(z, u, t=None, k=None, p=None, m=None, **kw):
    def dev(x, dt):
        return None if x is None else torch.as_tensor(np.asarray(x)).to("cuda", dt)
    return ls.sample(z, dev(u, torch.float32), dev(t, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32), **kw)


def settings(mode, rows, rng):
    t, k, p, m = (None,) * 4
    if mode in ("temperature", "mixed"):
        t = np.float32(rng.uniform(0.3, 2.0, rows))
    if mode in ("top_k", "mixed"):
        k = rng.choice([0, 1, 2, 5, 50, 1000, 10 ** 9], rows)
    if mode in ("top_p", "mixed"):
        p = np.float32(rng.choice([0.0, 1e-6, 0.1, 0.5, 0.9, 0.999, 1.0, 2.0], rows))
    if mode in ("min_p", "mixed"):
        m = np.float32(rng.choice([0.0, 1e-4, 0.02, 0.5, 1.0, 7.0], rows))
    if mode == "mixed":
        t[::7] = 0.0
    return t, k, p, m


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["plain", "temperature", "top_k", "top_p", "min_p", "mixed"])
@pytest.mark.parametrize("rows,V,dt", [(1, 1, "fp32"), (3, 2, "bf16"), (5, 31, "fp16"), (9, 513, "fp32"), (7, 4096, "bf16"), (4, 5003, "fp16"), (6, 32000, "fp32"),
                                       (40, 50001, "bf16"), (3, 128256, "fp32"), (2, 262144, "fp16"), (2, 262144, "fp32")])
def test_the_token_of_the_definition(mode, rows, V, dt):
    rng = np.random.default_rng(V + len(mode))
    z = rng.standard_normal((rows, V)) * 2.5
    z[np.arange(rows)[:, None], rng.integers(0, V, (rows, 8))] += rng.uniform(0, 9, (rows, 8))
    z = torch.from_numpy(z).to("cuda", DT[dt])
    u = np.float32(rng.random(rows) * 0.999999)
    u[0] = 0.0
    t, k, p, m = settings(mode, rows, rng)
    check(z, u, call(z, u, t, k, p, m), t, k, p, m)


@pytest.mark.gpu
@pytest.mark.parametrize("V,dt", [(50001, "bf16"), (128256, "fp32"), (20000, "fp32")])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 0.5, 6.0])
def test_cuts_that_leave_thousands_of_tokens(V, dt, spread):
    """Flat logits: top-k of thousands, a top-p that half of the vocabulary is needed for, and both."""
    rng = np.random.default_rng(V)
    rows = 12
    z = torch.from_numpy(rng.standard_normal((rows, V)) * spread).to("cuda", DT[dt])
    u = np.float32(rng.random(rows) * 0.99999)
    k = rng.choice([2049, 5000, V // 2, V - 1], rows)
    p = np.float32(rng.choice([0.3, 0.9, 0.9999], rows))
    m = np.float32(rng.choice([0.0, 0.01, 0.9], rows))
    for kw in ((None, k, None, None), (None, None, p, None), (None, k, p, m), (np.float32([0.01] * rows), k, p, None), (np.float32([50.0] * rows), k, p, None)):
        check(z, u, call(z, u, *kw), *kw)


@pytest.mark.gpu
@pytest.mark.parametrize("V,dt", [(128256, "fp32"), (50001, "bf16")])
def test_a_top_k_of_more_tokens_than_weigh_anything_with_min_p(V, dt):
    """Low temperatures: thousands of tokens weigh something, fewer than top-k would keep, and min-p has the last word; again and again, in clusters of
    every size."""
    rng = np.random.default_rng(V)
    for rows in (1, 3, 30, 80):
        z = torch.from_numpy(rng.standard_normal((rows, V))).to("cuda", DT[dt])
        u, t, k = np.float32(rng.random(rows) * 0.99999), np.float32([0.08] * rows), [V - 1] * rows
        for m in (np.float32([0.01] * rows), np.float32([1e-9] * rows), np.float32([1.0] * rows)):
            first = [x.clone() for x in call(z, u, t, k, None, m)]
            check(z, u, first, t, k, None, m)
            for _ in range(10):
                assert all(torch.equal(a, b) for a, b in zip(call(z, u, t, k, None, m), first))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V,dt", [(1, 50001, "fp32"), (20, 20011, "bf16"), (40, 9000, "fp16"), (160, 5003, "fp32"), (300, 700, "bf16")])
def test_a_small_k_wherever_its_tokens_lie(rows, V, dt):
    """The largest logits spread, side by side, at either end, many alike, or fewer that weigh anything than k."""
    rng = np.random.default_rng(V + rows)
    z = rng.standard_normal((rows, V))
    kind = (np.arange(rows) if rows > 1 else np.array([1])) % 6
    for r in range(rows):
        if kind[r] == 1:
            at = int(rng.integers(0, V - 300))
            z[r, at:at + 300] += 9
        elif kind[r] == 2:
            z[r, -200:] += 9
        elif kind[r] == 3:
            z[r] = np.round(z[r])
        elif kind[r] == 4:
            z[r, rng.random(V) < 0.999] -= 300
        elif kind[r] == 5:
            z[r] = 0.5
    z = torch.from_numpy(z).to("cuda", DT[dt])
    u = np.float32(rng.random(rows) * 0.99999)
    t, p = np.float32(rng.uniform(0.5, 1.5, rows)), np.float32(rng.choice([0.3, 0.9, 1.0], rows))
    for k in (1, 2, 24, 25, 96, 97, 192, 193):
        check(z, u, call(z, u, t, [k] * rows), t, [k] * rows)
        check(z, u, call(z, u, t, [k] * rows, p, np.float32([0.02] * rows)), t, [k] * rows, p, np.float32([0.02] * rows))


@pytest.mark.gpu
@pytest.mark.parametrize("V", [100, 20011])
def test_ties_go_to_the_lower_index(V):
    """Few distinct values: the cut of top-k and top-p lies among equal logits, which the lower indexes survive."""
    rng = np.random.default_rng(V)
    rows = 24
    z = torch.from_numpy(rng.integers(0, 3, (rows, V)).astype(np.float32)).cuda()
    z[0] = 1.0
    z[1] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0)  # equal, whatever the sign
    u = np.float32(rng.random(rows) * 0.99999)
    for k, p in (([7] * rows, None), (None, [0.37] * rows), (list(range(1, rows + 1)), [0.5] * rows), ([V - 1] * rows, [0.9999] * rows), ([V // 2] * rows, [0.3] * rows)):
        p32 = None if p is None else np.float32(p)
        check(z, u, call(z, u, None, k, p32, None), None, k, p32, None)
    half = np.float32([0.5] * rows)
    uniform = torch.zeros(rows, V, device="cuda")  # exactly half of the tokens carry half of the mass
    tok, prob = call(uniform, np.float32([1 - 2 ** -24] * rows), None, None, half, None)
    assert (tok == (V + 1) // 2 - 1).all() and (prob == np.float32(1 / ((V + 1) // 2))).all()
    tok, _ = call(uniform, np.float32([0.0] * rows), None, None, half, None)
    assert (tok == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 30000])
def test_masked_infinite_and_missing_logits(V):
    rng = np.random.default_rng(V)
    z = rng.standard_normal((10, V)).astype(np.float32)
    z[0, :] = -np.inf                       # nothing left
    z[1, :] = np.nan
    z[2, 1:] = -np.inf                      # one left
    z[3, ::2] = -np.inf
    z[4, ::2] = np.nan                      # counts as masked out
    z[5, [3, 17, 30]] = np.inf              # they share the weight
    z[6, :] = np.finfo(np.float32).min      # masks of the type's lowest value: a row of nothing else is uniform
    z[7, 5:] = np.finfo(np.float32).min
    z[8, :] = np.finfo(np.float32).max
    z[9, :] = 0.0
    u = np.float32(rng.random(10) * 0.9999)
    zt = torch.from_numpy(z).cuda()
    for t, k, p, m in ((None,) * 4, (np.float32([0.5] * 10), [3] * 10, None, None), (None, None, np.float32([0.9] * 10), None), (None, [V] * 10, None, np.float32([0.1] * 10)),
                       (np.float32([0.0] * 10),) + (None,) * 3, (np.float32([np.inf] * 10),) + (None,) * 3, (np.float32([1e-40] * 10),) + (None,) * 3):
        check(zt, u, call(zt, u, t, k, p, m), t, k, p, m)


@pytest.mark.gpu
def test_settings_that_switch_a_filter_off_and_uniforms_out_of_range():
    rng = np.random.default_rng(1)
    z = torch.from_numpy(rng.standard_normal((6, 700)).astype(np.float32)).cuda()
    u = np.float32(rng.random(6))
    want = [x.clone() for x in call(z, u)]
    nan = np.float32([np.nan] * 6)
    for t, k, p, m in ((None, [0] * 6, None, None), (None, [-3] * 6, None, None), (None, None, nan, nan), (None, None, np.float32([0, -1, 1, 5, np.inf, 0]), np.float32([0, -1, 0, 0, -np.inf, 0])),
                       (np.float32([1.0] * 6), [700, 701, 10 ** 9, 0, 0, 700], None, None)):
        got = call(z, u, t, k, p, m)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(call(z, u, nan)[0], z.argmax(1).int()) and torch.equal(call(z, u, np.float32([-1.0] * 6))[0], z.argmax(1).int())
    top = call(z, np.float32([1.0, 2.0, np.inf, -1.0, np.nan, -np.inf]))[0]
    assert top.tolist() == [699, 699, 699, 0, 0, 0]


@pytest.mark.gpu
def test_strides_alignment_streams_and_graphs():
    rng = np.random.default_rng(2)
    for dt in ("fp32", "bf16"):
        for V, off in ((1000, 0), (20001, 1), (20001, 3), (65536, 5)):
            wide = torch.full((5, V + 11), float("inf"), device="cuda", dtype=DT[dt])  # what lies around the rows must not enter
            z = wide[:, off:off + V]
            z.copy_(torch.from_numpy(rng.standard_normal((5, V)) * 3))
            u, p = np.float32(rng.random(5) * 0.9999), np.float32([0.8] * 5)
            check(z, u, call(z, u, None, [900] * 5, p), None, [900] * 5, p)
    z = torch.from_numpy(rng.standard_normal((4, 9000)).astype(np.float32)).cuda()
    ut, out, pr = torch.rand(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        ls.sample(z, ut, out=out, probs=pr)
    st.synchronize()
    check(z, ut, (out, pr))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ls.sample(z, ut, out=out, probs=pr)
    z.copy_(torch.randn(4, 9000))
    ut.copy_(torch.rand(4))
    graph.replay()
    torch.cuda.synchronize()
    check(z, ut, (out, pr))


@pytest.mark.gpu
def test_rows_follow_their_distribution():
    """20,000 draws of one filtered row against its probabilities: chi-square over the kept tokens, at 6 standard deviations."""
    rng = np.random.default_rng(3)
    z = torch.from_numpy((rng.standard_normal(300) * 1.5).astype(np.float32)).cuda().expand(20000, -1).contiguous()
    u = torch.from_numpy(rng.random(20000, dtype=np.float32)).cuda()
    n = 20000
    tok, _ = ls.sample(z, u, top_k=torch.full((n,), 40, dtype=torch.int32, device="cuda"), top_p=torch.full((n,), 0.8, device="cuda"))
    zs = z[0].double().cpu().numpy()
    order = np.argsort(-zs, kind="stable")[:40]
    w = np.exp(zs[order] - zs.max())
    c = np.cumsum(w)
    order = order[:int(np.searchsorted(c, float(np.float32(0.8)) * c[-1])) + 1]
    w = np.exp(zs[order] - zs.max())
    expect = n * w / w.sum()
    seen = np.bincount(tok.cpu().numpy(), minlength=300)
    assert seen.sum() == seen[order].sum()
    chi, df = ((seen[order] - expect) ** 2 / expect).sum(), len(order) - 1
    assert chi < df + 6 * math.sqrt(2 * df)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    V, rows = 262144, 3
    stride = 1 << 30
    store = torch.zeros(2 * stride + V, dtype=torch.float32, device="cuda")
    z = store.as_strided((rows, V), (stride, 1))
    z.copy_(torch.randn(rows, V))
    u = np.float32([0.1, 0.5, 0.9])
    check(z, u, call(z, u, None, None, np.float32([0.9] * 3)), None, None, np.float32([0.9] * 3))


def resolution(V):
    """(2^-S, V * 2^-(S + 1)): what weights are multiples of, in parts of the largest, and what a sum of V of them is off by at most."""
    S = min(48, 61 - max(0, (V - 1).bit_length()))
    return 2.0 ** -S, V * 2.0 ** -(S + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [2, 5000, 8193, 50001, 262144])
@pytest.mark.parametrize("t", [1.0, 0.3])
def test_tokens_below_half_a_step_of_the_largest_count_as_masked_out(V, t):
    """A uniform of 0 takes the first token that weighs anything.  Logits by 2 % of a weight to either side of half a step (a weight is off by 1.4e-13 of itself, a logit of
    that size by 2^-19 of the weight's logarithm)."""
    unit, _ = resolution(V)
    border = math.log(unit / 2) * t
    z = torch.full((4, V), -1e4, device="cuda")
    z[:, V - 1] = 0.0
    z[0, 0], z[1, 0] = border + 0.02 * t, border - 0.02 * t
    z[2, 0] = z[3, 0] = border - 0.02 * t
    if V > 2:
        z[2, V // 2] = border + 0.02 * t
    ts, u = np.float32([t] * 4), np.float32([0.0] * 4)
    for k, p, m in ((None,) * 3, ([0, V, 10 ** 9, V - 1] if V > 2 else [0, 2, 2, 2], None, None), (None, None, np.float32([1e-30] * 4))):
        tok, prob = call(z, u, ts, k, p, m)
        if m is None:
            assert tok.tolist() == [0, V - 1, V // 2, V - 1]
            assert prob[1] == 1.0 and prob[3] == 1.0 and prob[0] < unit
        else:
            assert tok[1] == V - 1 and tok[3] == V - 1  # (nor does min-p bring it back)
    masked = z.masked_fill(z < border, -math.inf)
    u = np.float32([0.0, 0.25, 0.5, 0.999])
    for a, b in zip(call(z, u, ts), call(masked, u, ts)):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [5000, 50001, 131072, 262144])
@pytest.mark.parametrize("off", [-0.6, -0.01, 0.0, 0.01, 0.4, 3.0])
def test_how_far_a_heavy_tail_moves_a_border(V, off):
    """Thousands of tokens about half a step of the largest weight: each rounds the same way.  The token drawn is the definition's or one whose border is
    nearer than a sum can be off: V * 2^-(S + 1) of the largest weight, and 1.4e-13 of the sum; and so is the last token that top-p keeps."""
    unit, bound = resolution(V)
    rng = np.random.default_rng(V)
    rows = 16
    z = np.full((rows, V), math.log(unit / 2) + off, np.float32)
    z[:, rng.integers(0, V, 40)] = rng.uniform(-12, -3, 40)
    z[:, V // 3] = 0.0
    w = np.exp(z[0].astype(np.float64))
    run = np.cumsum(w)
    bound = bound + 1.4e-13 * run[-1]
    at = run[rng.integers(0, V, rows)] / run[-1]
    at[:5] = run[V // 3 - 1] / run[-1] * np.array([0.3, 0.9, 1.0, 1.1, 3.0])  # (about the largest token's border)
    u = np.float32(np.clip(at, 0, 1 - 2.0 ** -24))
    tok = call(torch.from_numpy(z).cuda(), u)[0].cpu().numpy()
    at = u.astype(np.float64) * run[-1]
    want = np.minimum(np.searchsorted(run, at, side="right"), V - 1)
    edge = np.minimum(at - (run[want] - w[want]), run[want] - at)
    assert (tok == want)[edge > bound].all() and (edge[:5] > bound).any()
    assert (run[tok] - w[tok] <= at + bound).all() and (run[tok] >= at - bound).all()
    # the same weights in the order of the ranking: a uniform of 1 takes the last token kept
    z = -np.sort(-z, axis=1)
    w = np.exp(z[0].astype(np.float64))
    run = np.cumsum(w)
    p = np.float32(np.concatenate([1 - 2.0 ** -np.arange(8, 24), [0.5] * (rows - 16)]))
    last = call(torch.from_numpy(z).cuda(), np.float32([1.0] * rows), None, None, p)[0].cpu().numpy()
    goal = p.astype(np.float64) * run[-1]
    assert (run[last] >= goal - bound).all() and (run[last] - w[last] < goal + bound).all()


def test_no_cta_reaches_into_another_before_all_of_its_cluster_have_started():
    """Read off the source, for what it prevents is a fault: every CTA of a cluster arrives at its barrier, and waits there ahead of the first exchange (a
    reduction, or an address in another CTA's shared memory)."""
    body = (pathlib.Path(__file__).parents[1] / "paper_2609_17184_b200/csrc/op_sample.cuh").read_text().split("sample_kernel(const __grid_constant__ Params p)")[1]
    arrive, wait = body.find("barrier.cluster.arrive"), body.find("barrier.cluster.wait")
    assert 0 <= arrive < wait < min(body.find(x) for x in ("R.max(", "R.sum(", "R.scan(", "cl.sync(", "map_shared_rank("))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,V", [(1, 16384), (30, 2056), (3, 2049), (2, 262144)])
def test_clusters_that_begin_again_and_again(rows, V):
    """Slices of some 260 to 1000 tokens (and a long one), whose load leaves next to no time between a CTA's start and its first exchange."""
    rng = np.random.default_rng(rows)
    z = torch.from_numpy(rng.standard_normal((rows, V)).astype(np.float32)).cuda()
    u, k = torch.from_numpy(rng.random(rows, dtype=np.float32) * 0.9999).cuda(), torch.full((rows,), 20, dtype=torch.int32, device="cuda")
    plain, few = [x.clone() for x in ls.sample(z, u)], [x.clone() for x in ls.sample(z, u, top_k=k)]
    check(z, u.cpu().numpy(), plain)
    got = [(ls.sample(z, u), ls.sample(z, u, top_k=k)) for _ in range(200)]
    for a, b in got:
        assert all(torch.equal(x, y) for x, y in zip((*a, *b), (*plain, *few)))


def test_refusals():
    """EINVAL before anything is launched: the addresses here are never read."""
    A = 1 << 20

    def rc(z=A, dt=0, ld=100, rows=2, V=100, u=A, tok=A):
        return ls.lib.loopspec_op_sample(z, dt, ld, rows, V, u, None, None, None, None, tok, None, None)

    for kw in (dict(z=None), dict(z=A + 2), dict(z=A + 1, dt=1), dict(dt=-1), dict(dt=3), dict(ld=99), dict(rows=-1), dict(V=0), dict(V=262145, ld=262145), dict(u=None), dict(tok=None)):
        assert rc(**kw) == -1, kw
    assert rc(rows=0) == 0


@pytest.mark.gpu
def test_wrapper_refusals():
    z, u = torch.zeros(3, 50, device="cuda"), torch.zeros(3, device="cuda")
    for f in (lambda: ls.sample(z.double(), u), lambda: ls.sample(z[0], u), lambda: ls.sample(z.t(), u), lambda: ls.sample(z, u[:2]), lambda: ls.sample(z, u.half()), lambda: ls.sample(z, u.cpu()),
              lambda: ls.sample(z, u, top_k=u), lambda: ls.sample(z, u, temperature=u[:1]), lambda: ls.sample(z[:1].expand(3, -1), u), lambda: ls.sample(z, u, out=u),
              lambda: ls.sample(z.cpu(), u)):
        with pytest.raises(ls.LoopSpecError) as e:
            f()
        assert e.value.status == "EINVAL"
    out, probs = ls.sample(z[:0], u[:0])
    assert out.numel() == 0 and probs.numel() == 0
