"""prefix_attention: attention of a batch whose sequences share a prefix, over a paged cache."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2609_17184_b200 as ls
from .op_util import cu, pages_for

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def make(P, counts, lens, nq, nkv, d, page, dt, pad=0, seed=0, scale=2.0, dev="cuda", fill=float("nan")):
    """Inputs; what no row may see - other pages, slots behind the lengths, padded rows - holds `fill`."""
    rng = np.random.default_rng(seed)
    table, pages = pages_for([P] + list(lens), page, rng)
    kv = torch.full((pages, 2, nkv, page, d), fill, dtype=DT[dt])
    for i, n in enumerate([P] + list(lens)):
        for j in range(0, n, page):
            m = min(page, n - j)
            kv[int(table[i, j // page]), :, :, :m] = torch.from_numpy(rng.standard_normal((2, nkv, m, d)).astype(np.float32)).to(DT[dt])
    T = sum(counts) + pad
    q = torch.from_numpy(rng.standard_normal((T, nq, d)).astype(np.float32) * scale).to(DT[dt])
    if pad:
        q[-pad:] = fill
    s = dict(q=q.to(dev), kv=kv.to(dev), prefix=table[0, :-(-P // page)].clone().to(dev), P=P, table=table[1:].clone().to(dev),
             lens=torch.tensor(lens, dtype=torch.int32, device=dev), cu=cu(counts).to(dev), counts=list(counts), own=list(lens), page=page, pad=pad)
    return s


def call(s, **kw):
    return ls.prefix_attention(s["q"], s["kv"][:, 0], s["kv"][:, 1], s["prefix"], s["P"], s["table"], s["lens"], s["cu"], **kw)


def check(s, got, lse, scale=None, rows=None):
    """Against 64 bits.  How far: with w the softmax weights and A = sum w |v|, a weight is rounded by half a step, and off by the error of
    its score (a d-term fp32 sum of exact products: at most d / 2^24 of sum |q k| scale, twice: numerator and denominator) and 2^-21 for the
    exponentials and merges; fp32 sums of n keys in steps of 16 are off by n / 16 + 64 times 2^-23; the result is rounded by
    half a step.  In fp16 a weight below 2^-24 of the largest is off by 2^-25 of it."""
    T, nq, d = s["q"].shape
    nkv = s["kv"].size(2)
    G, page, P = nq // nkv, s["page"], s["P"]
    half = torch.finfo(s["q"].dtype).eps / 2
    sc = scale or d ** -0.5

    def take(pages, n):
        x = s["kv"][pages[:-(-n // page)].long()].double()  # [p][2][h][page][d]
        return x.permute(1, 2, 0, 3, 4).reshape(2, nkv, -1, d)[:, :, :n]

    pre = take(s["prefix"], P)
    row = 0
    for b, n in enumerate(s["counts"]):
        own = take(s["table"][b], s["own"][b])
        for j in range(n):
            see = max(s["own"][b] - (n - 1 - j), 0)
            k, v = torch.cat([pre, own[:, :, :see]], 2)
            if rows is None or row in rows:
                if k.size(1) == 0:
                    assert (got[row] == 0).all() and (lse[row] == -math.inf).all()
                else:
                    q = s["q"][row].double().view(nkv, G, d)
                    score = torch.einsum("hgd,hkd->hgk", q, k) * sc
                    err = torch.einsum("hgd,hkd->hgk", q.abs(), k.abs()).amax(-1, keepdim=True) * sc * d * 2.0 ** -24 + score.abs().amax(-1, keepdim=True) * 2.0 ** -22
                    want = torch.logsumexp(score, -1)
                    w = torch.exp(score - want[..., None])
                    o, a = torch.einsum("hgk,hkd->hgd", w, v), torch.einsum("hgk,hkd->hgd", w, v.abs())
                    c = half + 2 * err + 2.0 ** -21 + (k.size(1) / 16 + 64) * 2.0 ** -23
                    tol = half * o.abs() + a * c
                    if s["q"].dtype == torch.float16:
                        tol = tol + 2.0 ** -25 * w.amax(-1, keepdim=True) * v.abs().sum(1)[:, None] + 2.0 ** -25
                    far = (got[row].double().view(nkv, G, d) - o).abs()
                    assert (far <= tol).all(), (row, b, j, far.max().item(), (far / tol).max().item())
                    fl = (lse[row].double().view(nkv, G) - want).abs()
                    assert (fl <= err[..., 0] + 2.0 ** -21 * (1 + want.abs()) + (k.size(1) / 16 + 64) * 2.0 ** -23).all(), (row, fl.max().item())
            row += 1


CASES = [
    # P, counts, lens, nq, nkv, d, page, type, pad
    (0, [1], [1], 1, 1, 64, 16, "bf16", 0),
    (1, [1], [0], 1, 1, 128, 16, "fp16", 0),
    (512, [1], [33], 16, 16, 128, 64, "bf16", 0),
    (77, [1, 1, 1], [5, 0, 300], 8, 2, 64, 16, "fp16", 2),
    (0, [3, 1, 0, 2], [1, 0, 9, 2], 4, 4, 64, 8, "bf16", 1),          # rows that see nothing
    (130, [4, 1, 3], [20, 1, 66], 32, 8, 64, 16, "bf16", 0),
    (2001, [1, 2, 3, 4, 4, 3, 2, 1], [100, 130, 170, 200, 260, 290, 300, 101], 32, 8, 64, 16, "fp16", 0),
    (16, [5, 7], [5, 90], 6, 2, 128, 1, "bf16", 3),
    (100, [40, 3], [41, 3], 12, 3, 128, 2, "bf16", 0),
    (255, [1] * 40, list(range(40)), 8, 1, 128, 4, "fp16", 0),
    (5000, [1], [17], 4, 1, 64, 256, "bf16", 0),
    (3000, [2, 1], [700, 1300], 5, 1, 128, 32, "bf16", 0),
    (0, [1] * 300, [(7 * i) % 50 for i in range(300)], 4, 2, 64, 16, "fp16", 5),
    (1024, [1] * 150, [(11 * i) % 70 + 1 for i in range(150)], 4, 4, 128, 16, "bf16", 0),
    (700, [3] * 50, [(11 * i) % 70 + 3 for i in range(50)], 16, 4, 64, 64, "fp16", 0),
    (129, [130, 1], [131, 2], 2, 2, 128, 32, "bf16", 1),
    (4096, [1] * 64, [64] * 64, 8, 2, 128, 128, "fp16", 0),
    (639, [2] * 33, [5] * 33, 8, 2, 64, 8, "bf16", 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_64_bits(i):
    P, counts, lens, nq, nkv, d, page, dt, pad = CASES[i]
    s = make(P, counts, lens, nq, nkv, d, page, dt, pad, seed=i)
    out = torch.full_like(s["q"], 7.0)
    lse = torch.full(s["q"].shape[:2], 7.0, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, l = call(s, out=out, lse=lse, flag=flag)
    assert got is out and l is lse and flag.item() == 0
    check(s, got, l)
    if pad:  # rows behind the last sequence are left as they were
        assert (got[-pad:] == 7.0).all() and (l[-pad:] == 7.0).all()
    scratch = torch.full((ls.prefix_attention_scratch_bytes(s["q"].size(0), len(counts), nq, nkv, d, P),), 0xff, dtype=torch.uint8, device="cuda")
    again, _ = call(s, scratch=scratch)  # (whatever the scratch holds: NaN here)
    assert torch.equal(got[:sum(counts)], again[:sum(counts)])


@pytest.mark.gpu
@pytest.mark.parametrize("d,own", [(64, True), (128, False)])
def test_more_row_tiles_than_sms(d, own):
    """1200 rows of 16 query heads to a key head: 150 tiles of 128 rows for the prefix, two rounds of them."""
    s = make(270, [300] * 4, [310, 300, 305, 320] if own else [0] * 4, 32, 2, d, 16, "bf16", seed=11)
    check(s, *call(s), rows={0, 5, 299, 300, 599, 777, 1199})


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(d, bad):
    """The last of four new rows carries an infinity or NaN: the three before it do not see its key and value."""
    s = make(40, [4, 1], [21, 9], 8, 2, d, 16, "bf16", seed=3)
    page = int(s["table"][0, 20 // 16])
    s["kv"][page, 1, 1, 20 % 16, 3:9] = bad
    got, lse = call(s)
    check(s, got, lse, rows={0, 1, 2, 4})
    assert not got[3, 4:, 3:9].isfinite().any() and got[3, :4].isfinite().all() and got[3, 4:, 9:].isfinite().all()
    s["kv"][page, 0, 1, 20 % 16, 0] = bad  # ... and in its key
    got, lse = call(s)
    check(s, got, lse, rows={0, 1, 2, 4})


@pytest.mark.gpu
def test_a_prefix_with_not_a_number_in_one_head():
    s = make(300, [1] * 40, [3] * 40, 4, 2, 128, 16, "bf16", seed=4)
    s["kv"][int(s["prefix"][5]), 1, 0, 3, 7] = float("nan")
    got, _ = call(s)
    assert got[:, :2, 7].isnan().all() and got[:, :2, :7].isfinite().all() and got[:, 2:].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 60])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_key_that_is_no_number_shows_in_every_row(B, bad):
    """Each key of the prefix in turn (by its place in a tile), and an own one: scores that are no number leave none."""
    for at in list(range(0, 140, 9)) + [299]:
        s = make(300, [1] * B, [3] * B, 4, 2, 128, 16, "bf16", seed=4)
        s["kv"][int(s["prefix"][at // 16]), 0, 0, at % 16, 5:7] = bad  # (two elements: inf - inf or a sum of either sign)
        got, lse = call(s)
        q = s["q"][:, :2, 5:7].float()
        score = (q * bad).sum(-1)
        gone = ~(score == -math.inf)  # (-inf: a weight of nothing)
        assert got[:, :2][gone].isnan().all() and got[:, :2][~gone].isfinite().all() and got[:, 2:].isfinite().all()
        assert lse[:, 2:].isfinite().all() and not lse[:, :2][gone].isfinite().any()


@pytest.mark.gpu
def test_references_that_move_often():
    """Keys whose scores grow along the prefix, so that rows leave their reference behind again and again, and rows that never do."""
    for d, dt in ((64, "fp16"), (128, "bf16")):
        s = make(1300, [1] * 80, [40] * 80, 2, 1, d, 16, dt, seed=9, scale=1.0)
        for j in range(-(-1300 // 16)):
            s["kv"][int(s["prefix"][j]), 0] *= 1 + j / 8
        s["q"][::3] *= 0.01
        check(s, *call(s))


@pytest.mark.gpu
@pytest.mark.parametrize("B", [2, 70])
def test_scales_strides_streams_and_graphs(B):
    """Large scores (one key takes nearly all), a scale, rows inside wider ones, [page][slot][head] order, a stream of its own, a captured call
    replayed on other lengths and contents."""
    s = make(333, [1] * B, [5 + b for b in range(B)], 8, 2, 64, 16, "bf16", seed=5, scale=20.0)
    pool = s["kv"].permute(0, 1, 3, 2, 4).contiguous()
    s["kv"] = pool.permute(0, 1, 3, 2, 4)
    wide = torch.zeros(B, 8 * 64 + 16, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:-8] = s["q"].view(B, -1)
    s["q"] = wide[:, 8:-8].view(B, 8, 64)
    out = torch.zeros(B, 8 * 64 + 8, dtype=torch.bfloat16, device="cuda")[:, :512].view(B, 8, 64)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        _, lse = call(s, out=out, scale=0.3)
    st.synchronize()
    check(s, out, lse, scale=0.3)
    scratch = torch.empty(ls.prefix_attention_scratch_bytes(B, B, 8, 2, 64, 333), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, out=out, lse=lse, scratch=scratch)
    s["own"] = [5 + b // 2 for b in range(B)]
    s["lens"].copy_(torch.tensor(s["own"], dtype=torch.int32))
    s["q"].copy_(torch.randn(B, 8, 64))
    scratch.fill_(0xff)  # (whatever the scratch holds)
    graph.replay()
    torch.cuda.synchronize()
    check(s, out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 40])
def test_offsets_beyond_32_bits(n):
    s = make(20, [1] * n, [18] * n, 2, 1, 64, 16, "bf16", seed=6)
    pages = s["kv"].size(0)
    stride = ((1 << 31) // (pages - 2) + 4096) // 64 * 64  # the last pages begin beyond 2^31 elements
    store = torch.full(((pages - 1) * stride + 4096,), float("nan"), dtype=torch.bfloat16, device="cuda")
    far = store.as_strided(s["kv"].shape, (stride, 1024, 1024, 64, 1))
    far.copy_(s["kv"])
    s["kv"] = far
    check(s, *call(s))


@pytest.mark.gpu
def test_flags():
    """Pages outside the cache, row counts and lengths that cannot be: a bit each, other sequences as they should be."""
    for n in (1, 40):
        counts, lens = [2, 1, 3] * n, [20, 5, 33] * n
        rows = {r for r in range(6 * n) if r % 6 >= 2}

        def flagged(change, bit, ok=rows):
            s = make(100, counts, lens, 4, 2, 64, 16, "bf16", seed=7)
            change(s)
            flag = torch.zeros(1, dtype=torch.int32, device="cuda")
            got, lse = call(s, flag=flag)
            assert flag.item() == bit
            for b in range(0, 3 * n, 3):
                s["own"][b] = 20
            if ok:
                s["table"][::3] = make(100, counts, lens, 4, 2, 64, 16, "bf16", seed=7)["table"][::3]
                check(s, got, lse, rows=ok)

        def entry(value):
            return lambda s: s["table"][::3].fill_(value)

        flagged(entry(-1), 1)
        flagged(entry(2 ** 31 - 1), 1)
        flagged(lambda s: s["prefix"][2:3].fill_(10 ** 6), 1, ok=None)
        flagged(lambda s: s["lens"][::3].fill_(-1), 2)
        flagged(lambda s: s["lens"][::3].fill_(2 ** 30), 2)  # (taken as the table's capacity; its other entries are pages of the cache)
        flagged(lambda s: s["cu"][1:2].fill_(10 ** 6), 2, ok=None)
        flagged(lambda s: s["cu"][1:2].fill_(-3), 2, ok=None)
        flagged(lambda s: s["cu"].fill_(0)[1::2].fill_(6 * n), 2, ok=None)  # (rows that belong to several sequences)


def stopped(s, stop_tile, wait_us, flag, out, lse, scratch):
    """The call with its test hook, through the C ABI."""
    from paper_2609_17184_b200.binding import PagedKv
    T, nq, d = s["q"].shape
    pages, _, nkv, page, _ = s["kv"].shape
    kv = PagedKv(s["kv"][:, 0].data_ptr(), s["kv"][:, 1].data_ptr(), s["kv"].stride(0), s["kv"].stride(2), s["kv"].stride(3), pages, page, nkv, d,
                 1 if s["q"].dtype == torch.bfloat16 else 2)
    return ls.lib.loopspec_debug_prefix_attention(s["q"].data_ptr(), nq * d, T, nq, C.byref(kv), s["prefix"].data_ptr(), s["P"], s["table"].data_ptr(), s["table"].stride(0),
                                                  s["table"].size(1), s["lens"].data_ptr(), s["cu"].data_ptr(), len(s["counts"]), 0.0, out.data_ptr(), nq * d, lse.data_ptr(),
                                                  None if flag is None else flag.data_ptr(), scratch.data_ptr(), scratch.numel(),
                                                  torch.cuda.current_stream().cuda_stream, stop_tile, wait_us)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dt,P", [(64, "fp16", 1200), (128, "bf16", 3100), (128, "bf16", 100)])
def test_waits_that_run_out_leave_a_flag_and_no_numbers(d, dt, P):
    """The tensor cores' CTAs request no tile from the given one on (none at all, none beyond what the rings hold, none of the last ones).  The call ends, every
    row of the prefix is NaN, with a flag or without, and the next call is right."""
    B = 80
    s = make(P, [1] * B, [20] * B, 4, 2, d, 16, dt, seed=8)
    want, want_lse = call(s)
    scratch = torch.empty(ls.prefix_attention_scratch_bytes(B, B, 4, 2, d, P), dtype=torch.uint8, device="cuda")
    out, lse, flag = torch.empty_like(want), torch.empty_like(want_lse), torch.zeros(1, dtype=torch.int32, device="cuda")
    assert stopped(s, 10 ** 6, 200, flag, out, lse, scratch) == 0 and flag.item() == 0  # (beyond all tiles)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    for stop in (0, 1, 2, 4):
        for f in (flag.zero_(), None):
            assert stopped(s, stop, 200, f, out, lse, scratch) == 0
            torch.cuda.synchronize()
            if f is not None:
                dropped = f.item() == 4
                assert dropped or (f.item() == 0 and stop > 0)  # (a CTA has as many tiles as the roles leave it)
                assert dropped or torch.equal(out, want)
            if dropped:
                assert out.isnan().any(-1).any() and (out.isnan().all(-1) == lse.isnan()).all()
                assert stop > 0 or (out.isnan().all() and lse.isnan().all())
                fine = ~lse.isnan()
                assert torch.equal(out[fine], want[fine]) and torch.equal(lse[fine], want_lse[fine])
            got, l = call(s, flag=flag.zero_())
            assert flag.item() == 0 and torch.equal(got, want) and torch.equal(l, want_lse)


@pytest.mark.gpu
def test_dimensions_of_one_element_have_any_stride():
    s = make(13, [1], [9], 3, 1, 64, 1, "bf16", seed=12)
    for name in ("q", "kv"):
        x = s[name]
        s[name] = x.as_strided(x.shape, [3 if n == 1 else st for n, st in zip(x.shape, x.stride())])
    check(s, *call(s))


@pytest.mark.gpu
def test_nothing_to_do():
    s = make(10, [1], [3], 2, 1, 64, 16, "bf16")
    s["q"] = s["q"][:0]
    out, lse = call(s)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    s = make(10, [1], [3], 2, 1, 64, 16, "bf16")
    s["cu"].zero_()
    out = torch.full_like(s["q"], 3.0)
    call(s, out=out)
    assert (out == 3.0).all()


def test_refusals():
    """EINVAL or ECAPACITY before anything is launched: the addresses here are never read."""
    from paper_2609_17184_b200.binding import PagedKv
    A = 1 << 20

    def rc(kv=None, q=A, qld=128, T=3, nq=2, pages=A, P=20, table=A, tld=4, width=4, lens=A, cu_=A, B=2, scale=0.0, out=A, old=128, scratch=A, room=1 << 40):
        d = dict(k=A, v=A, ps=2048, hs=1024, ss=64, n=4, page=16, nkv=1, d=64, t=1)
        d.update(kv or {})
        return ls.lib.loopspec_op_prefix_attention(q, qld, T, nq, C.byref(PagedKv(*d.values())), pages, P, table, tld, width, lens, cu_, B, scale, out, old, None,
                                                   None, scratch, room, None)

    for kw in (dict(k=None), dict(v=A + 8), dict(ps=4), dict(page=24), dict(d=96), dict(d=256), dict(t=0), dict(nkv=3), dict(nkv=0)):
        assert rc(kv=kw) == -1, kw
    for kw in (dict(q=None), dict(q=A + 8), dict(qld=124), dict(qld=64), dict(T=-1), dict(nq=0), dict(pages=None), dict(P=-1), dict(table=None), dict(tld=3), dict(width=-1),
               dict(lens=None), dict(cu_=None), dict(B=-1), dict(B=2049), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(out=None),
               dict(out=A + 4), dict(old=64), dict(width=1 << 28, tld=1 << 28)):
        assert rc(**kw) == -1, kw
    need = ls.prefix_attention_scratch_bytes(3, 2, 2, 1, 64, 20)
    assert need > 0 and rc(room=need - 1) == -3 and rc(scratch=None) == -3 and rc(scratch=A + 128) == -3
    assert rc(T=0) == 0 and rc(B=0) == 0
    for bad in ((-1, 2, 2, 1, 64, 20), (3, 2, 3, 2, 64, 20), (3, 2, 2, 1, 80, 20), (3, 2, 2, 1, 64, -1), (3, 4000, 2, 1, 64, 20)):
        assert ls.prefix_attention_scratch_bytes(*bad) == 0


def test_sizes_that_cannot_be_counted_are_refused():
    """Positions and a grid's sequences x heads are counted in 32 bits, positions in tiles of up to 128."""
    from paper_2609_17184_b200.binding import PagedKv
    A = 1 << 20
    assert ls.prefix_attention_scratch_bytes(1, 2048, 1 << 20, 1, 64, 0) == 0
    for P in (2 ** 31 - 1, 2 ** 31 - 100):
        assert ls.prefix_attention_scratch_bytes(1, 1, 1, 1, 64, P) == 0
    for page, width in ((1, 2 ** 31 - 1), (2, 2 ** 30 - 1), (4, 2 ** 29 - 2)):
        assert ls.lib.loopspec_op_prefix_attention(A, 64, 1, 1, C.byref(PagedKv(A, A, 2048, 1024, 64, 4, page, 1, 64, 1)), None, 0, A, width, width, A, A, 1, 0.0, A, 64, None,
                                                   None, A, 1 << 40, None) == -1
    assert ls.prefix_attention_scratch_bytes(1, 2048, 1 << 18, 1, 64, 0) > 0 and ls.prefix_attention_scratch_bytes(1, 1, 1, 1, 64, 2 ** 31 - 256) > 0


@pytest.mark.gpu
def test_wrapper_refusals():
    def fails(status="EINVAL", call_kw={}, **kw):
        s = make(20, [2, 1], [4, 3], 4, 2, 64, 16, "bf16")
        for k, f in kw.items():
            s[k] = f(s[k])
        with pytest.raises(ls.LoopSpecError) as e:
            call(s, **call_kw)
        assert e.value.status == status

    fails(q=lambda x: x.half())
    fails(q=lambda x: x[..., :32])
    fails(q=lambda x: x[:, :3])
    fails(q=lambda x: x.cpu())
    fails(kv=lambda x: x.transpose(3, 4))
    fails(prefix=lambda x: x[:1])
    fails(prefix=lambda x: None)
    fails(table=lambda x: x.long())
    fails(lens=lambda x: x[:1])
    fails(cu=lambda x: x[:2])
    fails(call_kw=dict(out=torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")))
    fails(call_kw=dict(lse=torch.zeros(3, 3, device="cuda")))
    fails(call_kw=dict(scale=0.0))
    fails(call_kw=dict(scale=-1.0))
    fails("ECAPACITY", call_kw=dict(scratch=torch.zeros(256, dtype=torch.uint8, device="cuda")))
