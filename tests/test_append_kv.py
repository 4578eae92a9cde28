"""append_kv: norms and rotation of queries and keys, keys and values into a paged cache."""
import numpy as np
import pytest
import torch

import paper_2609_17184_b200 as ls
from .op_util import cu, inv_freq, pages_for

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def make(counts, cached, nq, nkv, d, page, tin, tc, rot, norm, pad=0, offset=None, seed=0, dev="cuda"):
    """Inputs on the CPU and, as the call takes them, on the device."""
    rng = np.random.default_rng(seed)
    table, pages = pages_for([a + b for a, b in zip(counts, cached)], page, rng)
    T = sum(counts) + pad
    x = torch.from_numpy(rng.standard_normal((T, (nq + 2 * nkv) * d))).to(DT[tin])
    kv = torch.from_numpy(rng.standard_normal((pages, 2, nkv, page, d)).astype(np.float32)).to(DT[tc])
    q = torch.from_numpy(rng.standard_normal((T, nq, d)).astype(np.float32)).to(DT[tc])
    gains = [torch.from_numpy(1 + 0.2 * rng.standard_normal(d).astype(np.float32)) if norm else None for _ in range(2)]
    s = dict(x=x, kv=kv, q=q, table=table, cached=torch.tensor(cached, dtype=torch.int32), cu=cu(counts), f=inv_freq(rot) if rot else None, qn=gains[0],
             kn=gains[1], off=None if offset is None else torch.tensor(offset, dtype=torch.int32), nq=nq, nkv=nkv, d=d, page=page, rot=rot, counts=counts)
    return s, {k: (v.to(dev) if isinstance(v, torch.Tensor) else v) for k, v in s.items()}


def call(g, **kw):
    return ls.append_kv(g["x"], g["kv"][:, 0], g["kv"][:, 1], g["table"], g["cached"], g["cu"], g["nq"], g["f"], q_norm=g["qn"], k_norm=g["kn"],
                        pos_offset=g["off"], out=g["q"], **kw)


def reference(s, eps=1e-6):
    """q and cache in 64 bits and how far the call may be from them: half a step of the rounding, and 2^-20 of the pair's size for what is done in 32
    bits (at most 14 additions for a sum of squares, root, quotient, gain, sine and cosine to 2 ulp of an angle that is 2^-25 of a
    turn off, two products and a sum: under 16 of 2^-24); in fp16 half of its smallest step, too."""
    nq, nkv, d, page, rot = s["nq"], s["nkv"], s["d"], s["page"], s["rot"]
    x = s["x"].double().view(-1, nq + 2 * nkv, d)
    q, kv = s["q"].double().clone(), s["kv"].double().clone()
    tq, tkv = torch.zeros_like(q), torch.zeros_like(kv)
    half = torch.finfo(s["kv"].dtype).eps / 2
    tiny = 2.0 ** -25 if s["kv"].dtype == torch.float16 else 0.0

    def turned(y, gain, index):
        if gain is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double()
        size = y.abs()
        if rot:
            h = rot // 2
            angle = index * s["f"]
            c, n = torch.cos(angle), torch.sin(angle)
            a, b = y[..., :h], y[..., h:rot]
            both = (a.abs() + b.abs())
            y, size = torch.cat([a * c - b * n, b * c + a * n, y[..., rot:]], -1), torch.cat([both, both, y[..., rot:].abs()], -1)
        return y, half * y.abs() + 2.0 ** -20 * size + tiny

    row = 0
    for b, n in enumerate(s["counts"]):
        for j in range(n):
            pos = int(s["cached"][b]) + j
            index = float(pos + (int(s["off"][b]) if s["off"] is not None else 0))
            at = int(s["table"][b, pos // page]), pos % page
            q[row], tq[row] = turned(x[row, :nq], s["qn"], index)
            kv[at[0], 0, :, at[1]], tkv[at[0], 0, :, at[1]] = turned(x[row, nq:nq + nkv], s["kn"], index)
            v = x[row, nq + nkv:]
            kv[at[0], 1, :, at[1]], tkv[at[0], 1, :, at[1]] = v, half * v.abs() + tiny
            row += 1
    return q, kv, tq, tkv


def check(s, g):
    q, kv, tq, tkv = reference(s)
    assert ((g["q"].double().cpu() - q).abs() <= tq).all()
    assert ((g["kv"].double().cpu() - kv).abs() <= tkv).all()  # (untouched places to the bit: their tolerance is 0)


CASES = [
    # counts, cached, nq, nkv, d, page, in, cache, rot, norm, pad, offset
    ([1], [0], 1, 1, 8, 1, "fp32", "bf16", 8, False, 0, None),
    ([1], [512], 16, 16, 128, 64, "bf16", "bf16", 128, False, 0, None),
    ([1] * 33, list(range(33)), 8, 2, 64, 16, "fp32", "fp16", 64, True, 0, None),
    ([3, 0, 17, 1, 0, 5], [0, 9, 31, 64, 0, 2], 6, 6, 64, 16, "fp16", "fp16", 32, True, 4, [0, 5, 100, 7, 1, 3]),
    ([0, 0, 2], [3, 4, 5], 4, 1, 128, 8, "bf16", "bf16", 128, True, 0, None),
    ([40], [3], 4, 4, 80, 4, "bf16", "bf16", 80, True, 1, None),
    ([5, 2], [0, 1], 5, 1, 256, 2, "fp32", "bf16", 64, True, 3, None),
    ([7], [0], 3, 3, 24, 32, "fp16", "fp16", 0, True, 0, None),
    ([7], [1], 3, 2, 96, 32, "bf16", "bf16", 16, False, 0, None),
    ([2, 3], [0, 8], 0, 2, 64, 16, "fp32", "bf16", 64, True, 0, None),
    ([1, 2], [10, 0], 32, 8, 128, 16, "fp32", "bf16", 128, True, 0, [1000003, 2 ** 30]),
    ([2, 1] * 700, [0, 1] * 700, 2, 1, 16, 2, "fp32", "bf16", 16, False, 7, None),
    ([1100, 0, 1299], [5, 7, 0], 3, 2, 64, 32, "bf16", "bf16", 32, True, 3, None),  # a warp per row
    ([2050], [1], 2, 1, 40, 16, "fp32", "fp16", 40, False, 1, [3]),
    ([1000], [0], 0, 3, 8, 1, "bf16", "bf16", 8, True, 5, None),
    ([700, 0, 401], [3, 2, 9], 9, 3, 128, 16, "fp16", "fp16", 128, True, 2, [9, 0, 1000003]),
    ([1001], [2], 7, 1, 256, 64, "fp32", "bf16", 256, True, 0, None),
    ([1, 998, 1], [0, 5, 0], 17, 5, 96, 8, "fp32", "fp16", 0, True, 0, None),
    ([1000], [7], 1, 1, 64, 32, "bf16", "bf16", 24, False, 0, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_append_against_64_bits(case):
    counts, cached, nq, nkv, d, page, tin, tc, rot, norm, pad, offset = case
    s, g = make(counts, cached, nq, nkv, d, page, tin, tc, rot, norm, pad, offset)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert call(g, flag=flag) is g["q"]
    check(s, g)
    assert flag.item() == 0


@pytest.mark.gpu
def test_one_gain_strides_and_other_streams():
    """A norm of the keys alone, rows of qkv and q inside wider ones, [page][slot][head] order, a stream of its own, and a captured call replayed
    on new contents."""
    s, g = make([4, 2], [5, 0], 4, 2, 64, 16, "bf16", "bf16", 64, True)
    s["qn"] = g["qn"] = None
    T = 6
    wide = torch.full((T, g["x"].size(1) + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:-16] = g["x"]
    g["x"] = wide[:, 8:-16]
    outer = torch.zeros(T, 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    outer[:, :256] = g["q"].view(T, -1)
    g["q"] = outer[:, :256].view(T, 4, 64)
    pool = g["kv"].permute(0, 1, 3, 2, 4).contiguous()  # [page][k|v][slot][head][d]
    g["kv"] = pool.permute(0, 1, 3, 2, 4)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call(g)
    st.synchronize()
    check(s, g)
    assert (outer[:, 256:] == 0).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(g)
    x2 = torch.randn(T, s["x"].size(1)).to(torch.bfloat16)
    s["x"] = x2
    g["x"].copy_(x2)
    s["cached"][0] = 6
    g["cached"].copy_(s["cached"])
    s["kv"], s["q"] = g["kv"].cpu().clone(), g["q"].cpu().clone()
    graph.replay()
    torch.cuda.synchronize()
    check(s, g)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    s, g = make([2], [15], 1, 1, 64, 16, "fp32", "bf16", 64, False)
    s["table"][0, :2] = torch.tensor([2, 1], dtype=torch.int32)
    g["table"].copy_(s["table"])
    stride = (1 << 31) // 2 + 1024  # page 2 begins beyond 2^31 elements
    store = torch.zeros(2 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    g["kv"] = store.as_strided((3, 2, 1, 16, 64), (stride, 1024, 1024, 64, 1))
    s["kv"] = torch.zeros(3, 2, 1, 16, 64, dtype=torch.bfloat16)
    call(g)
    check(s, g)


@pytest.mark.gpu
def test_bad_entries_leave_a_flag_and_nothing_else():
    """Pages outside the cache, a position beyond the table, a negative length: those rows are not appended, the others are."""
    s, g = make([2, 1, 1, 3], [0, 4, 0, 0], 2, 1, 32, 4, "bf16", "bf16", 32, False)
    before = g["kv"].clone()
    table, cached = g["table"].clone(), g["cached"].clone()
    for b, page in ((0, -1), (0, g["kv"].size(0)), (0, 2 ** 31 - 1)):
        g["table"].copy_(table)
        g["table"][b, 0] = page
        g["kv"].copy_(before)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(g, flag=flag)
        assert flag.item() == 1
        keep = int(s["table"][0, 0])
        assert torch.equal(g["kv"][keep], before[keep])
        last = int(s["table"][3, 0])
        assert not torch.equal(g["kv"][last], before[last])
    g["table"].copy_(table)
    for value in (-5, 2 ** 31 - 1, 4 * g["table"].size(1)):
        g["cached"].copy_(cached)
        g["cached"][1] = value
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(g, flag=flag)
        assert flag.item() == 1
        call(g)  # (no flag asked for)


@pytest.mark.gpu
@pytest.mark.parametrize("gains", [(True, False), (False, True)])
def test_a_prompt_with_bad_pages_one_gain_and_numbers_that_are_none(gains):
    s, g = make([600, 500], [1, 4], 6, 2, 64, 16, "bf16", "bf16", 64, True, pad=3)
    for key, keep in zip(("qn", "kn"), gains):
        if not keep:
            s[key] = g[key] = None
    bad = (0, 3)  # positions 48 .. 63 of the first sequence: rows 47 .. 62
    s["table"] = s["table"].clone()
    g["table"][bad] = g["kv"].size(0)
    g["x"][700] = float("nan")
    g["x"][-3:] = float("inf")  # (padding)
    before = g["kv"].clone()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(g, flag=flag)
    assert flag.item() == 1
    lost = int(s["table"][bad])
    assert torch.equal(g["kv"][lost], before[lost])
    at = int(s["table"][1, 104 // 16]), 104 % 16  # row 700: position 104 of the second sequence
    assert g["q"][700].isnan().all() and g["kv"][at[0], :, :, at[1]].isnan().all()
    q, kv, tq, tkv = reference(s)
    dq, dkv = (g["q"].double().cpu() - q).abs() <= tq, (g["kv"].double().cpu() - kv).abs() <= tkv
    dq[700], dkv[lost], dkv[at[0], :, :, at[1]] = True, True, True
    assert dq.all() and dkv.all()


def counted(cu_rows, T, cached, far=0):
    """Inputs of T rows and four or so sequences under these counts, whatever they say; every sequence has pages for `cached` positions and T more."""
    B = len(cu_rows) - 1
    s, g = make([T] + [0] * (B - 1), [cached] * B, 2, 1, 32, 4, "bf16", "bf16", 32, True)
    s["table"], pages = pages_for([cached + T + far] * B, 4, np.random.default_rng(1))
    s["kv"] = torch.randn(pages, 2, 1, 4, 32).to(torch.bfloat16)
    s["cu"] = torch.tensor(cu_rows, dtype=torch.int32)
    for k in ("table", "kv", "cu"):
        g[k] = s[k].cuda()
    return s, g


def positions_written(s, g):
    """[(sequence, position)] of the slots that are not what they were."""
    moved = (g["kv"].cpu() != s["kv"]).any(4).any(2).any(1)  # [page][slot]
    where = {int(p): (b, i) for b, row in enumerate(s["table"]) for i, p in enumerate(row)}
    return sorted((where[int(p)][0], where[int(p)][1] * 4 + int(slot)) for p, slot in moved.nonzero())


@pytest.mark.gpu
@pytest.mark.parametrize("many", [1, 100])  # (rows of either kernel)
@pytest.mark.parametrize("cu_rows,T", [([0, 5, 3, 8], 12), ([0, 6, 10, 2, 12], 12), ([0, 5, 20], 12), ([-3, 4, 12], 12), ([12, 9, 6, 3, 0], 12), ([2, 2, 1], 12), ([0, 4, 2 ** 31 - 1], 12),
                                       ([0, -2 ** 31, 12], 12)])
def test_row_counts_that_do_not_ascend_leave_a_flag_and_what_is_cached(cu_rows, T, many):
    cached = 7 * many
    s, g = counted([min(max(c * many, -2 ** 31), 2 ** 31 - 1) for c in cu_rows], T * many, cached, far=4 * many)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(g, flag=flag)
    assert flag.item() & 2
    assert all(pos >= cached for _, pos in positions_written(s, g))
    g["kv"].copy_(s["kv"])
    call(g)  # (no flag asked for)
    assert all(pos >= cached for _, pos in positions_written(s, g))


@pytest.mark.gpu
@pytest.mark.parametrize("many", [1, 100])
def test_row_counts_beyond_the_rows_leave_a_flag_and_append_what_there_is(many):
    s, g = counted([0, 5 * many, 20 * many], 12 * many, 3)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(g, flag=flag)
    assert flag.item() == 2
    assert positions_written(s, g) == [(0, 3 + j) for j in range(5 * many)] + [(1, 3 + j) for j in range(7 * many)]


@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 127, 128, 3000])
def test_row_counts_are_looked_at_to_the_last(B):
    """Good counts of any number leave no flag; one bad count in any place does."""
    s, g = make([1] + [0] * (B - 1), [0] * B, 1, 1, 8, 4, "bf16", "bf16", 8, False)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(g, flag=flag)
    assert flag.item() == 0
    for at in sorted({0, 1, B // 2, B - 1, B}):
        for bad in (-1, 2):
            flag.zero_()
            g["cu"].copy_(s["cu"])
            g["cu"][at] = bad
            call(g, flag=flag)
            assert flag.item() & 2, (at, bad)


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("tin,tc", [("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp16")])
@pytest.mark.parametrize("nq,nkv,d,rot", [(6, 2, 128, 128), (4, 4, 64, 32), (3, 1, 96, 96), (2, 1, 8, 8)])
def test_a_row_is_the_same_in_calls_of_any_number_of_rows(nq, nkv, d, rot, tin, tc, norm):
    """The same tokens among 1300 rows and among 900: queries, keys and values to the bit."""
    s, g = make([1300], [3], nq, nkv, d, 16, tin, tc, rot, norm)
    many = call(g).clone(), g["kv"].clone()
    g["kv"].copy_(s["kv"])
    g["x"], g["q"], g["cu"] = g["x"][:900], g["q"][:900], torch.tensor([0, 900], dtype=torch.int32, device="cuda")
    q = call(g)
    assert torch.equal(q, many[0][:900])
    pages = s["table"][0, :903 // 16].long()
    assert torch.equal(g["kv"][pages], many[1][pages])


@pytest.mark.gpu
def test_not_a_number_stays_in_its_row():
    s, g = make([3, 2], [0, 6], 2, 2, 64, 16, "fp32", "bf16", 64, True, pad=2)
    g["x"][1] = float("nan")
    g["x"][-1] = float("inf")  # (padding)
    call(g)
    q, kv, tq, tkv = reference(s)
    rows = [0, 2, 3, 4, 5, 6]
    assert ((g["q"].double().cpu() - q).abs() <= tq)[rows].all()
    assert g["q"][1].isnan().all()
    page = int(s["table"][0, 0])
    assert g["kv"][page, :, :, 1].isnan().all()
    g["kv"][page, :, :, 1] = s["kv"][page, :, :, 1].cuda()
    kv[page, :, :, 1] = s["kv"][page, :, :, 1].double()
    assert ((g["kv"].double().cpu() - kv).abs() <= tkv).all()


@pytest.mark.gpu
def test_dimensions_of_one_element_have_any_stride():
    s, g = make([1], [5], 3, 1, 64, 1, "fp32", "bf16", 64, True)
    for name in ("x", "q", "kv"):
        x = g[name]
        g[name] = x.as_strided(x.shape, [3 if n == 1 else st for n, st in zip(x.shape, x.stride())])
    call(g)
    check(s, g)


@pytest.mark.gpu
def test_no_rows_and_padding_only():
    s, g = make([2], [0], 2, 1, 64, 16, "bf16", "bf16", 64, False)
    kv, q = g["kv"].clone(), g["q"].clone()
    g["cu"].zero_()
    call(g)
    assert torch.equal(kv, g["kv"]) and torch.equal(q, g["q"])
    g["x"], g["q"] = g["x"][:0], g["q"][:0]
    assert call(g).shape == (0, 2, 64)


def test_refusals():
    """EINVAL before anything is launched: the addresses here are never read."""
    from paper_2609_17184_b200.binding import PagedKv
    import ctypes as C
    A = 1 << 20

    def rc(kv=None, dtype=1, ld=256, T=2, nq=2, table=A, tld=4, width=4, cached=A, cu_=A, B=1, f=A, rot=64, q=A, qld=128, x=A):
        kv = PagedKv(*(kv or ok()))
        return ls.lib.loopspec_op_append_kv(x, dtype, ld, T, nq, C.byref(kv), table, tld, width, cached, cu_, B, None, f, rot, None, None, 1e-6, q, qld, None, None)

    def ok(**kw):
        d = dict(k=A, v=A, ps=2048, hs=1024, ss=64, n=4, page=16, nkv=1, d=64, t=1)
        d.update(kw)
        return list(d.values())

    for kw in (dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(ps=2044), dict(hs=4), dict(ss=-64), dict(page=0), dict(page=12),
               dict(page=1 << 17), dict(nkv=0), dict(d=0), dict(d=20), dict(d=264), dict(t=0), dict(t=3), dict(n=-1)):
        assert rc(kv=ok(**kw)) == -1, kw
    for kw in (dict(dtype=-1), dict(dtype=3), dict(ld=250), dict(ld=248), dict(T=-1), dict(nq=-1), dict(table=None), dict(tld=3), dict(width=-1), dict(cached=None),
               dict(cu_=None), dict(B=-1), dict(f=None), dict(rot=12), dict(rot=72), dict(rot=-8), dict(q=None), dict(q=A + 8), dict(qld=120), dict(qld=132),
               dict(x=None), dict(x=A + 8)):
        assert rc(**kw) == -1, kw
    for qn, kn in ((A + 4, None), (None, A + 8)):
        kv = PagedKv(*ok())
        assert ls.lib.loopspec_op_append_kv(A, 1, 256, 2, 2, C.byref(kv), A, 4, 4, A, A, 1, None, A, 64, qn, kn, 1e-6, A, 128, None, None) == -1
    assert ls.lib.loopspec_op_append_kv(A, 1, 256, 2, 2, None, A, 4, 4, A, A, 1, None, A, 64, None, None, 1e-6, A, 128, None, None) == -1
    assert rc(T=0) == 0 and rc(B=0) == 0  # nothing to do


def test_more_rows_than_can_be_counted_are_refused():
    """Rows are counted in 32 bits, four to a CTA: the last numbers would come round to negative rows."""
    from paper_2609_17184_b200.binding import PagedKv
    import ctypes as C
    A = 1 << 20
    kv = PagedKv(A, A, 2048, 1024, 64, 4, 16, 1, 64, 1)
    for T in (2 ** 31 - 1, 2 ** 31 - 3):
        assert ls.lib.loopspec_op_append_kv(A, 1, 256, T, 2, C.byref(kv), A, 4, 4, A, A, 1, None, A, 64, None, None, 1e-6, A, 128, None, None) == -1


def test_wrapper_refuses_what_is_not_a_device_tensor():
    s, g = make([1], [0], 2, 1, 64, 16, "bf16", "bf16", 64, False, dev="cpu")
    with pytest.raises(ls.LoopSpecError) as e:
        call(g)
    assert e.value.status == "EINVAL"


@pytest.mark.gpu
def test_wrapper_refusals():
    def fails(**kw):
        s, g = make([2, 1], [0, 3], 2, 1, 64, 16, "bf16", "bf16", 64, True)
        for k, f in kw.items():
            g[k] = f(g[k])
        with pytest.raises(ls.LoopSpecError) as e:
            call(g)
        assert e.value.status == "EINVAL"

    fails(x=lambda x: x.double())
    fails(x=lambda x: x[:, :-8])
    fails(x=lambda x: x[:1].expand(3, -1))
    fails(x=lambda x: x.t().contiguous().t())
    fails(kv=lambda x: x.float())
    fails(kv=lambda x: x[..., :60])
    fails(kv=lambda x: x.transpose(3, 4))
    fails(table=lambda x: x.long())
    fails(table=lambda x: x[:1].expand(2, -1))
    fails(cached=lambda x: x[:1])
    fails(cached=lambda x: x.cpu())
    fails(cu=lambda x: x[:-1])
    fails(f=lambda x: x.float())
    fails(f=lambda x: x[:-2])
    fails(qn=lambda x: x[:-1])
    fails(kn=lambda x: x.half())
    fails(q=lambda x: x[:-1])
    fails(q=lambda x: x.half())
    fails(nq=lambda x: 3)
