"""GPU: append into paged storage and attention over its pages, against the
formulas in 64 bits (tests/paged_ref.py).  Every slot that holds no token is
NaN, so a kernel that let one through would show it."""
import ctypes
import math

import pytest
import torch

import paper_2609_26425_gb300 as qwm
from paged_ref import attend64, inv_freq, make_case, offsets, rope64, rope_bound, visible

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    qwm.lib()


def build(lens, Hk, D, dtype, page, pages, table):
    cache = qwm.PagedCache(Hk, pages.shape[0], page_tokens=page, head_dim=D, dtype=dtype)
    cache.pages.copy_(pages)
    batch = qwm.PagedBatch(offsets(lens).cuda(), torch.tensor([kv for _, kv in lens], dtype=torch.int32).cuda(),
                           table.cuda(), max(a for a, _ in lens), max(kv for _, kv in lens))
    return cache, batch


def compare(got, lse, want):
    out, l64, ob, lb = want
    g = got.double().cpu()
    assert bool(torch.isfinite(g).all())
    err = (g - out).abs()
    assert bool((err <= ob).all()), float((err / ob.clamp(min=1e-300)).max())
    le = lse.double().cpu()
    empty = torch.isinf(l64)
    assert torch.equal(torch.isinf(le) & (le < 0), empty)
    assert bool(((le - l64).abs()[~empty] <= lb[~empty]).all())
    assert bool((g[empty.t()] == 0).all())


def run_case(seed, lens, Hq, Hk, D, dtype, page, block, window, sinks):
    q, keys, values, pages, table = make_case(seed, lens, Hq, Hk, D, dtype, page)
    # pages that no row sees are given back
    for b, (ql, kv) in enumerate(lens):
        see = torch.zeros(kv, dtype=torch.bool)
        for i in range(ql):
            see |= visible(kv - ql + i, kv, block, window, sinks)
        for i in range((kv + page - 1) // page):
            if not bool(see[i * page:(i + 1) * page].any()):
                table[b, i] = -1
    cache, batch = build(lens, Hk, D, dtype, page, pages, table)
    want = attend64(q, keys, values, lens, block, window, sinks)
    for split in (False, True):
        ws = qwm.paged_attend_workspace(cache, batch, Hq, window, sinks, block) if split else None
        if split and ws is None:
            continue
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True,
                                        workspace=ws)
        compare(out, lse, want)
        again, _ = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True,
                                        workspace=ws)
        assert torch.equal(out, again)          # the same bits, whichever part ends last
    assert cache.status() == 0


STEP = [
    # lens (new, held), Hq, Hk, D, dtype, page, block, window, sinks
    ([(1, 1)], 1, 1, 128, BF, 16, 1, 0, 0),
    ([(1, 0), (1, 1), (0, 5), (1, 64), (1, 65)], 4, 4, 128, BF, 16, 1, 0, 0),      # nothing held; no new token
    ([(1, 127), (1, 128), (1, 129), (1, 1000)], 8, 2, 64, HF, 32, 1, 0, 0),
    ([(1, 700), (1, 33)], 40, 8, 128, BF, 64, 1, 100, 4),
    ([(1, 1500), (1, 1499)], 5, 1, 128, HF, 128, 1, 513, 70),
    ([(4, 300), (3, 3), (2, 1), (1, 90)], 8, 2, 64, BF, 16, 1, 17, 3),              # drafts; rows before the start
    ([(5, 777)], 6, 1, 128, HF, 32, 4, 64, 20),                                     # 30 rows, blocks of 4
    ([(7, 1037)], 4, 1, 128, BF, 16, 1, 0, 0),
    ([(1, 2900)], 32, 1, 64, HF, 64, 1, 0, 0),                                      # 32 heads on one cache head
    ([(8, 40)], 3, 3, 128, BF, 16, 8, 0, 0),                                        # a whole block at once
    ([(1, 1200)], 2, 2, 128, BF, 16, 1, 1, 0),                                      # a window of the token itself
    ([(1, 1200)], 2, 2, 128, BF, 16, 1, 40, 1100),                                  # sinks reach the window
]


@pytest.mark.parametrize("case", range(len(STEP)))
def test_step(case):
    run_case(100 + case, *STEP[case])


CHUNK = [
    ([(33, 33)], 1, 1, 128, BF, 16, 1, 0, 0),
    ([(128, 128)], 1, 1, 128, HF, 64, 1, 0, 0),
    ([(129, 700), (1, 5), (0, 9), (40, 20)], 2, 2, 64, BF, 32, 1, 0, 0),            # ragged; rows before the start
    ([(257, 300)], 1, 1, 128, BF, 128, 1, 50, 7),
    ([(100, 1000)], 3, 1, 64, HF, 16, 1, 130, 200),                                 # 300 rows of three grouped heads
    ([(90, 360)], 2, 1, 128, BF, 16, 90, 0, 0),                                     # frames of 90
    ([(90, 810)], 4, 2, 128, HF, 32, 90, 270, 45),                                  # frames, window of 3, half a frame kept
    ([(50, 500)], 1, 1, 128, BF, 16, 1 << 20, 0, 0),                                # no mask
    ([(70, 70), (300, 301)], 2, 2, 64, HF, 64, 64, 128, 10),
    ([(60, 7)], 1, 1, 64, BF, 16, 1, 0, 0),
    ([(45, 0)], 1, 1, 128, BF, 16, 1, 0, 0),                                        # nothing held: every row empty
    ([(35, 2100)], 7, 7, 128, BF, 64, 1, 0, 0),                                     # long and few rows: split
]


@pytest.mark.parametrize("case", range(len(CHUNK)))
def test_chunk(case):
    run_case(200 + case, *CHUNK[case])


@pytest.mark.parametrize("new,heads", [(4, 2), (60, 2)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype,D,page", [(BF, 128, 16), (HF, 64, 64)])
def test_nonfinite_tokens_reach_the_rows_that_see_them_only(new, heads, what, dtype, D, page):
    lens = [(new, 300)]
    q, keys, values, pages, table = make_case(7, lens, heads, 1, D, dtype, page)
    window, sinks = 200, 5
    odd_k, odd_v = 298, 300 - new + 1              # the last but one token's Key, the second new token's Value
    early = 300 - new - window + 2                 # a Value that the first rows see and later ones do not
    table_of = lambda j: (int(table[0, j // page]), j % page)
    pk, pv, pe = table_of(odd_k), table_of(odd_v), table_of(early)
    pages[pk[0], 0, 0, pk[1], 3] = math.nan
    pages[pv[0], 1, 0, pv[1], 9] = what
    pages[pe[0], 1, 0, pe[1], 11] = what
    cache, batch = build(lens, 1, D, dtype, page, pages, table)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, heads, window, sinks, 1)):
        out = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, workspace=ws).cpu()
        for i in range(new):
            p = 300 - new + i
            fine = torch.isfinite(out[i])
            if p >= odd_k:
                assert not bool(fine.any())
                continue
            want = torch.ones(heads, D, dtype=torch.bool)
            if p >= odd_v:
                want[:, 9] = False
            if early >= p + 1 - window:
                want[:, 11] = False
            assert torch.equal(fine, want), (i, p)
    k2, v2 = [keys[0].clone()], [values[0].clone()]
    ref = attend64(q, k2, v2, lens, 1, window, sinks)
    first = out[0].double()                        # the first row sees the early Value only
    ok = torch.arange(D) != 11
    assert bool(((first - ref[0][0]).abs() <= ref[2][0])[:, ok].all())


def test_strided_and_head_major_tensors():
    lens, Hq, Hk, D = [(40, 90), (9, 200)], 4, 2, 128
    q, keys, values, pages, table = make_case(11, lens, Hq, Hk, D, BF, 16)
    cache, batch = build(lens, Hk, D, BF, 16, pages, table)
    N = q.shape[0]
    ref = qwm.qwm_paged_attend(cache, batch, q.cuda())
    wide = torch.zeros(N, Hq + 3, D + 8, dtype=BF, device="cuda")
    wide[:, 1:1 + Hq, :D] = q.cuda()
    out = torch.full((Hq, N, D), 7.0, dtype=BF, device="cuda")
    got = qwm.qwm_paged_attend(cache, batch, wide[:, 1:1 + Hq, :D], out=out.permute(1, 0, 2))
    assert torch.equal(got, ref)
    small = qwm.PagedBatch(offsets([(2, 90), (1, 200)]).cuda(), torch.tensor([90, 200], dtype=torch.int32).cuda(),
                           table.cuda(), 2, 200)
    q3 = wide[:3, 1:1 + Hq, :D]
    a = qwm.qwm_paged_attend(cache, small, q3.contiguous())
    b = qwm.qwm_paged_attend(cache, small, q3, out=out.permute(1, 0, 2)[:3])
    assert torch.equal(a, b)


@pytest.mark.parametrize("rope_on,il,dtype,D,page,Hq,Hk", [
    (True, True, BF, 128, 16, 5, 5), (True, False, HF, 64, 64, 8, 2), (False, True, BF, 64, 128, 3, 1),
    (True, True, HF, 128, 32, 12, 4)])
def test_append_stores_each_token_once_and_nothing_else(rope_on, il, dtype, D, page, Hq, Hk):
    lens = [(1, 1), (37, 100), (0, 12), (130, 130), (5, 3), (1, 65)]
    g = torch.Generator().manual_seed(D + page)
    N = sum(a for a, _ in lens)
    qkv = torch.randn(N, Hq + 2 * Hk, D, generator=g).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    pos = torch.randint(0, 300, (N, 3), generator=g, dtype=torch.int32)
    pairs = (D // 2 - 2 * (D // 6), D // 6, D // 6)
    freq = inv_freq(pairs)
    _, _, _, pages, table = make_case(3, lens, 1, Hk, D, dtype, page)
    marks = torch.randn(pages.shape, generator=g).to(dtype)
    cache, batch = build(lens, Hk, D, dtype, page, marks, table)
    rope = qwm.Rope(freq.cuda(), pairs, interleaved=il) if rope_on else None
    dev = qkv.cuda()
    q_rot = qwm.qwm_paged_append(cache, batch, dev[:, Hq:Hq + Hk], dev[:, Hq + Hk:], rope=rope,
                                 pos=pos.cuda() if rope_on else None, q=dev[:, :Hq])
    k64 = rope64(k, pos, freq, pairs, il) if rope_on else k.double()
    kb = rope_bound(k, k64, dtype, pairs, il) if rope_on else torch.zeros_like(k64)
    q64 = rope64(q, pos, freq, pairs, il) if rope_on else q.double()
    qb = rope_bound(q, q64, dtype, pairs, il) if rope_on else torch.zeros_like(q64)
    assert bool(((q_rot.double().cpu() - q64).abs() <= qb).all())
    got, want, bound = cache.pages.double().cpu(), marks.double().clone(), torch.zeros(marks.shape, dtype=torch.float64)
    row = 0
    for b, (ql, kv) in enumerate(lens):
        for i in range(ql):
            p = kv - ql + i
            if p >= 0:
                at = int(table[b, p // page]), p % page
                want[at[0], 0, :, at[1]], bound[at[0], 0, :, at[1]] = k64[row], kb[row]
                want[at[0], 1, :, at[1]] = v[row].double()
            row += 1
    assert bool(((got - want).abs() <= bound).all())
    assert cache.status() == 0
    # without Queries, the same pages
    cache.pages.copy_(marks)
    assert qwm.qwm_paged_append(cache, batch, dev[:, Hq:Hq + Hk], dev[:, Hq + Hk:], rope=rope,
                                pos=pos.cuda() if rope_on else None) is None
    assert torch.equal(cache.pages.double().cpu(), got)


def test_offsets_beyond_32_bits():
    Hk, page, D = 8, 128, 128
    num = (1 << 31) // (2 * Hk * page * D) + 9              # the last pages start past 2^31 elements
    cache = qwm.PagedCache(Hk, num, page_tokens=page, head_dim=D)
    lens = [(40, 300), (1, 129)]
    ids = [num - 1, 0, num - 4, num - 2, num - 3]
    table = torch.tensor([ids[:3], [ids[3], ids[4], -1]], dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    total = [(kv, kv) for _, kv in lens]
    k = torch.randn(429, Hk, D, generator=g).to(BF)
    v = torch.randn(429, Hk, D, generator=g).to(BF)
    load = qwm.PagedBatch(offsets(total).cuda(), torch.tensor([300, 129], dtype=torch.int32).cuda(), table.cuda(), 300, 300)
    qwm.qwm_paged_append(cache, load, k.cuda(), v.cuda())
    q = torch.randn(41, Hk, D, generator=g).to(BF)
    batch = qwm.PagedBatch(offsets(lens).cuda(), torch.tensor([300, 129], dtype=torch.int32).cuda(), table.cuda(), 40, 300)
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True)
    compare(out, lse, attend64(q, [k[:300], k[300:]], [v[:300], v[300:]], lens, 1, 0, 0))
    one = qwm.PagedBatch(offsets([(1, 300), (1, 129)]).cuda(), torch.tensor([300, 129], dtype=torch.int32).cuda(),
                         table.cuda(), 1, 300)
    out, lse = qwm.qwm_paged_attend(cache, one, q[:2].cuda(), want_lse=True)
    compare(out, lse, attend64(q[:2], [k[:300], k[300:]], [v[:300], v[300:]], [(1, 300), (1, 129)], 1, 0, 0))
    assert cache.status() == 0


def test_another_stream_and_a_captured_graph():
    lens, Hq, Hk, D, page = [(1, 500), (1, 30)], 8, 2, 128, 16
    q, keys, values, pages, table = make_case(21, lens, Hq, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, Hq)
    dq, ref = q.cuda(), qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late = dq.clone()
        got = qwm.qwm_paged_attend(cache, batch, late, workspace=ws)
    side.synchronize()
    assert torch.equal(got, ref)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(dq)
    with torch.cuda.graph(graph):
        qwm.qwm_paged_attend(cache, batch, dq, out=out, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    batch.tensors[1].copy_(torch.tensor([437, 29], dtype=torch.int32))      # shorter sequences, the same graph
    graph.replay()
    torch.cuda.synchronize()
    short = [(1, 437), (1, 29)]
    want = attend64(q, [keys[0][:437], keys[1][:29]], [values[0][:437], values[1][:29]], short, 1, 0, 0)
    assert bool(((out.double().cpu() - want[0]).abs() <= want[2]).all())


def test_entries_out_of_range_are_recorded_and_not_followed():
    lens, Hk, D, page = [(1, 100), (40, 100)], 2, 128, 16
    q, keys, values, pages, table = make_case(31, lens, 2, Hk, D, BF, page)
    k = torch.zeros(41, Hk, D, dtype=BF, device="cuda")
    for bad in (pages.shape[0], -7, 1 << 30):
        broken = table.clone()
        broken[1, 6] = bad
        cache, batch = build(lens, Hk, D, BF, page, pages, broken)
        out = qwm.qwm_paged_attend(cache, batch, q.cuda())
        assert cache.status() == 1 and cache.status() == 0
        good = attend64(q[:1], keys[:1], values[:1], lens[:1], 1, 0, 0)     # the other sequence is as it should be
        assert bool(((out[:1].double().cpu() - good[0]).abs() <= good[2]).all())
        qwm.qwm_paged_append(cache, batch, k, k)
        assert cache.status() == 1
    cache, _ = build(lens, Hk, D, BF, page, pages, table)
    for off, kvl, mq, mkv in (([0, 1, 42], [100, 100], 41, 100), ([0, 50, 41], [100, 100], 50, 100),
                              ([0, 1, 41], [100, 101], 40, 100), ([0, 1, 41], [100, -1], 40, 100),
                              ([0, 1, 41], [100, 1 << 20], 40, 1 << 21), ([0, 1, 41], [100, 100], 39, 100)):
        batch = qwm.PagedBatch(torch.tensor(off, dtype=torch.int32).cuda(), torch.tensor(kvl, dtype=torch.int32).cuda(),
                               table.cuda(), mq, mkv)
        qwm.qwm_paged_attend(cache, batch, q.cuda())
        assert cache.status() == 1, (off, kvl)
        qwm.qwm_paged_append(cache, batch, k, k)
        assert cache.status() == 1, (off, kvl)


def test_refusals():
    lens, Hk, D, page = [(3, 40)], 2, 128, 16
    q, _, _, pages, table = make_case(41, lens, 4, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    dq = q.cuda()

    def status(fn):
        with pytest.raises(qwm.QwmError) as e:
            fn()
        return e.value.status

    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq[:, :3])) == 1                    # heads not grouped
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, block=0)) == 1
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, window=-1)) == 1
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, window=7, block=8)) == 1        # less than a block
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, sinks=-1)) == 1
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, sm_scale=0.0)) == 1
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, sm_scale=math.nan)) == 1
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, dq, out=dq[:1].expand(3, 4, D).clone()[:1].expand(3, 4, D))) == 1
    assert status(lambda: qwm.PagedCache(2, 4, page_tokens=24)) == 2
    assert status(lambda: qwm.PagedCache(2, 4, head_dim=96)) == 2
    assert status(lambda: qwm.PagedCache(0, 4)) == 2
    for bad in (dq.half(), dq[..., :64], dq.cpu(), dq[0]):
        with pytest.raises(ValueError):
            qwm.qwm_paged_attend(cache, batch, bad)
    k = torch.zeros(3, Hk, D, dtype=BF, device="cuda")
    rope = qwm.Rope(inv_freq((22, 21, 21)).cuda(), (22, 21, 21))
    with pytest.raises(ValueError):
        qwm.qwm_paged_append(cache, batch, k, k, rope=rope)                                      # no positions
    with pytest.raises(ValueError):
        qwm.qwm_paged_append(cache, batch, k, k[:2])
    assert status(lambda: qwm.qwm_paged_append(cache, batch, k[:, :1], k)) == 1
    with pytest.raises(ValueError):
        qwm.PagedBatch(batch.tensors[0].long(), batch.tensors[1], batch.tensors[2], 3, 40)
    none = torch.empty(0, 4, D, dtype=BF, device="cuda")
    assert qwm.qwm_paged_attend(cache, batch, none).shape == none.shape                          # no rows: nothing to do
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 60])
def test_a_wait_that_runs_out_is_recorded_and_the_next_call_is_exact(new):
    lens, Hk, D, page = [(new, 900)], 2, 128, 16
    q, keys, values, pages, table = make_case(51, lens, 2, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, 2)
    cache.set_wait_limit(1_000_000)                # 1 ms
    cache.set_idle_role(qwm.QWM_ROLE_PAGE_LOADS)
    qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws)
    torch.cuda.synchronize()
    assert cache.status() == 5
    cache.set_idle_role(0)
    cache.set_wait_limit(2_000_000_000)
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    compare(out, lse, attend64(q, keys, values, lens, 1, 0, 0))
    assert cache.status() == 0


@pytest.mark.parametrize("D,dtype,Hq,Hk,new", [(128, BF, 20, 4, 1), (64, HF, 24, 8, 1), (128, HF, 18, 9, 9)])
def test_step_over_many_sequences(D, dtype, Hq, Hk, new):
    """More groups than CTAs, of lengths from none to several ring turns."""
    g = torch.Generator().manual_seed(D + Hq)
    lens = []
    for i in range(61):
        q = int(torch.randint(0 if i % 7 == 3 else 1, new + 1, (1,), generator=g))
        lens.append((q, max(q, int(torch.randint(0, [5, 70, 700, 1800][i % 4], (1,), generator=g)))))
    run_case(300 + D, lens, Hq, Hk, D, dtype, 16, 1, 600, 9)


@pytest.mark.parametrize("new", [3, 150])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("order", ["rising", "falling", "peak late", "waves"])
def test_running_maxima_that_move(new, dtype, D, order):
    """Logits along one direction whose maximum moves by far more than a tile's
    probabilities span, up, down and in the middle of a tile, for some rows only."""
    kv, page = 700, 16
    lens = [(new, kv)]
    q, keys, values, pages, table = make_case(61, lens, 2, 1, D, dtype, page)
    j = torch.arange(kv, dtype=torch.float32)
    a = {"rising": j / 4, "falling": (kv - j) / 4, "peak late": 100 * ((j % 256) == 200) + 80 * (j == 610) + 0 * j,
         "waves": 60 * torch.sin(j / 37) + j / 20}[order]
    keys[0] = 0.05 * keys[0].float()
    keys[0][:, 0, 5] = a                                       # the direction is one channel
    keys[0] = keys[0].to(dtype)
    q = 0.2 * q.float()
    q[:, 0, 5] = torch.linspace(-1, 1, q.shape[0])             # some rows climb, some descend
    q[:, 1, 5] = 1.0
    q = q.to(dtype)
    for i in range((kv + page - 1) // page):
        n = min(page, kv - i * page)
        pages[int(table[0, i]), 0, :, :n] = keys[0][i * page:i * page + n].permute(1, 0, 2)
    cache, batch = build(lens, 1, D, dtype, page, pages, table)
    want = attend64(q, keys, values, lens, 1, 0, 0, scale=1.0)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, 2)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=1.0, want_lse=True, workspace=ws)
        compare(out, lse, want)


def test_more_sequences_than_threads():
    g = torch.Generator().manual_seed(77)
    lens = []
    for i in range(700):
        q = int(torch.randint(0, 2, (1,), generator=g))
        lens.append((q, max(q, int(torch.randint(0, 40, (1,), generator=g)))))
    run_case(401, lens, 2, 2, 64, BF, 16, 1, 20, 3)
    N = sum(a for a, _ in lens)
    k = torch.randn(N, 2, 64, generator=g).to(BF)
    _, _, _, pages, table = make_case(402, lens, 1, 2, 64, BF, 16)
    marks = torch.randn(pages.shape, generator=g).to(BF)
    cache, batch = build(lens, 2, 64, BF, 16, marks, table)
    qwm.qwm_paged_append(cache, batch, k.cuda(), (2 * k).cuda())
    want, row = marks.clone(), 0
    for b, (ql, kv) in enumerate(lens):
        for i in range(ql):
            p = kv - ql + i
            want[int(table[b, p // 16]), 0, :, p % 16] = k[row]
            want[int(table[b, p // 16]), 1, :, p % 16] = 2 * k[row]
            row += 1
    assert torch.equal(cache.pages.cpu(), want) and cache.status() == 0


def test_calls_of_any_sizes_take_turns_on_one_workspace():
    shapes = [([(1, 2000)], 40, 8, 128, BF), ([(1, 700)] * 37, 8, 8, 128, BF), ([(60, 1500)], 4, 2, 128, BF),
              ([(1, 900)] * 200, 12, 12, 128, BF), ([(300, 2500)], 1, 1, 128, BF), ([(1, 5000)] * 3, 8, 8, 128, BF),
              ([(2, 3000)] * 40, 8, 4, 64, HF)]
    made = []
    for i, (lens, Hq, Hk, D, dtype) in enumerate(shapes):
        q, keys, values, pages, table = make_case(500 + i, lens, Hq, Hk, D, dtype, 32)
        cache, batch = build(lens, Hk, D, dtype, 32, pages, table)
        made.append((cache, batch, q.cuda(), qwm.paged_attend_workspace(cache, batch, Hq)))
    sizes = [m[3].numel() for m in made if m[3] is not None]
    assert len(sizes) >= 4                          # (calls that are not split need none)
    shared = torch.zeros(max(sizes), dtype=torch.uint8, device="cuda")
    want = [qwm.qwm_paged_attend(c, b, q, workspace=own).clone() for c, b, q, own in made]
    for _ in range(2):
        for (c, b, q, _), w in list(zip(made, want)) + list(zip(made, want))[::-1]:
            assert torch.equal(qwm.qwm_paged_attend(c, b, q, workspace=shared), w)
    assert bool((shared[:65536] == 0).all())


@pytest.mark.parametrize("new,held", [(1, 90), (1, 900), (4, 6000), (60, 100), (60, 900), (300, 5000)])
@pytest.mark.parametrize("split", [False, True])
def test_a_limit_near_a_copys_latency_leaves_nothing_in_flight(new, held, split):
    """With the shortest limit some waits run out while their copies and MMAs are on
    the way.  A CTA lets them land before it ends (its last tiles' too, which no
    later wait of its own asks for), so the calls after it are exact."""
    lens, Hk, D, page = [(new, held)], 2, 128, 16
    q, keys, values, pages, table = make_case(71, lens, 4, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, 4) if split else None
    dq = q.cuda()
    want = qwm.qwm_paged_attend(cache, batch, dq, workspace=ws).clone()
    cold = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for _ in range(12):
        cold.zero_()                               # the pages leave the L2 cache
        cache.set_wait_limit(1000)
        qwm.qwm_paged_attend(cache, batch, dq, workspace=ws)
        cache.set_wait_limit(2_000_000_000)
        got = qwm.qwm_paged_attend(cache, batch, dq, workspace=ws)
        assert cache.status() in (0, 5)
        assert torch.equal(got, want)
    assert cache.status() == 0


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("b", [0, 1, 2])
@pytest.mark.parametrize("fault", ["offset", "long", "negative", "page"])
def test_step_calls_record_entries_out_of_range_of_every_sequence(fault, b, split):
    lens, Hk, D, page = [(1, 3000), (2, 3000), (1, 3000)], 2, 128, 16
    q, keys, values, pages, table = make_case(81, lens, 2, Hk, D, BF, page)
    off, held = offsets(lens), torch.tensor([kv for _, kv in lens], dtype=torch.int32)
    sound = {0, 1, 2} - {b}
    if fault == "offset":                          # b's end past its bound, or before its start
        off[b + 1 if b < 2 else b] += 9 if b < 2 else -9
        sound = {0, 1, 2} - ({b, b + 1} if b < 2 else {1, 2})
    elif fault == "page":
        table[b, 150] = pages.shape[0]
    else:
        held[b] = 3001 if fault == "long" else -1
    cache, _ = build(lens, Hk, D, BF, page, pages, table)
    batch = qwm.PagedBatch(off.cuda(), held.cuda(), table.cuda(), 2, 3000)
    ws = qwm.paged_attend_workspace(cache, batch, 2) if split else None
    assert (ws is not None) == split
    out = qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws).double().cpu()
    assert cache.status() == 1 and cache.status() == 0
    want = attend64(q, keys, values, lens, 1, 0, 0)
    for i in sound:                                # the others are as they should be
        r = slice(int(offsets(lens)[i]), int(offsets(lens)[i + 1]))
        assert bool(((out[r] - want[0][r]).abs() <= want[2][r]).all())


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("off", [(0, 1, -1), (1, 1, 0), (0, 0, None)])
@pytest.mark.parametrize("split", [False, True])
def test_rows_of_no_sequence_are_recorded(new, off, split):
    lens, Hk, D, page = [(new, 3000), (new, 3000)], 2, 128, 16
    q, _, _, pages, table = make_case(82, lens, 2, Hk, D, BF, page)
    cache, sound = build(lens, Hk, D, BF, page, pages, table)
    offs = [off[0], off[1] * new, 0 if off[2] is None else 2 * new + off[2]]
    batch = qwm.PagedBatch(torch.tensor(offs, dtype=torch.int32).cuda(), sound.tensors[1], sound.tensors[2], new, 3000)
    ws = qwm.paged_attend_workspace(cache, batch, 2) if split else None
    k = torch.zeros(2 * new, Hk, D, dtype=BF, device="cuda")
    qwm.qwm_paged_attend(cache, sound, q.cuda(), workspace=ws)
    assert cache.status() == 0
    qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws)
    assert cache.status() == 1 and cache.status() == 0
    qwm.qwm_paged_append(cache, batch, k, k)
    assert cache.status() == 1


@pytest.mark.parametrize("new,held", [(1, 40), (1, 3000), (3, 3000), (60, 3000)])
@pytest.mark.parametrize("split", [False, True])
def test_a_nan_logit_is_nan_in_the_lse(new, held, split):
    """Also where every logit of a row is NaN, so that it has no running maximum: its
    lse is not the -inf of a row that sees nothing."""
    lens, Hk, D, page = [(new, held)], 2, 128, 16
    q, keys, values, pages, table = make_case(83, lens, 4, Hk, D, BF, page)
    q[0, 1, 5] = math.nan                          # one row: all of its logits
    j = held - 1                                   # the last token's Key of head 1: the last rows' last logit
    pages[int(table[0, j // page]), 0, 1, j % page, 3] = math.nan
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, 4) if split else None
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    want = torch.zeros(new, 4, dtype=torch.bool)
    want[0, 1] = True
    want[-1, 2:] = True
    assert torch.equal(out.isnan().cpu(), want[..., None].expand(new, 4, D))
    assert torch.equal(lse.isnan().cpu(), want.t())
    assert bool(torch.isfinite(lse.cpu()[~want.t()]).all()) and cache.status() == 0


@pytest.mark.parametrize("new", [3, 150])
def test_large_values_under_a_rising_maximum(new):
    """Logits that rise by 2^38 over the keys, and Values of 2^100: a sum kept against
    a maximum that was left behind may not leave fp32's range."""
    kv, D, page = 700, 128, 16
    lens = [(new, kv)]
    q, keys, values, pages, table = make_case(84, lens, 2, 1, D, BF, page)
    keys[0] = 0.05 * keys[0].float()
    keys[0][:, 0, 5] = torch.arange(kv, dtype=torch.float32) / 17
    keys[0] = keys[0].to(BF)
    q = 0.2 * q.float()
    q[:, :, 5] = 1.0
    q = q.to(BF)
    values[0] = (values[0].float() * 2.0 ** 100).to(BF)
    for i in range((kv + page - 1) // page):
        n = min(page, kv - i * page)
        pages[int(table[0, i]), 0, :, :n] = keys[0][i * page:i * page + n].permute(1, 0, 2)
        pages[int(table[0, i]), 1, :, :n] = values[0][i * page:i * page + n].permute(1, 0, 2)
    cache, batch = build(lens, 1, D, BF, page, pages, table)
    want = attend64(q, keys, values, lens, 1, 0, 0, scale=1.0)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, 2)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=1.0, want_lse=True, workspace=ws)
        compare(out, lse, want)


@pytest.mark.parametrize("new,held", [(3, 40), (2, 3000), (70, 3000)])
def test_an_output_over_the_queries_is_refused_and_one_beside_them_is_not(new, held):
    lens, Hk, D, page = [(new, held)], 2, 128, 16
    q, keys, values, pages, table = make_case(91, lens, 4, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, 4)
    wide = torch.zeros(new, 12, D, dtype=BF, device="cuda")
    wide[:, :4] = q.cuda()
    for out in (wide[:, :4], wide[:, 1:5]):
        with pytest.raises(qwm.QwmError) as e:
            qwm.qwm_paged_attend(cache, batch, wide[:, :4], out=out, workspace=ws)
        assert e.value.status == 1
    want = qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws)
    for lo in (4, 8):                              # other heads of the same projection
        got = qwm.qwm_paged_attend(cache, batch, wide[:, :4], out=wide[:, lo:lo + 4], workspace=ws)
        assert torch.equal(got, want)
    assert torch.equal(wide[:, :4].cpu(), q) and cache.status() == 0


def test_a_bound_whose_row_tiles_pass_32_bits_is_refused():
    """1024 grouped heads under a bound of 2^30 + 1 tokens are 2^32 + 4 row tiles; cut to
    32 bits they would leave the second token's rows unwritten."""
    lens, D, page = [(2, 40)], 128, 16
    q, keys, values, pages, table = make_case(92, lens, 1024, 1, D, BF, page)
    cache, batch = build(lens, 1, D, BF, page, pages, table)
    with pytest.raises(qwm.QwmError) as e:
        qwm.qwm_paged_attend(cache, qwm.PagedBatch(*batch.tensors, (1 << 30) + 1, 40), q.cuda())
    assert e.value.status == 2
    loose = qwm.PagedBatch(*batch.tensors, 5000, 1 << 20)             # a loose bound is no matter
    assert torch.equal(qwm.qwm_paged_attend(cache, loose, q.cuda()), qwm.qwm_paged_attend(cache, batch, q.cuda()))
    assert cache.status() == 0


def test_parts_of_a_call_on_another_device_are_refused():
    lens, Hk, D, page = [(3, 40)], 2, 128, 16
    q, _, _, pages, table = make_case(93, lens, 4, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    rope = qwm.Rope(inv_freq((22, 21, 21)).cuda(), (22, 21, 21))
    pos, dq, k = torch.zeros(3, 3, dtype=torch.int32).cuda(), q.cuda(), torch.zeros(3, Hk, D, dtype=BF, device="cuda")
    for part in (cache, batch, rope):
        sound = part._key
        assert sound[-1] == dq.get_device()
        part._key = (*sound[:-1], 1)               # as on a second GPU
        calls = [] if part is rope else [lambda: qwm.qwm_paged_attend(cache, batch, dq)]
        calls += [lambda: qwm.qwm_paged_append(cache, batch, k, k, rope=rope, pos=pos, q=dq)]
        calls += [lambda: qwm.qwm_rope(rope, dq, pos)] if part is rope else []
        for call in calls:
            with pytest.raises(ValueError, match="on another device"):
                call()
        part._key = sound
        for call in calls:
            call()
    assert cache.status() == 0


@pytest.mark.parametrize("new,held", [(1, 40), (1, 3000), (4, 3000), (60, 3000)])
@pytest.mark.parametrize("split", [False, True])
def test_a_row_whose_logits_are_all_minus_infinity_is_an_empty_one(new, held, split):
    lens, Hk, D, page = [(new, held)], 1, 128, 16
    q, keys, values, pages, table = make_case(94, lens, 2, Hk, D, BF, page)
    for b in range(pages.shape[0]):
        pages[b, 0, 0, :, 3] = -math.inf           # every Key's, of every page
    q[:, 0, 3] = 0.5                               # head 0's logits are -inf,
    q[:, 1, 3] = -0.5                              # head 1's are inf
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    ws = qwm.paged_attend_workspace(cache, batch, 2) if split else None
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    assert bool((out[:, 0] == 0).all()) and bool((lse[0] == -math.inf).all())
    assert bool(out[:, 1].isnan().all()) and bool(lse[1].isnan().all()) and cache.status() == 0


def test_an_error_is_reported_by_the_call_that_met_it_only():
    """Reading the status on a stream that is being captured fails; the calls after it do
    not."""
    lens, Hk, D, page = [(1, 40)], 2, 128, 16
    q, _, _, pages, table = make_case(95, lens, 4, Hk, D, BF, page)
    cache, batch = build(lens, Hk, D, BF, page, pages, table)
    dq, k = q.cuda(), torch.zeros(1, Hk, D, dtype=BF, device="cuda")
    want = qwm.qwm_paged_attend(cache, batch, dq)
    torch.cuda.synchronize()
    runtime = ctypes.CDLL("libcudart.so.%d" % int(torch.version.cuda.split(".")[0]))   # loaded by PyTorch
    side, graph = torch.cuda.Stream(), ctypes.c_void_p()
    for call in (lambda: torch.equal(qwm.qwm_paged_attend(cache, batch, dq), want),
                 lambda: qwm.qwm_paged_append(cache, batch, k, k) is None):
        assert runtime.cudaStreamBeginCapture(ctypes.c_void_p(side.cuda_stream), 2) == 0
        with torch.cuda.stream(side), pytest.raises(qwm.QwmError) as e:
            cache.status()
        assert e.value.status == 4
        assert runtime.cudaStreamEndCapture(ctypes.c_void_p(side.cuda_stream), ctypes.byref(graph)) != 0
        runtime.cudaGetLastError()
        assert call()
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("split", [False, True])
def test_rows_of_no_sequence_leave_the_others_as_they_are(new, split):
    """A tensor with rows before the first sequence and after the last."""
    lens, Hk, D, page = [(new, 3000), (new, 2000)], 2, 128, 16
    q, keys, values, pages, table = make_case(96, lens, 2, Hk, D, BF, page)
    cache, sound = build(lens, Hk, D, BF, page, pages, table)
    pad = torch.ones(5, 2, D, dtype=BF)
    wide = torch.cat([pad[:3], q, pad]).cuda()
    batch = qwm.PagedBatch(sound.tensors[0] + 3, sound.tensors[1], sound.tensors[2], new, 3000)
    ws = qwm.paged_attend_workspace(cache, batch, 2) if split else None
    out, lse = qwm.qwm_paged_attend(cache, batch, wide, want_lse=True, workspace=ws)
    assert cache.status() == 1
    compare(out[3:-5], lse[:, 3:-5], attend64(q, keys, values, lens, 1, 0, 0))
