"""GPU: paged storage in 8 bits -- quantised append, read-back and attention over the
codes -- against the definitions in 64 bits (tests/codes_ref.py).  Every slot that holds
no token is NaN, so a kernel that let one through would show it."""
import math

import pytest
import torch

import paper_2609_26425_gb300 as qwm
from codes_ref import MOST, attend_codes64, make_code_case, quantise64, scale64, stands_for
from paged_ref import inv_freq, make_case, offsets, rope64, rope_bound, visible
from test_gpu_paged import CHUNK, STEP, compare

pytestmark = pytest.mark.gpu
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    qwm.lib()


def made(Hk, num, page, D, dtype, codes=None, scales=None):
    cache = qwm.PagedCache(Hk, num, page_tokens=page, head_dim=D, dtype=dtype, storage=E4)
    if codes is not None:
        cache.pages.view(torch.uint8).copy_(codes)
        cache.scales.copy_(scales)
    return cache


def batch_of(lens, table, **more):
    return qwm.PagedBatch(offsets(lens).cuda(), torch.tensor([kv for _, kv in lens], dtype=torch.int32).cuda(),
                          table.cuda(), max(a for a, _ in lens), max(kv for _, kv in lens), **more)


def held(cache):
    """What the pages stand for, in 64 bits."""
    return stands_for(cache.pages.view(torch.uint8).cpu(), cache.scales.cpu())


# ------------------------------------------------------------------ append and read-back
def tokens_of(lens, page, table):
    """(row, page id, slot) of every new token that is stored."""
    row = 0
    for b, (ql, kv) in enumerate(lens):
        for i in range(ql):
            p = kv - ql + i
            if p >= 0:
                yield row, int(table[b, p // page]), p % page
            row += 1


@pytest.mark.parametrize("rope_on,il,dtype,D,page,Hq,Hk,part", [
    (True, True, BF, 128, 16, 5, 5, 64), (True, False, HF, 64, 64, 8, 2, 24), (False, True, BF, 64, 128, 3, 1, 0),
    (True, True, HF, 128, 32, 12, 4, 36), (True, False, BF, 128, 128, 1, 3, 64), (True, False, BF, 128, 16, 2, 2, 8),
    (True, True, BF, 64, 16, 7, 7, 4)])
def test_append_quantises_each_token_once_and_nothing_else(rope_on, il, dtype, D, page, Hq, Hk, part):
    lens = [(1, 1), (37, 100), (0, 12), (130, 130), (5, 3), (1, 65)]
    g = torch.Generator().manual_seed(D + page)
    N = sum(a for a, _ in lens)
    size = torch.exp2(torch.rand(N, Hq + 2 * Hk, 1, generator=g) * 24 - 14)          # rows from 2^-14 to 2^10
    qkv = (torch.randn(N, Hq + 2 * Hk, D, generator=g) * size).to(dtype)
    qkv[3] = 0
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    pos = torch.randint(0, 300, (N, 3), generator=g, dtype=torch.int32)
    pairs = (part - 2 * (part // 3), part // 3, part // 3)
    freq = inv_freq(pairs)
    _, _, _, pages, table = make_case(3, lens, 1, Hk, D, dtype, page)
    marks = torch.randint(0, 256, pages.shape, generator=g, dtype=torch.uint8)
    smarks = torch.randn(pages.shape[:-1], generator=g).half()
    cache, batch = made(Hk, pages.shape[0], page, D, dtype, marks, smarks), batch_of(lens, table)
    rope = qwm.Rope(freq.cuda(), pairs, interleaved=il) if rope_on else None
    dev = qkv.cuda()
    q_rot = qwm.qwm_paged_append(cache, batch, dev[:, Hq:Hq + Hk], dev[:, Hq + Hk:], rope=rope,
                                 pos=pos.cuda() if rope_on else None, q=dev[:, :Hq])
    k64 = rope64(k, pos, freq, pairs, il) if rope_on else k.double()
    q64 = rope64(q, pos, freq, pairs, il) if rope_on else q.double()
    if rope_on:
        assert bool(((q_rot.double().cpu() - q64).abs() <= rope_bound(q, q64, dtype, pairs, il)).all())
        # the fp32 rotation's share of rope_bound: what it leaves of a pair's size
        eps = rope_bound(k, torch.zeros_like(k64), torch.bfloat16, pairs, il)
    else:
        assert torch.equal(q_rot.cpu(), q)
        eps = torch.zeros_like(k64)
    got_c, got_s = cache.pages.view(torch.uint8).cpu(), cache.scales.cpu()
    want_c, want_s = marks.clone(), smarks.clone()
    vc, vs = quantise64(v)
    most = k64.abs().amax(-1)
    for row, pid, slot in tokens_of(lens, page, table):
        want_c[pid, 1, :, slot], want_s[pid, 1, :, slot] = vc[row], vs[row].half()          # Values: the same bits
        s = got_s[pid, 0, :, slot].double()
        # a Key's scale: that of its largest magnitude, give or take the rotation's error
        e = eps[row].amax(-1)
        assert bool(((s >= scale64((most[row] - e)[:, None])) & (s <= scale64((most[row] + e)[:, None]))).all())
        got = stands_for(got_c[pid, 0, :, slot], got_s[pid, 0, :, slot])
        # half a step of e4m3 at that scale: 2^-4 of the value, 2^-10 of the scale below its normal numbers
        half = torch.maximum((k64[row].abs() + eps[row]) * 2.0 ** -4, s[:, None] * 2.0 ** -10)
        assert bool(((got - k64[row]).abs() <= half + eps[row]).all())
        if not rope_on:
            c0, s0 = quantise64(k[row])
            assert torch.equal(got_c[pid, 0, :, slot], c0) and torch.equal(s, s0)
        want_c[pid, 0, :, slot], want_s[pid, 0, :, slot] = got_c[pid, 0, :, slot], got_s[pid, 0, :, slot]
    assert torch.equal(got_c, want_c)
    assert torch.equal(got_s.view(torch.int16), want_s.view(torch.int16))
    assert cache.status() == 0
    # without Queries, the same pages
    cache.pages.view(torch.uint8).copy_(marks)
    cache.scales.copy_(smarks)
    assert qwm.qwm_paged_append(cache, batch, dev[:, Hq:Hq + Hk], dev[:, Hq + Hk:], rope=rope,
                                pos=pos.cuda() if rope_on else None) is None
    assert torch.equal(cache.pages.view(torch.uint8).cpu(), got_c)
    # read-back: what the codes stand for, exactly; zeros for tokens before the start
    rk, rv = qwm.qwm_paged_read(cache, batch, tokens=N)
    want = torch.zeros(2, N, Hk, D, dtype=torch.float64)
    for row, pid, slot in tokens_of(lens, page, table):
        for x in (0, 1):
            want[x, row] = stands_for(got_c[pid, x, :, slot], got_s[pid, x, :, slot])
    assert rk.dtype == rv.dtype == dtype
    assert torch.equal(rk.double().cpu(), want[0]) and torch.equal(rv.double().cpu(), want[1])


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_borders_of_the_quantiser(dtype, D):
    """Ties, the scale's borders, the smallest and the largest rows, both signs of zero."""
    rows = []
    for e in (-24, -15, -7, 0, 8, 15):
        for m in (1.0, 1.5, 1.75, 1.7578125, 1.9921875):                  # 448 = 1.75 x 2^8
            x = torch.zeros(D, dtype=torch.float64)
            x[0] = m * 2.0 ** e
            x[1:1 + 48] = x[0] * torch.arange(48) / 47.0
            x[50:60] = x[0] * 2.0 ** -torch.arange(10.0)
            x[60:] = -x[0] * (17 + 2 * torch.arange(D - 60)) / 2.0 ** 9       # halves of steps
            rows.append(x)
    x = torch.stack(rows).clamp(-65504, 65504).to(dtype)
    assert bool(torch.isfinite(x.double()).all())
    x[-1, 5] = -0.0
    N = x.shape[0]
    cache = made(1, 8, 16, D, dtype)
    table = torch.arange(8, dtype=torch.int32)[None]
    batch = batch_of([(N, N)], table, tokens=N)
    qwm.qwm_paged_append(cache, batch, x[:, None].cuda(), (-x)[:, None].cuda())
    c, s = quantise64(x)
    got_c = cache.pages.view(torch.uint8).cpu().permute(1, 2, 0, 3, 4).reshape(2, 128, D)[:, :N]
    got_s = cache.scales.cpu().permute(1, 2, 0, 3).reshape(2, 128)[:, :N]
    assert torch.equal(got_s[0].double(), s) and torch.equal(got_s[1].double(), s)
    assert torch.equal(got_c[0], c)
    assert torch.equal(got_c[1], c ^ 128)
    k, v = qwm.qwm_paged_read(cache, batch)
    assert torch.equal(k[:, 0].double().cpu(), stands_for(c, s)) and torch.equal(v, -k)
    assert cache.status() == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan, 65536.0, -3e38])
def test_values_beyond_the_range_saturate_and_are_recorded(dtype, where, what):
    N, Hk, D = 40, 3, 128
    g = torch.Generator().manual_seed(5)
    x = [torch.randn(N, Hk, D, generator=g).to(dtype) for _ in range(2)]
    w = int(where == "value")
    clean = [quantise64(t) for t in x]
    x[w][17, 1, 9] = what                                  # (binary16 makes an infinity of the largest)
    cache = made(Hk, 3, 16, D, dtype)
    batch = batch_of([(N, N)], torch.arange(3, dtype=torch.int32)[None], tokens=N)
    qwm.qwm_paged_append(cache, batch, x[0].cuda(), x[1].cuda())
    assert cache.status() == 6 and cache.status() == 0
    got = [t.double().cpu() for t in qwm.qwm_paged_read(cache, batch)]
    want = [stands_for(*t) for t in clean]
    row = x[w][17, 1].double()
    if math.isnan(what):
        row[9] = 0                                         # the others keep their scale
        want[w][17, 1] = stands_for(*quantise64(row))
        want[w][17, 1, 9] = math.nan
    else:
        want[w][17, 1] = stands_for(*quantise64(row))
        assert want[w][17, 1, 9] == math.copysign(MOST, what)
    for a, b in zip(got, want):
        assert torch.equal(a.nan_to_num(nan=7e7), b.nan_to_num(nan=7e7))


def test_the_largest_of_the_range_is_not_recorded():
    x = torch.zeros(1, 1, 64, dtype=HF)
    x[0, 0, 0], x[0, 0, 1] = 65504.0, -61440.0
    cache = made(1, 1, 16, 64, HF)
    batch = batch_of([(1, 1)], torch.zeros(1, 1, dtype=torch.int32), tokens=1)
    qwm.qwm_paged_append(cache, batch, x.cuda(), x.cuda())
    k, _ = qwm.qwm_paged_read(cache, batch)
    assert cache.status() == 0 and k[0, 0, :3].tolist() == [61440.0, -61440.0, 0.0]


@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("dtype,D,page,Hk", [(BF, 128, 16, 5), (HF, 64, 128, 2), (BF, 64, 32, 1)])
def test_read_back_of_any_tokens(codes, dtype, D, page, Hk):
    """Ragged parts of sequences, earlier tokens, either output alone, strided outputs; a copy of 16-bit pages."""
    lens = [(33, 70), (0, 5), (1, 1), (260, 300), (4, 2)]
    if codes:
        _, keys, values, c, s, table = make_code_case(13, lens, 1, Hk, D, dtype, page)
        cache = made(Hk, c.shape[0], page, D, dtype, c, s)
    else:
        _, keys, values, pages, table = make_case(13, lens, 1, Hk, D, dtype, page)
        cache = qwm.PagedCache(Hk, pages.shape[0], page_tokens=page, head_dim=D, dtype=dtype)
        cache.pages.copy_(pages)
    for cut in (0, 2):                                     # tokens left off the end: earlier ones are read
        at = [(ql, max(0, kv - cut)) for ql, kv in lens]
        N = sum(a for a, _ in at)
        want = torch.zeros(2, N, Hk, D, dtype=torch.float64)
        row = 0
        for (ql, kv), k, v in zip(at, keys, values):
            for i in range(ql):
                if kv - ql + i >= 0:
                    want[0, row], want[1, row] = k[kv - ql + i].double(), v[kv - ql + i].double()
                row += 1
        batch = batch_of(at, table)
        k, v = qwm.qwm_paged_read(cache, batch, tokens=N)
        assert k.dtype == dtype and k.shape == (N, Hk, D) and k.is_contiguous()
        assert torch.equal(k.double().cpu(), want[0]) and torch.equal(v.double().cpu(), want[1])
        wide = torch.full((N, 2 * Hk + 1, D + 8), 3.0, dtype=dtype, device="cuda")
        heads = torch.full((Hk, N, D), 3.0, dtype=dtype, device="cuda")
        k2, v2 = qwm.qwm_paged_read(cache, batch, k_out=heads.permute(1, 0, 2), v_out=wide[:, 1:1 + Hk, :D])
        assert k2.data_ptr() == heads.data_ptr() and torch.equal(k2, k) and torch.equal(v2, v)
        wide[:, 1:1 + Hk, :D] = 3.0
        assert bool((wide == 3.0).all())
        none, v3 = qwm.qwm_paged_read(cache, batch, tokens=N, keys=False)
        k3, none2 = qwm.qwm_paged_read(cache, batch, tokens=N, values=False)
        assert none is None and none2 is None and torch.equal(k3, k) and torch.equal(v3, v)
    assert cache.status() == 0
    empty = batch_of([(0, 5)], table[:1], tokens=0)
    k, v = qwm.qwm_paged_read(cache, empty)
    assert k.shape == v.shape == (0, Hk, D)


def test_read_back_records_entries_out_of_range():
    lens, Hk, D, page = [(20, 100), (40, 100)], 2, 128, 16
    _, keys, values, c, s, table = make_code_case(15, lens, 1, Hk, D, BF, page)
    for bad in (c.shape[0], -7, 1 << 30):
        broken = table.clone()
        broken[1, 5] = bad                                 # tokens 80 .. 95
        cache = made(Hk, c.shape[0], page, D, BF, c, s)
        k, v = qwm.qwm_paged_read(cache, batch_of(lens, broken), tokens=60)
        assert cache.status() == 1 and cache.status() == 0
        want = torch.cat([keys[0][80:], keys[1][60:]])
        want[20 + 20:20 + 36] = 0
        assert torch.equal(k.double().cpu(), want)
    for off, kvl, mq, mkv in (([0, 20, 61], [100, 100], 41, 100), ([0, 20, 60], [100, 101], 40, 100),
                              ([0, 20, 60], [100, -1], 40, 100), ([0, 20, 60], [100, 100], 39, 100)):
        batch = qwm.PagedBatch(torch.tensor(off, dtype=torch.int32).cuda(), torch.tensor(kvl, dtype=torch.int32).cuda(),
                               table.cuda(), mq, mkv)
        k, _ = qwm.qwm_paged_read(cache, batch, tokens=60)
        assert cache.status() == 1, (off, kvl)
        assert torch.equal(k[:20].double().cpu(), keys[0][80:]) and bool((k[20:] == 0).all())


# ------------------------------------------------------------------ attention
def run_case(seed, lens, Hq, Hk, D, dtype, page, block, window, sinks):
    q, keys, values, c, s, table = make_code_case(seed, lens, Hq, Hk, D, dtype, page)
    for b, (ql, kv) in enumerate(lens):                    # pages that no row sees are given back
        see = torch.zeros(kv, dtype=torch.bool)
        for i in range(ql):
            see |= visible(kv - ql + i, kv, block, window, sinks)
        for i in range((kv + page - 1) // page):
            if not bool(see[i * page:(i + 1) * page].any()):
                table[b, i] = -1
    cache, batch = made(Hk, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, block, window, sinks)
    for split in (False, True):
        ws = qwm.paged_attend_workspace(cache, batch, Hq, window, sinks, block) if split else None
        if split and ws is None:
            continue
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True,
                                        workspace=ws)
        compare(out, lse, want)
        again, _ = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True,
                                        workspace=ws)
        assert torch.equal(out, again)                     # the same bits, whichever part ends last
    assert cache.status() == 0


@pytest.mark.parametrize("case", range(len(STEP)))
def test_step(case):
    run_case(100 + case, *STEP[case])


@pytest.mark.parametrize("case", range(len(CHUNK)))
def test_chunk(case):
    run_case(200 + case, *CHUNK[case])


@pytest.mark.parametrize("D,dtype,Hq,Hk,new", [(128, BF, 20, 4, 1), (64, HF, 24, 8, 1), (128, HF, 18, 9, 9),
                                               (64, BF, 12, 4, 4)])
def test_step_over_many_sequences(D, dtype, Hq, Hk, new):
    """More groups than CTAs, of lengths from none to several ring turns."""
    g = torch.Generator().manual_seed(D + Hq)
    lens = []
    for i in range(61):
        q = int(torch.randint(0 if i % 7 == 3 else 1, new + 1, (1,), generator=g))
        lens.append((q, max(q, int(torch.randint(0, [5, 70, 700, 1800][i % 4], (1,), generator=g)))))
    run_case(300 + D, lens, Hq, Hk, D, dtype, 16, 1, 600, 9)


@pytest.mark.parametrize("Hq,Hk,new,lens", [
    (8, 4, 1, [(1, 501), (1, 900), (0, 700), (1, 255), (1, 257), (1, 1)]),          # 256-key tiles, whole groups
    (4, 4, 2, [(2, 7000), (1, 6400), (2, 511), (2, 2), (1, 3000)]),                 # shared out
    (12, 4, 4, [(4, 6100), (3, 6144), (1, 256), (4, 4)] + [(2, 30 + 97 * i) for i in range(16)]),   # 12 rows
])
@pytest.mark.parametrize("dtype,page,window,sinks", [(BF, 16, 0, 0), (HF, 128, 0, 0), (BF, 32, 2600, 70)])
def test_wide_tiles(Hq, Hk, new, lens, dtype, page, window, sinks):
    run_case(700 + Hq, lens, Hq, Hk, 64, dtype, page, 1, window, sinks)


@pytest.mark.parametrize("Hq,Hk,new,lens,window,sinks", [
    (10, 2, 4, [(4, 900), (1, 300), (3, 3), (0, 5), (2, 777)], 0, 0),               # 20, 5, 15, 0 and 10 rows
    (3, 3, 32, [(32, 40), (17, 1100), (8, 2600), (9, 9), (1, 4000), (31, 31)], 0, 0),
    (24, 4, 5, [(5, 1 + 61 * i) if i % 3 else (1 + i % 5, 5 + 150 * i) for i in range(40)], 600, 33),
    (17, 1, 1, [(1, 5000), (1, 1), (1, 64)], 0, 0),
])
@pytest.mark.parametrize("dtype,D,page", [(BF, 128, 64), (HF, 64, 16), (BF, 64, 32), (HF, 128, 128)])
def test_rows_in_blocks(Hq, Hk, new, lens, window, sinks, dtype, D, page):
    """More rows of a cache head than one block of the step's, of another number in each sequence."""
    lens = [(q, max(q, kv)) for q, kv in lens]
    run_case(800 + Hq, lens, Hq, Hk, D, dtype, page, 1, window, sinks)


@pytest.mark.parametrize("D,dtype,B,Hk,new", [(128, BF, 10, 8, 40), (64, HF, 20, 8, 33), (128, HF, 4, 20, 300)])
def test_groups_past_a_full_wave_are_cut(D, dtype, B, Hk, new):
    """A little more work than the GPU has places for: the first groups whole, the rest in parts."""
    lens = [(new, 1500 - 7 * i) for i in range(B)]
    q, keys, values, c, s, table = make_code_case(41, lens, Hk, Hk, D, dtype, 64)
    cache, batch = made(Hk, c.shape[0], 64, D, dtype, c, s), batch_of(lens, table)
    ws = qwm.paged_attend_workspace(cache, batch, Hk)
    assert ws is not None
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    again, _ = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    assert torch.equal(out, again)
    # every sequence's first and last rows against 64 bits, all of them against the call that is not split
    plain, plain_lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True)
    u = 2.0 ** -8 if dtype == BF else 2.0 ** -11
    size = torch.cat([v.abs().amax(0)[None].expand(new, -1, -1) for v in values])
    assert bool(((out.double() - plain.double()).abs().cpu() <= 4 * u * size).all())
    assert bool(((lse - plain_lse).abs() <= 2.0 ** -18 * (1 + plain_lse.abs())).all())
    for b, (_, kv) in enumerate(lens):
        for r in (0, new - 1):
            i, p = b * new + r, kv - new + r + 1
            want = attend_codes64(q[i:i + 1], [keys[b][:p]], [values[b][:p]], [(1, p)], 1, 0, 0)
            compare(out[i:i + 1], lse[:, i:i + 1], want)
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 3, 150])
@pytest.mark.parametrize("q_size,k_size", [(2.0 ** 100, 1e-3), (2.0 ** -100, 6e4), (2.0 ** 20, 1.0), (2.0 ** -126, 1.0)])
def test_queries_of_any_size(new, q_size, k_size):
    """bf16 Queries far outside binary16's range, with a scale that brings the logits back."""
    lens, Hq, Hk, D, page = [(new, 300)], 4, 2, 128, 16
    q, _, values, c, s, table = make_code_case(17, lens, Hq, Hk, D, BF, page)
    g = torch.Generator().manual_seed(3)
    kc, ks = quantise64((torch.randn(300, Hk, D, generator=g).clamp(-2.5, 2.5) * k_size / 2.5).to(BF))
    for i in range(19):
        n = min(page, 300 - i * page)
        c[int(table[0, i]), 0, :, :n] = kc[i * page:i * page + n].permute(1, 0, 2)
        s[int(table[0, i]), 0, :, :n] = ks[i * page:i * page + n].t().half()
    q = (q.double() * q_size).to(BF)
    q[0, 0] = 0
    q[0, 1, 3:] = 0
    scale = 0.05 / (q_size * k_size)
    if not scale < 1e38:
        scale = 1e38
    keys = [stands_for(kc, ks)]
    cache, batch = made(Hk, c.shape[0], page, D, BF, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, 1, 0, 0, scale=scale)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, Hq)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=scale, want_lse=True, workspace=ws)
        compare(out, lse, want)


@pytest.mark.parametrize("new,heads", [(4, 2), (60, 2)])
@pytest.mark.parametrize("dtype,D,page", [(BF, 128, 16), (HF, 64, 64)])
@pytest.mark.parametrize("by", ["code", "scale"])
def test_nan_tokens_reach_the_rows_that_see_them_only(new, heads, dtype, D, page, by):
    lens = [(new, 300)]
    q, keys, values, c, s, table = make_code_case(7, lens, heads, 1, D, dtype, page)
    window, sinks = 200, 5
    odd_k, odd_v = 298, 300 - new + 1              # the last but one token's Key, the second new token's Value
    early = 300 - new - window + 2                 # a Value that the first rows see and later ones do not
    at = lambda j: (int(table[0, j // page]), j % page)
    (pk, sk), (pv, sv), (pe, se) = at(odd_k), at(odd_v), at(early)
    if by == "code":
        c[pk, 0, 0, sk, 3] = 127
        c[pv, 1, 0, sv, 9] = 255
        c[pe, 1, 0, se, 11] = 127
    else:                                          # a caller's scale: every channel of the token
        s[pk, 0, 0, sk] = math.nan
        s[pv, 1, 0, sv] = math.inf
        s[pe, 1, 0, se] = math.nan
        c[pv, 1, 0, sv] = 9
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, 1, window, sinks)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, heads, window, sinks, 1)):
        out = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, workspace=ws).cpu()
        for i in range(new):
            p = 300 - new + i
            fine = torch.isfinite(out[i])
            if p >= odd_k:
                assert not bool(fine.any())
                continue
            ok = torch.ones(heads, D, dtype=torch.bool)
            if p >= odd_v:
                ok[:, 9 if by == "code" else slice(None)] = False
            if early >= p + 1 - window:
                ok[:, 11 if by == "code" else slice(None)] = False
            assert torch.equal(fine, ok), (i, p)
            err = (out[i].double() - want[0][i]).abs()
            assert bool((err <= want[2][i])[ok].all()), (i, p)
    if by == "code":
        return
    # infinities from scales read back as they are
    k, v = qwm.qwm_paged_read(cache, batch_of([(300, 300)], table), tokens=300)
    assert bool(k[odd_k].isnan().all()) and bool((v[odd_v] == math.inf).all())


@pytest.mark.parametrize("new", [3, 150])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("order", ["rising", "falling", "peak late", "waves"])
def test_running_maxima_that_move(new, dtype, D, order):
    """Logits along one direction whose maximum moves by far more than a tile's
    probabilities span, up, down and in the middle of a tile, for some rows only."""
    kv, page = 700, 16
    lens = [(new, kv)]
    q, keys, values, c, s, table = make_code_case(61, lens, 2, 1, D, dtype, page)
    j = torch.arange(kv, dtype=torch.float64)
    a = {"rising": j / 4, "falling": (kv - j) / 4, "peak late": 100.0 * ((j % 256) == 200) + 80 * (j == 610),
         "waves": 60 * torch.sin(j / 37) + j / 20}[order]
    x = 0.05 * keys[0]
    x[:, 0, 5] = a                                             # the direction is one channel
    kc, ks = quantise64(x.to(dtype))
    keys[0] = stands_for(kc, ks)
    q = 0.2 * q.float()
    q[:, 0, 5] = torch.linspace(-1, 1, q.shape[0])             # some rows climb, some descend
    q[:, 1, 5] = 1.0
    q = q.to(dtype)
    for i in range((kv + page - 1) // page):
        n = min(page, kv - i * page)
        c[int(table[0, i]), 0, :, :n] = kc[i * page:i * page + n].permute(1, 0, 2)
        s[int(table[0, i]), 0, :, :n] = ks[i * page:i * page + n].t().half()
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, 1, 0, 0, scale=1.0)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, 2)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=1.0, want_lse=True, workspace=ws)
        compare(out, lse, want)


@pytest.mark.parametrize("new,G,gap", [(1, 2, 16.0), (3, 2, 16.0), (5, 3, 16.0), (150, 2, 11.0)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_many_keys_beside_one_that_draws_most_of_the_weight(new, G, gap, dtype, D):
    """A first token whose Value is zero and whose logit is above all others by 16 (steps:
    P 2^-23 of the largest) or 11 (chunks: 2^-15.9): the others are the output.  Their P keeps
    all its bits (2^-12 relative of binary16), so the output is off by that, its own
    rounding, and 2^-14 for the exponentials of arguments below 32 in fp32 and the sums."""
    kv, page = 900, 16
    lens = [(new, kv)]
    q, keys, values, c, s, table = make_code_case(67, lens, G, 1, D, dtype, page)
    q = torch.zeros_like(q)
    q[:, :, 5] = 1.0                                           # a logit is one channel of the Key
    keys[0][:, 0, 5] = 0.0
    keys[0][0, 0, 5] = gap
    values[0] = values[0].abs() + 0.5
    values[0][0] = 0.0
    for x, rows in enumerate((keys, values)):
        cc, cs = quantise64(rows[0].to(dtype))
        rows[0] = stands_for(cc, cs)
        for i in range((kv + page - 1) // page):
            n = min(page, kv - i * page)
            c[int(table[0, i]), x, :, :n] = cc[i * page:i * page + n].permute(1, 0, 2)
            s[int(table[0, i]), x, :, :n] = cs[i * page:i * page + n].t().half()
    assert float(keys[0][0, 0, 5]) == gap
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, 1, 0, 0, scale=1.0)[0]
    bound = want.abs() * (2.0 ** -12 + torch.finfo(dtype).eps / 2 * 1.01 + 2.0 ** -14) + (2.0 ** -25 if dtype == HF else 0)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, G)):
        out = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=1.0, workspace=ws)
        out = out[0] if isinstance(out, tuple) else out
        assert bool(((out.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("new", [1, 40])
def test_attention_over_codes_is_attention_over_what_they_stand_for(new):
    """The same bits' worth of tokens in 8-bit and in 16-bit pages."""
    lens, Hq, Hk, D, page = [(new, 2500), (new, 90)], 8, 2, 128, 64
    q, keys, values, c, s, table = make_code_case(23, lens, Hq, Hk, D, HF, page)
    cache, batch = made(Hk, c.shape[0], page, D, HF, c, s), batch_of(lens, table)
    wide = qwm.PagedCache(Hk, c.shape[0], page_tokens=page, head_dim=D, dtype=HF)
    wide.pages.copy_(stands_for(c, s).half())
    a, la = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True)
    b, lb = qwm.qwm_paged_attend(wide, batch, q.cuda(), want_lse=True)
    want = attend_codes64(q, keys, values, lens, 1, 0, 0)
    assert bool(((a.double() - b.double()).abs().cpu() <= 2 * want[2]).all())
    assert bool(((la - lb).abs().cpu() <= 2 * want[3]).all())


def test_every_pass_gives_the_same_bits():
    """Tiles at the mask's edges (first tokens, then the window's start) amid a long list of
    tiles, whose making takes longer than their neighbours', in more groups than the SMs hold."""
    new, kv, H, D, page = 4680, 23400, 20, 128, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    num = (kv + page - 1) // page
    cache = qwm.PagedCache(H, num, page_tokens=page, head_dim=D, dtype=BF, storage=torch.float8_e4m3fn)
    cache.pages.copy_(torch.randn(cache.pages.shape, generator=g, device="cuda").to(torch.float8_e4m3fn))
    cache.scales.copy_(torch.exp2(torch.randint(-2, 2, cache.scales.shape, generator=g, device="cuda").float()))
    table = torch.randperm(num, generator=torch.Generator().manual_seed(6)).int()[None]
    batch = batch_of([(new, kv)], table)
    q = torch.randn(new, H, D, generator=g, device="cuda").to(BF)
    mask = dict(window=18720, sinks=1560, block=new)
    ws = qwm.paged_attend_workspace(cache, batch, H, **mask)
    first, first_lse = qwm.qwm_paged_attend(cache, batch, q, want_lse=True, workspace=ws, **mask)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    out, lse = torch.empty_like(first), torch.empty_like(first_lse)
    for _ in range(400):
        qwm.qwm_paged_attend(cache, batch, q, out=out, lse=lse, workspace=ws, **mask)
        differ += (out.view(torch.int16) != first.view(torch.int16)).any() | (lse != first_lse).any()
    assert int(differ) == 0
    assert cache.status() == 0


def test_offsets_beyond_32_bits():
    Hk, page, D = 8, 128, 128
    num = (1 << 32) // (2 * Hk * page * D) + 9                 # the last pages' codes start past 2^32 bytes
    cache = made(Hk, num, page, D, BF)
    lens = [(40, 300), (1, 129)]
    ids = [num - 1, 0, num - 4, num - 2, num - 3]
    table = torch.tensor([ids[:3], [ids[3], ids[4], -1]], dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(429, Hk, D, generator=g).to(BF) for _ in range(2))
    load = batch_of([(300, 300), (129, 129)], table, tokens=429)
    qwm.qwm_paged_append(cache, load, k.cuda(), v.cuda())
    keys, values = (stands_for(*quantise64(x)).split([300, 129]) for x in (k, v))
    rk, rv = qwm.qwm_paged_read(cache, load)
    assert torch.equal(rk.double().cpu(), torch.cat(keys)) and torch.equal(rv.double().cpu(), torch.cat(values))
    q = torch.randn(41, Hk, D, generator=g).to(BF)
    for new in (40, 1):
        at = [(new, 300), (1, 129)]
        out, lse = qwm.qwm_paged_attend(cache, batch_of(at, table), q[:new + 1].cuda(), want_lse=True)
        compare(out, lse, attend_codes64(q[:new + 1], keys, values, at, 1, 0, 0))
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 60])
def test_a_wait_that_runs_out_is_recorded_and_the_next_call_is_exact(new):
    lens, Hk, D, page = [(new, 900)], 2, 128, 16
    q, keys, values, c, s, table = make_code_case(51, lens, 2, Hk, D, BF, page)
    cache, batch = made(Hk, c.shape[0], page, D, BF, c, s), batch_of(lens, table)
    ws = qwm.paged_attend_workspace(cache, batch, 2)
    cache.set_wait_limit(1_000_000)                # 1 ms
    cache.set_idle_role(qwm.QWM_ROLE_PAGE_LOADS)
    qwm.qwm_paged_attend(cache, batch, q.cuda(), workspace=ws)
    torch.cuda.synchronize()
    assert cache.status() == 5
    cache.set_idle_role(0)
    cache.set_wait_limit(2_000_000_000)
    out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
    compare(out, lse, attend_codes64(q, keys, values, lens, 1, 0, 0))
    assert cache.status() == 0


@pytest.mark.parametrize("new,held_", [(1, 90), (1, 900), (4, 6000), (60, 100), (60, 900), (300, 5000)])
@pytest.mark.parametrize("split", [False, True])
def test_a_limit_near_a_loads_latency_leaves_nothing_in_flight(new, held_, split):
    lens, Hk, D, page = [(new, held_)], 2, 128, 16
    q, keys, values, c, s, table = make_code_case(71, lens, 4, Hk, D, BF, page)
    cache, batch = made(Hk, c.shape[0], page, D, BF, c, s), batch_of(lens, table)
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


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("split", [False, True])
def test_entries_out_of_range_are_recorded_and_not_followed(new, split):
    lens, Hk, D, page = [(new, 3000), (new, 3000)], 2, 128, 16
    q, keys, values, c, s, table = make_code_case(31, lens, 2, Hk, D, BF, page)
    want = attend_codes64(q[:new], keys[:1], values[:1], lens[:1], 1, 0, 0)
    for bad in (c.shape[0], -7, 1 << 30):
        broken = table.clone()
        broken[1, 6] = bad
        cache, batch = made(Hk, c.shape[0], page, D, BF, c, s), batch_of(lens, broken)
        ws = qwm.paged_attend_workspace(cache, batch, 2) if split else None
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
        assert cache.status() == 1 and cache.status() == 0
        compare(out[:new], lse[:, :new], want)             # the other sequence is as it should be
    k = torch.zeros(2 * new, Hk, D, dtype=BF, device="cuda")
    broken = table.clone()
    broken[1, 2999 // page] = c.shape[0]
    before = cache.pages.view(torch.uint8).clone()
    qwm.qwm_paged_append(cache, batch_of([(0, 3000), (2 * new, 3000)], broken), k, k)
    assert cache.status() == 1
    first = 3000 - 2 * new                                 # what was in range is stored, nothing else
    for b in range(c.shape[0]):
        mine = [i for i in range(first // page, 2999 // page) if int(table[1, i]) == b]
        if not mine:
            assert torch.equal(cache.pages.view(torch.uint8)[b], before[b])


def test_steps_of_a_stream_append_attend_and_read_as_they_would_be_used():
    """A prompt, single tokens, a frame read back as it leaves the window; one captured step replayed over the rest."""
    Hq, Hk, D, page, T = 8, 2, 128, 16, 200
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn(T, Hq + 2 * Hk, D, generator=g).to(BF)
    pairs = (22, 21, 21)
    freq, pos = inv_freq(pairs), torch.stack([torch.arange(T) // 40, torch.arange(T) % 40 // 8, torch.arange(T) % 8], 1).int()
    rope = qwm.Rope(freq.cuda(), pairs)
    cache = made(Hk, 14, page, D, BF)
    table = torch.randperm(14, generator=g).int()[None, :13]
    dev, dpos, dtable = qkv.cuda(), pos.cuda(), table.cuda()
    outs = torch.empty(T, Hq, D, dtype=BF, device="cuda")
    window = 96

    def step(first, n, out):
        b = qwm.PagedBatch(torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([first + n], dtype=torch.int32).cuda(),
                           dtable, n, 208, tokens=n)
        x = dev[first:first + n]
        q = qwm.qwm_paged_append(cache, b, x[:, Hq:Hq + Hk], x[:, Hq + Hk:], rope=rope, pos=dpos[first:first + n], q=x[:, :Hq])
        ws = qwm.paged_attend_workspace(cache, b, Hq, window=window, sinks=4)
        qwm.qwm_paged_attend(cache, b, q, window=window, sinks=4, out=out, workspace=ws)

    step(0, 120, outs[:120])
    for t in range(120, 150):
        step(t, 1, outs[t:t + 1])
    # the rest by one captured step, its inputs in place
    x, p = torch.empty_like(dev[:1]), torch.empty_like(dpos[:1])
    kv, off, out = torch.empty(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.empty_like(outs[:1])
    b = qwm.PagedBatch(off, kv, dtable, 1, 208, tokens=1)
    ws = qwm.paged_attend_workspace(cache, b, Hq, window=window, sinks=4)
    rk, rv = torch.empty(1, Hk, D, dtype=BF, device="cuda"), torch.empty(1, Hk, D, dtype=BF, device="cuda")

    def fill(t):
        x.copy_(dev[t:t + 1])
        p.copy_(dpos[t:t + 1])
        kv.fill_(t + 1)

    def one():
        q = qwm.qwm_paged_append(cache, b, x[:, Hq:Hq + Hk], x[:, Hq + Hk:], rope=rope, pos=p, q=x[:, :Hq])
        qwm.qwm_paged_attend(cache, b, q, window=window, sinks=4, out=out, workspace=ws)
        qwm.qwm_paged_read(cache, b, k_out=rk, v_out=rv)

    fill(150)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    torch.cuda.current_stream().wait_stream(side)
    outs[150:151].copy_(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    reads = []
    for t in range(151, T):
        fill(t)
        graph.replay()
        outs[t:t + 1].copy_(out)
        reads.append((rk.clone(), rv.clone()))
    assert cache.status() == 0
    whole = qwm.PagedBatch(torch.tensor([0, T], dtype=torch.int32).cuda(), torch.tensor([T], dtype=torch.int32).cuda(),
                           dtable, T, 208, tokens=T)
    k, v = qwm.qwm_paged_read(cache, whole)
    for i, (a, c) in enumerate(reads):
        assert torch.equal(a[0], k[151 + i]) and torch.equal(c[0], v[151 + i])
    frame = qwm.PagedBatch(torch.tensor([0, 40], dtype=torch.int32).cuda(), torch.tensor([80], dtype=torch.int32).cuda(),
                           dtable, 40, 208, tokens=40)
    fk, fv = qwm.qwm_paged_read(cache, frame)                  # tokens 40 .. 79
    assert torch.equal(fk, k[40:80]) and torch.equal(fv, v[40:80])
    # Keys and Values: the quantised rotation and projection; the outputs: attention over them
    assert torch.equal(v.double().cpu(), stands_for(*quantise64(qkv[:, Hq + Hk:])))
    k64 = rope64(qkv[:, Hq:Hq + Hk], pos, freq, pairs, True)
    eps = rope_bound(qkv[:, Hq:Hq + Hk], torch.zeros_like(k64), BF, pairs, True)
    s = scale64(k64)[..., None]
    assert bool(((k.double().cpu() - k64).abs() <= torch.maximum((k64.abs() + eps) * 2.0 ** -4, s * 2.0 ** -10) + eps).all())
    q64 = qwm.qwm_rope(rope, dev[:, :Hq], dpos).cpu()
    want = attend_codes64(q64, [k.double().cpu()], [v.double().cpu()], [(T, T)], 1, window, 4)
    assert bool(((outs.double().cpu() - want[0]).abs() <= want[2]).all())


def test_another_stream_and_two_graphs_on_one_workspace():
    lens, Hq, Hk, D, page = [(1, 6000), (1, 30)], 8, 2, 128, 16
    q, keys, values, c, s, table = make_code_case(21, lens, Hq, Hk, D, BF, page)
    cache, batch = made(Hk, c.shape[0], page, D, BF, c, s), batch_of(lens, table, tokens=2)
    ws = qwm.paged_attend_workspace(cache, batch, Hq)
    dq = q.cuda()
    ref = qwm.qwm_paged_attend(cache, batch, dq, workspace=ws).clone()
    rk, rv = (t.clone() for t in qwm.qwm_paged_read(cache, batch))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late = dq.clone()
        got = qwm.qwm_paged_attend(cache, batch, late, workspace=ws)
        k, v = qwm.qwm_paged_read(cache, batch)
    side.synchronize()
    assert torch.equal(got, ref) and torch.equal(k, rk) and torch.equal(v, rv)
    graphs, outs = [], []
    for _ in range(2):
        g, out = torch.cuda.CUDAGraph(), torch.empty_like(dq)
        with torch.cuda.graph(g):
            qwm.qwm_paged_attend(cache, batch, dq, out=out, workspace=ws)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):                             # by turns on one stream
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ref) and torch.equal(outs[1], ref)


@pytest.mark.parametrize("compress", [False, True])
def test_the_streaming_example_runs_on_8_bit_pages(compress):
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import streaming_window as ex
    out, _ = ex.run(heads=2, frames=4, tokens=2, compress=compress, storage=E4)
    wide, _ = ex.run(heads=2, frames=4, tokens=2, compress=compress)
    assert out.shape == wide.shape and bool(torch.isfinite(out).all())
    # the first frame sees itself only: Keys' relative error of at most 2^-4 a channel, independent, of logits that
    # spread by 1, and Values' of 2^-4 (uniform in sign): well under half of the outputs' size
    assert (out - wide)[:ex.FRAME].float().norm() <= 0.5 * wide[:ex.FRAME].float().norm()


def test_refusals():
    cache = made(2, 4, 16, 128, BF)
    table = torch.arange(4, dtype=torch.int32)[None]
    batch = batch_of([(3, 40)], table)

    def status(fn):
        with pytest.raises(qwm.QwmError) as e:
            fn()
        return e.value.status

    with pytest.raises(ValueError, match="not known"):
        qwm.qwm_paged_read(cache, batch)
    with pytest.raises(ValueError):
        qwm.qwm_paged_read(cache, batch_of([(3, 40)], table, tokens=3), tokens=4)
    with pytest.raises(ValueError):
        qwm.PagedCache(2, 4, storage=torch.int8)
    with pytest.raises(ValueError):
        qwm.PagedCache(2, 4, dtype=BF, storage=HF)
    assert qwm.PagedCache(2, 4, dtype=BF, storage=BF).scales is None
    k = torch.zeros(3, 2, 128, dtype=BF, device="cuda")
    for bad in (k.half(), k[..., :64], k.cpu(), k[0], k[:2]):
        with pytest.raises(ValueError):
            qwm.qwm_paged_read(cache, batch, tokens=3, k_out=bad)
        with pytest.raises(ValueError):
            qwm.qwm_paged_append(cache, batch, k, bad)
    assert status(lambda: qwm.qwm_paged_read(cache, batch, k_out=k[:, :1])) == 1                 # heads
    assert status(lambda: qwm.qwm_paged_read(cache, batch, tokens=3, keys=False, values=False)) == 1
    assert status(lambda: qwm.qwm_paged_read(cache, batch, k_out=k, v_out=k)) == 1               # one place for both
    assert status(lambda: qwm.qwm_paged_read(cache, batch, k_out=k[:1].expand(3, 2, 128))) == 1  # rows on rows
    over = cache.buffer[256:256 + 3 * 2 * 128 * 2].view(BF).view(3, 2, 128)
    assert status(lambda: qwm.qwm_paged_read(cache, batch, k_out=over)) == 1                     # the pages themselves
    sound = cache._key
    cache._key = (*sound[:-1], 1)                                                                # as on a second GPU
    with pytest.raises(ValueError, match="on another device"):
        qwm.qwm_paged_read(cache, batch, tokens=3)
    cache._key = sound
    assert status(lambda: qwm.PagedCache(2, 4, page_tokens=24, storage=E4)) == 2
    assert status(lambda: qwm.PagedCache(2, 4, head_dim=96, storage=E4)) == 2
    q = torch.zeros(3, 4, 128, dtype=BF, device="cuda")
    assert status(lambda: qwm.qwm_paged_attend(cache, batch, q[:, :3])) == 1
    assert cache.status() == 0
