"""GPU: paged storage in 8 bits at its edges -- rings that turn many times, ranges, scales of a
caller's own, and the paths that only large calls take -- against the definitions in 64 bits
(tests/codes_ref.py)."""
import math

import pytest
import torch

import paper_2609_26425_gb300 as qwm
from codes_ref import (VALUE, alternating_case, attend_codes64, attend_codes64_close, make_code_case, quantise64, scale64,
                       stands_for)
from paged_ref import inv_freq, offsets, rope64, rope_bound
from test_gpu_paged import compare

pytestmark = pytest.mark.gpu
BF, HF, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    qwm.lib()


def batch_of(lens, table, **more):
    return qwm.PagedBatch(offsets(lens).cuda(), torch.tensor([kv for _, kv in lens], dtype=torch.int32).cuda(),
                          table.cuda(), max(a for a, _ in lens), max(kv for _, kv in lens), **more)


def made(Hk, num, page, D, dtype, codes=None, scales=None):
    cache = qwm.PagedCache(Hk, num, page_tokens=page, head_dim=D, dtype=dtype, storage=E4)
    if codes is not None:
        cache.pages.view(torch.uint8).copy_(codes)
        cache.scales.copy_(scales)
    return cache


def filled(seed, Hk, num, page, D, dtype, codes):
    """A cache whose every slot holds a random token, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = qwm.PagedCache(Hk, num, page_tokens=page, head_dim=D, dtype=dtype, storage=E4 if codes else None)
    for p in cache.pages:
        p.copy_(torch.randn(p.shape, generator=g, device="cuda").to(cache.storage))
    if codes:
        cache.scales.copy_(torch.exp2(torch.randint(-2, 2, cache.scales.shape, generator=g, device="cuda").float()))
    return cache


# ------------------------------------------------------------------ rings
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("dtype,D,Hq,Hk,new,window", [(BF, 128, 20, 4, 1, 0), (HF, 128, 12, 4, 4, 2600), (BF, 64, 8, 8, 1, 0),
                                                      (HF, 64, 12, 4, 4, 0), (BF, 128, 2, 1, 10, 0)])
def test_every_step_gives_the_same_bits(codes, dtype, D, Hq, Hk, new, window):
    """Rings that turn many times, with tiles at the mask's edges among whole ones: a slot that went back before
    its loads were done would show in some pass."""
    lens = [(1 + i % new, 3000 + 977 * i) for i in range(12)]
    page = 64
    width = -(-lens[-1][1] // page)
    cache = filled(11, Hk, width, page, D, dtype, codes)
    table = torch.stack([torch.randperm(width, generator=torch.Generator().manual_seed(i)) for i in range(len(lens))]).int()
    batch = batch_of(lens, table)
    q = torch.randn(sum(a for a, _ in lens), Hq, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    mask = dict(window=window, sinks=70 if window else 0)
    ws = qwm.paged_attend_workspace(cache, batch, Hq, **mask)
    assert ws is not None
    first, first_lse = qwm.qwm_paged_attend(cache, batch, q, want_lse=True, workspace=ws, **mask)
    assert bool(torch.isfinite(first_lse).all()) and bool(torch.isfinite(first).all())
    out, lse = torch.empty_like(first), torch.empty_like(first_lse)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(500):
        qwm.qwm_paged_attend(cache, batch, q, out=out, lse=lse, workspace=ws, **mask)
        differ += (out.view(torch.int16) != first.view(torch.int16)).any() | (lse != first_lse).any()
    assert int(differ) == 0
    assert cache.status() == 0


# ------------------------------------------------------------------ ranges
def in_pages(page, table, lens, rows, which, codes, scales):
    """Writes the codes and scales of `rows` (per sequence, [kv][heads][channels], 64 bits) into their pages;
    returns what they stand for."""
    held = []
    for b, ((_, kv), x) in enumerate(zip(lens, rows)):
        c, s = quantise64(x)
        held.append(stands_for(c, s))
        for i in range(-(-kv // page)):
            n = min(page, kv - i * page)
            codes[int(table[b, i]), which, :, :n] = c[i * page:i * page + n].permute(1, 0, 2)
            scales[int(table[b, i]), which, :, :n] = s[i * page:i * page + n].t().half()
    return held


@pytest.mark.parametrize("new,G,kv,B", [(1, 2, 300, 1), (3, 2, 300, 1), (5, 2, 300, 1), (5, 2, 200, 80), (2, 2, 9000, 1),
                                        (5, 2, 9000, 1), (5, 2, 2600, 80), (150, 2, 300, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("side", [1.0, -1.0])
def test_products_beyond_fp32_with_a_scale_that_brings_them_back(new, G, kv, B, D, side):
    """q k^T about 2^131 (fp32 ends at 2^128), logits about 32 side: the maxima that warps, CTAs and parts
    hand on have to be those of the logits."""
    lens, page, scale = [(new, kv - i) for i in range(B)], 16, 2.0 ** -126
    q, _, values, c, s, table = make_code_case(19, lens, G, 1, D, BF, page)
    g = torch.Generator().manual_seed(kv + D)
    x = [torch.randn(n, 1, D, generator=g).clamp(-3, 3).double() * 2.0 ** 8 for _, n in lens]
    for y in x:
        y[..., 0] = 2.0 ** 11
    keys = in_pages(page, table, lens, x, 0, c, s)
    q = torch.randn(new * B, G, D, generator=g).clamp(-3, 3).double() * 2.0 ** 117
    q[..., 0] = side * 2.0 ** 120
    q = q.to(BF)
    cache, batch = made(1, c.shape[0], page, D, BF, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, 1, 0, 0, scale=scale)
    assert float((want[1].abs() > 4).float().mean()) > 0.99    # (log-sum-exps: |q k^T| > 2^128 at the maxima)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, G)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), sm_scale=scale, want_lse=True, workspace=ws)
        compare(out, lse, want)
    assert cache.status() == 0


# ------------------------------------------------------------------ scales that a caller wrote
ODD = [0.1, 1 / 3, 3.0, 0.75, 1000.3, 512.0, 65504.0, 2.0 ** -16, 3 * 2.0 ** -24, 2.0 ** -24, 0.00123, -1.0, -0.3, 0.0, math.inf,
       -math.inf, math.nan, 1.0, 256.0, 2.0 ** -15]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
def test_read_back_with_any_scale_rounds_once(dtype, D):
    """Every code with scales of every kind: the product of the two, rounded to the cache's type."""
    rows = 256 // D                                            # tokens for all codes, of each scale
    N, page = rows * len(ODD), 16
    scales = torch.tensor(ODD).half().repeat_interleave(rows)
    codes = torch.arange(256, dtype=torch.uint8).view(rows, D).repeat(len(ODD), 1)
    num = -(-N // page)
    pc, ps = torch.full((num * page, D), 127, dtype=torch.uint8), torch.zeros(num * page).half()
    pc[:N], ps[:N] = codes, scales
    cache = made(1, num, page, D, dtype)
    for x in (0, 1):
        cache.pages.view(torch.uint8)[:, x, 0].copy_(pc.view(num, page, D))
        cache.scales[:, x, 0].copy_(ps.view(num, page))
    k, v = qwm.qwm_paged_read(cache, batch_of([(N, N)], torch.arange(num, dtype=torch.int32)[None], tokens=N))
    # 4 x 11 bits: the product is a number of fp32, so this rounds once
    exact = stands_for(codes, scales)
    assert torch.equal(exact.float().double().nan_to_num(), exact.nan_to_num())
    want = exact.float().to(dtype)
    for got in (k[:, 0].cpu(), v[:, 0].cpu()):
        nan = want.isnan()
        assert torch.equal(got.isnan(), nan)
        assert torch.equal(got.view(torch.int16)[~nan], want.view(torch.int16)[~nan])


@pytest.mark.parametrize("new,G", [(1, 2), (3, 2), (5, 2), (6, 4), (150, 2)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (HF, 128), (HF, 64)])
@pytest.mark.parametrize("kv,B,some", [(300, 1, False), (300, 1, True), (200, 80, False), (6500, 1, True)])
def test_attention_over_any_scale_is_one_rule(new, G, dtype, D, kv, B, some):
    """Products of scales that are no power of two, or below 2^-15, are rounded to binary16 before they enter,
    in steps and chunks alike; `some`: one token in 40 has one, the others as appended."""
    if new == 150:
        B = min(B, 2)
    lens, page = [(new, kv - i) for i in range(B)], 16
    q, _, _, c, s, table = make_code_case(29, lens, G, 1, D, dtype, page)
    g = torch.Generator().manual_seed(kv)
    pool = torch.tensor([0.1, 1 / 3, 0.37, 0.0123, -0.21, 2.0 ** -17, 3 * 2.0 ** -18])
    held = [[], []]
    for b, (_, n) in enumerate(lens):
        for x in (0, 1):
            codes, sc = quantise64(torch.randn(n, 1, D, generator=g).double())
            codes = torch.where(VALUE[codes.long()].abs() > 240, codes ^ 8, codes)      # (so that q k^T stays moderate)
            odd = pool[torch.randint(0, len(pool), (n, 1), generator=g)] / 16
            use = torch.rand(n, 1, generator=g) < (1 / 40 if some else 1.0)
            sc = torch.where(use, odd, sc.float()).half()
            held[x].append(stands_for(codes, sc).half().double())
            for i in range(-(-n // page)):
                m = min(page, n - i * page)
                c[int(table[b, i]), x, :, :m] = codes[i * page:i * page + m].permute(1, 0, 2)
                s[int(table[b, i]), x, :, :m] = sc[i * page:i * page + m].t()
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, held[0], held[1], lens, 1, 0, 0)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, G)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
        compare(out, lse, want)


@pytest.mark.parametrize("new,G", [(1, 2), (4, 2), (5, 2), (150, 2)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_a_product_beyond_binary16_is_an_infinity_in_steps_and_chunks(new, G, dtype, D):
    """Code 448 at scale 512 of one Key's channel: +inf times q there, so the rows of head 0 (q > 0) are NaN and
    those of head 1 (q < 0) do not see the token."""
    lens, kv, page, at = [(new, 400)], 400, 16, 37
    q, keys, values, c, s, table = make_code_case(33, lens, G, 1, D, dtype, page)
    q[:, 0, 3], q[:, 1, 3] = 0.5, -0.5
    pid, slot = int(table[0, at // page]), at % page
    c[pid, 0, 0, slot] = 0
    c[pid, 0, 0, slot, 3] = 126                                # 448
    s[pid, 0, 0, slot] = 512.0
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    keys[0][at] = 0
    keys[0][at, 0, 3] = 1e6                                    # (its weight in 64 bits: exp(-1e6 / 2 / sqrt(D)) = 0)
    want = attend_codes64(q[:, 1:], keys, values, lens, 1, 0, 0)
    keys[0][at, 0, 3] = 0                                      # (the bounds, without it)
    bound = attend_codes64(q[:, 1:], keys, values, lens, 1, 0, 0)[2:]
    for ws in (None, qwm.paged_attend_workspace(cache, batch, G)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), want_lse=True, workspace=ws)
        assert bool(out[:, 0].isnan().all()) and bool(lse[0].isnan().all())
        compare(out[:, 1:], lse[1:], (*want[:2], *bound))


# ------------------------------------------------------------------ paths that only large calls take
@pytest.mark.parametrize("dtype,D,il,Hq,Hk,part,lens", [
    (BF, 128, True, 3, 2, 64, [(4680, 4999), (0, 7), (31, 40)]),               # 7 tokens a CTA
    (HF, 64, False, 1, 1, 24, [(1, 1), (12007, 12100), (903, 903)]),           # 16, the most
    (BF, 64, True, 40, 1, 32, [(2500, 2500), (77, 5000)]),                     # 3
    (HF, 128, False, 0, 5, 64, [(1217, 1300)]),                                # without Queries
])
def test_append_of_many_tokens_a_block(dtype, D, il, Hq, Hk, part, lens):
    """Blocks of threads with several tokens each, their tables of angles and of places among them."""
    N, page = sum(a for a, _ in lens), 32
    g = torch.Generator().manual_seed(N)
    qkv = (torch.randn(N, Hq + 2 * Hk, D, generator=g) * torch.exp2(torch.rand(N, Hq + 2 * Hk, 1, generator=g) * 12 - 8)).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    pos = torch.randint(0, 3000, (N, 3), generator=g, dtype=torch.int32)
    pairs = (part - 2 * (part // 3), part // 3, part // 3)
    freq = inv_freq(pairs)
    width = max(-(-kv // page) for _, kv in lens)
    num = len(lens) * width + 2
    table = torch.randperm(num, generator=g)[:len(lens) * width].int().view(len(lens), width)
    marks = torch.randint(0, 256, (num, 2, Hk, page, D), generator=g, dtype=torch.uint8)
    smarks = torch.randn(num, 2, Hk, page, generator=g).half()
    cache, batch = made(Hk, num, page, D, dtype, marks, smarks), batch_of(lens, table, tokens=N)
    dev = qkv.cuda()
    rot = qwm.qwm_paged_append(cache, batch, dev[:, Hq:Hq + Hk], dev[:, Hq + Hk:], rope=qwm.Rope(freq.cuda(), pairs, interleaved=il),
                               pos=pos.cuda(), q=dev[:, :Hq] if Hq else None)
    if Hq:
        q64 = rope64(q, pos, freq, pairs, il)
        assert bool(((rot.double().cpu() - q64).abs() <= rope_bound(q, q64, dtype, pairs, il)).all())
    at = torch.cat([torch.arange(kv - ql, kv) for ql, kv in lens])
    seq = torch.cat([torch.full((ql,), b) for b, (ql, _) in enumerate(lens)])
    pid, slot = table[seq, at // page].long(), at % page
    got_c, got_s = cache.pages.view(torch.uint8).cpu(), cache.scales.cpu()
    # Values: the same bits
    vc, vs = quantise64(v)
    assert torch.equal(got_c[pid, 1, :, slot], vc) and torch.equal(got_s[pid, 1, :, slot].double(), vs)
    # Keys: the scale of the largest magnitude give or take the rotation's error, codes within half a step and that
    k64 = rope64(k, pos, freq, pairs, il)
    eps = rope_bound(k, torch.zeros_like(k64), BF, pairs, il)
    most, e = k64.abs().amax(-1), eps.amax(-1)
    s = got_s[pid, 0, :, slot].double()
    assert bool(((s >= scale64((most - e)[..., None])) & (s <= scale64((most + e)[..., None]))).all())
    got = stands_for(got_c[pid, 0, :, slot], got_s[pid, 0, :, slot])
    half = torch.maximum((k64.abs() + eps) * 2.0 ** -4, s[..., None] * 2.0 ** -10)
    assert bool(((got - k64).abs() <= half + eps).all())
    # and nothing else
    mine = torch.zeros(num, page, dtype=torch.bool)
    mine[pid, slot] = True
    keep = ~mine[:, None, None, :].expand(num, 2, Hk, page)
    assert torch.equal(got_c[keep], marks[keep])
    assert torch.equal(got_s.view(torch.int16)[keep], smarks.view(torch.int16)[keep])
    assert cache.status() == 0


@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("dtype,D,page,Hk,lens", [
    (BF, 128, 16, 37, [(2111, 2500), (0, 3), (41, 41)]),                       # 1215 turns
    (HF, 64, 32, 3, [(5, 5), (60011, 60020), (70, 100)]),                      # rows of a token across turns
    (HF, 128, 128, 1, [(40003, 40003)]),
    (BF, 64, 64, 80, [(2009, 2010), (60, 70)]),
])
def test_read_back_of_more_rows_than_the_grid_takes_at_once(codes, dtype, D, page, Hk, lens):
    N = sum(a for a, _ in lens)
    assert 2 * N * Hk > 2 * 608 * 256 * 4 // (D // 16) or Hk == 1
    width = max(-(-kv // page) for _, kv in lens)
    cache = filled(5, Hk, len(lens) * width, page, D, dtype, codes)
    table = torch.randperm(len(lens) * width, generator=torch.Generator().manual_seed(2)).int().view(len(lens), width)
    at = torch.cat([torch.arange(kv - ql, kv) for ql, kv in lens])
    seq = torch.cat([torch.full((ql,), b) for b, (ql, _) in enumerate(lens)])
    pid, slot = table[seq, at // page].long().cuda(), (at % page).cuda()
    batch = batch_of(lens, table, tokens=N)
    k, v = qwm.qwm_paged_read(cache, batch)
    none, v1 = qwm.qwm_paged_read(cache, batch, keys=False)
    k1, none2 = qwm.qwm_paged_read(cache, batch, values=False)
    assert none is None and none2 is None
    for x, gots in enumerate(((k, k1), (v, v1))):
        if codes:
            want = stands_for(cache.pages.view(torch.uint8)[pid, x, :, slot].cpu(), cache.scales[pid, x, :, slot].cpu())
        else:
            want = cache.pages[pid, x, :, slot].double().cpu()
        for got in gots:
            assert torch.equal(got.double().cpu(), want)
    assert cache.status() == 0


def full_case(seed, lens, Hq, Hk, D, dtype, page, block, window, sinks, cut=None):
    """Attention of every row against 64 bits, with the closer bounds of codes; `cut`: whether some groups are in parts."""
    q, keys, values, c, s, table = make_code_case(seed, lens, Hq, Hk, D, dtype, page)
    cache, batch = made(Hk, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64(q, keys, values, lens, block, window, sinks)
    ws = qwm.paged_attend_workspace(cache, batch, Hq, window, sinks, block)
    for w in (None, ws):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True, workspace=w)
        compare(out, lse, want)
    assert cache.status() == 0
    return ws


@pytest.mark.parametrize("case", [
    # lens, Hq, Hk, D, dtype, page, block, window, sinks: several groups of 512 (256) rows of a head
    ([(700, 900), (1, 5), (513, 513)], 1, 1, 128, BF, 16, 1, 0, 0),
    ([(301, 640), (40, 700)], 4, 1, 128, HF, 64, 1, 333, 21),                   # 1204 rows of four heads
    ([(600, 1200)], 2, 2, 128, BF, 128, 600, 900, 100),
    ([(257, 300), (511, 800)], 3, 1, 64, HF, 32, 1, 200, 5),
])
def test_several_groups_of_rows(case):
    full_case(401, *case)


@pytest.mark.parametrize("case", [
    # a little more groups than the SMs (pairs of them) hold
    ([(40, 1500 - 7 * i) for i in range(10)], 24, 8, 128, BF, 64, 1, 1100, 33),
    ([(33, 1500 - 7 * i) for i in range(20)], 16, 8, 64, HF, 16, 1, 1200, 70),
    ([(30, 1500 - 60 * i) for i in range(20)], 8, 4, 128, HF, 128, 30, 0, 0),
])
def test_cut_groups_under_windows_first_tokens_and_grouped_heads(case):
    lens, Hq, Hk, D = case[:4]
    ws = full_case(403, *case)
    rows = 512 if D == 128 else 256
    # parts are kept for the last groups only: fewer bytes than one part of every group
    assert ws is not None and ws.numel() < len(lens) * Hk * rows * (4 * D + 8)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_append_stores_what_is_in_range_and_nothing_else(new, dtype, D):
    """One entry of the table out of range: the tokens of its page are left out, all others stored, bit for bit."""
    Hk, page, kv = 2, 16, 3000
    lens = [(new, kv), (20 + new, kv), (0, 50), (3, 700)]      # the second has tokens before, in and after the broken page
    N = sum(a for a, _ in lens)
    g = torch.Generator().manual_seed(new)
    width = -(-kv // page)
    num = len(lens) * width
    table = torch.randperm(num, generator=g).int().view(len(lens), width)
    k, v = ((torch.randn(N, Hk, D, generator=g) * torch.exp2(torch.rand(N, Hk, 1, generator=g) * 8 - 4)).to(dtype) for _ in range(2))
    for bad in (num, -7, 1 << 30):
        broken = table.clone()
        broken[1, (kv - 10) // page] = bad
        marks = torch.randint(0, 256, (num, 2, Hk, page, D), generator=g, dtype=torch.uint8)
        smarks = torch.randn(num, 2, Hk, page, generator=g).half()
        cache = made(Hk, num, page, D, dtype, marks, smarks)
        qwm.qwm_paged_append(cache, batch_of(lens, broken, tokens=N), k.cuda(), v.cuda())
        assert cache.status() == 1 and cache.status() == 0
        stored = 0
        for x, rows in enumerate((k, v)):
            codes, scales = quantise64(rows)
            row = 0
            for b, (ql, n) in enumerate(lens):
                for p in range(n - ql, n):
                    if 0 <= broken[b, p // page] < num:
                        at = int(broken[b, p // page])
                        marks[at, x, :, p % page], smarks[at, x, :, p % page] = codes[row], scales[row].half()
                        stored += 1
                    row += 1
        assert 0 < stored < 2 * N
        assert torch.equal(cache.pages.view(torch.uint8).cpu(), marks)
        assert torch.equal(cache.scales.cpu().view(torch.int16), smarks.view(torch.int16))


# ------------------------------------------------------------------ the products' own rounding
@pytest.mark.parametrize("new,G,B", [(1, 2, 1), (4, 2, 3), (5, 2, 1), (5, 2, 80), (12, 2, 2), (150, 2, 1)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (HF, 128), (HF, 64)])
def test_probabilities_keep_binary16s_bits(new, G, B, dtype, D):
    """Differences of two probabilities, whatever the tensors' type is."""
    lens, page = [(new, new + 40 + i) for i in range(B)], 16
    q, keys, values, c, s, table = alternating_case(lens, G, D, dtype, page)
    cache, batch = made(1, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64_close(q, keys, values, lens, 1, 2, 0, step=new * G <= 32)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, G, 2, 0, 1)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=2, want_lse=True, workspace=ws)
        compare(out, lse, want)


@pytest.mark.parametrize("case", [
    # lens, Hq, Hk, D, dtype, page, block, window, sinks
    ([(1, 2900), (1, 17), (0, 5)], 8, 1, 128, BF, 16, 1, 0, 0),
    ([(1, 7000)], 4, 4, 64, BF, 64, 1, 0, 0),
    ([(4, 5000), (3, 40)], 3, 1, 128, BF, 32, 1, 2100, 9),
    ([(5, 4000)], 4, 2, 64, BF, 16, 1, 0, 0),
    ([(9, 2500)], 2, 1, 128, HF, 128, 1, 0, 0),
    ([(90, 1300)], 2, 1, 128, BF, 16, 90, 0, 0),
    ([(70, 900), (40, 20)], 3, 1, 64, BF, 32, 1, 500, 30),
    ([(150, 1000)], 1, 1, 128, HF, 64, 1, 0, 0),
])
def test_attention_within_the_closer_bounds(case):
    lens, Hq, Hk, D, dtype, page, block, window, sinks = case
    q, keys, values, c, s, table = make_code_case(87, lens, Hq, Hk, D, dtype, page)
    cache, batch = made(Hk, c.shape[0], page, D, dtype, c, s), batch_of(lens, table)
    want = attend_codes64_close(q, keys, values, lens, block, window, sinks, step=max(a for a, _ in lens) * (Hq // Hk) <= 32)
    for ws in (None, qwm.paged_attend_workspace(cache, batch, Hq, window, sinks, block)):
        out, lse = qwm.qwm_paged_attend(cache, batch, q.cuda(), window=window, sinks=sinks, block=block, want_lse=True, workspace=ws)
        compare(out, lse, want)
