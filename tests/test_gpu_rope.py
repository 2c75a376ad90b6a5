"""GPU: rotary positions over three axes against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2609_26425_gb300 as qwm
from paged_ref import inv_freq, rope64, rope_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    qwm.lib()


def positions(seed, n, most=5000):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, most, (n, 3), generator=g, dtype=torch.int32)


def check(got, x, pos, freq, pairs, il, sign):
    want = rope64(x, pos, freq, pairs, il, sign)
    bound = rope_bound(x, want, x.dtype, pairs, il)
    assert bool(((got.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("il", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,hq,hk,d,pairs", [
    (1, 1, 1, 128, (22, 21, 21)), (7, 5, 1, 128, (22, 21, 21)), (33, 12, 12, 64, (12, 10, 10)),
    (129, 3, 2, 128, (16, 16, 16)), (5, 2, 2, 256, (44, 42, 42)), (4, 40, 8, 128, (64, 0, 0)),
    (3, 2, 1, 40, (0, 8, 0)), (2, 33, 7, 8, (4, 0, 0)), (4099, 3, 1, 64, (8, 8, 8)),
])
def test_rope_matches_the_formula(n, hq, hk, d, pairs, dtype, il, backward):
    if sum(pairs) % (4 if il else 8):
        pytest.skip("pairs of this layout come in eights")
    g = torch.Generator().manual_seed(n * 131 + d)
    q, k = torch.randn(n, hq, d, generator=g).to(dtype), torch.randn(n, hk, d, generator=g).to(dtype)
    pos, freq = positions(n, n), inv_freq(pairs)
    rope = qwm.Rope(freq.cuda(), pairs, interleaved=il)
    if backward:
        a, b = qwm.qwm_rope_backward(rope, q.cuda(), pos.cuda(), dk=k.cuda())
    else:
        a, b = qwm.qwm_rope(rope, q.cuda(), pos.cuda(), k=k.cuda())
    sign = -1.0 if backward else 1.0
    check(a, q, pos, freq, pairs, il, sign)
    check(b, k, pos, freq, pairs, il, sign)
    rest = slice(2 * sum(pairs), None)
    assert torch.equal(a.cpu()[..., rest], q[..., rest])      # channels that are not rotated


@pytest.mark.parametrize("il", [True, False])
def test_large_and_negative_positions(il):
    # angles up to 2^31: the reduction keeps the fp32 accuracy of the reduced
    # angle while it is below 2^24, and 2^-17 of a turn beyond
    pairs = (32, 16, 16)
    pos = torch.tensor([[0, 0, 0], [-5, -70000, 3], [1 << 20, -(1 << 20), 12345677], [(1 << 24) + 3, 16777215, -16777217]],
                       dtype=torch.int32)
    x = torch.randn(4, 2, 128, generator=torch.Generator().manual_seed(3)).to(torch.float16)
    freq = inv_freq(pairs)
    rope = qwm.Rope(freq.cuda(), pairs, interleaved=il)
    check(qwm.qwm_rope(rope, x.cuda(), pos.cuda()), x, pos, freq, pairs, il, 1.0)
    far = torch.tensor([[(1 << 31) - 1, -(1 << 31), 1 << 30]], dtype=torch.int32)
    want = rope64(x[:1], far, freq, pairs, il)
    got = qwm.qwm_rope(rope, x[:1].cuda(), far.cuda()).double().cpu()
    assert bool(((got - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -14 * x[:1].double().abs().max()).all())


def test_strides_in_place_and_empty():
    pairs, d = (22, 21, 21), 128
    freq = inv_freq(pairs)
    rope = qwm.Rope(freq.cuda(), pairs)
    g = torch.Generator().manual_seed(9)
    n, hq, hk = 19, 6, 2
    qkv = torch.randn(n, hq + 2 * hk, d, generator=g).to(torch.bfloat16)
    pos = positions(4, n)
    dev = qkv.cuda()
    a, b = qwm.qwm_rope(rope, dev[:, :hq], pos.cuda(), k=dev[:, hq:hq + hk])       # slices of a projection
    check(a, qkv[:, :hq], pos, freq, pairs, True, 1.0)
    check(b, qkv[:, hq:hq + hk], pos, freq, pairs, True, 1.0)
    ht = qkv.permute(1, 0, 2).contiguous().cuda()                                  # head-major
    out = torch.empty(hq, n, d, dtype=torch.bfloat16, device="cuda")
    c = qwm.qwm_rope(rope, ht[:hq].permute(1, 0, 2), pos.cuda(), q_out=out.permute(1, 0, 2))
    assert torch.equal(c, a)
    x, y = dev[:, :hq], dev[:, hq:hq + hk]
    keep = dev[:, hq + hk:].clone()
    qwm.qwm_rope(rope, x, pos.cuda(), k=y, q_out=x, k_out=y)                       # in place
    assert torch.equal(x, a) and torch.equal(y, b) and torch.equal(dev[:, hq + hk:], keep)
    none = torch.empty(0, hq, d, dtype=torch.bfloat16, device="cuda")
    assert qwm.qwm_rope(rope, none, torch.empty(0, 3, dtype=torch.int32, device="cuda")).shape == (0, hq, d)


def test_gradient_against_the_formula_and_differences():
    pairs, d, n, h = (12, 10, 10), 64, 5, 3
    freq, pos = inv_freq(pairs), positions(1, n)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(n, h, d, generator=g).to(torch.float16)
    dy = torch.randn(n, h, d, generator=g).to(torch.float16)
    for il in (True, False):
        rope = qwm.Rope(freq.cuda(), pairs, interleaved=il)
        dx = qwm.qwm_rope_backward(rope, dy.cuda(), pos.cuda()).double().cpu()
        # autograd of the formula
        z = x.double().requires_grad_(True)
        axis = [a for a in range(3) for _ in range(pairs[a])]
        t = (pos[:, axis].double() * freq.double())[:, None]
        P = len(axis)
        ia = torch.arange(P) * (2 if il else 1)
        ib = ia + (1 if il else P)
        loss = (torch.cat([z[..., ia] * t.cos() - z[..., ib] * t.sin(), z[..., ia] * t.sin() + z[..., ib] * t.cos()], -1)
                * torch.cat([dy[..., ia], dy[..., ib]], -1).double()).sum()
        loss.backward()
        bound = rope_bound(dy, z.grad, torch.float16, pairs, il)
        assert bool(((dx - z.grad).abs() <= bound).all())
        # central differences of the 64-bit formula (linear in x: exact to rounding)
        for idx in ((0, 0, 0), (1, 2, 5), (4, 1, d - 1), (2, 0, 33)):
            e = torch.zeros(n, h, d, dtype=torch.float64)
            e[idx] = 1e-3
            f = lambda v: float((rope64(v, pos, freq, pairs, il) * dy.double()).sum())
            num = (f(x.double() + e) - f(x.double() - e)) / 2e-3
            assert abs(num - float(dx[idx])) <= float(bound[idx]) + 1e-8


def test_nonfinite_values_stay_in_their_pairs():
    pairs, d = (22, 21, 21), 128
    rope = qwm.Rope(inv_freq(pairs).cuda(), pairs)
    x = torch.ones(2, 2, d, dtype=torch.bfloat16, device="cuda")
    x[1, 0, 10] = math.inf
    x[0, 1, 3] = math.nan
    y = qwm.qwm_rope(rope, x, torch.ones(2, 3, dtype=torch.int32, device="cuda"))
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, 10:12] = True
    want[0, 1, 2:4] = True
    assert torch.equal(bad, want)


def test_refusals():
    pairs = (22, 21, 21)
    rope = qwm.Rope(inv_freq(pairs).cuda(), pairs)
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        qwm.qwm_rope(rope, x.float(), pos)
    with pytest.raises(ValueError):
        qwm.qwm_rope(rope, x, pos[:3])
    with pytest.raises(ValueError):
        qwm.qwm_rope(rope, x, pos.long())
    with pytest.raises(ValueError):
        qwm.qwm_rope(rope, x, pos, k=x.half())
    with pytest.raises(ValueError):
        qwm.qwm_rope(rope, x.transpose(1, 2), pos)                      # channels not contiguous
    with pytest.raises(qwm.QwmError) as e:
        qwm.qwm_rope(rope, x[..., :64].contiguous(), pos)               # 64 pairs in 64 channels
    assert e.value.status == 2
    odd = torch.zeros(4 * 2 * 132, dtype=torch.bfloat16, device="cuda").as_strided((4, 2, 128), (264, 132, 1))
    with pytest.raises(qwm.QwmError) as e:
        qwm.qwm_rope(rope, odd, pos)                                    # strides that are no multiple of 8
    assert e.value.status == 1
    with pytest.raises(qwm.QwmError) as e:
        qwm.qwm_rope(rope, x, pos, q_out=x[:1].expand(4, 2, 128))       # rows that share memory
    assert e.value.status == 1
    with pytest.raises(ValueError):
        qwm.Rope(inv_freq(pairs), pairs)                                # not on the GPU
    with pytest.raises(ValueError):
        qwm.Rope(inv_freq(pairs).cuda(), (22, 21, 20))


@pytest.mark.parametrize("token,head,heads,n", [
    (256, 128, 2, 5), (128, 640, 2, 5), (264, 136, 2, 5),      # token-major, head-major, padded
    (384, 256, 2, 4), (136, 272, 2, 2),                        # rows of one axis between those of the other
    (8, 8, 1, 1), (128, 0, 1, 5)])                             # a stride that is never used
def test_outputs_of_any_order_whose_rows_are_apart(token, head, heads, n):
    pairs = (22, 21, 21)
    freq, pos = inv_freq(pairs), positions(6, n)
    rope = qwm.Rope(freq.cuda(), pairs)
    x = torch.randn(n, heads, 128, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    flat = torch.full(((n - 1) * token + (heads - 1) * head + 128,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = flat.as_strided((n, heads, 128), (token, head, 1))
    assert qwm.qwm_rope(rope, x.cuda(), pos.cuda(), q_out=out) is out
    check(out, x, pos, freq, pairs, True, 1.0)
    assert int((flat == 7.0).sum()) >= flat.numel() - x.numel()


@pytest.mark.parametrize("il", [True, False])
@pytest.mark.parametrize("span,fastest", [(1 << 31, 1.0), (1 << 24, 1.0), (1 << 22, 900.0), (5000, 3.0e6), (1 << 31, 1e-7)])
def test_every_position_is_turned_to_fp32_accuracy(span, fastest, il):
    """The same bound as for small positions; the 64-bit formula's own product of a
    position and a frequency is good to 2^-23 here."""
    pairs, n = (32, 16, 16), 64
    g = torch.Generator().manual_seed(5)
    pos = torch.randint(-span, span, (n, 3), generator=g).to(torch.int32)
    pos[0] = torch.tensor([span - 1, -span, 0])
    x = torch.randn(n, 4, 128, generator=g).to(torch.float16)
    freq = inv_freq(pairs) * fastest
    freq[3] = -freq[3]
    got = qwm.qwm_rope(qwm.Rope(freq.cuda(), pairs, interleaved=il), x.cuda(), pos.cuda())
    check(got, x, pos, freq, pairs, il, 1.0)


def test_a_frequency_that_is_not_finite_is_nan_in_its_pairs():
    pairs = (22, 21, 21)
    freq = inv_freq(pairs)
    freq[3], freq[9] = math.inf, math.nan
    x = torch.ones(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    y = qwm.qwm_rope(qwm.Rope(freq.cuda(), pairs), x, torch.ones(2, 3, dtype=torch.int32, device="cuda"))
    bad = torch.zeros(128, dtype=torch.bool)
    bad[6:8] = bad[18:20] = True
    assert torch.equal(y.isnan().cpu(), bad.expand(2, 2, 128))


def test_a_call_that_fails_gives_back_what_it_made():
    """Keys too large to allocate an output for, after the Queries' output was made."""
    pairs, n = (4, 0, 0), 1 << 20
    rope = qwm.Rope(inv_freq(pairs).cuda(), pairs)
    x = torch.zeros(1, 1, 8, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(n, 3, dtype=torch.int32, device="cuda")
    before = torch.cuda.memory_allocated()
    with pytest.raises(MemoryError):
        qwm.qwm_rope(rope, x.expand(n, 1, 8), pos, k=x.expand(n, n, 8))
    with pytest.raises(qwm.QwmError):
        qwm.qwm_rope(qwm.Rope(rope.inv_freq, (4, 0, 0), interleaved=False), x.expand(n, 1, 8), pos)
    assert torch.cuda.memory_allocated() == before


def formula(x, pos, freq, pairs, il):
    """The rotation in torch operations in 64 bits, for autograd."""
    axis = [a for a in range(3) for _ in range(pairs[a])]
    t, P = (pos[:, axis].double() * freq.double())[:, None], sum(pairs)
    ia = torch.arange(P) * (2 if il else 1)
    ib = ia + (1 if il else P)
    y = x.clone()
    y[..., ia] = x[..., ia] * t.cos() - x[..., ib] * t.sin()
    y[..., ib] = x[..., ia] * t.sin() + x[..., ib] * t.cos()
    return y


@pytest.mark.parametrize("il", [True, False])
@pytest.mark.parametrize("wants", ["q", "k", "both"])
@pytest.mark.parametrize("layout", ["dense", "slices", "head-major"])
def test_autograd_records_the_rotation(layout, wants, il):
    pairs, d, n, hq, hk = (12, 10, 10), 72, 7, 3, 2
    freq, pos = inv_freq(pairs), positions(31, n)
    rope = qwm.Rope(freq.cuda(), pairs, interleaved=il)
    g = torch.Generator().manual_seed(32)
    qkv = torch.randn(n, hq + hk, d, generator=g).to(torch.float16)
    dy = torch.randn(n, hq + hk, d, generator=g).to(torch.float16)
    q, k = qkv[:, :hq].clone(), qkv[:, hq:].clone()
    if layout == "slices":
        base = qkv.cuda()
        dq, dk = base[:, :hq], base[:, hq:]
    elif layout == "head-major":
        dq, dk = (t.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2) for t in (q, k))
    else:
        dq, dk = q.cuda(), k.cuda()
    dq, dk = dq.detach().requires_grad_(wants != "k"), dk.detach().requires_grad_(wants != "q")
    a, b = qwm.qwm_rope(rope, dq, pos.cuda(), k=dk)
    with torch.no_grad():
        plain = qwm.qwm_rope(rope, dq, pos.cuda(), k=dk)
    assert torch.equal(a, plain[0]) and torch.equal(b, plain[1])
    assert not plain[0].requires_grad and a.requires_grad and b.requires_grad
    ((a * dy[:, :hq].cuda()).sum() + (b * dy[:, hq:].cuda()).sum()).backward()
    for x, got, w in ((q, dq.grad, dy[:, :hq]), (k, dk.grad, dy[:, hq:])):
        if got is None:
            continue
        z = x.double().requires_grad_(True)
        (formula(z, pos, freq, pairs, il) * w.double()).sum().backward()
        bound = rope_bound(w, z.grad, torch.float16, pairs, il)
        assert bool(((got.double().cpu() - z.grad).abs() <= bound).all())
    assert (dq.grad is None) == (wants == "k") and (dk.grad is None) == (wants == "q")


def test_autograd_in_place_and_through_expanded_gradients():
    pairs, d, n, h = (22, 21, 21), 128, 5, 3
    freq, pos = inv_freq(pairs), positions(33, n).cuda()
    rope = qwm.Rope(freq.cuda(), pairs)
    x = torch.randn(n, h, d, generator=torch.Generator().manual_seed(34)).to(torch.bfloat16).cuda().requires_grad_(True)
    qwm.qwm_rope(rope, x, pos).sum().backward()                        # a gradient whose strides are 0
    want, x.grad = x.grad, None
    assert torch.equal(want, qwm.qwm_rope_backward(rope, torch.ones_like(x).detach(), pos))
    y = x * 1.0
    assert qwm.qwm_rope(rope, y, pos, q_out=y) is y                    # in place
    y.sum().backward()
    assert torch.equal(x.grad, want)
    x.grad = None
    z, given = x * 1.0, torch.empty_like(x).detach()
    assert qwm.qwm_rope(rope, z, pos, q_out=given) is given            # into a tensor of the caller's
    given.sum().backward()
    assert torch.equal(x.grad, want)
    with pytest.raises(RuntimeError, match="leaf"):
        qwm.qwm_rope(rope, x, pos, q_out=x)
    y = x * 1.0
    square = y * y
    with torch.no_grad():
        qwm.qwm_rope(rope, y, pos, q_out=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        square.sum().backward()


def test_the_gradient_has_a_gradient():
    pairs, d, n, h = (8, 8, 8), 64, 4, 2
    pos, rope = positions(35, n).cuda(), qwm.Rope(inv_freq(pairs).cuda(), pairs, interleaved=False)
    g = torch.Generator().manual_seed(36)
    x, v, w = (torch.randn(n, h, d, generator=g).to(torch.float16).cuda() for _ in range(3))
    x.requires_grad_(True), v.requires_grad_(True)
    back, = torch.autograd.grad(qwm.qwm_rope(rope, x, pos), x, v, create_graph=True)
    assert torch.equal(back, qwm.qwm_rope_backward(rope, v.detach(), pos))
    again, = torch.autograd.grad(back, v, w)
    assert torch.equal(again, qwm.qwm_rope(rope, w, pos))
