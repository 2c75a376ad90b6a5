"""GPU: paged storage in 8 bits at its edges -- rings that turn many times, ranges, scales of a
caller's own, and the paths that only large calls take -- against the definitions in 64 bits
(tests/codes_ref.py)."""
import math

import pytest
import torch

import paper_2609_26425_gb300 as qwm
from paged_ref import offsets

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
