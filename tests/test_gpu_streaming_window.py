"""GPU: the streaming example, pages and 2-bit history together."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import streaming_window
    return streaming_window


def test_stream_in_pages_is_plain_attention(ex):
    """bf16 rotation (two roundings), P and output: 2^-8 each of values below 1."""
    out, _ = ex.run(heads=2, frames=4, compress=False)
    want = ex.plain(2, 4, 3, 3)
    assert (out.float() - want).abs().max().item() <= 4 * 2.0 ** -8
    assert (out.float() - want).abs().mean().item() <= 2.0 ** -10


def test_compressed_history_changes_the_outputs_little_and_only_where_it_is_seen(ex):
    full, _ = ex.run(heads=2, frames=5, window=3, compress=True)
    pages, _ = ex.run(heads=2, frames=5, window=5, compress=False)      # every frame in pages
    first = 3 * ex.FRAME                                                # frames whose history is all in pages
    assert torch.equal(full[:first], pages[:first])
    err = (full[first:].float() - pages[first:].float())
    # about half the keys are 2-bit ones: their Values' error (a group of 32's range
    # over 3, uniform: 0.4 of the Values' spread) averages out like the Values do
    assert err.norm().item() <= 0.6 * pages[first:].float().norm().item()
    assert bool(torch.isfinite(full).all())


@pytest.mark.parametrize("frames,window,tokens", [(5, 3, 3), (4, 2, 5), (2, 3, 2)])
def test_pages_and_history_are_the_whole_stream(ex, frames, window, tokens):
    """With Queries of zeros every token counts the same: a row's log-sum-exp is the log
    of the number of tokens it sees, to a few fp32 roundings (one token of 4400 more or
    less is 2.3e-4), and Values of one mark the tokens at the pages' lower end."""
    s = ex.Stream(2, frames, window, True)
    edge = max(0, frames - window) * ex.FRAME              # the first token that is never compressed
    for i in range(frames):
        q, k, v = ex.projected(i, ex.FRAME, 2)
        at = torch.arange(i * ex.FRAME, (i + 1) * ex.FRAME, device="cuda")
        v = ((at >= edge) & (at < edge + 8)).to(v.dtype)[:, None, None].expand_as(v).contiguous()
        s.step(torch.zeros_like(q), k, v, ex.FRAME)
        assert (s.lse - math.log(s.len)).abs().max().item() <= 1e-5
        if i + 1 < frames:
            s.leave()
    for t in range(tokens):
        q, k, v = ex.projected(1000 + t, 1, 2)
        out = s.step(torch.zeros_like(q), k, torch.zeros_like(v), 1, keep=False)
        assert (out.float() * s.len - 8).abs().max().item() <= 8 * 2.0 ** -7
        assert (s.lse - math.log(s.len)).abs().max().item() <= 1e-5
    assert s.cache.status() == 0 and s.history.status() == 0
