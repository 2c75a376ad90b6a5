"""GPU: the streaming example, pages and 2-bit history together."""
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
