"""Host-only checks of the 8-bit paged storage: sizes, refusals that need no GPU (every call
here returns before anything is launched), and the 64-bit reference itself."""
import ctypes as ct
import types

import pytest
import torch

from codes_ref import MOST, VALUE, quantise64, scale64, stands_for
from paper_2609_26425_gb300 import paged


@pytest.fixture(scope="module")
def L():
    from paper_2609_26425_gb300 import build
    build.build()
    import paper_2609_26425_gb300 as qwm
    return qwm.lib()


def rows(heads=2, data=4096, token=256, head=128):
    return paged.QwmRows(data, token, head, heads)


def test_buffer_holds_a_header_the_codes_and_the_scales(L):
    for hk, d, t, n in ((8, 128, 64, 5), (1, 64, 16, 1), (40, 128, 128, 1000)):
        assert L.qwm_paged_bytes_e4m3(paged.QwmPagedConfig(hk, d, t, 0, n)) == 256 + n * 2 * hk * t * (d + 2)
    for hk, d, t, dt, n in ((0, 128, 64, 0, 5), (8, 96, 64, 0, 5), (8, 128, 24, 0, 5), (8, 128, 256, 0, 5),
                            (8, 128, 64, 2, 5), (8, 128, 64, 0, 0), (4096, 128, 16, 0, 1 << 19)):
        assert L.qwm_paged_bytes_e4m3(paged.QwmPagedConfig(hk, d, t, dt, n)) == 0


def test_calls_without_a_cache_a_batch_or_an_output_are_refused(L):
    b = paged.QwmPagedBatch(1, 1, 1, 1, 1, 4096, 4096, 4096)
    assert L.qwm_paged_read(None, b, rows(), rows(), None) == 1
    cfg, h = paged.QwmPagedConfig(8, 128, 64, 0, 5), ct.c_void_p()
    assert L.qwm_paged_init_e4m3(ct.byref(h), cfg, None, 1 << 30, None) == 1
    assert L.qwm_paged_init_e4m3(ct.byref(h), paged.QwmPagedConfig(8, 80, 64, 0, 5), 4096, 1 << 30, None) == 2
    assert L.qwm_paged_init_e4m3(ct.byref(h), cfg, 4097, 1 << 30, None) == 1
    n = L.qwm_paged_bytes_e4m3(cfg)
    assert L.qwm_paged_init_e4m3(ct.byref(h), cfg, 4096, n - 1, None) == 3
    assert L.qwm_paged_bytes(cfg) > n                      # (and 16-bit pages do not fit it)
    assert L.qwm_paged_init(ct.byref(h), cfg, 4096, n, None) == 3 and not h.value


def test_storage_is_the_dtype_or_e4m3():
    for bad in (torch.int8, torch.float8_e5m2, torch.float16):
        with pytest.raises(ValueError, match="storage"):
            paged.PagedCache(2, 4, dtype=torch.bfloat16, storage=bad, device="cuda:0")


def test_a_read_of_unknown_length_or_of_wrong_outputs_is_refused():
    read = paged.binding().read
    cache = types.SimpleNamespace(_key=(0, 128, 0, 0), kv_heads=2)
    b = paged.QwmPagedBatch(1, 1, 1, 1, 1, 4096, 4096, 4096)
    at = ct.addressof(b)
    any_rows, three = (at, -1, 0), (at, 3, 0)
    with pytest.raises(ValueError, match="not known"):
        read(cache._key, any_rows, 2, -1, None, None)
    with pytest.raises(ValueError, match="another device"):
        read(cache._key, (at, 3, 1), 2, -1, None, None)
    for bad in (7, "k", torch.zeros(3, 2, 128)):           # not a tensor; not on the GPU
        with pytest.raises(ValueError):
            read(cache._key, any_rows, 2, 3, bad, False)
    with pytest.raises(ValueError):
        read(cache._key, three, 2, -2, None, None)
    with pytest.raises(TypeError):
        read(cache._key, three, 2, 3, None)


def test_reference_quantiser():
    """Pins of the reference: hand-made rows, its bound, and PyTorch's own conversion."""
    x = torch.zeros(4, 64, dtype=torch.float64)
    x[0, :4] = torch.tensor([448.0, 17.0, 19.0, -1.0])     # scale 1: 17 and 19 are ties (16, 18, 20)
    x[1, :2] = torch.tensor([449.0, 2.0 ** -9])            # scale 2: 2^-10 is half the least code, a tie with 0
    x[2, 0] = 1e9
    c, s = quantise64(x)
    v = stands_for(c, s)
    assert s.tolist() == [1.0, 2.0, 256.0, 2.0 ** -15]
    assert v[0, :4].tolist() == [448.0, 16.0, 20.0, -1.0] and v[1, :2].tolist() == [448.0, 0.0]
    assert v[2, 0] == MOST and not bool(v[3].any())
    g = torch.Generator().manual_seed(1)
    y = torch.randn(500, 64, generator=g).double() * torch.exp2(torch.rand(500, 1, generator=g) * 30 - 20)
    c, s = quantise64(y)
    y = y.clamp(-MOST, MOST)
    assert torch.equal((y / s[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8), c)
    assert bool(((stands_for(c, s) - y).abs() <= torch.maximum(y.abs() * 2.0 ** -4, s[:, None] * 2.0 ** -10)).all())
    for t in (torch.bfloat16, torch.float16):              # every code at every scale is exact in both types
        for e in range(-15, 9):
            w = VALUE[:127] * 2.0 ** e
            ok = w <= MOST
            assert torch.equal(w[ok].to(t).double(), w[ok])
    assert torch.equal(scale64(y), s)
