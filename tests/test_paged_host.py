"""Host-only checks of the rotary and paged entry points: sizes and refusals that
need no GPU (every call here returns before anything is launched)."""
import contextlib
import ctypes as ct
import types

import pytest
import torch

from paper_2609_26425_gb300 import paged


@pytest.fixture(scope="module")
def L():
    from paper_2609_26425_gb300 import build
    build.build()
    import paper_2609_26425_gb300 as qwm
    return qwm.lib()


def rows(heads=2, data=4096, token=256, head=128):
    return paged.QwmRows(data, token, head, heads)


def test_buffer_holds_a_header_and_the_pages(L):
    for hk, d, t, n in ((8, 128, 64, 5), (1, 64, 16, 1), (40, 128, 128, 1000)):
        assert L.qwm_paged_bytes(paged.QwmPagedConfig(hk, d, t, 0, n)) == 256 + n * 2 * hk * t * d * 2
    for hk, d, t, dt, n in ((0, 128, 64, 0, 5), (8, 96, 64, 0, 5), (8, 128, 24, 0, 5), (8, 128, 256, 0, 5),
                            (8, 128, 64, 2, 5), (8, 128, 64, 0, 0), (4096, 128, 16, 0, 1 << 19)):
        assert L.qwm_paged_bytes(paged.QwmPagedConfig(hk, d, t, dt, n)) == 0


def test_rope_refusals(L):
    def call(pairs=(22, 21, 21), d=128, dt=0, il=1, n=4, q=None, qo=None, k=None, ko=None, freq=4096, pos=4096):
        cfg = paged.QwmRopeConfig(d, dt, (ct.c_int32 * 3)(*pairs), il)
        return L.qwm_rope(cfg, freq, pos, n, q or rows(), qo or rows(), k, ko, None)

    assert call(n=0) == 0                                   # nothing to do
    assert call(n=0, freq=None, pos=None) == 0
    assert call(freq=None) == 1 and call(pos=None) == 1 and call(n=-1) == 1
    assert call(pairs=(22, 21, 22)) == 2                    # more channels than there are
    assert call(pairs=(0, 0, 0)) == 2 and call(pairs=(1, 1, 1)) == 2
    assert call(pairs=(4, 4, 4), il=0) == 2                 # halves come in eights
    assert call(pairs=(-4, 4, 4)) == 1
    assert call(d=264) == 2 and call(d=100) == 2 and call(dt=2) == 2
    assert call(q=rows(3)) == 1                             # heads differ
    assert call(q=rows(data=4098)) == 1 and call(q=rows(token=252)) == 1 and call(q=rows(head=-128)) == 1
    assert call(qo=rows(token=0)) == 1                      # written rows that share memory
    assert call(k=rows()) == 1                              # Keys in, none out


def test_calls_without_a_cache_or_a_batch_are_refused(L):
    b = paged.QwmPagedBatch(1, 1, 1, 1, 1, 4096, 4096, 4096)
    m = paged.QwmMask(1, 0, 0)
    assert L.qwm_paged_append(None, b, rows(), rows(), None, None, None, None, None, None) == 1
    assert L.qwm_paged_attend(None, b, rows(), m, 1.0, rows(), None, None, 0, None) == 1
    assert L.qwm_paged_attend_workspace_bytes(None, b, 2, m) == 0
    assert L.qwm_paged_set_wait_limit(None, 2000) == 1 and L.qwm_paged_set_idle_role(None, 0) == 1
    h = ct.c_void_p()
    assert L.qwm_paged_init(ct.byref(h), paged.QwmPagedConfig(8, 128, 64, 0, 5), None, 1 << 30, None) == 1
    assert L.qwm_paged_init(ct.byref(h), paged.QwmPagedConfig(8, 80, 64, 0, 5), 4096, 1 << 30, None) == 2
    assert L.qwm_paged_init(ct.byref(h), paged.QwmPagedConfig(8, 128, 64, 0, 5), 4097, 1 << 30, None) == 1
    assert L.qwm_paged_init(ct.byref(h), paged.QwmPagedConfig(8, 128, 64, 0, 5), 4096, 256, None) == 3


def test_written_rows_that_share_memory_are_refused(L):
    def call(token, head, heads, n):
        cfg = paged.QwmRopeConfig(128, 0, (ct.c_int32 * 3)(22, 21, 21), 1)
        return L.qwm_rope(cfg, 4096, 4096, n, rows(heads), rows(heads, token=token, head=head), None, None, None)

    assert call(128, 128, 2, 4) == 1                        # (n, 1) is (n + 1, 0)
    assert call(256, 128, 3, 4) == 1                        # (n, 2) is (n + 1, 0)
    assert call(128, 384, 2, 4) == 1                        # head-major, the last token is the next head's first
    assert call(384, 256, 4, 4) == 1                        # (2, 0) is (0, 3)
    assert call(120, 512, 2, 4) == 1 and call(512, 120, 2, 4) == 1


def test_outputs_over_their_inputs_are_refused(L):
    def call(at, token=256, head=128, token_out=256, head_out=128, n=4):
        cfg = paged.QwmRopeConfig(128, 0, (ct.c_int32 * 3)(22, 21, 21), 1)
        return L.qwm_rope(cfg, 4096, 4096, n, rows(2, data=1 << 20, token=token, head=head),
                          rows(2, data=(1 << 20) + 2 * at, token=token_out, head=head_out), None, None, None)

    assert call(128) == 1 and call(-256) == 1 and call(8) == 1         # a head, a token, a vector on
    assert call(0, token_out=512) == 1                                 # the same place, other strides
    assert call(64, token=1024, token_out=1024) == 1
    assert call(128, token=128, head=1024, token_out=128, head_out=1024) == 1


class Calls:
    """Stand-in for the library and for CUDA: which device was current in each call."""

    def __init__(self):
        self.current, self.seen = 0, []

    def qwm_paged_bytes(self, cfg):
        return 4096

    def qwm_paged_free(self, handle):
        pass

    def qwm_paged_init(self, handle, cfg, buf, n, stream):
        self.seen.append(("init", self.current, stream))
        handle._obj.value = 1
        return 0

    def qwm_paged_status(self, handle, v, stream):
        self.seen.append(("status", self.current, stream))
        return 0


class Buffer:
    device = torch.device("cuda:1")

    def data_ptr(self):
        return 1 << 20

    def view(self, *a):
        return self

    __getitem__ = view


def test_a_cache_is_made_and_read_with_its_own_device_current(monkeypatch):
    calls = Calls()

    @contextlib.contextmanager
    def device(d):
        before, calls.current = calls.current, torch.device(d).index
        yield
        calls.current = before

    monkeypatch.setattr(paged, "_C", calls)
    monkeypatch.setattr(torch, "empty", lambda *a, device, **k: Buffer() if device == Buffer.device else None)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d: types.SimpleNamespace(cuda_stream=0))
    cache = paged.PagedCache(2, 4, device="cuda:1")
    assert cache.status() == 0
    assert calls.seen == [("init", 1, 0), ("status", 1, 0)] and calls.current == 0
    cache.handle = None


class OnDevice(torch.Tensor):
    """An int32 tensor that is said to be on a device."""

    @staticmethod
    def __new__(cls, device, *shape):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=torch.int32, device=device)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError


@pytest.mark.parametrize("other", [0, 1, 2])
def test_a_batchs_tensors_are_on_one_device(other):
    t = [OnDevice("cuda:%d" % int(i == other), *shape) for i, shape in enumerate(((3,), (2,), (2, 5)))]
    with pytest.raises(ValueError, match="one device"):
        paged.PagedBatch(*t, 1, 64)


def test_a_binding_of_another_pytorch_is_built_again(L, monkeypatch):
    from paper_2609_26425_gb300 import build
    assert build.up_to_date()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.0")
        assert not build.up_to_date()
    with monkeypatch.context() as m:
        m.setattr(torch, "__file__", "/elsewhere/torch/__init__.py")
        assert not build.up_to_date()
    assert build.up_to_date()
