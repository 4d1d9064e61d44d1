"""What the binding of the calls on lists checks before it hands raw addresses on: streams, devices, storage."""
import gc
import types
import weakref

import numpy as np
import pytest
import torch

from paper_2302_08545_amd import api

from .test_tensors_host import NORM, SCALE, WS, _Gpu, _gpu, _p


def _calls(t, **kw):
    p = _p()
    return (lambda: api.thc_grad_norm(t, 0, 1.0, NORM, SCALE, WS, **kw), lambda: api.thc_grad_clip(t, 0, 1.0, NORM, SCALE, WS, **kw),
            lambda: api.thc_gather(p, t, None, 1 << 44, **kw), lambda: api.thc_scatter(p, 1 << 44, None, t, **kw))


def _current(monkeypatch, device):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: device, raising=False)


def _stream(handle, device):
    return types.SimpleNamespace(cuda_stream=handle, device=torch.device("cuda", device))


def test_streams_of_another_device_than_the_lists_are_refused(monkeypatch):
    """The null stream is the current device's, whoever hands it on; other streams say whose they are."""
    _current(monkeypatch, 0)
    t = api.make_tensors([_gpu(torch.zeros(4), at=1)])
    for stream in (0, _stream(0, 1), _stream(0, 0), _stream(4096, 0)):
        for call in _calls(t, stream=stream):
            with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
                call()


def test_buffers_of_an_empty_list_have_to_be_on_the_streams_device(monkeypatch):
    _current(monkeypatch, 0)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    here, there = _gpu(torch.zeros(1)), _gpu(torch.zeros(1), at=1)
    ws = _gpu(torch.zeros(api.thc_norm_workspace_bytes(), dtype=torch.uint8))
    for call in (api.thc_grad_norm, api.thc_grad_clip):
        for norm, scale in ((there, here), (here, there)):
            for stream in (_stream(4096, 0), _stream(0, 0), 0):
                with pytest.raises(ValueError, match="cuda:0"):
                    call([], 0, 1.0, norm, scale, ws, stream=stream)


def test_buffers_whose_memory_holds_their_negative_are_refused():
    x = _gpu(torch.view_as_complex(torch.ones(1, 2)).conj().imag)          # one float, -1, stored as 1
    assert x.is_neg() and x.is_contiguous() and float(x) == -1.0
    t, one, p = api.make_tensors([]), _gpu(torch.zeros(1)), _p()
    ws = _gpu(torch.zeros(api.thc_norm_workspace_bytes(), dtype=torch.uint8))
    flat = _gpu(torch.zeros(1 << 12))
    for call in (api.thc_grad_norm, api.thc_grad_clip):
        with pytest.raises(ValueError, match="norm_out"):
            call(t, 0, 1.0, x, one, ws, stream=0)
        with pytest.raises(ValueError, match="scale_out"):
            call(t, 0, 1.0, one, x, ws, stream=0)
    with pytest.raises(ValueError, match="scale"):
        api.thc_gather(p, t, x, flat, stream=0)
    with pytest.raises(ValueError, match="scale"):
        api.thc_scatter(p, flat, x, t, stream=0)


def test_a_list_keeps_the_memory_that_it_describes():
    """A tensor that is given other storage leaves its addresses in the list: the memory there has to stay allocated."""
    memory = np.zeros(64, dtype=np.float32)
    seen, at = weakref.ref(memory), memory.ctypes.data
    g = torch.Tensor._make_subclass(_Gpu, torch.from_numpy(memory))        # no view, which would keep the tensor it is of
    t = api.make_tensors([g])
    del memory
    g.data = torch.ones(64)
    gc.collect()
    alive = seen() is not None
    assert alive and t.data[0] == at
    del t
    gc.collect()
    alive = seen() is not None
    assert not alive
