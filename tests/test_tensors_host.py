"""Lists of tensors on the host: what the calls that take them refuse, before anything reaches a GPU."""
import ctypes as C
import os
import shutil
import subprocess
import types

import pytest
import torch

from paper_2302_08545_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, OK = -1, 0
NORM, SCALE, WS = 1 << 45, (1 << 45) + 4, 1 << 46      # addresses that no list here comes near
INF, NAN = float("inf"), float("nan")
T430 = [0, 3, 5, 7, 9, 11, 13, 14, 15, 17, 19, 21, 23, 25, 27, 30]


def _raw(data, numel, dtype):
    n = len(numel)
    return api.thc_tensors(n, (C.c_void_p * n)(*data), (C.c_uint64 * n)(*numel), (C.c_uint32 * n)(*dtype))


def _p(**kw):
    base = dict(d=1 << 12, block=1 << 10, n=4, b=4, g=30, t_p=2.1538746, seed=7, table=T430, agg_bits=8)
    base.update(kw)
    return api.make_params(**base)


def _every(t, p=None, want=EINVAL):
    """All four calls with this list and otherwise good arguments."""
    L, p = api.lib(), p or _p()
    r = C.byref(t) if t is not None else None
    assert L.thc_grad_norm(r, 0, 1.0, NORM, SCALE, WS, None) == want
    assert L.thc_grad_clip(r, 0, 1.0, NORM, SCALE, WS, None) == want
    assert L.thc_gather(C.byref(p), r, None, 1 << 44, None) == want
    assert L.thc_scatter(C.byref(p), 1 << 44, None, r, None) == want


def test_bad_lists_are_refused_by_every_call():
    _every(None)
    _every(_raw([0], [4], [0]))                               # no memory
    _every(_raw([4096, 4098], [4, 4], [0, 0]))                # binary32 on two bytes
    _every(_raw([4097], [4], [1]))                            # bf16 on one byte
    _every(_raw([4096], [4], [3]))                            # no such type
    _every(_raw([1 << 48], [4], [0]))                         # no device address
    _every(_raw([4096], [1 << 40], [0]))                      # too long, alone and together
    _every(_raw([4096, 1 << 43], [1 << 39, 1 << 39], [1, 1]))
    n = C.c_uint64(4)
    _every(api.thc_tensors(1, None, C.pointer(n), (C.c_uint32 * 1)(0)))
    _every(api.thc_tensors(1, (C.c_void_p * 1)(4096), None, (C.c_uint32 * 1)(0)))
    _every(api.thc_tensors(1, (C.c_void_p * 1)(4096), C.pointer(n), None))


@pytest.mark.parametrize("call", ["thc_grad_norm", "thc_grad_clip"])
def test_arguments_of_the_norm_calls(call):
    f, t = getattr(api.lib(), call), C.byref(_raw([4096], [4], [0]))
    assert f(t, 2, 1.0, NORM, SCALE, WS, None) == EINVAL and f(t, -1, 1.0, NORM, SCALE, WS, None) == EINVAL
    assert f(t, 0, -1.0, NORM, SCALE, WS, None) == EINVAL and f(t, 0, NAN, NORM, SCALE, WS, None) == EINVAL
    assert f(t, 0, 1.0, None, SCALE, WS, None) == EINVAL and f(t, 0, 1.0, NORM + 2, SCALE + 4, WS, None) == EINVAL
    assert f(t, 0, 1.0, NORM, SCALE + 2, WS, None) == EINVAL
    assert f(t, 0, 1.0, NORM, SCALE, None, None) == EINVAL and f(t, 0, 1.0, NORM, SCALE, WS + 8, None) == EINVAL
    # what is written lies apart: from each other, and from the tensors
    assert f(t, 0, 1.0, NORM, NORM, WS, None) == EINVAL
    end = WS + api.thc_norm_workspace_bytes() - 4
    assert f(t, 0, 1.0, end, SCALE, WS, None) == EINVAL and f(t, 0, 1.0, NORM, end, WS, None) == EINVAL
    assert f(t, 0, 1.0, 4096, SCALE, WS, None) == EINVAL and f(t, 0, 1.0, NORM, 4096 + 12, WS, None) == EINVAL
    assert f(t, 0, 1.0, NORM, None, 4096, None) == EINVAL


def test_arguments_of_the_flat_calls():
    L, p, t = api.lib(), C.byref(_p()), C.byref(_raw([4096], [4], [0]))
    assert L.thc_gather(p, t, None, None, None) == EINVAL and L.thc_gather(p, t, None, (1 << 44) + 8, None) == EINVAL
    assert L.thc_gather(p, t, 18, 1 << 44, None) == EINVAL
    assert L.thc_gather(p, t, (1 << 44) + 8, 1 << 44, None) == EINVAL          # a factor inside what is written
    assert L.thc_scatter(p, 1 << 44, 4096 + 12, t, None) == EINVAL
    assert L.thc_scatter(p, None, None, t, None) == EINVAL and L.thc_scatter(p, (1 << 44) + 8, None, t, None) == EINVAL
    assert L.thc_scatter(p, 1 << 44, 18, t, None) == EINVAL
    # one element more than the vector holds
    _full = _raw([4096], [(1 << 12) + 1], [0])
    assert L.thc_gather(p, C.byref(_full), None, 1 << 44, None) == EINVAL
    assert L.thc_scatter(p, 1 << 44, None, C.byref(_full), None) == EINVAL
    # parameters are validated as everywhere
    for bad, code in ((dict(d=1000), -1), (dict(table=[1] + T430[1:]), -2), (dict(n=9), -3), (dict(in_dtype=2), -1)):
        q = C.byref(_p(**bad))
        assert L.thc_gather(q, t, None, 1 << 44, None) == code and L.thc_scatter(q, 1 << 44, None, t, None) == code
    assert L.thc_gather(None, t, None, 1 << 44, None) == EINVAL and L.thc_scatter(None, 1 << 44, None, t, None) == EINVAL


@pytest.mark.parametrize("data,numel,dtype", [
    ([4096, 4096], [8, 8], [0, 0]),                           # the same tensor twice
    ([8192, 4096, 8190], [8, 2050, 8], [1, 1, 1]),            # not in the order of addresses, one byte pair shared
    ([4096, 4104], [3, 4], [0, 1]),                           # different types
    ([4096 * 400 + 8] + [4096 * (i + 300) for i in range(300)], [1] + [1024] * 300, [0] * 301),
])
def test_memory_written_twice_is_refused(data, numel, dtype):
    L, t = api.lib(), _raw(data, numel, dtype)
    assert L.thc_grad_clip(C.byref(t), 0, 1.0, NORM, SCALE, WS, None) == EINVAL
    assert L.thc_scatter(C.byref(_p(d=1 << 20)), 1 << 44, None, C.byref(t), None) == EINVAL


def test_tensors_that_overlap_the_flat_vector_are_refused():
    L, p = api.lib(), _p()
    flat, end = 1 << 20, (1 << 20) + (4 << 12)
    for at in (flat, flat - 4, end - 4):
        t = _raw([at], [4], [0])
        assert L.thc_gather(C.byref(p), C.byref(t), None, flat, None) == EINVAL
        assert L.thc_scatter(C.byref(p), flat, None, C.byref(t), None) == EINVAL
    half = _p(in_dtype=1)                                     # a bf16 vector ends earlier
    t = _raw([end - 4], [4], [0])
    assert L.thc_gather(C.byref(half), C.byref(_raw([flat + (2 << 12) - 2], [1], [1])), None, flat, None) == EINVAL
    assert L.thc_scatter(C.byref(half), flat, None, C.byref(t), None) == EINVAL   # the estimate is binary32 all the same


def test_workspace_of_a_norm():
    assert api.lib().thc_norm_workspace_bytes(None) == EINVAL
    assert 0 < api.thc_norm_workspace_bytes() <= 1 << 20


def test_struct_layout():
    assert C.sizeof(api.thc_tensors) == 32
    assert [getattr(api.thc_tensors, f).offset for f in ("count", "data", "numel", "dtype")] == [0, 8, 16, 24]


class _Gpu(torch.Tensor):
    """A CPU tensor that says it is on a GPU: the checks of make_tensors read no memory."""
    is_cuda = True

    def get_device(self):
        return getattr(self, "at", 0)


def _gpu(t, at=0):
    t = t.as_subclass(_Gpu)
    t.at = at
    return t


def test_make_tensors_takes_runs_of_memory_only():
    x = _gpu(torch.zeros(4, 6, 5))
    for ok in (x, x.permute(2, 0, 1), x[1:3], x[:, :1, :1][:1], _gpu(torch.zeros(2, 3, 4, 5).to(memory_format=torch.channels_last)),
               _gpu(torch.zeros(())), _gpu(torch.zeros(0)), _gpu(torch.zeros(7, dtype=torch.bfloat16))):
        t = api.make_tensors([_gpu(ok)])
        assert t.count == 1 and t.numel[0] == ok.numel()
    for bad in (x[:, :3], x[..., ::2], _gpu(torch.zeros(1).expand(4)), _gpu(torch.zeros(4, dtype=torch.float64)), torch.zeros(4),
                _gpu(torch.zeros(3, dtype=torch.int32)), 4096, types.SimpleNamespace(is_cuda=True)):
        with pytest.raises(ValueError):
            api.make_tensors([bad if not isinstance(bad, _Gpu) else _gpu(bad)])
    with pytest.raises(ValueError):
        api.make_tensors([_gpu(torch.zeros(4)), _gpu(torch.zeros(4), at=1)])
    assert api.make_tensors([]).count == 0


def test_lists_of_another_device_than_the_current_one_are_refused(monkeypatch):
    t = api.make_tensors([_gpu(torch.zeros(4), at=1)])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    for call in (lambda: api.thc_grad_norm(t, 0, 1.0, NORM, SCALE, WS), lambda: api.thc_grad_clip(t, 0, 1.0, NORM, SCALE, WS),
                 lambda: api.thc_gather(_p(), t, None, 1 << 44), lambda: api.thc_scatter(_p(), 1 << 44, None, t)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()


def test_buffers_of_another_type_size_or_place_are_refused():
    t, one = api.make_tensors([]), _gpu(torch.zeros(1))
    ws = _gpu(torch.zeros(api.thc_norm_workspace_bytes(), dtype=torch.uint8))
    bad = [torch.zeros(1), _gpu(torch.zeros(0)), _gpu(torch.zeros(1, dtype=torch.float64))]
    for b in bad:
        for call in (api.thc_grad_norm, api.thc_grad_clip):
            with pytest.raises(ValueError, match="norm_out"):
                call(t, 0, 1.0, b, one, ws, stream=0)
            with pytest.raises(ValueError, match="scale_out"):
                call(t, 0, 1.0, one, b, ws, stream=0)
    with pytest.raises(ValueError, match="ws"):
        api.thc_grad_norm(t, 0, 1.0, one, None, ws[:-1], stream=0)
    p = _p()
    for flat in (torch.zeros(1 << 12), _gpu(torch.zeros((1 << 12) - 1)), _gpu(torch.zeros(1 << 12, dtype=torch.bfloat16)),
                 _gpu(torch.zeros(1 << 13))[::2]):
        with pytest.raises(ValueError, match="grad_out"):
            api.thc_gather(p, t, None, flat, stream=0)
        with pytest.raises(ValueError, match="flat"):
            api.thc_scatter(p, flat, None, t, stream=0)
    with pytest.raises(ValueError, match="grad_out"):
        api.thc_gather(_p(in_dtype=1), t, None, _gpu(torch.zeros(1 << 12)), stream=0)


def test_buffers_of_another_device_than_the_lists_are_refused(monkeypatch):
    here, there = _gpu(torch.zeros(1)), _gpu(torch.zeros(1), at=1)
    ws = _gpu(torch.zeros(api.thc_norm_workspace_bytes(), dtype=torch.uint8))
    far_ws = _gpu(torch.zeros(api.thc_norm_workspace_bytes(), dtype=torch.uint8), at=1)
    flat, far = _gpu(torch.zeros(1 << 12)), _gpu(torch.zeros(1 << 12), at=1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    p = _p()
    full = api.make_tensors([_gpu(torch.zeros(4))])
    for t, stream in ((full, 0), (full, None), (api.make_tensors([]), None)):
        for call in (api.thc_grad_norm, api.thc_grad_clip):
            for norm, scale, work in ((there, here, ws), (here, there, ws), (here, None, far_ws)):
                with pytest.raises(ValueError, match="cuda:0"):
                    call(t, 0, 1.0, norm, scale, work, stream=stream)
        for scale, vector in ((there, flat), (None, far)):
            with pytest.raises(ValueError, match="cuda:0"):
                api.thc_gather(p, t, scale, vector, stream=stream)
            with pytest.raises(ValueError, match="cuda:0"):
                api.thc_scatter(p, vector, scale, t, stream=stream)


def test_a_tensor_whose_memory_holds_its_negative_is_refused():
    x = torch.view_as_complex(torch.ones(1, 2)).conj().imag          # one element, -1, stored as 1
    assert x.is_neg() and float(x) == -1.0
    with pytest.raises(ValueError, match="negative"):
        api.make_tensors([_gpu(x)])


def test_tables_of_a_list_are_clean_under_asan_and_ubsan(tmp_path):
    """The tables that travel with the launches, walked on the CPU as the kernels walk them: every element once, nothing outside."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "san_tensors"
    subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
                    "-static-libubsan", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2302_08545_amd", "csrc"), os.path.join(ROOT, "tests", "san_tensors.cpp"), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "0 problem(s)" in res.stdout
