"""Clipping of lists above 128 MB, whose scaling is a launch of its own that reads the factor back from device memory, from the caller's
place or from the workspace; odd starts, mixed types, several tables; and the same list in another place.

Bars, derived from the definitions:
  norm    L2: a thread adds at most 1024 + 32 squares one after another (lists of up to 2^28 bytes: 32 units of 32 KB a workgroup, at most
          32 elements of a unit a thread, and edges), then come at most 6 + 8 joins in the workgroup, 2 launches and 4 + 6 of the partials.
          All terms are positive, so each of fewer than 2^11 additions costs at most 2^-53 relative: 2^-42, halved by the root.  The
          reference adds up 2^16 squares at a time in binary64, in whatever order (2^-37, halved), and these sums exactly.  Then the
          rounding to binary32: half a step, 2^-24.  MAX: no rounding at all.
  factor  limit / norm in binary64, rounded once: the same.
  moves   round(fl32(x * c)) with the factor that the call itself used: the same bits.
"""
import math

import numpy as np
import pytest
import torch

from paper_2302_08545_amd import api

from .test_gpu_tensors import BF16, DEV, F16, F32, NAN, Tensors

pytestmark = pytest.mark.gpu
REL = 2.0 ** -24 + 2.0 ** -36
MOST = 128 << 20                      # bytes up to which a list is scaled behind its norm
GUARD = 170


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "these tests need the GPU"
    api.lib()
    yield
    torch.cuda.synchronize()


def _sizes(lists, types):
    """Sizes of tensors that take a little more than 128 MB together."""
    wide = sum(t.itemsize for t in types) / len(types)
    if lists == "few":
        return [int(MOST / types[0].itemsize) + 1003, 17, 250, 3]
    return [int(MOST / wide / 300) + 500 + (i * 37) % 300 for i in range(300)]


def _list(lists, types, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    parts = []
    for i, n in enumerate(_sizes(lists, types)):
        x = torch.randn(n, generator=gen, device=DEV) * 10.0 ** ((i * 7) % 5 - 2)
        parts.append(x.to(types[i % len(types)]))
    X = Tensors(parts, (1, 3, 0, 7, 2))
    assert MOST < sum(x.numel() * x.element_size() for x in parts) <= 1 << 28
    return X


def _norm64(parts, kind):
    if kind == api.THC_NORM_MAX:
        return max(float(x.abs().max()) for x in parts)
    sums = []
    for x in parts:
        q = x.double().square()
        cut = q.numel() >> 16 << 16
        sums += q[:cut].reshape(-1, 1 << 16).sum(dim=1).tolist() + [float(q[cut:].sum())]
    return math.sqrt(math.fsum(sums))


def _buffers():
    """norm, factor, and a workspace of exactly the size asked for, with guard bytes before and behind it"""
    size = api.thc_norm_workspace_bytes()
    whole = torch.full((size + 512,), GUARD, dtype=torch.uint8, device=DEV)
    return torch.full((1,), NAN, device=DEV), torch.full((1,), NAN, device=DEV), whole[256:256 + size], whole


def _guards(whole):
    assert bool((whole[:256] == GUARD).all()) and bool((whole[-256:] == GUARD).all())


@pytest.mark.parametrize("kind", [api.THC_NORM_L2, api.THC_NORM_MAX], ids=["l2", "max"])
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (F32, BF16, F16)], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("lists", ["few", "tables"])
def test_clipping_with_and_without_a_place_for_the_factor(lists, types, kind):
    for given in (True, False):
        X = _list(lists, types, seed=51)
        v = _norm64(X.cpu, kind)
        limit = float(np.float32(v * 0.37))
        norm, scale, ws, whole = _buffers()
        api.thc_grad_clip(X.gpu, kind, limit, norm, scale if given else None, ws)
        assert abs(float(norm) - v) <= (0.0 if kind == api.THC_NORM_MAX else v * REL)
        if given:
            c = float(scale)
            assert abs(c - limit / v) <= limit / v * REL
        for x, g in zip(X.cpu, X.gpu):
            assert torch.equal(g, (x.float() * torch.tensor(c, dtype=F32, device=DEV)).to(x.dtype))
        X.guards_hold()
        _guards(whole)
        norm, scale, ws, whole = _buffers()           # below the limit: nothing is written
        before = [g.clone() for g in X.gpu]
        api.thc_grad_clip(X.gpu, kind, limit * 2.0, norm, scale if given else None, ws)
        assert not given or float(scale) == 1.0
        assert all(torch.equal(a, g) for a, g in zip(before, X.gpu))
        X.guards_hold()
        _guards(whole)


def test_a_long_list_clipped_in_a_captured_graph_without_a_place_for_the_factor():
    X = _list("few", (F32, BF16), seed=52)
    t = api.make_tensors(X.gpu)
    norm, _, ws, whole = _buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.thc_grad_clip(t, api.THC_NORM_L2, 2.5, norm, None, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.thc_grad_clip(t, api.THC_NORM_L2, 2.5, norm, None, ws)
    del t
    for k in range(3):
        for x, g in zip(X.cpu, X.gpu):
            g.copy_((x.float() * (k + 1)).to(x.dtype))
        Y = [g.clone() for g in X.gpu]
        graph.replay()
        n2, c2, w2, _ = _buffers()
        api.thc_grad_norm(X.gpu, api.THC_NORM_L2, 2.5, n2, c2, w2)
        torch.cuda.synchronize()
        v = _norm64(Y, api.THC_NORM_L2)
        assert abs(float(norm) - v) <= v * REL
        c = norm.new_tensor(float(np.float32(2.5 / v)))
        # the factor of the call is within half a step and the sums' slack of 2.5 / v: itself, or a neighbour of its rounding
        near = [torch.nextafter(c, c * 0), c, torch.nextafter(c, c * 2)]
        hits = [all(torch.equal((y.float() * f).to(y.dtype), g) for y, g in zip(Y, X.gpu)) for f in near]
        assert any(hits)
        assert abs(float(n2) - 2.5) <= 2.5 * 2.0 ** -7          # clipped to the limit, up to the roundings of bf16
        X.guards_hold()
        _guards(whole)


def test_the_same_list_further_on_has_the_same_norm():
    """Values whose sum depends on its order in every bit that counts: beside 2^24 squares of 2^-3 are lost one by one and kept together.
    The tensors keep their addresses modulo 128 bytes and what adjoins; everything else about their places changes."""
    sizes, gaps = [9000, 777, 0, 20_011, 5, 33_000, 64], [0, 0, 0, 32, 0, 3, 96]
    values = [torch.full((n,), 2.0 ** -3) for n in sizes]
    values[0][[5, 4000, 4001, 8000]] = torch.tensor([2.0 ** 24, 2.0 ** 12, 2.0 ** 12, 1.0])
    found = []
    for shift, wider in ((0, 0), (32, 0), (4096, 0), (96, 320), (32 * 1001, 32 * 77)):
        buf = torch.full((300_000,), 55.0, device=DEV)
        at, parts = shift, []
        for n, gap, x in zip(sizes, gaps, values):
            at += gap + (wider if gap else 0)
            buf[at:at + n] = x.to(DEV)
            parts.append(buf[at:at + n])
            at += n
        for call in (api.thc_grad_norm, api.thc_grad_clip):
            norm, scale, ws, _ = _buffers()
            call(parts, api.THC_NORM_L2, 2.0 ** 26, norm, scale, ws)
            found.append(float(norm))
            assert float(scale) == 1.0
    assert len(set(found)) == 1 and abs(found[0] - 2.0 ** 24) <= 2.0


def test_streams_by_handle_and_by_object():
    x = torch.full((1000,), 2.0, device=DEV)
    for stream in (0, torch.cuda.default_stream(), torch.cuda.current_stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        norm, scale, ws, _ = _buffers()
        torch.cuda.synchronize()
        api.thc_grad_norm([x], api.THC_NORM_L2, 1.0, norm, scale, ws, stream=stream)
        torch.cuda.synchronize()
        assert abs(float(norm) - 2.0 * math.sqrt(1000)) <= 2.0 * math.sqrt(1000) * REL
        norm.fill_(NAN)
        torch.cuda.synchronize()
        api.thc_grad_norm([], api.THC_NORM_L2, 1.0, norm, scale, ws, stream=stream)
        torch.cuda.synchronize()
        assert float(norm) == 0.0 and float(scale) == 1.0
