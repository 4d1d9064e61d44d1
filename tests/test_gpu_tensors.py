"""Lists of tensors on the GPU: the global norm, clipping by it, gathering into a flat vector, scattering over the tensors.

Bars, derived from the definitions:
  norm    the root of a sum of exact squares, added up in binary64 (any order is within N * 2^-53 of it, N < 2^30 here, so within
          2^-22 * 2^-1 of the sum's own half step at most for 2^30 terms and below 2^-33 for the sizes here), rounded once to
          binary32: half a step, 2^-24 relative, and 2^-33 for what precedes it.
  factor  max_norm / norm in binary64, rounded once: the same.
  moves   round(fl32(x * c)) with the factor that the call itself used: the same bits.
"""
import math

import numpy as np
import pytest
import torch

from oracle import thc_oracle as o
from paper_2302_08545_amd import api

from .test_gpu_parity import assert_indices_match, both_params, rel_l2, to_np32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")
NORM_REL = 2.0 ** -24 + 2.0 ** -33


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "these tests need the GPU"
    api.lib()
    yield
    torch.cuda.synchronize()


class Tensors:
    """CPU tensors and their copies on the GPU, each with guard elements before and behind it (`lead` shifts its start)."""

    GUARD = 77.0

    def __init__(self, cpu, leads=(0,)):
        self.cpu, self.whole, self.gpu = cpu, [], []
        for i, x in enumerate(cpu):
            lead = 64 + leads[i % len(leads)]
            w = torch.full((lead + x.numel() + 64,), self.GUARD, dtype=x.dtype, device=DEV)
            w[lead:lead + x.numel()] = x.to(DEV)
            self.whole.append(w)
            self.gpu.append(w[lead:lead + x.numel()])

    def guards_hold(self):
        for x, w, g in zip(self.cpu, self.whole, self.gpu):
            lead = (g.data_ptr() - w.data_ptr()) // w.element_size() if x.numel() else w.numel()
            assert bool((w[:lead] == self.GUARD).all()) and bool((w[lead + x.numel():] == self.GUARD).all())


def _values(sizes, types, seed=1):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=gen) * 10.0 ** ((i * 7) % 5 - 2)).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def _scalars():
    return (torch.full((1,), NAN, device=DEV), torch.full((1,), NAN, device=DEV),
            torch.full((api.thc_norm_workspace_bytes(),), 255, dtype=torch.uint8, device=DEV))


def _norm64(cpu, kind):
    if kind == api.THC_NORM_MAX:
        return max((float(x.double().abs().max()) for x in cpu if x.numel()), default=0.0)
    return math.sqrt(math.fsum(float(x.double().square().sum()) for x in cpu))


def _factor64(v, limit):
    return 1.0 if v <= limit else limit / v


def _scaled(x, c):
    return (x.float() * torch.tensor(c, dtype=F32)).to(x.dtype)


SIZES = {
    "none": [], "empty": [0, 0], "one": [1], "few": [0, 1, 2, 0, 3, 5, 8, 13], "unit": [8191, 8192, 8193],
    "odd": [7, 40001, 1, 129, 16385, 250, 3, 65537], "many": [1 + (i * 37) % 300 for i in range(700)],
    "table": [33] * 192, "table_and_one": [33] * 193, "63": [21] * 63, "64": [21] * 64, "244": [33] * 244, "245": [33] * 245, "489": [5] * 489,
    "one_group": [32_768 - 32], "two_units_a_wave": [1000] * 32, "and_one": [1000] * 33, "fused": [3_000_000, 145_000], "large": [3_000_001, 17, 1_500_000],
}
LEADS = {"aligned": (0,), "odd": (1, 3, 0, 7, 2)}


@pytest.mark.parametrize("lead", LEADS)
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (BF16, F32, F16)], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_norm_and_factor(sizes, types, lead):
    X = Tensors(_values(SIZES[sizes], types), LEADS[lead])
    t = api.make_tensors(X.gpu)
    for kind in (api.THC_NORM_L2, api.THC_NORM_MAX):
        v = _norm64(X.cpu, kind)
        for limit in (v * 0.37, v * 1.7 + 1e-3, INF, 0.0):
            norm, scale, ws = _scalars()
            api.thc_grad_norm(t, kind, limit, norm, scale, ws)
            limit = float(np.float32(limit))
            assert abs(float(norm) - v) <= v * NORM_REL
            assert abs(float(scale) - _factor64(v, limit)) <= _factor64(v, limit) * (NORM_REL + 2.0 ** -33)
        again, _, ws = _scalars()
        api.thc_grad_norm(t, kind, 1.0, again, None, ws)      # no factor wanted, and the same bits again
        assert float(again) == float(norm)
    X.guards_hold()


@pytest.mark.parametrize("lead", LEADS)
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (BF16, F32, F16)], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_clip_in_place(sizes, types, lead):
    for kind in (api.THC_NORM_L2, api.THC_NORM_MAX):
        for part in (0.37, 1.7):
            X = Tensors(_values(SIZES[sizes], types, seed=3), LEADS[lead])
            v = _norm64(X.cpu, kind)
            norm, scale, ws = _scalars()
            api.thc_grad_clip(X.gpu, kind, v * part, norm, scale, ws)       # a plain sequence of tensors
            c, limit = float(scale), float(np.float32(v * part))
            assert abs(float(norm) - v) <= v * NORM_REL
            assert abs(c - _factor64(v, limit)) <= _factor64(v, limit) * (NORM_REL + 2.0 ** -33)
            assert (c == 1.0) == (part > 1 or v == 0.0)
            for x, g in zip(X.cpu, X.gpu):
                assert torch.equal(g.cpu(), _scaled(x, c))
            X.guards_hold()


@pytest.mark.parametrize("lead", LEADS)
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (BF16, F32, F16)], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("out", [F32, BF16], ids=["to_f32", "to_bf16"])
@pytest.mark.parametrize("sizes", SIZES)
def test_gather_then_scatter(sizes, out, types, lead):
    X = Tensors(_values(SIZES[sizes], types, seed=5), LEADS[lead])
    total = sum(SIZES[sizes])
    exact = max(1, -(-total // 1024)) * 1024
    for d in (exact, exact + 9 * 1024):
        p = api.make_params(d, 1024, 1, 4, 15, 2.0, 7, range(16), in_dtype=api.THC_DTYPE_BF16 if out == BF16 else api.THC_DTYPE_F32)
        for c in (None, 0.3712345):
            flat = torch.full((d + 64,), 5.0, dtype=out, device=DEV)
            scale = None if c is None else torch.tensor([c], dtype=F32, device=DEV)
            api.thc_gather(p, X.gpu, scale, flat[:d])
            want = torch.cat([torch.zeros(0)] + [x.float() * torch.tensor(1.0 if c is None else c, dtype=F32) for x in X.cpu]).to(out)
            got = flat.cpu()
            assert torch.equal(got[:total], want) and not bool(got[total:d].any()) and bool((got[d:] == 5.0).all())
            X.guards_hold()
            est = torch.randn(d, generator=torch.Generator().manual_seed(6))
            Y = Tensors([torch.zeros_like(x) for x in X.cpu], LEADS[lead])
            api.thc_scatter(p, est.to(DEV), scale, Y.gpu)
            pos = 0
            for y, g in zip(Y.cpu, Y.gpu):
                part = est[pos:pos + y.numel()] * torch.tensor(1.0 if c is None else c, dtype=F32)
                assert torch.equal(g.cpu(), part.to(y.dtype))
                pos += y.numel()
            Y.guards_hold()


def test_tensors_without_gaps_between_them():
    """Views of one buffer, one behind the other, also between tensors that are not: what the library may treat as one run."""
    buf, other = torch.randn(50_000, device=DEV), torch.randn(1000, device=DEV).to(BF16)
    views = [buf[0:7], buf[7:20_000], buf[20_000:20_000], buf[20_000:20_001], other[:1], other[1:500], buf[30_000:50_000], buf[20_001:30_000],
             other[500:]]
    want = torch.cat([v.float().cpu() for v in views])
    p = api.make_params(51 * 1024, 1024, 1, 4, 15, 2.0, 7, range(16))
    flat = torch.full((51 * 1024,), 3.0, device=DEV)
    api.thc_gather(p, views, None, flat)
    assert torch.equal(flat[:51_000].cpu(), want) and not bool(flat[51_000:].any())
    norm, scale, ws = _scalars()
    api.thc_grad_clip(views, api.THC_NORM_L2, 1.0, norm, scale, ws)
    v = math.sqrt(math.fsum(want.double().square().tolist()))
    assert abs(float(norm) - v) <= v * NORM_REL
    assert torch.equal(torch.cat([x.float().cpu() for x in views]),
                       torch.cat([(w * scale.cpu()).to(x.dtype).float() for w, x in zip(want.split([x.numel() for x in views]), views)]))


def test_dimensions_in_another_order():
    x = torch.randn(6, 5, 4, 3, device=DEV).to(memory_format=torch.channels_last)
    y = torch.randn(30, 40, device=DEV).t()
    p = api.make_params(2048, 1024, 1, 4, 15, 2.0, 7, range(16))
    flat = torch.empty(2048, device=DEV)
    api.thc_gather(p, [x, y], None, flat)
    assert torch.equal(flat[:360], x.permute(0, 2, 3, 1).reshape(-1)) and torch.equal(flat[360:1560], y.t().reshape(-1))
    x2, y2 = torch.empty_like(x), torch.empty_like(y)          # in the order that the vector was gathered in
    api.thc_scatter(p, flat, None, [x2, y2])
    assert torch.equal(x2, x) and torch.equal(y2, y)


@pytest.mark.parametrize("place", [0, 1, 4099, 8192, 20_000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_infinities_and_nan(dtype, place):
    base = torch.randn(20_001, generator=torch.Generator().manual_seed(9)).to(dtype)
    for kind in (api.THC_NORM_L2, api.THC_NORM_MAX):
        for planted, v, c in (([NAN], NAN, NAN), ([INF], INF, 0.0), ([-INF], INF, 0.0), ([NAN, -INF], NAN, NAN)):
            x = base.clone()
            for k, z in enumerate(planted):
                x[(place + 500 * k) % 20_001] = z
            g = x.to(DEV)
            norm, scale, ws = _scalars()
            api.thc_grad_clip([g], kind, 1.0, norm, scale, ws)
            assert np.array_equal([float(norm), float(scale)], [v, c], equal_nan=True)
            want = _scaled(x, c)
            assert np.array_equal(g.float().cpu().numpy(), want.float().numpy(), equal_nan=True)
            norm, scale, ws = _scalars()
            api.thc_grad_norm([x.to(DEV)], kind, INF, norm, scale, ws)      # no limit: an infinite norm is not above it
            assert np.array_equal([float(norm), float(scale)], [v, NAN if v != v else 1.0], equal_nan=True)


def test_magnitudes_at_the_ends_of_binary32():
    for values, v in (([3.0e38, -3.0e38], math.sqrt(2) * float(np.float32(3.0e38))), ([2.0 ** -149] * 9, 3 * 2.0 ** -149),
                      ([2.0 ** -140, 2.0 ** -149], math.sqrt(2.0 ** -280 + 2.0 ** -298))):
        x = torch.tensor(values)
        norm, scale, ws = _scalars()
        g = x.to(DEV)
        api.thc_grad_clip([g], api.THC_NORM_L2, v / 4, norm, scale, ws)
        with np.errstate(over="ignore"):
            assert float(norm) == float(np.float32(v))          # infinite where it exceeds binary32
        c = float(np.float32(v / 4)) / v
        assert abs(float(scale) - c) <= c * (NORM_REL + 2.0 ** -33)   # and the factor is that of the norm itself
        assert torch.equal(g.cpu(), _scaled(x, float(scale)))


def test_a_tensor_of_more_than_2_to_the_32_elements():
    n = (1 << 32) + 8195
    x = torch.zeros(n + 3, dtype=BF16, device=DEV)[1:n + 1]     # not on 16 bytes
    spots = {0: 3.0, (1 << 31) + 5: -4.0, (1 << 32) - 1: 5.0, (1 << 32) + 1: -7.0, n - 1: 1.0}
    for k, v in spots.items():
        x[k] = v
    norm, scale, ws = _scalars()
    api.thc_grad_norm([x], api.THC_NORM_L2, 1.0, norm, scale, ws)
    assert float(norm) == 10.0
    d = n + (-n) % 1024
    p = api.make_params(d, 1024, 1, 4, 15, 2.0, 7, range(16), in_dtype=api.THC_DTYPE_BF16)
    flat = torch.full((d,), 9.0, dtype=BF16, device=DEV)
    api.thc_gather(p, [x], scale, flat)
    c = float(scale)
    for k, v in spots.items():
        assert float(flat[k]) == float(_scaled(torch.tensor(v, dtype=BF16), c))
    assert int(torch.count_nonzero(flat)) == 5
    api.thc_grad_clip([x], api.THC_NORM_MAX, 3.5, norm, scale, ws)
    assert float(norm) == 7.0 and float(scale) == 0.5
    assert [float(x[k]) for k in spots] == [v / 2 for v in spots.values()] and int(torch.count_nonzero(x)) == 5


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16, F32)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("over", [-1, 0, 1], ids=["below", "at", "above"])
@pytest.mark.parametrize("tensors", [1, 250])
def test_lists_around_128_mb(tensors, over, types):
    left, parts = (128 << 20) + 4 * over, []
    for i in range(tensors):
        dtype = types[i % len(types)]
        n = left // dtype.itemsize if i == tensors - 1 else (128 << 20) // tensors // dtype.itemsize - 5 * (i % 3)
        left -= n * dtype.itemsize
        # the same steps from a start of its own, so that no two places hold the same
        parts.append(((torch.arange(n, device=DEV, dtype=torch.int32) * 40_503 + i * 977) % 2039 - 1019).to(F32).mul_(2.0 ** -12).to(dtype))
    assert left < 4
    before = [x.clone() for x in parts]
    v = math.sqrt(math.fsum(float(x.double().square().sum()) for x in parts))
    norm, scale, ws = _scalars()
    total = sum(x.numel() for x in parts)
    for out in (F32, BF16):
        d = -(-total // 1024) * 1024 + 4096
        p = api.make_params(d, 1024, 1, 4, 15, 2.0, 7, range(16), in_dtype=api.THC_DTYPE_BF16 if out == BF16 else api.THC_DTYPE_F32)
        flat = torch.full((d,), 5.0, dtype=out, device=DEV)
        api.thc_grad_norm(parts, api.THC_NORM_L2, v * 0.37, norm, scale, ws)
        assert abs(float(norm) - v) <= v * NORM_REL
        api.thc_gather(p, parts, scale, flat)
        pos = 0
        for x in before:
            assert torch.equal(flat[pos:pos + x.numel()], (x.float() * scale).to(out))
            pos += x.numel()
        assert not bool(flat[total:].any())
    api.thc_grad_clip(parts, api.THC_NORM_L2, v * 1.01, norm, scale, ws)
    assert float(scale) == 1.0 and all(torch.equal(x, y) for x, y in zip(parts, before))
    api.thc_grad_clip(parts, api.THC_NORM_L2, v * 0.37, norm, scale, ws)
    assert all(torch.equal(x, (y.float() * scale).to(y.dtype)) for x, y in zip(parts, before))
    est = torch.randn(d, device=DEV)
    api.thc_scatter(p, est, scale, parts)
    pos = 0
    for x in parts:
        assert torch.equal(x, (est[pos:pos + x.numel()] * scale).to(x.dtype))
        pos += x.numel()


def test_captured_and_replayed_with_eager_work_between():
    cpu = _values([5000, 7, 90_000, 1, 8192], (F32, BF16), seed=11)
    X = Tensors(cpu)
    t = api.make_tensors(X.gpu)
    p = api.make_params(104 * 1024, 1024, 1, 4, 15, 2.0, 7, range(16))
    norm, scale, ws = _scalars()
    flat = torch.zeros(104 * 1024, device=DEV)
    back = Tensors([torch.zeros_like(x) for x in cpu])
    tb = api.make_tensors(back.gpu)

    def calls(norm, scale, ws, flat, tb):
        api.thc_grad_norm(t, api.THC_NORM_L2, 2.5, norm, scale, ws)
        api.thc_gather(p, t, scale, flat)
        api.thc_scatter(p, flat, None, tb)
        api.thc_grad_clip(tb, api.THC_NORM_L2, 1.25, norm, scale, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(norm, scale, ws, flat, tb)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(norm, scale, ws, flat, tb)
    del tb
    for k in range(4):
        for x, g in zip(cpu, X.gpu):
            g.copy_((x.float() * (k + 1) ** 2).to(x.dtype))
        graph.replay()
        n2, s2, w2 = _scalars()
        f2 = torch.full_like(flat, 8.0)
        b2 = Tensors([torch.zeros_like(x) for x in cpu])
        calls(n2, s2, w2, f2, api.make_tensors(b2.gpu))
        torch.cuda.synchronize()
        assert torch.equal(norm, n2) and torch.equal(scale, s2) and torch.equal(flat, f2)
        assert all(torch.equal(a, b) for a, b in zip(back.gpu, b2.gpu))
        assert float(n2) == pytest.approx(2.5, rel=1e-2)       # bf16 tensors among them: a rounding of 2^-9 each


def test_two_streams_with_workspaces_of_their_own():
    cpu = [_values([400_000, 3, 70_001], (BF16,), seed=k) for k in (1, 2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    X = [Tensors(c) for c in cpu]
    S = [_scalars() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for k in (0, 1):
            api.thc_grad_norm(X[k].gpu, api.THC_NORM_L2, 1.0, *S[k], stream=sides[k])
    torch.cuda.synchronize()
    for k in (0, 1):
        v = _norm64(cpu[k], api.THC_NORM_L2)
        assert abs(float(S[k][0]) - v) <= v * NORM_REL


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_a_training_step_of_four_workers(dtype):
    """Clip, gather, compress, aggregate, decompress, scatter; the oracle works from the gathered vectors and the GPU's range."""
    sizes, n, block = [30_000, 250, 9, 20_001, 0, 1000], 4, 1 << 14
    total = sum(sizes)
    d = -(-total // block) * block
    P, L = both_params(d, block, n, bf16=dtype == BF16)
    grads, vectors = [], []
    for w in range(n):
        cpu = _values(sizes, (dtype, F32), seed=20 + w)
        X = Tensors(cpu, (0, 3))
        norm, scale, ws = _scalars()
        vec = torch.full((d,), 9.0, dtype=dtype, device=DEV)
        api.thc_grad_norm(X.gpu, api.THC_NORM_L2, 1.0, norm, scale, ws)
        api.thc_gather(L, X.gpu, scale, vec)
        want = torch.cat([x.float() * scale.cpu() for x in cpu] + [torch.zeros(d - total)]).to(dtype)
        assert torch.equal(vec.cpu(), want)
        grads.append(want)
        vectors.append(vec)
    work = torch.zeros(api.thc_workspace_bytes(L), dtype=torch.uint8, device=DEV)
    M = torch.zeros(d // block, device=DEV)
    packed = [torch.zeros(d * L.b // 8, dtype=torch.uint8, device=DEV) for _ in range(n)]
    agg, out = torch.zeros(d, dtype=torch.uint8, device=DEV), torch.zeros(d, device=DEV)
    api.thc_compress_all(L, 3, vectors, None, M, packed, work)
    api.thc_aggregate(L, packed, agg)
    api.thc_decompress(L, 3, agg, M, out, work)
    Y = Tensors([torch.zeros_like(x) for x in cpu], (2, 0))
    api.thc_scatter(L, out, None, Y.gpu)
    torch.cuda.synchronize()
    refs = [o.compress(P, w, 3, to_np32(grads[w]), None, M.cpu().numpy())[0] for w in range(n)]
    for w in range(n):
        assert_indices_match(packed[w].cpu().numpy(), refs[w], L.b)
    est = o.decompress(P, 3, o.aggregate(P, refs), M.cpu().numpy())
    assert rel_l2(out.cpu().numpy(), est) <= 1e-5
    pos = 0
    for y, g in zip(Y.cpu, Y.gpu):
        assert torch.equal(g.cpu(), out[pos:pos + y.numel()].cpu().to(y.dtype))
        pos += y.numel()
    Y.guards_hold()


@pytest.mark.parametrize("sizes", [[5000], [300_000, 17], [9_000_000, 33, 4_000_000], [600] * 300], ids=["one_group", "fused", "launches", "tables"])
def test_clipping_without_a_place_for_the_factor(sizes):
    cpu = _values(sizes, (F32, BF16), seed=31)
    X, Y = Tensors(cpu, (1, 0)), Tensors(cpu, (1, 0))
    v = _norm64(cpu, api.THC_NORM_L2)
    norm, scale, ws = _scalars()
    api.thc_grad_clip(X.gpu, api.THC_NORM_L2, v / 3, norm, scale, ws)
    n2, _, w2 = _scalars()
    api.thc_grad_clip(Y.gpu, api.THC_NORM_L2, v / 3, n2, None, w2)
    assert torch.equal(norm, n2) and abs(float(norm) - v) <= v * NORM_REL
    for x, a, b in zip(cpu, X.gpu, Y.gpu):
        assert torch.equal(a, b) and torch.equal(a.cpu(), _scaled(x, float(scale)))
    X.guards_hold()
    Y.guards_hold()


@pytest.mark.parametrize("sizes", [[7, 300], [1000] * 33, [9_000_001, 13], [33_600_000, 5], [40] * 300 + [33_600_000]], ids=lambda s: f"{len(s)}x{s[-1]}")
def test_norm_and_clip_give_the_same_bits(sizes):
    for kind in (api.THC_NORM_L2, api.THC_NORM_MAX):
        X = Tensors(_values(sizes, (F32,), seed=17))
        one, c1, ws = _scalars()
        two, c2, _ = _scalars()
        api.thc_grad_norm(X.gpu, kind, 0.7, one, c1, ws)
        api.thc_grad_clip(X.gpu, kind, 0.7, two, c2, ws)
        assert torch.equal(one, two) and torch.equal(c1, c2) and 0.0 < float(c1) < 1.0


def test_a_tensor_listed_twice_is_read_twice():
    x = torch.randn(10_000, generator=torch.Generator().manual_seed(8))
    g = x.to(DEV)
    t = api.make_tensors([g, g[:100], g])
    norm, scale, ws = _scalars()
    api.thc_grad_norm(t, api.THC_NORM_L2, INF, norm, scale, ws)
    v = _norm64([x, x[:100], x], api.THC_NORM_L2)
    assert abs(float(norm) - v) <= v * NORM_REL
    p = api.make_params(20 * 1024, 1024, 1, 4, 15, 2.0, 7, range(16))
    flat = torch.empty(20 * 1024, device=DEV)
    api.thc_gather(p, t, None, flat)
    assert torch.equal(flat[:20_100].cpu(), torch.cat([x, x[:100], x]))
    for call in (lambda: api.thc_grad_clip(t, api.THC_NORM_L2, 1.0, norm, scale, ws), lambda: api.thc_scatter(p, flat, None, t)):
        with pytest.raises(api.ThcError) as e:
            call()
        assert e.value.status == -1
    torch.cuda.synchronize()
    assert torch.equal(g.cpu(), x)


def test_estimates_beyond_f16_and_in_its_subnormal_range():
    est = torch.tensor([1e5, -7e4, 65504.0, 65519.0, 65520.0, 3e-8, 2.0 ** -25, 3 * 2.0 ** -25, -1e-30, 0.1, NAN, INF] + [0.0] * 1012)
    y = torch.full((12,), 5.0, dtype=F16, device=DEV)
    z = torch.full((12,), 5.0, dtype=BF16, device=DEV)
    p = api.make_params(1024, 1024, 1, 4, 15, 2.0, 7, range(16))
    api.thc_scatter(p, est.to(DEV), None, [y])
    api.thc_scatter(p, est.to(DEV), None, [z])
    assert np.array_equal(y.float().cpu().numpy(), est[:12].to(F16).float().numpy(), equal_nan=True)
    assert np.array_equal(z.float().cpu().numpy(), est[:12].to(BF16).float().numpy(), equal_nan=True)


def test_on_a_stream_of_the_callers_own():
    side = torch.cuda.Stream()
    cpu = _values([70_000, 5], (BF16, F32), seed=41)
    X = Tensors(cpu)
    norm, scale, ws = _scalars()
    p = api.make_params(69 * 1024, 1024, 1, 4, 15, 2.0, 7, range(16))
    flat = torch.zeros(69 * 1024, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                    # the current stream, and the same one by name
        api.thc_grad_norm(X.gpu, api.THC_NORM_L2, 1.0, norm, scale, ws)
    api.thc_gather(p, X.gpu, scale, flat, stream=side)
    side.synchronize()
    assert torch.equal(flat[:70_005].cpu(), torch.cat([x.float() * scale.cpu() for x in cpu]))
