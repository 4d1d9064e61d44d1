"""Gathers by a factor where their form changes: around 12 MB, around one launch's tensors with and without zeros behind the list."""
import pytest
import torch

from paper_2302_08545_amd import api

from .test_gpu_tensors import BF16, DEV, F16, F32, Tensors

pytestmark = pytest.mark.gpu
MB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "these tests need the GPU"
    api.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (BF16, F16)], ids=["f32", "bf16", "f16", "bf16_f16"])
@pytest.mark.parametrize("mb", [9, 12, 13, 40])
@pytest.mark.parametrize("tensors", [3, 63, 64, 243, 244, 245])
def test_gather_by_a_factor(tensors, mb, types):
    gen = torch.Generator(device=DEV).manual_seed(tensors + mb)
    size, out = types[0].itemsize, F32 if types[0] == F32 else BF16
    n = [mb * MB // size // tensors + (i * 37) % 91 - 45 for i in range(tensors)]
    n[-1] += -sum(n) % 1024                                  # with nothing behind the list: exactly the vector's size
    X = Tensors([torch.randn(k, generator=gen, device=DEV).to(types[i % len(types)]) for i, k in enumerate(n)], (1, 3, 0, 7, 2))
    total = sum(n)
    scale = torch.tensor([0.3712345], device=DEV)
    want = torch.cat([x.float() * scale for x in X.cpu]).to(out)
    for zeros in (0, 1024 * 33):
        d = total + zeros
        p = api.make_params(d, 1024, 1, 4, 15, 2.0, 7, range(16), in_dtype=api.THC_DTYPE_BF16 if out == BF16 else api.THC_DTYPE_F32)
        flat = torch.full((d + 64,), 5.0, dtype=out, device=DEV)
        api.thc_gather(p, X.gpu, scale, flat[:d])
        assert torch.equal(flat[:total], want) and not bool(flat[total:d].any()) and bool((flat[d:] == 5.0).all())
        X.guards_hold()
