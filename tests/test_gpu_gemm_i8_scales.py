"""ssm_gemm_i8 with scales whose product leaves the normal float32 range."""
import pytest
import torch

import _i8_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"


def _codes(seed, *size):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(-128, 128, size, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)


def _gemm(a, sa, w, sw, dtype):
    from paper_2608_23167_amd import api
    m, n, k = a.shape[0], w.shape[0], a.shape[1]
    ws = torch.empty(api.ssm_gemm_i8_workspace_size(m, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty(m, n, dtype=dtype, device=DEV)
    api.ssm_gemm_i8(a, sa, w, sw, out, ws)
    return out


# few rows, any alignment, a tile whole and at its edge, sums of splits
PRODUCTS = [(3, 70, 256), (20, 70, 101), (130, 64, 1024), (130, 67, 1024), (18, 66, 3216)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ea,ew", [(-100, -40), (-40, -100), (-107, -25), (90, -20), (-60, 110)])
def test_scales_whose_product_is_small_or_large(gpu, m, n, k, dtype, ea, ew):
    """Scales whose product leaves the normal float32 range, on results that do not."""
    a, w = _codes(m, m, k), _codes(n, n, k)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    sa = (torch.rand(m, generator=g, device=DEV) + 1) * 2.0 ** ea
    sw = (torch.rand(n, generator=g, device=DEV) + 1) * 2.0 ** ew
    R.check_gemm(_gemm(a, sa, w, sw, dtype), a, sa, w, sw)


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_a_sum_of_zero_is_zero_at_any_scales(gpu, m, n, k):
    a, w = _codes(m, m, k), _codes(n, n, k)
    a[1], w[2] = 0, 0
    sa, sw = torch.full((m,), 2.0 ** 100, device=DEV), torch.full((n,), 2.0 ** 100, device=DEV)
    out = _gemm(a, sa, w, sw, F32)
    zero = (a.double() @ w.double().t()) == 0
    assert bool(zero[1].all()) and bool(zero[:, 2].all())
    assert not bool(out[zero].any()) and bool(torch.isinf(out[~zero]).all())
