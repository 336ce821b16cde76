"""ssm_norm_i8 on rows whose squares add up to about the largest float32."""
import pytest
import torch

import _i8_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("d", [1, 96, 1000, 1001, 4096, 8192, 12288, 20001, 32768, 40000])
def test_norm_of_rows_near_the_largest_sum_of_squares(gpu, d):
    """A row's squares add up to a float32 or the row is marked by a NaN scale: its codes
    and scale never say that it is zero."""
    from paper_2608_23167_amd import api
    limit = 2.0 ** 64 / d ** 0.5
    x = torch.empty(7, d, device=DEV)
    x[0] = 0.98 * limit                    # squares add up to 0.96 x 2^128
    x[1] = 1.02 * limit                    # 1.04 x 2^128
    x[2] = 0.0
    x[2, d - 1] = 2.0 ** 63.9              # one large value: its square is 0.87 x 2^128
    x[3] = 1.0
    x[3, d // 2] = -(2.0 ** 64.1)
    x[4] = 3e38
    x[5] = 0.0
    x[6] = 1.0
    gain = torch.ones(d, device=DEV)
    q, s = torch.full((7, d), 99, dtype=torch.int8, device=DEV), torch.full((7,), -1.0, device=DEV)
    resid = torch.empty_like(x)
    api.ssm_norm_i8(x, gain, 1e-5, q, s, resid=resid)
    assert torch.equal(resid, x)
    bad = torch.tensor([1, 3, 4], device=DEV)
    assert bool(torch.isnan(s[bad]).all()) and not bool(q[bad].any())
    assert float(s[5]) == 0 and not bool(q[5].any())
    ok = torch.tensor([0, 2, 6], device=DEV)
    R.check_codes(q[ok], s[ok], R.norm(x[ok], gain, 1e-5), R.norm_rel(d))
