"""As many rows as a 32-bit count holds."""
import pytest
import torch

from tests.dense_util import E4M3, ctx, status


@pytest.mark.gpu
def test_quant_of_the_most_rows():
    n = 2 ** 31 - 1
    x = torch.ones(n, 1, device="cuda", dtype=torch.float16)
    x[::2] = -0.25
    x[n - 1] = 3.0
    codes, scale = torch.empty(n, 1, device="cuda", dtype=E4M3), torch.empty(n, device="cuda")
    ctx().quant_rows(x, codes, scale)
    for rows in (slice(0, 4096), slice(0, n, 10007), slice(n - 4096, n)):
        v, s = x[rows].float(), scale[rows]
        assert torch.equal(s, v.abs()[:, 0] / 448) and torch.equal(codes[rows].float(), v.sign() * 448)
    assert status() == 0
