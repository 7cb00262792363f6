"""The root-mean-square norm of as many rows as a matrix may have."""
import pytest
import torch

from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [(1 << 27) - 1, (1 << 27) + 5, (1 << 28) + 3])
def test_more_rows_than_8_bit_floating_point_has(rows):
    # columns rounded up to 32: below 2^34 elements, which the norm takes; rounded up to 128, as rows in 8-bit floating point would be, from 2^27 rows on they are not
    some = 1000
    x = torch.zeros(rows, 3, dtype=torch.float16, device="cuda")
    x[:some], x[-some:] = (torch.randn(some, 3, device="cuda") for _ in range(2))
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    B.adatopk_rmsnorm_forward(x, None, 1e-5, y, rstd)
    for part in (slice(0, some), slice(rows - some, rows)):
        want, want_rstd = torch.empty(some, 3, dtype=torch.float16, device="cuda"), torch.empty(some, device="cuda")
        B.adatopk_rmsnorm_forward(x[part], None, 1e-5, want, want_rstd)
        assert torch.equal(y[part], want) and torch.equal(rstd[part], want_rstd)
    assert bool((rstd[some:-some] == rstd[some]).all()) and not bool(y[some:-some].any())
    if rows >= 1 << 27:  # and there they are refused
        with pytest.raises((ValueError, B.AdaTopKError)):
            B.adatopk_rmsnorm_forward(x, None, 1e-5, y, rstd, fp8=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
