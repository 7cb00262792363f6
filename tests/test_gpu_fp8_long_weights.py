"""Weights put into 8-bit floating point in the one orientation in which they fit."""
import pytest
import torch

from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("across", [False, True])
def test_a_row_that_has_no_room_as_a_column(across):
    # 2^27 + 5 elements in a row are 2^27 + 128 in 8 bits; in a column, 128 to each, 2^34 and more
    n, some = (1 << 27) + 5, 128 * 9 + 5
    w = torch.zeros((n, 1) if across else (1, n), dtype=torch.float16, device="cuda")
    w.view(-1)[-some:] = torch.randn(some, device="cuda")
    buffer, back, want, few = B.new_fp8(1, n), torch.empty(1, n, dtype=torch.float16, device="cuda"), torch.empty(1, some, dtype=torch.float16, device="cuda"), B.new_fp8(1, some)
    B.adatopk_fp8_store_weight(w, None if across else buffer, buffer if across else None)
    B.adatopk_fp8_load(buffer, back)
    B.adatopk_fp8_store(w.view(1, n)[:, -some:], few)  # one row: a tile of 128 x 128 holds as many of its elements as a block of 128
    B.adatopk_fp8_load(few, want)
    assert n % 128 == some % 128 and torch.equal(back[:, -some:], want) and not bool(back[:, :-some].any())
    with pytest.raises((ValueError, B.AdaTopKError)):
        B.adatopk_fp8_store_weight(w, buffer, buffer)
