"""Calls of a stage's training step at the edges of what their description allows: tensors without elements."""
import pytest
import torch

from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[True, False], ids=["extension", "python"])
def either_way(request, monkeypatch):
    """The calls with their arguments read by the extension, and by Python."""
    if request.param:
        assert B._load_marshal() is not None
    else:
        monkeypatch.setattr(B, "_marshal", False)


@pytest.mark.parametrize("shape", [(0, 64), (3, 0), (3, 0, 64), (0, 3, 64), (2, 3, 0), (0, 0, 64)])
def test_tensors_without_elements(shape, either_way):
    rows, cols = int(torch.Size(shape[:-1]).numel()), shape[-1]
    for x in (torch.empty(shape, device="cuda"), torch.empty(tuple(size + 2 for size in shape), device="cuda")[tuple(slice(0, size) for size in shape)]):
        buffer, f = torch.full((16,), 7, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
        B.adatopk_act8_store(x, buffer)
        B.adatopk_act8_load(buffer, x)
        B.adatopk_gelu_forward(x, x, buffer, buffer)
        B.adatopk_gelu_backward(x, buffer, x)
        B.adatopk_layernorm_forward(x, None, None, 1e-5, x, f, f, residual=x, sum_out=x, act8=buffer)
        dw, db = torch.full((cols,), 3.0, device="cuda"), torch.full((cols,), 3.0, device="cuda")
        ws = torch.empty(1 << 12, dtype=torch.uint8, device="cuda")
        for source in ((x, None), (None, buffer)):
            B.adatopk_layernorm_backward(x, *source, f, f, None, x, dw, db, ws, accumulate=True)
            assert bool((dw == 3.0).all()) and bool((db == 3.0).all())
        B.adatopk_layernorm_backward(x, x, None, f, f, None, x, dw, db, ws)
        assert bool((dw == 0.0).all()) and bool((db == 0.0).all())
        of_x, of_b = torch.full((cols, 32), 3.0, device="cuda"), torch.full((cols,), 3.0, device="cuda")
        if rows == 0:
            B.adatopk_weight_grad(x, buffer, of_x, of_b, ws)
            assert bool((of_x == 0.0).all()) and bool((of_b == 0.0).all())
        torch.cuda.synchronize()
        assert bool((buffer == 7).all())
