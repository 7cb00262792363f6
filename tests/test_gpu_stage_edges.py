"""Calls of a stage's training step at the edges of what their description allows: tensors without elements, values without a scale, the smallest
values, precision as described."""
import numpy as np
import pytest
import torch

import stage_reference as ref
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_numbers_of_groups_without_a_scale_are_zeros(dtype):
    # groups that hold a NaN or an infinity, and rows that layer norm makes NaN from end to end: E = 255, and the buffer is the same
    # whatever the values were; behind a row's end there are zeros in any case
    rows = 5
    for cols in (1, 31, 33, 40, 64, 100, 700, 1601, 3000):
        gen = torch.Generator(device="cuda").manual_seed(cols)
        x = torch.randn(rows, cols, device="cuda", generator=gen).to(dtype)
        x[1, cols // 2], x[3, cols - 1], x[3, 0] = float("nan"), float("inf"), -float("inf")
        whole = torch.tensor([False, True, False, True, False], device="cuda")
        groups, n = (cols + 31) // 32, B.adatopk_act8_bytes(rows, cols)
        marked = torch.zeros(rows, groups, dtype=torch.bool, device="cuda")
        marked[1, cols // 2 // 32] = marked[3, (cols - 1) // 32] = marked[3, 0] = True

        def split(buffer):
            q = buffer[:rows * groups * 32].view(torch.int8).view(rows, groups, 32)
            return q, buffer[n - rows * groups:].view(rows, groups)

        def check(buffer, where):
            q, e = split(buffer)
            assert torch.equal(e == 255, where), cols
            assert bool((q[where] == 0).all()), cols
            assert bool((q.reshape(rows, -1)[:, cols:] == 0).all()), cols

        buffers = [torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda") for _ in range(2)]
        B.adatopk_act8_store(x, buffers[0])
        check(buffers[0], marked)
        y = torch.empty_like(x)
        B.adatopk_gelu_forward(x.abs(), y, *buffers)  # (GELU of an infinity is one)
        check(buffers[0], marked)
        check(buffers[1], marked)
        B.adatopk_layernorm_forward(x, None, None, 1e-5, y, None, None, act8=buffers[0])
        check(buffers[0], whole[:, None].expand(rows, groups))
        B.adatopk_layernorm_forward(torch.full_like(x, 2.0), None, None, 0.0, y, None, None, act8=buffers[0])  # no variance and no eps: 0 / 0
        check(buffers[0], torch.ones_like(marked))


def test_groups_below_the_smallest_step():
    # E stops at 7, so a step is 2^-126 at least: a group below 2^-120 is held with errors of up to 2^-127, whatever its largest magnitude
    rng = np.random.default_rng(11)
    for top in range(-149, -112):
        x = ref.rounded(np.ldexp(1 + rng.random((3, 64)), top) * rng.choice([-1.0, 1.0], size=(3, 64)), torch.float32)
        x[0, 0] = 2.0 ** top
        buffer, y = B.new_act8(3, 64), torch.empty(3, 64, device="cuda")
        B.adatopk_act8_store(ref.on_device(x, torch.float32), buffer)
        B.adatopk_act8_load(buffer, y)
        amax = np.abs(x).reshape(3, 2, 32).max(axis=2).repeat(32, axis=1)
        assert (np.abs(ref.host(y) - x) <= np.maximum(amax / 127.5, 2.0 ** -127)).all(), top


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_down_to_the_smallest(dtype):
    # one token, an input of ones or of 64: the result is the gradient, to the bit for 16-bit types and from 2^-110 on for fp32; below that what
    # lies under 2^-133, the smallest number of its bf16 pieces, is cut off
    rng = np.random.default_rng(12)
    if dtype == torch.float32:
        dy = torch.from_numpy((np.ldexp(1 + rng.random(8192), rng.integers(-149, 0, size=8192)) * rng.choice([-1.0, 1.0], size=8192)).astype(np.float32))
    else:
        dy = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
        dy = dy[torch.isfinite(dy) & (dy.float().abs() < 2.0 ** 100)]
    dy = dy.view(1, -1).cuda()
    n = dy.shape[1]
    for value in (1.0, 64.0):
        buffer = torch.from_numpy(ref.act8_buffer(np.full((1, 2), value))).cuda()
        dw, db = torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda")
        ws = torch.empty(B.adatopk_weight_grad_workspace_bytes(1, n, 2, dtype), dtype=torch.uint8, device="cuda")
        B.adatopk_weight_grad(dy, buffer, dw, db, ws)
        want = dy[0].double()
        error = torch.zeros_like(want) if dtype != torch.float32 else torch.where(want.abs() < 2.0 ** -110, 2.0 ** -133, 0.0)
        assert bool(((db.double() - want).abs() <= error).all())
        for column in range(2):
            assert bool(((dw[:, column].double() - value * want).abs() <= value * error).all())


@pytest.mark.parametrize("tanh", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_slope_of_gelu_as_closely_as_it_is_described(dtype, tanh):
    # what the header says: 2^-21 of dy for fp32 and 2^-20 for 16-bit types, 2^-18 with the hyperbolic tangent, and the result's rounding.  Inputs: the
    # grids of the 8-bit form from 2^-8 to 8, among them what lies next to the slope's zero
    for scale in range(-8, 4):
        x = np.arange(-127, 128).repeat(5)[:1280 - 5] * 2.0 ** (scale - 6)
        x = np.concatenate([x, np.full(5, 127 * 2.0 ** (scale - 6))]).reshape(40, 32)
        x[:, 0] = 2.0 ** scale * 127 / 64  # (every group has this grid)
        held = ref.act8_encode(x)[2]
        assert np.array_equal(held, x)
        dy = ref.rounded(np.random.default_rng(scale + 20).uniform(1, 2, size=x.shape), dtype)
        dx = torch.empty(x.shape, dtype=dtype, device="cuda")
        B.adatopk_gelu_backward(ref.on_device(dy, dtype), torch.from_numpy(ref.act8_buffer(x)).cuda(), dx, tanh=tanh)
        want = dy * ref.gelu_slope(x, tanh)
        bound = dy * (2.0 ** -18 if tanh else 2.0 ** -21 if dtype == torch.float32 else 2.0 ** -20)
        assert (np.abs(ref.host(dx) - want) <= bound + ref.HALF_ULP[dtype] * (np.abs(want) + bound) + ref.SMALLEST[dtype]).all(), scale
