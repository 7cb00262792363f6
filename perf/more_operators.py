"""The operators of a stage's training step whose projections run in 8-bit floating point, and what they are timed on.

A stage normalises its rows, multiplies them with weights and, when all micro-batches' gradients have come back, changes the weights:

  rmsnorm_forward    rows divided by their root mean square and weighted, with the residual added before where there is one; the divided rows kept in
                     8-bit whole numbers for the backward pass, the weighted ones in 8-bit floating point for the product that reads them
  rmsnorm_backward   the gradients of input and weight, from the input or from the 8-bit rows
  fp8_store          activations or gradients put into 8-bit floating point and read back
  fp8_store_weight   a weight matrix put into 8-bit floating point, as it is and transposed, and read back
  fp8_product        x W^T of two matrices in 8-bit floating point, with bias and a summand
  muon_update        a weight matrix changed by its gradient, with momentum, orthogonalised by Newton-Schulz products

8-bit floating point: 128 consecutive elements of a row (of a weight matrix: a tile of 128 x 128) share a scale 2^(S - 127), the smallest power of two
with which the largest magnitude is at most 448, S at least 1; an element is held as the nearest number of four significand bits, exponents from -6 to 8
and subnormals (e4m3, ties to even) to its quotient with the scale.  One buffer holds the numbers, row by row, every row padded with zeros to a
multiple of 128, and from the next multiple of 256 bytes on the S: those of the rows' first 128 columns, padded to a multiple of 256, then those of the next.
The 8-bit whole numbers are those of perf/operators.py.

Newton-Schulz: X = U / (|U| + eps) with the Frobenius norm; then in each step A = X X^T, X = a X + (b A + c A A) X.

Fields of a case:
  op        one of the above
  dtype     "f32", "bf16", "f16": of activations, gradients and weights; statistics, momentum and gradients of weights are 32-bit
  rows, cols   tokens and features; of a weight matrix its rows and columns; fp8_product: tokens and input features, `out` the output features
  slack     elements between one row's end and the next row's start in the dense inputs (views into a wider tensor)
  residual  rmsnorm: a second summand of the input; its gradient is added to the input's.  fp8_product: a summand of the result
  keep      rmsnorm: the rows in whole numbers are written (forward) or read in place of the input (backward)
  eight     rmsnorm_forward: the weighted rows in 8-bit floating point are written
  bias      fp8_product: added to every row
  dense     fp8_product: the left matrix is put into 8 bits within the pass
  steps     muon_update: Newton-Schulz steps
  momentum  muon_update: the gradient goes through a momentum of 0.95 and Nesterov's look ahead; the weights decay and move by the result.
            Without it the orthogonalised gradient itself is asked for
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
GROUP, BLOCK = 32, 128
NS_A, NS_B, NS_C, NS_EPS = 3.4445, -4.7750, 2.0315, 1e-7
MOMENTUM, RATE, DECAY = 0.95, 0.02, 0.1


def _case(name, op, dtype, rows, cols, out=0, slack=0, residual=False, keep=False, eight=False, bias=False, dense=False, steps=0, momentum=False):
    c = dict(op=op, dtype=dtype, rows=rows, cols=cols, out=out, slack=slack, residual=residual, keep=keep, eight=eight, bias=bias, dense=dense,
             steps=steps, momentum=momentum)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The hidden state of 4 x 128 tokens of a small model, fp32: one call's latency.
        _case("rms_fwd_4x128x768_f32", "rmsnorm_forward", "f32", 512, 768),
        # An XL block's 16 x 1024 tokens in training: residual added, rows kept for the backward pass, and in 8 bits for the projection behind.
        _case("rms_fwd_16x1024x1600_bf16", "rmsnorm_forward", "bf16", 16384, 1600, residual=True, keep=True, eight=True),
        # Ragged rows whose input was kept as it is.
        _case("rms_bwd_1000x1601_f16", "rmsnorm_backward", "f16", 1000, 1601),
        # The XL block's backward pass from the 8-bit rows, the residual path's gradient added.
        _case("rms_bwd_16x1024x1600_bf16", "rmsnorm_backward", "bf16", 16384, 1600, residual=True, keep=True),
        # A ragged tail of a batch of gradients, a view into a wider tensor, on its way into the product that gives the input's gradient.
        _case("fp8_store_777x1001_f16", "fp8_store", "f16", 777, 1001, slack=23),
        # The first projection of an XL block's feed-forward half, after its update: for the forward pass, and transposed for the backward pass.
        _case("fp8_weight_6400x1600_bf16", "fp8_store_weight", "bf16", 6400, 1600),
        # One token through that projection, as when a model answers: latency and the weights' bytes.
        _case("fp8_product_1x1600x6400_bf16", "fp8_product", "bf16", 1, 1600, out=6400, bias=True),
        # An attention output projection of a small model on 4 x 128 tokens, fp32.
        _case("fp8_product_512x768x768_f32", "fp8_product", "f32", 512, 768, out=768, bias=True, residual=True),
        # Ragged in all three sizes, from dense activations.
        _case("fp8_product_2049x777x1000_f16", "fp8_product", "f16", 2049, 777, out=1000, slack=8, dense=True),
        # The XL projection on 16 x 1024 tokens in training, its input as the norm before it wrote it.
        _case("fp8_product_16x1024x1600x6400_bf16", "fp8_product", "bf16", 16384, 1600, out=6400, bias=True),
        # A small model's square weights: the orthogonalised gradient alone.
        _case("muon_768x768_f32", "muon_update", "f32", 768, 768, steps=5),
        # The step of the XL projection's weights.
        _case("muon_6400x1600_bf16", "muon_update", "bf16", 6400, 1600, steps=5, momentum=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rmsnorm_forward", "rmsnorm_backward", "fp8_store", "fp8_store_weight", "fp8_product", "fp8_product", "muon_update"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    slack = rng.choice([0, 0, 0, rng.randint(1, 64), 8 * rng.randint(1, 64)])
    even = rng.random() < 0.5  # features are multiples of 64 in most models

    def features(lo, hi):
        n = _log_uniform(rng, lo, hi)
        return max(64, n // 64 * 64) if even else n

    if op == "fp8_product":
        cols, out = features(32, 6400), features(32, 6400)
        rows = _log_uniform(rng, 1, max(1, min(16384, 160_000_000_000 // (cols * out))))
        dense = rng.random() < 0.5
        return _case(None, op, dtype, rows, cols, out=out, slack=slack if dense else 0, residual=rng.random() < 0.3, bias=rng.random() < 0.5, dense=dense)
    if op == "muon_update":
        less = features(16, 1600)
        more = features(less, min(6400, max(less, 10_000_000 // less)))
        rows, cols = (less, more) if rng.random() < 0.5 else (more, less)
        return _case(None, op, dtype, rows, cols, slack=slack, steps=rng.choice([3, 5, 5, 5]), momentum=rng.random() < 0.6)
    if op == "fp8_store_weight":
        return _case(None, op, dtype, features(32, 6400), features(32, 6400), slack=slack)
    most = 26_000_000 if op.startswith("rmsnorm") else 100_000_000
    cols = features(16, 8192)
    rows = _log_uniform(rng, 1, min(65536, most // cols))
    norm, forward = op.startswith("rmsnorm"), op == "rmsnorm_forward"
    return _case(None, op, dtype, rows, cols, slack=slack, residual=norm and rng.random() < 0.5, keep=norm and rng.random() < 0.5,
                 eight=forward and rng.random() < 0.5)


# ---------------------------------------------------------------- 8-bit whole numbers, a scale for 32, in torch operations
def _up(n, to):
    return (n + to - 1) // to * to


def _whole_bytes(rows, cols):
    return _up(rows * _up(cols, GROUP), 256) + rows * _up(cols, GROUP) // GROUP


def _whole_encode(x):
    rows, cols = x.shape
    g = torch.nn.functional.pad(x, (0, _up(cols, GROUP) - cols)).view(rows, -1, GROUP)
    E = (g.abs().amax(-1).view(torch.int32) >> 23).clamp(min=7)
    inverse = ((260 - E.clamp(max=254)) << 23).view(torch.float32)
    q = torch.round(g * inverse[..., None]).clamp(-127, 127)
    return torch.where(E[..., None] == 255, torch.zeros_like(q), q), E


def _whole_values(q, E, cols):
    v = q * ((E.clamp(max=254) - 6) << 23).view(torch.float32)[..., None]
    v = torch.where(E[..., None] == 255, torch.full_like(v, math.nan), v)
    return v.reshape(v.shape[0], -1)[:, :cols]


def _whole_pack(x):
    rows, cols = x.shape
    q, E = _whole_encode(x)
    at = _up(q.numel(), 256)
    buffer = torch.zeros(_whole_bytes(rows, cols), dtype=torch.uint8, device=x.device)
    buffer[:q.numel()] = q.to(torch.int8).view(-1).view(torch.uint8)
    buffer[at:] = E.view(-1).to(torch.uint8)
    return buffer


def _whole_unpack(buffer, rows, cols):
    width = _up(cols, GROUP)
    q = buffer[:rows * width].view(torch.int8).view(rows, -1, GROUP).to(torch.float32)
    return _whole_values(q, buffer[_up(rows * width, 256):].view(rows, -1).to(torch.int32), cols)


# ---------------------------------------------------------------- 8-bit floating point, a scale for 128
def _float_bytes(rows, cols):
    return _up(rows * _up(cols, BLOCK), 256) + _up(cols, BLOCK) // BLOCK * _up(rows, 256)


def _float_encode(x, tile):
    """Numbers [rows, groups, 128] as 8-bit floats and S [rows, groups] of 32-bit values; tile: the rows that share an S."""
    rows, cols = x.shape
    g = torch.nn.functional.pad(x, (0, _up(cols, BLOCK) - cols)).view(rows, -1, BLOCK)
    most = g.abs().amax(-1)
    if tile > 1:
        padded = torch.nn.functional.pad(most, (0, 0, 0, _up(rows, tile) - rows)).view(-1, tile, most.shape[1])
        most = padded.amax(1, keepdim=True).expand_as(padded).reshape(-1, most.shape[1])[:rows]
    # the exponent of the next power of two above the largest magnitude's quotient with 1.75
    S = (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    S = torch.where(torch.isfinite(most), S, torch.full_like(S, 255))
    inverse = ((254 - S.clamp(max=253)) << 23).view(torch.float32)
    q = g * inverse[..., None]
    return torch.where(S[..., None] == 255, torch.full_like(q, math.nan), q).to(torch.float8_e4m3fn), S


def _float_values(q, S, cols):
    v = q.to(torch.float32) * (S.clamp(max=254) << 23).view(torch.float32)[..., None]
    return v.reshape(v.shape[0], -1)[:, :cols]


def _float_kept(x, tile):
    return _float_values(*_float_encode(x, tile), x.shape[1])


def _float_pack(x, tile):
    rows, cols = x.shape
    q, S = _float_encode(x, tile)
    at = _up(q.numel(), 256)
    buffer = torch.zeros(_float_bytes(rows, cols), dtype=torch.uint8, device=x.device)
    buffer[:q.numel()] = q.view(-1).view(torch.uint8)
    buffer[at:].view(-1, _up(rows, 256))[:, :rows] = S.t().to(torch.uint8)
    return buffer


def _float_unpack(buffer, rows, cols):
    width = _up(cols, BLOCK)
    q = buffer[:rows * width].view(torch.float8_e4m3fn).view(rows, -1, BLOCK)
    return _float_values(q, buffer[_up(rows * width, 256):].view(-1, _up(rows, 256))[:, :rows].t().to(torch.int32), cols)


# ---------------------------------------------------------------- inputs
def _dense(case, cols, values):
    """`values` as the case's type, in rows with the case's slack between them."""
    wide = torch.zeros(values.shape[0], cols + case["slack"], dtype=DTYPES[case["dtype"]], device="cuda")
    wide[:, :cols] = values
    return wide[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, cols, dtype = case["op"], case["rows"], case["cols"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def gradient(n):  # heavy-tailed: 1e-3 times Student's t of 3 degrees of freedom
        g = normal(rows, n).mul_(1e-3)
        chi = torch.zeros_like(g)
        for _ in range(3):
            chi.add_(normal(rows, n).square_())
        return g.div_(chi.div_(3.0).sqrt_())

    def hidden():  # a residual stream: a few features are much larger than the others
        scale = torch.where(torch.rand(cols, device="cuda", generator=gen) < 0.01, 12.0, 1.0)
        return normal(rows, cols) * scale + 0.1 * normal(cols)

    def new(*shape, dtype=dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def buffer(size):
        return new(size, dtype=torch.uint8)

    state = {"case": case, "rows": rows, "cols": cols}
    if op == "rmsnorm_forward":
        state["weight"] = (1.0 + 0.2 * normal(cols)).to(dtype)
        state["x"] = _dense(case, cols, hidden())
        state["residual"] = _dense(case, cols, normal(rows, cols)) if case["residual"] else None
        state["sum"] = new(rows, cols) if case["residual"] else None
        state["y"], state["rstd"] = new(rows, cols), new(rows, dtype=torch.float32)
        state["whole"] = buffer(_whole_bytes(rows, cols)) if case["keep"] else None
        state["eight"] = buffer(_float_bytes(rows, cols)) if case["eight"] else None
        state["kept"] = [new(rows, cols, dtype=torch.bfloat16) for _ in range(2)]
    elif op == "rmsnorm_backward":
        state["weight"] = (1.0 + 0.2 * normal(cols)).to(dtype)
        x = _dense(case, cols, hidden())
        rstd = torch.rsqrt(x.float().square().mean(-1) + EPS)
        state["x"] = None if case["keep"] else x
        state["whole"] = _whole_pack(x.float() * rstd[:, None]) if case["keep"] else None
        state["rstd"], state["dy"] = rstd, _dense(case, cols, gradient(cols))
        state["dsum"] = _dense(case, cols, gradient(cols)) if case["residual"] else None
        state["dx"], state["dweight"] = new(rows, cols), new(cols, dtype=torch.float32)
    elif op == "fp8_store":
        state["x"], state["eight"] = _dense(case, cols, gradient(cols)), buffer(_float_bytes(rows, cols))
        state["y"] = new(rows, cols, dtype=torch.bfloat16)
    elif op == "fp8_store_weight":
        state["w"] = _dense(case, cols, normal(rows, cols) * cols ** -0.5)
        state["eight"], state["across"] = buffer(_float_bytes(rows, cols)), buffer(_float_bytes(cols, rows))
        state["y"], state["yt"] = new(rows, cols, dtype=torch.bfloat16), new(cols, rows, dtype=torch.bfloat16)
    elif op == "fp8_product":
        x, out = _dense(case, cols, normal(rows, cols)), case["out"]
        state["x"] = x if case["dense"] else None
        state["eight"] = buffer(_float_bytes(rows, cols)) if case["dense"] else _float_pack(x.float(), 1)
        state["w"] = _float_pack((normal(out, cols) * cols ** -0.5).to(dtype).float(), BLOCK)
        state["bias"] = (0.1 * normal(out)).to(dtype) if case["bias"] else None
        state["add"] = normal(rows, out).to(dtype) if case["residual"] else None
        state["y"] = new(rows, out)
    else:
        # a gradient has a few strong directions and noise beside them
        strong = max(1, min(rows, cols) // 16)
        g = normal(rows, strong) @ normal(strong, cols) * strong ** -0.5 + 0.5 * normal(rows, cols)
        wide = torch.zeros(rows, cols + case["slack"], device="cuda")
        wide[:, :cols] = 1e-3 * g
        state["grad"] = wide[:, :cols]
        state["momentum"] = 1e-2 * normal(rows, cols) if case["momentum"] else None
        state["w"] = (normal(rows, cols) * cols ** -0.5).to(dtype) if case["momentum"] else new(rows, cols)
    return state


# ---------------------------------------------------------------- one pass
def _newton_schulz(u, steps):
    """Of 32-bit values, the longer side last."""
    x = u / (u.square().sum(dtype=torch.float64).sqrt() + NS_EPS).float()
    for _ in range(steps):
        a = torch.mm(x, x.t())
        x = NS_A * x + torch.mm(NS_B * a + NS_C * torch.mm(a, a), x)
    return x


def _plain(s):
    case, op, rows, cols = s["case"], s["case"]["op"], s["rows"], s["cols"]
    dtype = DTYPES[case["dtype"]]
    if op == "rmsnorm_forward":
        x, out = s["x"].float(), {}
        if s["residual"] is not None:  # the sum is kept in the type, for the next block, and normalised as kept
            out["sum"] = (x + s["residual"].float()).to(dtype)
            x = out["sum"].float()
        rstd = 1.0 / torch.sqrt(x.square().mean(-1) + EPS)
        h = x * rstd[:, None]
        y = h * s["weight"].float()
        out.update(y=y.to(dtype), rstd=rstd)
        if case["keep"]:
            out["whole"] = _whole_values(*_whole_encode(h), cols).to(torch.bfloat16)
        if case["eight"]:
            out["eight"] = _float_kept(y, 1).to(torch.bfloat16)
        return out
    if op == "rmsnorm_backward":
        dy = s["dy"].float()
        h = _whole_unpack(s["whole"], rows, cols) if case["keep"] else s["x"].float() * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = (g - h * (g * h).mean(-1)[:, None]) * s["rstd"][:, None]
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(dtype), "dweight": (dy * h).sum(0)}
    if op == "fp8_store":
        return _float_kept(s["x"].float(), 1).to(torch.bfloat16)
    if op == "fp8_store_weight":
        kept = _float_kept(s["w"].float(), BLOCK).to(torch.bfloat16)
        return {"w": kept, "across": kept.t().contiguous()}
    if op == "fp8_product":
        x = _float_kept(s["x"].float(), 1) if case["dense"] else _float_unpack(s["eight"], rows, cols)
        y = torch.mm(x, _float_unpack(s["w"], case["out"], cols).t())
        if s["bias"] is not None:
            y = y + s["bias"].float()
        if s["add"] is not None:
            y = y + s["add"].float()
        return y.to(dtype)
    u, out = s["grad"], {}
    if s["momentum"] is not None:
        out["momentum"] = s["momentum"].mul_(MOMENTUM).add_(u)
        u = u + MOMENTUM * out["momentum"]
    o = _newton_schulz(u, case["steps"]) if rows <= cols else _newton_schulz(u.t().contiguous(), case["steps"]).t()
    if s["momentum"] is None:
        out["w"] = o.to(dtype).contiguous()
        return out
    out["w"] = s["w"].copy_((1.0 - RATE * DECAY) * s["w"].float() - RATE * o)
    return out


def _scratch(s, size):
    """The workspace, which a program keeps from step to step."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(size(), 256), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own(s):
    from paper_2410_12707_amd import binding as B

    case, op, rows, cols = s["case"], s["case"]["op"], s["rows"], s["cols"]
    if op == "rmsnorm_forward":
        B.adatopk_rmsnorm_forward(s["x"], s["weight"], EPS, s["y"], s["rstd"], residual=s["residual"], sum_out=s["sum"], act8=s["whole"], fp8=s["eight"])
        out = {"y": s["y"], "rstd": s["rstd"]}
        if case["residual"]:
            out["sum"] = s["sum"]
        if case["keep"]:
            B.adatopk_act8_load(s["whole"], s["kept"][0])
            out["whole"] = s["kept"][0]
        if case["eight"]:
            B.adatopk_fp8_load(s["eight"], s["kept"][1])
            out["eight"] = s["kept"][1]
        return out
    if op == "rmsnorm_backward":
        ws = _scratch(s, lambda: B.adatopk_rmsnorm_backward_workspace_bytes(rows, cols))
        B.adatopk_rmsnorm_backward(s["dy"], s["x"], s["whole"], s["rstd"], s["weight"], s["dx"], s["dweight"], ws, dsum=s["dsum"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if op == "fp8_store":
        B.adatopk_fp8_store(s["x"], s["eight"])
        B.adatopk_fp8_load(s["eight"], s["y"])
        return s["y"]
    if op == "fp8_store_weight":
        B.adatopk_fp8_store_weight(s["w"], s["eight"], s["across"])
        B.adatopk_fp8_load(s["eight"], s["y"])
        B.adatopk_fp8_load(s["across"], s["yt"])
        return {"w": s["y"], "across": s["yt"]}
    if op == "fp8_product":
        if case["dense"]:
            B.adatopk_fp8_store(s["x"], s["eight"])
        ws = _scratch(s, lambda: B.adatopk_fp8_product_workspace_bytes(rows, case["out"], cols))
        B.adatopk_fp8_product(s["eight"], s["w"], cols, s["y"], ws, bias=s["bias"], add=s["add"])
        return s["y"]
    ws = _scratch(s, lambda: B.adatopk_muon_update_workspace_bytes(rows, cols))
    if s["momentum"] is None:
        B.adatopk_muon_update(s["grad"], None, 0.0, False, s["w"], 1.0, 0.0, ws, steps=case["steps"], eps=NS_EPS)
        return {"w": s["w"]}
    B.adatopk_muon_update(s["grad"], s["momentum"], MOMENTUM, True, s["w"], -RATE, 1.0 - RATE * DECAY, ws, steps=case["steps"], eps=NS_EPS)
    return {"momentum": s["momentum"], "w": s["w"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Each input read once and each output written once; what is kept in 8 bits is written, and read where the pass reads it back."""
    rows, cols, out, op = case["rows"], case["cols"], case["out"], case["op"]
    n, e = rows * cols, 4 if case["dtype"] == "f32" else 2
    whole = rows * _up(cols, GROUP) // GROUP * (GROUP + 1)
    eight = rows * _up(cols, BLOCK) // BLOCK * (BLOCK + 1)
    if op == "rmsnorm_forward":
        read_back = (2 * whole + 2 * n if case["keep"] else 0) + (2 * eight + 2 * n if case["eight"] else 0)
        return {"bytes": n * e * (4 if case["residual"] else 2) + cols * e + 4 * rows + read_back, "flops": 4 * n}
    if op == "rmsnorm_backward":
        return {"bytes": n * e * (3 if case["residual"] else 2) + (whole if case["keep"] else n * e) + 4 * rows + cols * (e + 4), "flops": 9 * n}
    if op == "fp8_store":
        return {"bytes": n * e + 2 * eight + 2 * n, "flops": 2 * n}
    if op == "fp8_store_weight":
        return {"bytes": n * e + 4 * eight + 4 * n, "flops": 2 * n}
    if op == "fp8_product":
        weight = out * _up(cols, BLOCK) // BLOCK * (BLOCK + 1)
        return {"bytes": weight + (n * e + 2 * eight if case["dense"] else eight) + rows * out * e * (2 if case["residual"] else 1) + (out * e if case["bias"] else 0),
                "flops": 2 * n * out}
    less, more = min(rows, cols), max(rows, cols)
    # X X^T and A A are symmetric: half of each
    return {"bytes": n * (4 + e) + (n * (8 + e) if case["momentum"] else 0), "flops": case["steps"] * (3 * less * less * more + less ** 3)}


# ---------------------------------------------------------------- the definition in 64 bits
def _two_to(e):
    """2^e in 64 bits, from its bits (a power function need not be exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _whole64(x):
    """x / step, rounded and clamped, times step, with step a 64th of the power of two at or below the group's largest magnitude."""
    kept = torch.empty_like(x)
    for lo in range(0, x.shape[1], GROUP):  # group by group
        part = x[:, lo:lo + GROUP]
        _, exponent = torch.frexp(part.abs().amax(1, keepdim=True))  # magnitude = m * 2^exponent, m in [1/2, 1)
        step = _two_to((exponent - 1).clamp(min=-120) - 6)
        kept[:, lo:lo + GROUP] = torch.clamp(torch.round(part / step), -127, 127) * step
    return kept


def _float64(x, tile):
    """The nearest multiples of each number's own step, an eighth of the power of two at or below it, at least 2^-9 scales."""
    kept = torch.empty_like(x)
    for lo in range(0, x.shape[1], BLOCK):
        part = x[:, lo:lo + BLOCK]
        most = part.abs().amax(1)
        if tile > 1:
            most = torch.cat([piece.amax().expand(piece.numel()) for piece in most.split(tile)])
        m, exponent = torch.frexp(most)  # m * 2^exponent <= 448 scales = 0.875 * 2^9 scales
        scale = (exponent - 9 + (m > 0.875).int()).clamp(min=-126)
        _, own_exponent = torch.frexp(part)
        step = _two_to(torch.maximum(own_exponent - 4, scale.unsqueeze(1) - 9))
        kept[:, lo:lo + BLOCK] = torch.round(part / step) * step
    return kept


def _read_whole(buffer, rows, cols):
    width = -(-cols // GROUP)
    numbers = buffer[:rows * width * GROUP].view(torch.int8).double().view(rows, width * GROUP)
    start = -(-(rows * width * GROUP) // 256) * 256
    scale = _two_to(buffer[start:start + rows * width].long() - 133).view(rows, width)
    return (numbers * scale.repeat_interleave(GROUP, 1))[:, :cols]


def _read_float(buffer, rows, cols):
    """Sign, exponent and significand of every byte taken apart."""
    width, high = -(-cols // BLOCK), -(-rows // 256) * 256
    byte = buffer[:rows * width * BLOCK].long().view(rows, width * BLOCK)
    exponent, fraction = (byte >> 3) & 15, (byte & 7).double()
    value = torch.where(exponent > 0, (8.0 + fraction) * _two_to(exponent - 10), fraction * 2.0 ** -9)
    value = torch.where(byte > 127, -value, value)
    start = -(-(rows * width * BLOCK) // 256) * 256
    scale = _two_to(buffer[start:start + width * high].long().view(width, high)[:, :rows] - 127).t()
    return (value * scale.repeat_interleave(BLOCK, 1))[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op, rows, cols, dtype = case["op"], case["rows"], case["cols"], DTYPES[case["dtype"]]
    if op == "rmsnorm_forward":
        x, out = s["x"].double(), {}
        if case["residual"]:
            out["sum"] = x + s["residual"].double()
            x = out["sum"].to(dtype).double()
        rstd = (torch.linalg.vecdot(x, x) / cols + EPS).pow(-0.5)
        h = x * rstd.unsqueeze(1)
        out.update(y=h * s["weight"].double(), rstd=rstd)
        if case["keep"]:
            out["whole"] = _whole64(h)
        if case["eight"]:
            out["eight"] = _float64(out["y"], 1)
        return out
    if op == "rmsnorm_backward":
        dy, rstd, w = s["dy"].double(), s["rstd"].double().unsqueeze(1), s["weight"].double()
        h = _read_whole(s["whole"], rows, cols) if case["keep"] else s["x"].double() * rstd
        dx = rstd * (dy * w) - h * (rstd * torch.linalg.vecdot(dy * w, h).unsqueeze(1) / cols)  # without its part along the row
        if case["residual"]:
            dx = dx + s["dsum"].double()
        return {"dx": dx, "dweight": torch.ones(rows, dtype=torch.float64, device="cuda") @ (dy * h)}
    if op == "fp8_store":
        return _float64(s["x"].double(), 1)
    if op == "fp8_store_weight":
        kept = _float64(s["w"].double(), BLOCK)
        return {"w": kept, "across": kept.t().contiguous()}
    if op == "fp8_product":
        x = _float64(s["x"].double(), 1) if case["dense"] else _read_float(s["eight"], rows, cols)
        y = (_read_float(s["w"], case["out"], cols) @ x.t().contiguous()).t()
        for more in ("bias", "add"):
            if s[more] is not None:
                y = y + s[more].double()
        return y.contiguous()
    g, out = s["grad"].double(), {}
    if case["momentum"]:
        out["momentum"] = MOMENTUM * s["momentum"].double() + g
        g = g + MOMENTUM * out["momentum"]
    x = g / (torch.linalg.matrix_norm(g) + NS_EPS)
    one = torch.eye(min(rows, cols), dtype=torch.float64, device="cuda")
    for _ in range(case["steps"]):  # the polynomial of the smaller of X X^T and X^T X, on its side
        gram = x @ x.t().contiguous() if rows <= cols else x.t().contiguous() @ x
        factor = NS_A * one + gram @ (NS_B * one + NS_C * gram)
        x = factor @ x if rows <= cols else x @ factor
    out["w"] = (1.0 - RATE * DECAY) * s["w"].double() - RATE * x if case["momentum"] else x
    return out
