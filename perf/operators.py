"""The server-side operators of a wide MLP's iteration, as cases to be timed and compared.

Four operators:

  orthogonalize  a matrix (or a batch of them) pushed towards its nearest semi-orthogonal one by Newton-Schulz steps
                 X <- a X + (b A + c A^2) X, A = X X^T, from X = G / (||G||_F + eps)
  muon           one optimiser step of a weight matrix: momentum, Nesterov look-ahead, orthogonalised direction,
                 decoupled weight decay
  mx_quantize    microscaled 4-bit floating point (E2M1 elements, one power-of-two scale per 32 of a row) and back
  mx_gemm        product of two such matrices, D = A B^T

`run` computes them in elementary torch operations while `own` is false, and through the library's entry points
while it is true.
"""
import math

import torch

own = False

STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # output layer of the 784-200-10 network, and its hidden layer: calls where latency counts
        {"name": "orth-10x200-f32", "op": "orthogonalize", "batch": 1, "rows": 10, "cols": 200, "type": "f32"},
        {"name": "orth-200x784-f32", "op": "orthogonalize", "batch": 1, "rows": 200, "cols": 784, "type": "f32"},
        # a ragged batch of tall matrices, as the blocks of a split layer
        {"name": "orth-8x650x257-bf16", "op": "orthogonalize", "batch": 8, "rows": 650, "cols": 257, "type": "bf16"},
        # square hidden layer of the 1024-4096-4096-1000 network, gradients kept in 16 bits
        {"name": "orth-4096x4096-bf16", "op": "orthogonalize", "batch": 1, "rows": 4096, "cols": 4096, "type": "bf16"},
        # one optimiser step of the same network's first layer, fp32 master weights
        {"name": "muon-4096x1024-f32", "op": "muon", "rows": 4096, "cols": 1024, "type": "f32", "grad": "f32"},
        # and of its output layer with 16-bit weights and gradients
        {"name": "muon-1000x4096-bf16", "op": "muon", "rows": 1000, "cols": 4096, "type": "bf16", "grad": "bf16"},
        # one group's minibatch rows; and the upload factors of all 256 groups of 128 rows, quantised along the batch
        {"name": "quant-64x784-f32", "op": "mx_quantize", "rows": 64, "cols": 784, "transpose": False, "type": "f32"},
        {"name": "quant-32768x4096t-bf16", "op": "mx_quantize", "rows": 32768, "cols": 4096, "transpose": True,
         "type": "bf16"},
        # one sample through a hidden layer whose weights are kept in 4 bits
        {"name": "linear-1x4096x4096-bf16", "op": "mx_linear", "m": 1, "n": 4096, "k": 4096, "type": "bf16"},
        # a ragged batch through the output layer
        {"name": "linear-333x1000x4096-f32", "op": "mx_linear", "m": 333, "n": 1000, "k": 4096, "type": "f32"},
        # an evaluation slab of rows through a hidden layer
        {"name": "linear-4096x4096x4096-bf16", "op": "mx_linear", "m": 4096, "n": 4096, "k": 4096, "type": "bf16"},
        # the aggregate of a hidden layer's weight gradient over all groups' 4-bit upload factors
        {"name": "gemm-4096x4096x32768-f32", "op": "mx_gemm", "m": 4096, "n": 4096, "k": 32768, "type": "f32"},
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; mostly not a round number."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["orthogonalize", "orthogonalize", "muon", "muon", "mx_quantize", "mx_linear", "mx_linear",
                     "mx_gemm"])
    kind = rng.choice(["f32", "bf16"])
    if op == "orthogonalize":
        rows, cols = _size(rng, 1, 4096), _size(rng, 1, 4096)
        batch = 1 if rng.random() < 0.6 else _size(rng, 1, max(1, min(16, 4096 * 4096 // (rows * cols))))
        return {"op": op, "batch": batch, "rows": rows, "cols": cols, "type": kind}
    if op == "muon":
        return {"op": op, "rows": _size(rng, 1, 4096), "cols": _size(rng, 1, 4096), "type": kind,
                "grad": rng.choice(["f32", "bf16"])}
    if op == "mx_quantize":
        return {"op": op, "rows": _size(rng, 1, 32768), "cols": _size(rng, 1, 4096),
                "transpose": rng.random() < 0.5, "type": kind}
    m = 1 if op == "mx_linear" and rng.random() < 0.3 else _size(rng, 1, 4096)
    return {"op": op, "m": m, "n": _size(rng, 8, 4096), "k": _size(rng, 16, 4096 if op == "mx_linear" else 32768),
            "type": kind}


# ------------------------------------------------------------------------------------------------ inputs
def _gradient(gen, batch, rows, cols, dtype):
    """A weight gradient as a network meets it: errors^T x activations over a minibatch, features of uneven scale
    (the singular values fall off), and the noise floor that momentum leaves."""
    k = min(512, 2 * max(rows, cols))
    scale = lambda n: torch.exp(torch.randn(n, generator=gen, device="cuda"))  # noqa: E731
    dz = torch.randn(batch, k, rows, generator=gen, device="cuda") * scale(rows)
    act = torch.relu(torch.randn(batch, k, cols, generator=gen, device="cuda")) * scale(cols)
    g = dz.mT @ act / k
    g += 0.3 * g.square().mean().sqrt() * torch.randn(g.shape, generator=gen, device="cuda")
    return (1e-3 * g).to(dtype)


def _matrix(gen, rows, cols, dtype):
    """Activations or weights: normal values, rows of uneven size."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    dt = TYPES[case["type"]]
    op = case["op"]
    s = {"case": case}
    if op == "orthogonalize":
        g = _gradient(gen, case["batch"], case["rows"], case["cols"], dt)
        s["g"] = g if case["batch"] > 1 else g[0]
    elif op == "muon":
        r, c = case["rows"], case["cols"]
        s["w"] = (torch.randn(r, c, generator=gen, device="cuda") / math.sqrt(c)).to(dt)
        s["m"] = _gradient(gen, 1, r, c, torch.float32)[0]
        s["g"] = _gradient(gen, 1, r, c, TYPES[case["grad"]])[0]
    elif op == "mx_quantize":
        s["x"] = _matrix(gen, case["rows"], case["cols"], dt)
    elif op == "mx_linear":  # the weights are kept in 4 bits, the samples arrive as they are
        s["x"] = _matrix(gen, case["m"], case["k"], dt)
        s["b"] = _packed(_matrix(gen, case["n"], case["k"], torch.float32) / math.sqrt(case["k"]))
    else:
        s["a"] = _packed(_matrix(gen, case["m"], case["k"], torch.float32))
        s["b"] = _packed(_matrix(gen, case["n"], case["k"], torch.float32))
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _orthogonalize(g):
    """g: [..., rows, cols] in 32 or 64 bits."""
    a, b, c = COEF
    x = g / (g.square().sum((-2, -1), keepdim=True).sqrt() + EPS)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT
    for _ in range(STEPS):
        A = x @ x.mT
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.mT if tall else x


def _muon_scale(rows, cols):
    return math.sqrt(max(1.0, rows / cols))


LR, BETA, DECAY = 1e-3, 0.95, 0.01


def _blocks(x):
    """x [rows, cols] as blocks of 32 along the rows (zeros behind the end), and each block's scale exponent:
    floor(log2(largest magnitude)) - 2, the largest exponent of an element being 2."""
    r, c = x.shape
    nb = -(-c // 32)
    x = torch.nn.functional.pad(x, (0, nb * 32 - c)).view(r, nb, 32)
    top = x.abs().amax(-1)
    e = (torch.frexp(top).exponent - 3).clamp(-127, 127)
    return x, torch.where(top > 0, e, -127)


def _round_e2m1(x, e):
    """Magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6; ties to the even code; larger ones to 6."""
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), y)


def _mx_values(x):
    """The values that the 4-bit form of x stands for."""
    b, e = _blocks(x)
    v = torch.ldexp(_round_e2m1(b, e), e[..., None])
    return v.reshape(x.shape[0], -1)[:, :x.shape[1]]


def _packed(x):
    """The 4-bit form as the library lays it out: codes two to a byte, the even column in the low half, rows of whole
    blocks of 32; scales (exponent + 127) in tiles of 128 rows x 256 columns: [row tile][column tile][half][row % 32]
    [row % 128 / 32][block % 4]."""
    r, c = x.shape
    b, e = _blocks(x)
    q = _round_e2m1(b, e)
    a = q.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, 2 + a, 4 + a / 2)).to(torch.uint8)
    code |= torch.signbit(q).to(torch.uint8) << 3
    code = code.view(r, -1, 2)
    rt, ct = -(-r // 128), -(-c // 256)
    s = torch.zeros(rt * 128, ct * 8, dtype=torch.uint8, device=x.device)
    s[:r, :e.shape[1]] = (e + 127).to(torch.uint8)
    s = s.view(rt, 4, 32, ct, 2, 4).permute(0, 3, 4, 2, 1, 5).contiguous()
    return {"rows": r, "cols": c, "codes": (code[..., 0] | (code[..., 1] << 4)).contiguous(), "scales": s}


def _unpacked(q, dtype):
    r, c = q["rows"], q["cols"]
    codes = torch.stack((q["codes"] & 15, q["codes"] >> 4), -1).view(r, -1)
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype,
                         device=codes.device)
    s = q["scales"]
    rt, ct = s.shape[:2]
    e = s.permute(0, 4, 3, 1, 2, 5).reshape(rt * 128, ct * 8)[:r, :codes.shape[1] // 32].to(torch.int32) - 127
    v = torch.ldexp(table[codes.to(torch.int32)].view(r, -1, 32), e[..., None].to(dtype))
    return v.view(r, -1)[:, :c]


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        return _run_own(state, case, op)
    dt = TYPES[case["type"]]
    if op == "orthogonalize":
        return _orthogonalize(state["g"].float()).to(dt)
    if op == "muon":
        m, g, w = state["m"], state["g"].float(), state["w"]
        m.mul_(BETA).add_(g, alpha=1 - BETA)
        o = _orthogonalize((1 - BETA) * g + BETA * m)
        w.copy_(w.float() * (1 - LR * DECAY) - LR * _muon_scale(*w.shape) * o)
        return {"w": w, "m": m}
    if op == "mx_quantize":
        x = state["x"].float()
        return _mx_values(x.T if case["transpose"] else x).to(torch.bfloat16)
    b = _unpacked(state["b"], torch.float32)
    a = _mx_values(state["x"].float()) if op == "mx_linear" else _unpacked(state["a"], torch.float32)
    return (a @ b.T).to(dt)


def _run_own(state, case, op):
    from paper_2201_04301_b200 import binding
    dt = TYPES[case["type"]]
    if op == "orthogonalize":
        return binding.orthogonalize(state["g"], steps=STEPS, coef=COEF, eps=EPS)
    if op == "muon":
        w = state["w"]
        binding.muon_update(w, state["m"], state["g"], lr=LR, beta=BETA, weight_decay=DECAY, nesterov=True,
                            scale=_muon_scale(*w.shape), steps=STEPS, coef=COEF, eps=EPS)
        return {"w": w, "m": state["m"]}
    if op == "mx_quantize":
        return binding.mx_quantize(state["x"], transpose=case["transpose"]).dequantize(torch.bfloat16)
    b = binding.MxMatrix(**state["b"])
    a = binding.mx_quantize(state["x"]) if op == "mx_linear" else binding.MxMatrix(**state["a"])
    return binding.mx_gemm(a, b, dtype=dt)


# ------------------------------------------------------------------------------------------------ accounting
def _matrix_bytes(rows, cols):
    return rows * cols / 2 + rows * cols / 32


def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2}
    if op in ("orthogonalize", "muon"):
        n, r, c = case.get("batch", 1), min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # A and A^2 are symmetric: half of their entries are enough
        flops = n * STEPS * (r * r * c + r ** 3 + 2 * r * r * c)
        if op == "orthogonalize":
            return {"bytes": 2 * n * r * c * size[case["type"]], "flops": flops}
        return {"bytes": r * c * (2 * size[case["type"]] + 8 + size[case["grad"]]), "flops": flops}
    if op == "mx_quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * size[case["type"]] + n * 2, "flops": 4 * n}
    m, n, k = case["m"], case["n"], case["k"]
    a = m * k * size[case["type"]] if op == "mx_linear" else _matrix_bytes(m, k)
    return {"bytes": a + _matrix_bytes(n, k) + m * n * size[case["type"]], "flops": 2 * m * n * k}


def _exact_e2m1(x):
    """Values of the 4-bit form in 64 bits, straight from the definition: the nearest of the 15 values times the
    block's scale, the even code on a tie."""
    r, c = x.shape
    nb = -(-c // 32)
    p = torch.zeros(r, nb * 32, dtype=torch.float64, device=x.device)
    p[:, :c] = x
    p = p.view(r, nb, 32)
    top = p.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
    e = torch.where(torch.exp2(e) > top, e - 1, torch.where(torch.exp2(e + 1) <= top, e + 1, e))  # the logarithm is rounded
    scale = torch.exp2((e - 2).clamp(-127, 127))
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    y = (p / scale).abs()
    hi = torch.searchsorted(grid, y.clamp(max=6)).clamp(max=7)  # smallest value that is not below y
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - y, y - grid[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0)) | (y >= 6)
    v = torch.where(take_hi, grid[hi], grid[lo]) * torch.sign(p) * scale
    return v.view(r, -1)[:, :c]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("orthogonalize", "muon"):
        g = s["g"].double()
        if op == "muon":
            m = BETA * s["m"].double() + (1 - BETA) * g
            g = (1 - BETA) * g + BETA * m
        a, b, c = COEF
        x = g / (torch.linalg.matrix_norm(g)[..., None, None] + EPS)
        eye = torch.eye(min(x.shape[-2:]), dtype=torch.float64, device=x.device)
        for _ in range(STEPS):
            if x.shape[-2] > x.shape[-1]:
                A = x.mT @ x
                x = x @ (a * eye + b * A + c * (A @ A))
            else:
                A = x @ x.mT
                x = (a * eye + b * A + c * (A @ A)) @ x
        if op == "orthogonalize":
            return x
        w = s["w"].double() * (1 - LR * DECAY) - LR * math.sqrt(max(1.0, g.shape[0] / g.shape[1])) * x
        return {"w": w, "m": m}
    if op == "mx_quantize":
        x = s["x"].double()
        if x.numel() > 1 << 26:  # the whole at once would not fit beside the inputs: the columns in parts
            parts = [_exact_e2m1(p) for p in (x.T if case["transpose"] else x).split(256)]
            return torch.cat(parts)
        return _exact_e2m1(x.T if case["transpose"] else x)
    b = _unpacked(s["b"], torch.float64)
    a = _exact_e2m1(s["x"].double()) if op == "mx_linear" else _unpacked(s["a"], torch.float64)
    return a @ b.T
