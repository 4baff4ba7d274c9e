"""The matrix operators against 64-bit forms: orthogonalised updates, 4-bit quantisation and product."""
import math

import numpy as np
import pytest
import torch

from oracle import matrix as om
from paper_2201_04301_b200 import binding

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}         # half a step of the output type, relative
# HALF: a step rounds three operands (X, A, the polynomial) to fp16, each by at most 2^-11 of its norm; that reaches
# the new iterate through the polynomial, |b s^2 + c s^4| <= 2.81 on the iterates' range, and later steps contract
# errors of singular values near one by |p'| , p / s <= 0.72: sum <= 3 * 2^-11 * 2.81 / (1 - 0.72).
HALF_TOL = 3 * 2.0 ** -11 * 2.81 / 0.28
# FULL: the iterate is kept in 22 bits; rounding into directions of tiny singular values grows 3.4445-fold a step:
# 3.4445^4 * 2^-22 * 3.4445 of X_0's unit norm (the results here have norms of at least one).
FULL_TOL = 3.4445 ** 5 * 2.0 ** -22


def rel(x, y):
    return np.linalg.norm(x - y) / max(np.linalg.norm(y), 1e-300)


def num(t):
    return t.detach().double().cpu().numpy()


def spectrum(rows, cols, kind, seed=0):
    gen = np.random.default_rng(seed)
    if kind == "gauss":
        return gen.standard_normal((rows, cols))
    u, _, v = np.linalg.svd(gen.standard_normal((rows, cols)), full_matrices=False)
    i = np.arange(1, min(rows, cols) + 1)
    s = {"power": 1.0 / i ** 2, "rank": (i <= max(1, len(i) // 3)).astype(float)}[kind]
    return (u * s) @ v


# ------------------------------------------------------------------------------------------- refusals (no device work)
def c_orth(lib, **kw):
    a = dict(g=4096, o=8192, type=0, batch=1, rows=4, cols=4, ld_g=4, sg=0, ld_o=4, so=0, prec=0, steps=5, eps=1e-7,
             work=4096, bytes=1 << 30, coef=None)
    a.update(kw)
    buf = binding.C.create_string_buffer(256)
    VP = binding._VP
    coef = (binding.C.c_double * 3)(*a["coef"]) if a["coef"] else None
    st = lib.gcada_orthogonalize(VP(a["g"]), VP(a["o"]), a["type"], a["batch"], a["rows"], a["cols"], a["ld_g"], a["sg"],
                                 a["ld_o"], a["so"], a["prec"], a["steps"], coef, a["eps"], VP(a["work"]), a["bytes"],
                                 None, None, buf, 256)
    return st, buf.value.decode()


@pytest.mark.parametrize("bad", [
    dict(type=2), dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 20) + 1), dict(batch=65536),
    dict(prec=2), dict(steps=-1), dict(steps=101), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(coef=(17.0, 0.0, 0.0)), dict(coef=(1.0, float("nan"), 0.0)), dict(g=0), dict(o=0), dict(g=4098),
    dict(ld_g=3), dict(ld_o=3), dict(batch=2, sg=16, so=15), dict(batch=2, sg=-1, so=16), dict(work=0),
    dict(work=4097), dict(bytes=8)])
def test_orthogonalize_refuses(lib, bad):
    st, text = c_orth(lib, **bad)
    assert st == binding.EINVAL and text


@pytest.mark.parametrize("bad", [dict(sg=0), dict(sg=17), dict(ld_g=5, sg=20), dict(ld_o=5, so=20, sg=20)])
def test_orthogonalize_refuses_batches_in_place_of_another_layout(lib, bad):
    """One matrix, three times, with the first result in its place: the others might read the result."""
    st, text = c_orth(lib, **{**dict(batch=3, g=8192, o=8192, sg=16, so=16), **bad})
    assert st == binding.EINVAL and "layout" in text


def test_empty_matrices_are_no_error(lib):
    for kw in (dict(batch=0), dict(rows=0), dict(cols=0)):
        assert c_orth(lib, g=0, o=0, work=0, bytes=0, **kw)[0] == binding.OK
    n = binding.C.c_size_t(7)
    assert lib.gcada_orthogonalize_work(1, 0, 5, binding.C.byref(n)) == binding.OK and n.value == 0


def c_muon(lib, **kw):
    a = dict(w=4096, m=8192, g=4096 * 3, wt=0, gt=0, rows=4, cols=4, ld=(4, 4, 4), lr=0.1, beta=0.9, wd=0.0, scale=1.0,
             work=4096, bytes=1 << 30)
    a.update(kw)
    buf = binding.C.create_string_buffer(256)
    VP = binding._VP
    st = lib.gcada_muon_update(VP(a["w"]), a["wt"], VP(a["m"]), VP(a["g"]), a["gt"], a["rows"], a["cols"], *a["ld"],
                               a["lr"], a["beta"], 1, a["wd"], a["scale"], 0, 5, None, 1e-7, VP(a["work"]), a["bytes"],
                               None, None, buf, 256)
    return st, buf.value.decode()


@pytest.mark.parametrize("bad", [
    dict(wt=3), dict(gt=-1), dict(rows=-1), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta=1.0), dict(beta=-0.1),
    dict(wd=float("inf")), dict(scale=float("nan")), dict(w=0), dict(m=0), dict(g=0), dict(m=8194), dict(ld=(3, 4, 4)),
    dict(ld=(4, 3, 4)), dict(ld=(4, 4, 3)), dict(work=0), dict(bytes=100), dict(m=4096), dict(g=4096), dict(g=8192)])
def test_muon_refuses(lib, bad):
    st, text = c_muon(lib, **bad)
    assert st == binding.EINVAL and text


def test_mx_refuses(lib):
    VP, C = binding._VP, binding.C
    buf = C.create_string_buffer(256)

    def quant(x=4096, t=0, rows=4, cols=4, ld=4, codes=4096, scales=4096):
        return lib.gcada_mx_quantize(VP(x), t, rows, cols, ld, 0, VP(codes), VP(scales), None, buf, 256)

    def dequant(x=4096, t=0, rows=4, cols=4, ld=4, codes=4096, scales=4096):
        return lib.gcada_mx_dequantize(VP(codes), VP(scales), rows, cols, VP(x), t, ld, None, buf, 256)

    for f in (quant, dequant):
        for bad in (dict(x=0), dict(x=4098), dict(t=5), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 22) + 1), dict(ld=3),
                    dict(codes=0), dict(scales=0), dict(codes=4100), dict(scales=4104)):
            assert f(**bad) == binding.EINVAL, bad
            assert buf.value
        assert f(x=0, rows=0) == binding.OK and f(x=0, cols=0) == binding.OK

    def gemm(a=4096, sa=4096, m=4, b=4096, sb=4096, n=4, k=32, d=4096, t=0, ld=4, alpha=1.0, beta=0.0, bias=0):
        return lib.gcada_mx_gemm(VP(a), VP(sa), m, VP(b), VP(sb), n, k, VP(d), t, ld, alpha, beta, VP(bias), None, None, buf, 256)

    for bad in (dict(a=0), dict(sa=0), dict(b=0), dict(sb=0), dict(d=0), dict(d=4098), dict(bias=2), dict(k=0), dict(m=-1),
                dict(n=-1), dict(t=2), dict(ld=3), dict(alpha=float("nan")), dict(beta=float("inf")), dict(a=4100)):
        assert gemm(**bad) == binding.EINVAL, bad
    assert gemm(m=0, a=0) == binding.OK and gemm(n=0, b=0, ld=0) == binding.OK
    n, s = C.c_size_t(), C.c_size_t()
    assert lib.gcada_mx_size(-1, 4, C.byref(n), C.byref(s)) == binding.EINVAL
    assert lib.gcada_mx_size(130, 257, C.byref(n), C.byref(s)) == binding.OK and (n.value, s.value) == (130 * 144, 4 * 1024)


def test_without_a_device_the_operators_fail(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    st, text = c_orth(lib)
    assert st == binding.ECUDA and text
    st, text = c_muon(lib)
    assert st == binding.ECUDA and text
    buf = binding.C.create_string_buffer(256)
    VP = binding._VP
    assert lib.gcada_mx_quantize(VP(4096), 0, 4, 4, 4, 0, VP(4096), VP(8192), None, buf, 256) == binding.ECUDA and buf.value
    assert lib.gcada_mx_gemm(VP(4096), VP(4096), 4, VP(4096), VP(4096), 4, 32, VP(4096), 0, 4, 1.0, 0.0, None, None, None, buf, 256) == binding.ECUDA
    assert lib.gcada_mx_gemm(VP(4096), VP(4096), 4, VP(4096), VP(4096), 4, 32, VP(4096), 0, 4, 1.0, 0.0, None, None, None, None, 0) == binding.ECUDA


def test_python_refusals():
    x = torch.zeros(4, 4)
    for call in (lambda: binding.orthogonalize(x), lambda: binding.mx_quantize(x), lambda: binding.muon_update(x, x, x, 0.1),
                 lambda: binding.orthogonalize(x.double()), lambda: binding.MxMatrix(4, 4, x, x)):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------------------------------- orthogonalisation
SHAPES = [(1, 1), (1, 300), (300, 1), (2, 3), (10, 200), (63, 65), (64, 64), (129, 127), (200, 784), (257, 130), (96, 1000),
          (384, 256), (513, 520)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gauss", "power", "rank"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize(shape, kind):
    for t, precision in (("f32", "full"), ("bf16", "half"), ("f32", "half"), ("bf16", "full")):
        g = torch.from_numpy(spectrum(*shape, kind)).to(TYPES[t]).cuda()
        o = binding.orthogonalize(g, precision=precision)
        want = om.newton_schulz(num(g))
        assert rel(num(o), want) <= (FULL_TOL if precision == "full" else HALF_TOL) + OUT[t], (t, precision)
    binding.check_operators()


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_orthogonalize_batches_strides_and_places(t):
    tol = FULL_TOL if t == "f32" else HALF_TOL
    gen = torch.Generator(device="cuda").manual_seed(3)
    base = torch.randn(5, 70, 211, generator=gen, device="cuda").to(TYPES[t])
    g = base[1:4, 3:68, 5:206]                               # unaligned rows, a gap behind every row and matrix
    out = torch.full((3, 65, 203), 7.0, device="cuda").to(TYPES[t])
    binding.orthogonalize(g, out=out[:, :, 1:202])
    for i in range(3):
        assert rel(num(out[i, :, 1:202]), om.newton_schulz(num(g[i]))) <= tol + OUT[t]
    assert (out[:, :, 0] == 7).all() and (out[:, :, 202] == 7).all()
    one = binding.orthogonalize(g[0].clone())
    same = binding.orthogonalize(g[0].expand(3, 65, 201))   # the same matrix three times, without copies
    assert all(torch.equal(same[i], one) for i in range(3))
    place = g[0].clone()
    binding.orthogonalize(place, out=place)
    assert torch.equal(place, one)


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(12, 520, 700), (12, 700, 520), (40, 530, 610), (2, 1100, 900), (1, 300, 4000), (30, 128, 256)])
def test_orthogonalize_many_tiles(shape, t):
    gen = torch.Generator(device="cuda").manual_seed(7)
    g = torch.randn(shape, generator=gen, device="cuda").to(TYPES[t])
    o = binding.orthogonalize(g)
    for i in sorted({0, shape[0] // 2, shape[0] - 1}):
        assert rel(num(o[i]), om.newton_schulz(num(g[i]))) <= (FULL_TOL if t == "f32" else HALF_TOL) + OUT[t]
    assert torch.equal(o, binding.orthogonalize(g))
    binding.check_operators()


@pytest.mark.gpu
def test_orthogonalize_steps_coefficients_and_scale():
    g = torch.from_numpy(spectrum(40, 90, "gauss")).float().cuda()
    for steps in (0, 1, 2, 9):
        assert rel(num(binding.orthogonalize(g, steps=steps)), om.newton_schulz(num(g), steps)) <= FULL_TOL
    cubic = (1.5, -0.5, 0.0)
    o = binding.orthogonalize(g, steps=30, coef=cubic)
    assert rel(num(o), om.newton_schulz(num(g), 30, cubic)) <= FULL_TOL
    assert np.abs(num(o) @ num(o).T - np.eye(40)).max() < 1e-5
    for factor in (1e-30, 1e-6, 1e25):                       # the squares alone would leave fp32's range
        h = g * factor
        assert rel(num(binding.orthogonalize(h)), om.newton_schulz(num(h))) <= FULL_TOL
    z = torch.zeros(33, 70, device="cuda")
    assert (binding.orthogonalize(z) == 0).all()
    for bad in (float("nan"), float("inf")):
        h = g.clone()
        h[3, 4] = bad
        assert binding.orthogonalize(h).isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_orthogonalize_extremes(t):
    """What test_orthogonalize_steps_coefficients_and_scale checks for matrices that stay on chip, for larger ones."""
    tol = (FULL_TOL if t == "f32" else HALF_TOL) + OUT[t]
    for shape in ((100, 150), (150, 100), (700, 300)):
        g = torch.from_numpy(spectrum(*shape, "gauss")).to(TYPES[t]).cuda()
        for factor in (1e-30, 1e-9, 1e-6, 1e25):
            h = g * factor
            assert rel(num(binding.orthogonalize(h)), om.newton_schulz(num(h))) <= tol, (shape, factor)
        for steps in (0, 1, 2, 9):
            assert rel(num(binding.orthogonalize(g, steps=steps)), om.newton_schulz(num(g), steps)) <= tol
        assert (binding.orthogonalize(torch.zeros_like(g)) == 0).all()
        for bad in (float("nan"), float("inf"), -float("inf")):
            h = g.clone()
            h[3, 4] = bad
            assert binding.orthogonalize(h).isnan().all()
    assert binding.orthogonalize(g[:0]).shape == (0, 300) and binding.orthogonalize(g[:, :0]).shape == (700, 0)
    assert binding.orthogonalize(g[None][:0]).shape == (0, 700, 300)
    assert binding.mx_quantize(g[:0]).dequantize().shape == (0, 300)
    q = binding.mx_quantize(g)
    assert binding.mx_gemm(binding.mx_quantize(g[:0]), q).shape == (0, 700)
    with pytest.raises(binding.GCadaError):
        binding.mx_gemm(binding.mx_quantize(g[:, :0]), binding.mx_quantize(g[:, :0]))
    for bad in (g.T, g[:, ::2], g.double()):
        with pytest.raises(ValueError):
            binding.orthogonalize(bad)


def exact_orthogonalize(g, steps=5):
    """The 64-bit form on the device, for sweeps."""
    x = g.double()
    x = x / (torch.linalg.matrix_norm(x)[..., None, None] + 1e-7)
    a, b, c = om.COEF
    for _ in range(steps):
        s = x @ x.mT if x.shape[-2] <= x.shape[-1] else x.mT @ x
        p = b * s + c * (s @ s)
        x = a * x + (p @ x if x.shape[-2] <= x.shape[-1] else x @ p)
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_orthogonalize_sweep(seed):
    rng = np.random.default_rng(seed)
    for _ in range(25):
        rows, cols = (int(round(np.exp(rng.uniform(0, np.log(1500))))) for _ in range(2))
        batch = int(rng.integers(1, 4))
        t = ("f32", "bf16")[int(rng.integers(2))]
        gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
        g = torch.randn(batch, rows, cols, generator=gen, device="cuda")
        g *= torch.exp(torch.randn(batch, rows, 1, generator=gen, device="cuda"))
        g = g.to(TYPES[t])
        want = exact_orthogonalize(g)
        for precision, tol in (("full", FULL_TOL), ("half", HALF_TOL)):
            o = binding.orthogonalize(g, precision=precision)
            err = torch.linalg.matrix_norm(o.double() - want) / torch.linalg.matrix_norm(want)
            assert (err <= tol + OUT[t]).all(), (batch, rows, cols, t, precision, err)
    binding.check_operators()


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(4))
def test_product_sweep(seed):
    rng = np.random.default_rng(seed)
    for _ in range(25):
        m, n, k = (int(round(np.exp(rng.uniform(0, np.log(top))))) for top in (1500, 1500, 6000))
        gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
        x, y = (torch.randn(s, k, generator=gen, device="cuda") * torch.exp(2 * torch.randn(s, 1, generator=gen, device="cuda")) for s in (m, n))
        a, b = binding.mx_quantize(x), binding.mx_quantize(y.T.contiguous(), transpose=True)
        av, bv = a.dequantize().double(), b.dequantize().double()
        d = binding.mx_gemm(a, b).double()
        assert ((d - av @ bv.T).abs() <= (k / 32 + 3) * 2.0 ** -23 * (av.abs() @ bv.abs().T)).all(), (m, n, k)
    binding.check_operators()


@pytest.mark.gpu
def test_orthogonalize_streams_graphs_and_repeats():
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = torch.randn(150, 333, generator=gen, device="cuda")
    want = binding.orthogonalize(g)
    assert torch.equal(binding.orthogonalize(g), want)       # the order of every sum is fixed
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = binding.orthogonalize(g, stream=side)
    side.synchronize()
    assert torch.equal(other, want)
    raw = binding.orthogonalize(g, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(raw, want)
    work = torch.empty(binding.orthogonalize_work(g), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(g)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.orthogonalize(g, out=out, work=work)
    g.copy_(torch.randn(150, 333, generator=gen, device="cuda"))
    want = binding.orthogonalize(g)
    for _ in range(2):
        out.zero_()
        work.random_(0, 256)                                 # what the work area holds before a call means nothing
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    with pytest.raises(binding.GCadaError):
        binding.orthogonalize(g, work=work[:1024])


# ------------------------------------------------------------------------------------------- optimiser step
@pytest.mark.gpu
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(1, 1), (7, 50), (130, 33), (200, 300)])
@pytest.mark.parametrize("wt,gt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_muon_update(shape, wt, gt, nesterov):
    gen = torch.Generator(device="cuda").manual_seed(11)
    pad = lambda dt: torch.randn(shape[0] + 2, shape[1] + 3, generator=gen, device="cuda").to(dt)  # noqa: E731
    wb, mb, gb = pad(TYPES[wt]), pad(torch.float32), pad(TYPES[gt])
    w, m, g = (t[1:-1, 2:-1] for t in (wb, mb, gb))
    keep = [t.clone() for t in (wb, mb, gb)]
    kw = dict(lr=0.05, beta=0.9, weight_decay=0.1, scale=1.3)
    rw, rm = num(w), num(m)
    for _ in range(2):
        rw, rm = om.muon(rw, rm, num(g), nesterov=nesterov, **kw)
        binding.muon_update(w, m, g, nesterov=nesterov, **kw)
        if wt == "bf16":
            # the stored weights are rounded after every step: half a step of bf16, plus the direction's error
            step = kw["lr"] * kw["scale"] * 1.3 * math.sqrt(min(shape))
            assert np.abs(num(w) - rw).max() <= 2.0 ** -8 * np.abs(rw).max() + HALF_TOL * step
            rw = num(w)
        else:
            # fp32: the direction's error times the step, and a few roundings of the weight
            assert np.linalg.norm(num(w) - rw) <= FULL_TOL * kw["lr"] * kw["scale"] * 1.3 * math.sqrt(min(shape)) + 2.0 ** -22 * np.linalg.norm(rw)
        assert rel(num(m), rm) <= 2.0 ** -22
    for t, k in zip((wb, mb, gb), keep):                     # nothing outside the matrices
        edge = torch.ones_like(t, dtype=torch.bool)
        edge[1:-1, 2:-1] = False
        assert torch.equal(t[edge], k[edge])


# ------------------------------------------------------------------------------------------- 4-bit matrices
def special_matrix(rows, cols, seed=0):
    gen = np.random.default_rng(seed)
    x = gen.standard_normal((rows, cols)) * np.exp2(gen.integers(-20, 20, (rows, 1)))
    x = x.astype(np.float32)
    if rows > 3 and cols > 8:
        x[0] = 0
        x[1, :8] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]       # ties, and 5 between 4 and 6
        x[2, :8] = [7.9, 6, -7, -0.25, -0.75, 0.0, -0.0, 4]       # beyond the largest value
        x[3, :4] = [1e-45, 3e-39, -2e-42, 0]                      # subnormals
        x[3, 4:] = 0
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 31), (5, 32), (4, 33), (31, 256), (128, 257), (129, 64), (70, 500), (300, 130)])
def test_quantize_and_read_back(shape, t):
    x = torch.from_numpy(special_matrix(*shape)).to(TYPES[t]).cuda()
    codes, exps = om.mx_quantize(num(x))
    packed, scales = om.mx_pack(codes, exps)
    wide = torch.full((shape[1], shape[0] + 3), 5.0, device="cuda").to(TYPES[t])
    wide[:, 1:-2] = x.T
    for transpose, src in ((False, x), (True, x.T.contiguous()), (True, wide[:, 1:-2])):
        q = binding.mx_quantize(src, transpose=transpose)
        assert (q.rows, q.cols) == shape
        assert np.array_equal(q.codes.cpu().numpy(), packed) and np.array_equal(q.scales.cpu().numpy(), scales)
    want = om.mx_values(codes, exps, shape[1])
    assert np.array_equal(num(q.dequantize(torch.float32)), want)
    back = num(q.dequantize(torch.bfloat16))
    normal = np.abs(want) >= 2.0 ** -126
    assert np.array_equal(back[normal], want[normal])
    padded = torch.full((shape[0], shape[1] + 5), 9.0, device="cuda")
    q.dequantize(out=padded[:, 2:-3])
    assert np.array_equal(num(padded[:, 2:-3]), want) and (padded[:, :2] == 9).all() and (padded[:, -3:] == 9).all()


@pytest.mark.gpu
def test_infinities_and_nan_take_their_block_only():
    x = torch.randn(130, 96, device="cuda")
    x[3, 40], x[129, 0], x[5, 95] = float("inf"), float("nan"), -float("inf")
    for transpose in (False, True):
        q = binding.mx_quantize(x.T.contiguous() if transpose else x, transpose=transpose)
        v = q.dequantize()
        hole = torch.zeros_like(x, dtype=torch.bool)
        hole[3, 32:64] = hole[129, :32] = hole[5, 64:] = True
        assert v[hole].isnan().all() and v[~hole].isfinite().all()
    b = binding.mx_quantize(torch.randn(70, 96, device="cuda"))
    d = binding.mx_gemm(q, b)
    rows = torch.zeros(130, dtype=torch.bool)
    rows[[3, 129, 5]] = True
    assert d[rows].isnan().all() and d[~rows].isfinite().all()


GEMMS = [(1, 1, 1), (1, 8, 32), (3, 5, 33), (1, 300, 1000), (2, 257, 96), (8, 130, 513), (16, 64, 64), (17, 1000, 300), (64, 40, 4096),
         (128, 128, 256), (129, 127, 257), (130, 333, 700), (300, 260, 64), (1, 4096, 128), (1500, 2100, 160), (200, 500, 3000), (257, 1025, 2050), (2600, 2300, 1030), (4000, 5000, 300)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", GEMMS)
def test_product(shape):
    m, n, k = shape
    gen = torch.Generator(device="cuda").manual_seed(m * 1000 + n)
    a = binding.mx_quantize(torch.randn(m, k, generator=gen, device="cuda") * torch.exp(torch.randn(m, 1, generator=gen, device="cuda")))
    b = binding.mx_quantize(torch.randn(n, k, generator=gen, device="cuda"))
    av, bv = a.dequantize().double(), b.dequantize().double()
    exact, mass = av @ bv.T, av.abs() @ bv.abs().T
    # fp32 sums of exact products: one rounding (or cut) of at most 2^-23 of the sum of magnitudes per 32 products
    tol = (k / 32 + 3) * 2.0 ** -23 * mass
    d = binding.mx_gemm(a, b)
    assert ((d.double() - exact).abs() <= tol).all()
    d = binding.mx_gemm(a, b, dtype=torch.bfloat16)
    assert ((d.double() - exact).abs() <= tol + 2.0 ** -8 * exact.abs()).all()
    bias = torch.randn(n, generator=gen, device="cuda")
    for t in ("f32", "bf16"):
        c = torch.randn(m, n + 3, generator=gen, device="cuda").to(TYPES[t])
        before = c.clone()
        binding.mx_gemm(a, b, out=c[:, 2:-1], alpha=0.5, beta=-1.5, bias=bias)
        want = 0.5 * exact + bias.double() - 1.5 * before[:, 2:-1].double()
        size = mass + bias.double().abs() + 2 * before[:, 2:-1].double().abs()
        assert ((c[:, 2:-1].double() - want).abs() <= (k / 32 + 6) * 2.0 ** -23 * size + OUT[t] * want.abs()).all()
        assert torch.equal(c[:, :2], before[:, :2]) and torch.equal(c[:, -1], before[:, -1])
    nan = torch.full((m, n), float("nan"), device="cuda")    # beta = 0: what was there is not read
    assert torch.equal(binding.mx_gemm(a, b, out=nan), binding.mx_gemm(a, b))
    binding.check_operators()


@pytest.mark.gpu
def test_product_streams_and_graphs():
    x, w = torch.randn(77, 500, device="cuda"), torch.randn(90, 500, device="cuda")
    b = binding.mx_quantize(w)
    want = binding.mx_gemm(binding.mx_quantize(x), b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q = binding.mx_quantize(x, stream=side)
    d = binding.mx_gemm(q, b, stream=side)
    side.synchronize()
    assert torch.equal(d, want)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mx_gemm(binding.mx_quantize(x), b, out=out)
    x.mul_(-2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, -2 * want)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 64, 486), (1, 64, 492), (1, 64, 733), (1, 740, 64), (16, 64, 480), (17, 64, 480), (64, 40, 300),
                                   (65, 40, 300), (130, 64, 64), (200, 30, 500), (500, 12, 33), (300, 70, 64)])
def test_orthogonalize_narrow_batches(shape):
    """Both sides of what decides, by work and batch, whether a narrow matrix stays on chip."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    for t in ("f32", "bf16"):
        g = torch.randn(shape, generator=gen, device="cuda").to(TYPES[t])
        work = torch.empty(binding.orthogonalize_work(g), dtype=torch.uint8, device="cuda")
        for precision, tol in (("full", FULL_TOL), ("half", HALF_TOL)):
            o = binding.orthogonalize(g, precision=precision, work=work)
            for i in sorted({0, shape[0] // 3, shape[0] - 1}):
                assert rel(num(o[i]), om.newton_schulz(num(g[i]))) <= tol + OUT[t], (t, precision, i)
            if min(shape[1:]) <= 64:                              # narrow matrices have fp32 accuracy either way
                assert rel(num(o[0]), om.newton_schulz(num(g[0]))) <= FULL_TOL + OUT[t], (t, precision)
    binding.check_operators()


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    """Chains of large and small calls side by side, each with its own work area, then two captured chains replayed
    side by side: the same bits as one after the other."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    mats = [torch.randn(s, generator=gen, device="cuda").to(t) for s in ((300, 900), (40, 200), (2, 520, 260), (10, 90))
            for t in (torch.float32, torch.bfloat16)]
    x, w = torch.randn(200, 640, generator=gen, device="cuda"), torch.randn(333, 640, generator=gen, device="cuda")
    b = binding.mx_quantize(w)

    def chain(order, outs, works):
        for i in order:
            binding.orthogonalize(mats[i], out=outs[i], work=works[i])
            binding.mx_gemm(binding.mx_quantize(x), b, out=outs[-1])

    def buffers():
        return ([torch.zeros_like(g) for g in mats] + [torch.zeros(200, 333, device="cuda")],
                [torch.empty(binding.orthogonalize_work(g), dtype=torch.uint8, device="cuda") for g in mats])

    want, works = buffers()
    chain(range(len(mats)), want, works)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    orders = [list(range(len(mats))), list(reversed(range(len(mats))))]
    places = [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(3):
        for side, order, place in zip(sides, orders, places):
            with torch.cuda.stream(side):
                chain(order, *place)
    torch.cuda.synchronize()
    for outs, _ in places:
        assert all(torch.equal(o, r) for o, r in zip(outs, want))
    graphs = []
    for order, (outs, works) in zip(orders, places):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            chain(order, outs, works)
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for side, graph in zip(sides, graphs):
            with torch.cuda.stream(side):
                graph.replay()
    torch.cuda.synchronize()
    for outs, _ in places:
        assert all(torch.equal(o, r) for o, r in zip(outs, want))
    binding.check_operators()


@pytest.mark.gpu
def test_rows_whose_offsets_pass_32_bits():
    rows, cols, ld = 70, 130, 36_000_000                       # the last row starts 2.5e9 elements behind the first
    far = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    g = far.as_strided((rows, cols), (ld, 1))
    out = far.as_strided((rows, cols), (ld, 1), 1001)
    g.copy_(torch.from_numpy(spectrum(rows, cols, "gauss")))
    near = g.contiguous()
    binding.orthogonalize(g, out=out)
    assert torch.equal(out, binding.orthogonalize(near))
    q = binding.mx_quantize(near)
    far_q = binding.mx_quantize(g)
    assert torch.equal(far_q.codes, q.codes) and torch.equal(far_q.scales, q.scales)
    assert torch.equal(binding.mx_quantize(g, transpose=True).codes, binding.mx_quantize(near, transpose=True).codes)
    q.dequantize(out=out)
    assert torch.equal(out, q.dequantize(torch.bfloat16))
    binding.mx_gemm(q, q, out=far.as_strided((rows, rows), (ld, 1), 2000))
    assert torch.equal(far.as_strided((rows, rows), (ld, 1), 2000), binding.mx_gemm(q, q, dtype=torch.bfloat16))
    m = torch.zeros(rows, cols, device="cuda")
    w, w2, m2 = out, out.contiguous(), m.clone()
    binding.muon_update(w, m, g, lr=0.1)
    binding.muon_update(w2, m2, near, lr=0.1)
    assert torch.equal(w, w2) and torch.equal(m, m2)
    binding.check_operators()


# ------------------------------------------------------------------------------------------- together
@pytest.mark.gpu
def test_an_iteration_of_the_server():
    """Three groups upload the factors of a weight gradient in 4 bits; their aggregate is one product over all rows;
    the weights move along its orthogonalised momentum."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    n_out, n_in, rows = 130, 200, 3 * 64
    w = torch.randn(n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)
    m = torch.zeros_like(w)
    rw, rm = num(w), num(m)
    for _ in range(3):
        dz = (torch.randn(rows, n_out, generator=gen, device="cuda") / rows).bfloat16()
        act = torch.relu(torch.randn(rows, n_in, generator=gen, device="cuda")).bfloat16()
        a, b = binding.mx_quantize(dz, transpose=True), binding.mx_quantize(act, transpose=True)
        agg = binding.mx_gemm(a, b)
        binding.muon_update(w, m, agg, lr=0.02, weight_decay=0.01)
        da, db = (om.mx_values(*om.mx_quantize(num(t).T), rows) for t in (dz, act))
        ra = da @ db.T
        assert (np.abs(num(agg) - ra) <= (rows / 32 + 3) * 2.0 ** -23 * (np.abs(da) @ np.abs(db).T)).all()
        rw, rm = om.muon(rw, rm, ra, 0.02, 0.95, True, 0.01, 1.0)
    assert np.linalg.norm(num(w) - rw) <= 3 * (FULL_TOL * 0.02 * 1.3 * math.sqrt(n_out) + 2.0 ** -22 * np.linalg.norm(rw))


# ------------------------------------------------------------------------------------------- accuracy
def even_spectrum(kind, rows, cols, seed=0):
    """Matrices whose singular values are all alike: nothing averages their roundings out."""
    gen = np.random.default_rng(seed)
    r = min(rows, cols)
    if kind == "identity":
        return np.eye(rows, cols)
    if kind == "permutation":
        x = np.zeros((rows, cols))
        x[gen.permutation(rows)[:r], gen.permutation(cols)[:r]] = gen.choice([-1.0, 1.0], r)
        return x
    u = np.linalg.qr(gen.standard_normal((max(rows, cols), r)))[0]
    return u if rows >= cols else np.ascontiguousarray(u.T)


def even_bound(r, operand, kept, steps=5):
    """First-order bound of the relative error where all r singular values are s_0 = r^-1/2.  A step rounds what it keeps (X, A,
    the polynomial's terms: `kept`, relative) and its products' operands (`operand`): with q = b A + c A^2
        dA <= 2 operand A,   dq <= |b + 2 c A| dA + 2 operand |c| A^2 + operand max(|q|, |q - b - c|)
        dx <= s (dq + operand |q| + kept (|a| + |b| A + |c| A^2 + 2))
    An error of a multiple of an orthogonal matrix grows by |p'(s)| in its symmetric and by p(s) / s in its other part."""
    a, b, c = om.COEF
    s, e = 1 / math.sqrt(r), 0.0
    for _ in range(steps):
        worst = max(max(abs(a + 3 * b * t * t + 5 * c * t ** 4), abs(a + b * t * t + c * t ** 4)) for t in (s - e, s, s + e))
        A = s * s
        q = b * A + c * A * A
        dq = abs(b + 2 * c * A) * 2 * operand * A + 2 * operand * abs(c) * A * A + operand * max(abs(q), abs(q - b - c))
        e = worst * e + s * (dq + operand * abs(q) + kept * (a + abs(b) * A + abs(c) * A * A + 2))
        s = s * (a + q)
    return e / s


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["identity", "permutation", "orthogonal"])
@pytest.mark.parametrize("shape", [(65, 65), (92, 92), (100, 180), (151, 151), (308, 308), (500, 398), (400, 400), (1024, 1024)])
def test_accuracy_where_all_singular_values_are_alike(shape, kind):
    """The accuracy that a caller gets without asking is that of fp32 arithmetic, whatever the type and the matrix: below
    half a step of bf16 too, which the products of 11-bit operands can miss by more than its half."""
    x = even_spectrum(kind, *shape)
    for t in ("f32", "bf16"):
        g = torch.from_numpy(x * 0.5).to(TYPES[t]).cuda()
        want = om.newton_schulz(num(g))
        # (a rounded orthogonal matrix has singular values within 2^-8 of each other: the bound's slope hardly moves)
        full = 1.1 * even_bound(min(shape), 2.0 ** -22, 2.0 ** -22) + OUT[t]
        assert rel(num(binding.orthogonalize(g)), want) <= full, t
        assert rel(num(binding.orthogonalize(g, precision="full")), want) <= full, t
        assert rel(num(binding.orthogonalize(g, precision="half")), want) <= 1.1 * even_bound(min(shape), 2.0 ** -11, 2.0 ** -22) + OUT[t], t
        assert rel(num(binding.orthogonalize(g, precision="half")), want) <= 0.04 + OUT[t], t      # what the header says
    w, m = torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, device="cuda")
    binding.muon_update(w, m, g, lr=-1.0, beta=0.0, scale=1.0)
    assert rel(num(w), want) <= full
    binding.check_operators()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(66, 700), (100, 150), (200, 784), (513, 520), (700, 300)])
def test_accuracy_of_either_precision_for_spread_spectra(shape):
    """The figures that the header gives for random matrices."""
    for kind in ("gauss", "power"):
        g = torch.from_numpy(spectrum(*shape, kind, seed=4)).float().cuda()
        want = om.newton_schulz(num(g))
        assert rel(num(binding.orthogonalize(g, precision="half")), want) <= (2e-3 if min(shape) >= 100 else 4e-3), kind
        assert rel(num(binding.orthogonalize(g, precision="full")), want) <= 2e-5, kind


@pytest.mark.gpu
def test_the_precision_is_full_unless_half_is_asked_for():
    gen = torch.Generator(device="cuda").manual_seed(8)
    for t in TYPES.values():
        g = torch.randn(130, 300, generator=gen, device="cuda").to(t)
        assert torch.equal(binding.orthogonalize(g), binding.orthogonalize(g, precision="full"))
        results = []
        for precision in (None, "full", "half"):
            w, m = torch.zeros(130, 300, dtype=t, device="cuda"), torch.zeros(130, 300, device="cuda")
            binding.muon_update(w, m, g, lr=0.1, precision=precision)
            results.append(w)
        assert torch.equal(results[0], results[1]) and not torch.equal(results[0], results[2])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(100, 150), (150, 100), (300, 300), (10, 200), (60, 40), (4, 4)])
def test_norms_far_below_eps(shape):
    """The largest eps with matrices so small that X_0 is beyond fp32's range: results of the formula's size, not NaN, and no
    digits lost on the way to results that are in range again."""
    g = torch.from_numpy(spectrum(*shape, "gauss")).float().cuda()
    grow = (1.875, -1.25, 0.375)                                # a tiny iterate grows 1.875-fold a step, 2e27-fold in a hundred
    for factor, eps in ((1e-20, 1e30), (1e-30, 1e20), (1e-38, 1e30), (1e-12, 1e30), (1.0, 1e30), (1e-38, 1e-7), (3e-44, 1e-7), (1e-25, 1e-20)):
        h = g * factor
        for steps, coef in ((0, om.COEF), (1, om.COEF), (5, om.COEF), (100, grow)):
            o = num(binding.orthogonalize(h, steps=steps, coef=coef, eps=eps))
            want = om.newton_schulz(num(h), steps, coef, eps)
            # every step rounds the iterate to 22 bits; numbers below fp32's normal range have its smallest step, 2^-149, and a
            # last factor in that range 2^-149 of 1.2e-38 / 2^10
            tol = (FULL_TOL + steps * 2.0 ** -21) * np.linalg.norm(want) + 2.0 ** -138 * np.sqrt(want.size)
            assert np.linalg.norm(o - want) <= tol, (factor, eps, steps)
    binding.check_operators()


# ------------------------------------------------------------------------------------------- status, memory, autograd
@pytest.mark.gpu
@pytest.mark.parametrize("device", [None, "cuda", 0, "cuda:0"])
def test_a_wait_that_gave_up_is_reported_once(device):
    """The word is set from the host; no wait runs out."""
    binding.orthogonalize(torch.ones(4, 4, device="cuda"))
    binding.check_operators(device)
    binding._status_word(0).fill_(1)
    with pytest.raises(binding.GCadaError) as e:
        binding.check_operators(device if device is None or isinstance(device, int) else torch.device(device))
    assert e.value.status == binding.ETIMEOUT
    binding.check_operators(device)


FIRST_CALL_CAPTURED = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2201_04301_b200 import binding
x = torch.randn(130, 200, device="cuda")
n = torch.randn(10, 90, device="cuda")
out, small, prod = torch.zeros_like(x), torch.zeros_like(n), torch.zeros(130, 130, device="cuda")
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    binding.orthogonalize(n, out=small)
    binding.orthogonalize(x, out=out)
    q = binding.mx_quantize(x)
    binding.mx_gemm(q, q, out=prod)
graph.replay()
torch.cuda.synchronize()
binding.check_operators("cuda")
word = binding._status_words[0]
assert word, "the captured kernels have no status word"
assert torch.equal(out, binding.orthogonalize(x)) and torch.equal(small, binding.orthogonalize(n))
q = binding.mx_quantize(x)
assert torch.equal(prod, binding.mx_gemm(q, q))
assert binding._status_words[0] == word
print("same")
"""


@pytest.mark.gpu
def test_the_first_calls_of_a_process_may_be_captured():
    """... and their kernels know the status word that check_operators reads."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_CAPTURED.format(root=root)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


BUSY = """
// Lets the kernels behind it start at once, then keeps one thread asleep for `ns` nanoseconds (ten seconds at most).
__global__ void busy_kernel(long long ns) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  long long t0, t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  do {
    __nanosleep(1000);
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  } while (t - t0 < ns && t - t0 < 10000000000LL);
}
extern "C" int busy(void* stream, long long ns) {
  busy_kernel<<<1, 1, 0, static_cast<cudaStream_t>(stream)>>>(ns);
  return (int)cudaGetLastError();
}
"""


@pytest.mark.gpu
def test_a_long_predecessor_that_lets_them_start_early(tmp_path):
    """The kernels' bounded waits (a second or so) begin when their predecessor has finished: one that runs for longer, but lets
    the next kernels become resident meanwhile, is no failure."""
    import subprocess
    from paper_2201_04301_b200 import build
    src, so = tmp_path / "busy.cu", tmp_path / "busy.so"
    src.write_text(BUSY)
    subprocess.run(["nvcc", *build.NVCC_FLAGS, "-shared", "-o", str(so), str(src)], check=True, capture_output=True)
    busy = binding.C.CDLL(str(so)).busy
    busy.argtypes = [binding.C.c_void_p, binding.C.c_longlong]
    gen = torch.Generator(device="cuda").manual_seed(1)
    mats = [torch.randn(s, generator=gen, device="cuda") for s in ((130, 300), (600, 700), (10, 200))]
    a, b = (binding.mx_quantize(torch.randn(s, generator=gen, device="cuda")) for s in ((300, 4000), (500, 4000)))
    calls = [lambda g=g: binding.orthogonalize(g) for g in mats] + [lambda: binding.mx_gemm(a, b)]
    want = [f() for f in calls]
    binding.check_operators()
    for f, w in zip(calls, want):
        assert busy(torch.cuda.current_stream().cuda_stream, 2_500_000_000) == 0
        o = f()
        binding.check_operators()
        assert torch.equal(o, w)


NOTHING_KEPT_OF_A_CAPTURE = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2201_04301_b200 import binding
x = torch.randn(10, 90, device="cuda")
out, graph = torch.zeros_like(x), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    binding.orthogonalize(x, out=out)
    binding.muon_update(torch.zeros_like(x), torch.zeros_like(x), x, lr=0.1)
graph.replay()
torch.cuda.synchronize()
private = [s for s in torch.cuda.memory_snapshot() if tuple(s["segment_pool_id"]) != (0, 0)]
assert private, "the capture had no memory of its own"
del graph
torch.cuda.empty_cache()
assert not [s for s in torch.cuda.memory_snapshot() if tuple(s["segment_pool_id"]) != (0, 0)], "a part of the graph's memory is held"
first = binding.orthogonalize(x)
assert torch.equal(first, out) and binding._unused_work
print("same")
"""


@pytest.mark.gpu
def test_nothing_of_a_graph_s_memory_outlives_it():
    """The area that narrow matrices hand over but do not use is kept for later calls, unless a graph's memory pool made it."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", NOTHING_KEPT_OF_A_CAPTURE.format(root=root)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@pytest.mark.gpu
def test_written_tensors_have_their_versions_raised():
    """Autograd then refuses a backward pass through a tensor that an operator has overwritten meanwhile."""
    x = torch.randn(20, 40, device="cuda")
    w = torch.randn(20, 40, device="cuda", requires_grad=True)
    m, before = torch.zeros_like(x), w._version
    loss = w.square().sum()                                     # keeps w for its backward pass
    binding.muon_update(w, m, x, lr=0.1)
    assert w._version > before and m._version > 0
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    q = binding.mx_quantize(x)
    other = binding.MxMatrix(20, 40, q.codes.clone(), q.scales.clone())
    for out, call in ((torch.zeros_like(x), lambda o: binding.orthogonalize(x, out=o)), (torch.zeros_like(x), lambda o: q.dequantize(out=o)),
                      (torch.zeros(20, 20, device="cuda"), lambda o: binding.mx_gemm(q, q, out=o))):
        version, of_x = out._version, x._version
        call(out)
        assert out._version > version and x._version == of_x
    versions = other.codes._version, other.scales._version
    binding.mx_quantize(x, out=other)
    assert other.codes._version > versions[0] and other.scales._version > versions[1]
    codes = q.codes._version
    binding.mx_quantize(x, out=q)
    assert q.codes._version > codes
    with torch.inference_mode():                                # tensors without a version counter
        y = torch.zeros(20, 40, device="cuda")
        assert torch.equal(binding.orthogonalize(x, out=y), binding.orthogonalize(x))


@pytest.mark.gpu
def test_results_carry_no_gradient():
    x = torch.randn(20, 40, device="cuda", requires_grad=True)
    q = binding.mx_quantize(x)
    for r in (binding.orthogonalize(x), binding.orthogonalize(x.T.contiguous()), q.codes, q.dequantize(), binding.mx_gemm(q, q)):
        assert not r.requires_grad and r.grad_fn is None
