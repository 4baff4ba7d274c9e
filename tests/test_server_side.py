"""Contexts whose server side uses the matrix operators: update rule Muon, 4-bit uploads, and both together.

Every step is checked against 64-bit forms of its own inputs (iterate, momentum and aggregate before and after,
read from the context)."""
import math

import numpy as np
import pytest
import torch

from oracle import matrix as om
from oracle.models import MLP, round_to_bf16
from oracle.philox import batch_indices
from paper_2201_04301_b200 import binding, build
from paper_2201_04301_b200.workloads import make_workload

from parity import TOL_BF16, rel_l2, to_cuda
from test_matrix_operators import FULL_TOL, HALF_TOL

pytestmark = pytest.mark.gpu

FP32 = dict(name="cfg4", rows=5 * 90, dims=(20, 12, 5), M=10, M_G=2, D=3, batch=16, c=0.3, alpha=0.01)
WIDE = dict(name="cfg4", rows=3 * 120, dims=(150, 90, 70, 7), M=3, M_G=1, D=2, batch=33, c=0.3, alpha=0.01)
BF16 = dict(name="cfg5", rows=3000, dims=(64, 128, 96, 40), M=6, M_G=2, D=3, batch=128, c=0.3)
ODD16 = dict(name="cfg5", rows=2100, dims=(75, 130, 33), M=5, M_G=1, D=2, batch=200, c=0.3)


def workload(kw):
    kw = dict(kw)
    return make_workload(kw.pop("name"), **kw)


def layers(dims):
    """(rows, cols, slice of W, slice of b) of every layer."""
    o, out = 0, []
    for n_in, n_out in zip(dims[:-1], dims[1:]):
        out.append((n_out, n_in, slice(o, o + n_out * n_in), slice(o + n_out * n_in, o + n_out * n_in + n_out)))
        o += n_out * n_in + n_out
    return out


def state(g):
    return [np.asarray(t, dtype=np.float64) for t in (g.get_theta(), g.get_debug(binding.DBG_H), g.get_debug(binding.DBG_VHAT),
                                                      g.get_debug(binding.DBG_AGG))]


@pytest.mark.parametrize("kw", [FP32, WIDE, BF16, ODD16], ids=["fp32", "fp32-wide", "bf16", "bf16-odd"])
@pytest.mark.parametrize("rule", [dict(), dict(weight_decay=0.5, scale=0.2, nesterov=False, steps=3)], ids=["default", "other"])
def test_muon_steps(kw, rule):
    w = workload(kw)
    st = torch.cuda.Stream()
    g = binding.from_workload(to_cuda(w), stream=st, server_rule=dict(rule="muon", **rule), schedule=("poly", 2.0, 0.5))
    tol = FULL_TOL if w["compute"] == "fp32" else HALF_TOL
    wd, scale, nest, steps = (rule.get(k, d) for k, d in (("weight_decay", 0.0), ("scale", 1.0), ("nesterov", True), ("steps", 5)))
    theta, h, vh, _ = state(g)
    for k in range(6):
        g.step(1)
        theta1, h1, vh1, agg = state(g)
        alpha = w["alpha"] / math.sqrt(1 + k / 2.0)
        assert rel_l2(h1, w["beta1"] * h + (1 - w["beta1"]) * agg) < 2.0 ** -21
        for rows, cols, W, b in layers(w["dims"]):
            A, H = agg[W].reshape(rows, cols), h[W].reshape(rows, cols)
            s = scale * math.sqrt(max(1.0, rows / cols))
            want, _ = om.muon(theta[W].reshape(rows, cols), H, A, alpha, w["beta1"], nest, wd, s, steps=steps)
            err = np.linalg.norm(theta1[W].reshape(rows, cols) - want)
            assert err <= tol * alpha * s * 1.3 * math.sqrt(min(rows, cols)) + 2.0 ** -22 * np.linalg.norm(want)
            assert np.array_equal(vh1[W], vh[W])
            v = np.maximum(vh[b], w["beta2"] * vh[b] + (1 - w["beta2"]) * agg[b] ** 2)
            assert rel_l2(vh1[b], v) < 2.0 ** -20
            assert rel_l2(theta1[b], theta[b] - alpha * h1[b] / np.sqrt(w["eps"] + v)) < 2.0 ** -19
        norm = np.sum((theta1 - theta) ** 2)
        # the step itself is formed in fp32: its entries carry half a step of the iterate's
        slack = 4 * 2.0 ** -24 * np.linalg.norm(theta1) * math.sqrt(norm)
        assert abs(g.get_debug(binding.DBG_SRING)[k % w["D"]] - norm) <= slack + 2.0 ** -20 * norm
        theta, h, vh = theta1, h1, vh1
    assert np.isfinite(theta).all()
    g.close()


@pytest.mark.parametrize("kw", [BF16, ODD16, WIDE], ids=["bf16", "bf16-odd", "fp32-wide"])
def test_the_rule_s_precision_is_full_unless_half_is_asked_for(kw):
    """The first step from the same iterate: weights, momentum and aggregate are fp32, so fp32 accuracy is what a network gets
    without asking, whatever its own products round to."""
    w = workload(kw)
    theta = w["theta0"].numpy().astype(np.float64)
    moved = {}
    for name, options in (("default", {}), ("full", {binding.OPT_SERVER_PRECISION: 0}), ("half", {binding.OPT_SERVER_PRECISION: 1})):
        g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), options=options, server_rule=dict(rule="muon"))
        g.step(1)
        moved[name], h, vh, agg = state(g)
        g.close()
        for rows, cols, W, b in layers(w["dims"]):
            s = math.sqrt(max(1.0, rows / cols))
            want, _ = om.muon(theta[W].reshape(rows, cols), np.zeros((rows, cols)), agg[W].reshape(rows, cols), w["alpha"],
                              w["beta1"], True, 0.0, s)
            err = np.linalg.norm(moved[name][W].reshape(rows, cols) - want)
            tol = HALF_TOL if name == "half" else FULL_TOL
            assert err <= tol * w["alpha"] * s * 1.3 * math.sqrt(min(rows, cols)) + 2.0 ** -22 * np.linalg.norm(want), (name, rows, cols)
    assert np.array_equal(moved["default"], moved["full"]) and not np.array_equal(moved["full"], moved["half"])
    g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream())
    for bad in (2, -1, 0.5):
        with pytest.raises(binding.GCadaError) as e:
            g.set_option(binding.OPT_SERVER_PRECISION, bad)
        assert e.value.status == binding.EINVAL
    g.close()
    lin = binding.from_workload(to_cuda(make_workload("cfg1", rows=300)), stream=torch.cuda.Stream())
    with pytest.raises(binding.GCadaError) as e:
        lin.set_option(binding.OPT_SERVER_PRECISION, 1)
    assert e.value.status == binding.EINVAL
    lin.close()

@pytest.mark.parametrize("kw", [FP32, BF16], ids=["fp32", "bf16"])
def test_the_aggregate_under_muon_is_the_sum_of_uploads(kw):
    w = workload(kw)
    g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), server_rule=dict(rule="muon"))
    for mask in ([1] * g.G, [1] + [0] * (g.G - 1), [0] * g.G, [0, 1] + [0] * (g.G - 2)):
        g.step_forced(np.array([mask], dtype=np.uint8))
        total = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64).sum(axis=0)
        assert rel_l2(g.get_debug(binding.DBG_AGG), total) < 2.0 ** -16
    g.close()


def run(w, n, **kw):
    g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), **kw)
    g.step(n)
    out = g.get_theta(), g.get_selection_mask(0, n), g.get_comm_count(), g.get_debug(binding.DBG_AGG)
    g.close()
    return out


@pytest.mark.parametrize("kw,options", [(FP32, {}), (WIDE, {}), (BF16, {}), (BF16, {binding.OPT_UPLOAD: 1}), (ODD16, {binding.OPT_UPLOAD: 1})],
                         ids=["fp32", "fp32-wide", "bf16", "bf16-mx", "bf16-odd-mx"])
@pytest.mark.parametrize("rule", ["muon", "amsgrad"])
def test_replayed_and_plain_launches_agree(kw, options, rule):
    w = workload(kw)
    a = run(w, 37, options=options, server_rule=dict(rule=rule))
    b = run(w, 37, options={**options, binding.OPT_GRAPH: 0.0}, server_rule=dict(rule=rule))
    for x, y in zip(a, b):
        assert np.array_equal(np.asarray(x), np.asarray(y))
    assert np.isfinite(a[0]).all() and a[1].any()


@pytest.mark.parametrize("kw,options", [(FP32, {}), (BF16, {binding.OPT_UPLOAD: 1})], ids=["fp32", "bf16-mx"])
def test_checkpoints_continue_bit_for_bit(kw, options):
    w = to_cuda(workload(kw))
    make = lambda: binding.from_workload(w, stream=torch.cuda.Stream(), options=options, server_rule=dict(rule="muon"))  # noqa: E731
    a = make()
    a.step(9)
    saved = a.checkpoint_save()
    a.step(8)
    b = make()
    b.checkpoint_load(saved)
    b.step(8)
    assert np.array_equal(a.get_theta(), b.get_theta()) and a.get_comm_count() == b.get_comm_count()
    plain = binding.from_workload(w, stream=torch.cuda.Stream())
    if options:                       # another upload form has other state
        with pytest.raises(binding.GCadaError) as e:
            plain.checkpoint_load(saved)
        assert e.value.status == binding.EINVAL
    for g in (a, b, plain):
        g.close()


def factors(model, theta, X, y):
    """(dz_l, a_{l-1}) of every layer, operands rounded as the bf16 MLP rounds them."""
    ls, acts, zs = model._forward(theta, X)
    s = zs[-1] - zs[-1].max(axis=1, keepdims=True)
    dz = np.exp(s)
    dz /= dz.sum(axis=1, keepdims=True)
    dz[np.arange(len(y)), y.astype(np.int64)] -= 1.0
    dz /= len(y)
    out = []
    for l in range(len(ls) - 1, -1, -1):
        dz = round_to_bf16(dz)
        out.append((dz, acts[l]))
        if l:
            dz = (dz @ ls[l][0]) * (zs[l - 1] > 0)
    return out[::-1]


def four_bits(x):
    """Blocks of 32 rows (zeros behind the end) down every column."""
    return om.mx_values(*om.mx_quantize(x.T), x.shape[0]).T


@pytest.mark.parametrize("kw", [BF16, ODD16], ids=["bf16", "bf16-odd"])
def test_uploads_in_four_bits(kw):
    w = workload(kw)
    n_g = w["N"] // (w["M"] // w["M_G"])
    model = MLP(w["dims"], bf16=True)
    g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), options={binding.OPT_UPLOAD: binding.UPLOAD_MXFP4})
    full = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream())
    theta = w["theta0"].numpy().astype(np.float64)
    g.step(1)
    full.step(1)
    assert np.array_equal(g.get_selection_mask(0, 1), full.get_selection_mask(0, 1))      # every group
    assert np.array_equal(g.get_debug(binding.DBG_LHS), full.get_debug(binding.DBG_LHS))  # the test is not quantised
    uploads = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64)
    exact = np.asarray(full.get_debug(binding.DBG_GLAST), dtype=np.float64)
    X = w["X"][:, :w["dims"][0]].float().numpy().astype(np.float64)
    for grp in range(g.G):
        rows = batch_indices(w["seed"], 0, grp, w["batch"], n_g)
        for (n_out, n_in, W, b), (dz, act) in zip(layers(w["dims"]), factors(model, theta, X[rows], w["y"].numpy()[rows])):
            want = (four_bits(dz).T @ four_bits(act)).ravel()
            got = uploads[grp][W]
            # a bf16 rounding that falls the other way moves a factor's entry by 2^-8, and now and then its 4-bit value
            # to the next one: far less than the quantisation itself, which is worth 5 to 25 % of the gradient
            assert rel_l2(got, want) < TOL_BF16, (grp, n_out, n_in, rel_l2(got, want))
            assert 0.03 < rel_l2(got, exact[grp][W]) < 0.3
            assert rel_l2(uploads[grp][b], exact[grp][b]) == 0.0
    assert rel_l2(g.get_debug(binding.DBG_AGG), uploads.sum(axis=0)) < 2.0 ** -18
    # later uploads replace the earlier ones and leave the others' alone
    for mask in ([0, 1] + [0] * (g.G - 2), [0] * g.G, [1] + [0] * (g.G - 1)):
        before = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64)
        g.step_forced(np.array([mask], dtype=np.uint8))
        after = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64)
        for grp in range(g.G):
            assert np.array_equal(before[grp], after[grp]) == (not mask[grp])
        assert rel_l2(g.get_debug(binding.DBG_AGG), after.sum(axis=0)) < 2.0 ** -18
    g.close()
    full.close()


@pytest.mark.parametrize("batch", [200, 129, 31])
def test_padding_rows_take_no_part_in_an_uploads_scales(batch):
    """A minibatch that ends inside a block of 32 rows: the block's scale is that of its own rows.  The kernels pad a
    minibatch with zero features, whose activations are relu(b); here those are far above every sample's, and in the later
    steps the biases are what the updates have made of them."""
    w = workload(dict(ODD16, batch=batch))
    dims, n_g = w["dims"], w["N"] // (w["M"] // w["M_G"])
    w["X"][:, :dims[0]] = w["X"][:, :dims[0]].abs()
    rows, cols, W, b = layers(dims)[0]
    w["theta0"][W] = -w["theta0"][W].abs()
    x = w["X"][:, :cols].double()
    drop = (x @ w["theta0"][W].view(rows, cols).double().T).max(dim=0).values      # the sample that is lowered least
    w["theta0"][b] = (-drop + 0.02 * drop.abs()).float()                           # a little above zero, for that one
    model, X = MLP(dims, bf16=True), w["X"][:, :dims[0]].float().numpy().astype(np.float64)
    g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), options={binding.OPT_UPLOAD: binding.UPLOAD_MXFP4})
    for k in range(3):
        theta = np.asarray(g.get_theta(), dtype=np.float64)
        g.step_forced(np.ones((1, g.G), dtype=np.uint8))
        uploads = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64)
        for grp in range(g.G):
            pick = batch_indices(w["seed"], k, grp, batch, n_g)
            for (n_out, n_in, W, b), (dz, act) in zip(layers(dims), factors(model, theta, X[pick], w["y"].numpy()[pick])):
                want = (four_bits(dz).T @ four_bits(act)).ravel()
                assert rel_l2(uploads[grp][W], want) < TOL_BF16, (k, grp, n_out, n_in, rel_l2(uploads[grp][W], want))
    g.close()


def test_settings_made_after_the_plans_leave_no_second_set_of_buffers():
    """Timing the gradient builds the plans; a rule, lag weights or smoothness constants set then replace them."""
    w = to_cuda(workload(dict(BF16, rows=64 * 300, dims=(256, 1024, 1024, 40), M=64, M_G=1, batch=256)))
    g = binding.from_workload(w, stream=torch.cuda.Stream())
    theta = g.get_theta()
    g.time_gradient(1)
    free = []
    for setting in (lambda: g.set_server_rule("muon"), lambda: g.set_lag_weights([0.3] * w["D"]), lambda: g.set_smoothness([1.0] * g.G),
                    lambda: g.set_server_rule("muon", scale=0.5), lambda: g.set_server_rule("amsgrad"), lambda: g.set_server_rule("muon", scale=0.5)):
        setting()
        g.time_gradient(1)
        torch.cuda.synchronize()
        free.append(torch.cuda.mem_get_info()[0])
    assert free[0] - min(free) < 64 << 20, free               # the plans' buffers are 0.6 GB
    assert np.array_equal(g.get_theta(), theta)
    g.step(2)
    other = binding.from_workload(w, stream=torch.cuda.Stream(), server_rule=dict(rule="muon", scale=0.5))
    other.step(2)
    assert np.array_equal(g.get_theta(), other.get_theta())
    g.close()
    other.close()

def test_refusals():
    lin = binding.from_workload(to_cuda(make_workload("cfg1", rows=300)), stream=torch.cuda.Stream())
    fp32 = binding.from_workload(to_cuda(workload(FP32)), stream=torch.cuda.Stream())
    for call in (lambda: lin.set_server_rule("muon"), lambda: lin.set_option(binding.OPT_UPLOAD, 1),
                 lambda: fp32.set_option(binding.OPT_UPLOAD, 1), lambda: fp32.set_option(binding.OPT_UPLOAD, 2),
                 lambda: fp32.set_server_rule(2), lambda: fp32.set_server_rule("muon", steps=0),
                 lambda: fp32.set_server_rule("muon", steps=101), lambda: fp32.set_server_rule("muon", scale=0.0),
                 lambda: fp32.set_server_rule("muon", weight_decay=-1.0), lambda: fp32.set_server_rule("muon", scale=float("nan"))):
        with pytest.raises(binding.GCadaError) as e:
            call()
        assert e.value.status == binding.EINVAL
    fp32.step(1)
    with pytest.raises(binding.GCadaError) as e:
        fp32.set_server_rule("muon")
    assert e.value.status == binding.ESTATE
    lin.close()
    fp32.close()


def test_printed_rule_and_inspection_with_the_new_server_side():
    w = workload(BF16)
    for options in ({binding.OPT_RULE: 1.0, binding.OPT_UPLOAD: 1}, {binding.OPT_KEEP_STALE: 1.0, binding.OPT_UPLOAD: 1},
                    {binding.OPT_TIMING: 1.0, binding.OPT_UPLOAD: 1}):
        g = binding.from_workload(to_cuda(w), stream=torch.cuda.Stream(), options=options, smoothness=[1.0] * 3,
                                  server_rule=dict(rule="muon"))
        n0 = g.get_launch_count()
        g.step(20)
        assert np.isfinite(g.get_theta()).all() and g.get_iteration() == 20 and g.get_launch_count() > n0
        if options.get(binding.OPT_RULE):
            uploads = np.asarray(g.get_debug(binding.DBG_GLAST), dtype=np.float64)
            assert rel_l2(g.get_debug(binding.DBG_AGG), uploads.sum(axis=0)) < 2.0 ** -18
        g.time_empty_chain(16)
        g.eval_loss(0, 100)
        g.close()


def test_no_index_check_fires():
    build.build(debug=True)
    binding.load(binding.DEBUG_LIB_PATH)
    try:
        for kw, options in ((FP32, {}), (BF16, {binding.OPT_UPLOAD: 1}), (ODD16, {binding.OPT_UPLOAD: 1})):
            g = binding.from_workload(to_cuda(workload(kw)), stream=torch.cuda.Stream(), options=options, server_rule=dict(rule="muon"))
            g.step(21)
            assert np.isfinite(g.get_theta()).all()
            g.close()
    finally:
        binding.load(binding.LIB_PATH)
