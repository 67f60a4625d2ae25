"""Global gradient norm, clipping and the clipped step over many tensors, against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

SIZES = {
    "one": [1], "few": [5, 1, 0, 130], "odd": [1000, 16383, 16384, 16385, 3, 40001], "many": [(i * 37) % 977 for i in range(400)],
    "long": [3_000_001, 70_000], "none": [0, 0], "chunks": [16384 * 5],
}


def packed(sizes, dtypes, seed, scale=0.1):
    """gradients and weights one behind the other, so that they start anywhere; dtypes in turn"""
    g = torch.Generator().manual_seed(seed)
    grads, weights = [], []
    total = sum(sizes) + 1
    flat = {d: (torch.randn(total, generator=g) * scale).to(d).cuda() for d in dtypes}
    flat_w = torch.randn(total, generator=g).cuda()
    at = 1
    for i, n in enumerate(sizes):
        grads.append(flat[dtypes[i % len(dtypes)]][at:at + n])
        weights.append(flat_w[at:at + n])
        at += n
    return grads, weights, flat, flat_w


def norm_of(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


@pytest.mark.parametrize("dtypes", [[torch.float32], [torch.bfloat16], [torch.float32, torch.bfloat16]])
@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("clips", [True, False])
def test_norm_clip_and_step_match_the_formulas(name, dtypes, clips):
    grads, weights, flat, flat_w = packed(SIZES[name], dtypes, len(name))
    keep_g, keep_w = {d: t.clone() for d, t in flat.items()}, flat_w.clone()
    old_g, old_w = [g.double() for g in grads], [w.double() for w in weights]
    want = norm_of(grads)
    max_norm = 0.3 * want if clips and want else 2 * want + 1
    eta, lam = 0.25, 0.02
    tensors = api.wpsgd_tensor_list(grads, weights)
    near = lambda v: abs(float(v) - want) <= 2.0 ** -23 * want  # noqa: E731  (fp64 sums, rounded once)
    assert near(api.wpsgd_grad_norm(tensors))
    assert near(api.wpsgd_clipped_step(tensors, eta, lam, max_norm))
    factor = min(1.0, max_norm / want) if want else 1.0
    for w, ow, og in zip(weights, old_w, old_g):
        ideal = (1 - eta * lam) * ow - eta * factor * og
        # two factors, a product and a sum rounded to fp32
        assert ((w.double() - ideal).abs() <= 2.0 ** -22 * (ow.abs() + eta * factor * og.abs()) + 1e-40).all()
    assert flat_w[0] == keep_w[0] and all(torch.equal(flat[d], keep_g[d]) for d in flat)      # nothing beside the tensors, no gradient
    if sum(SIZES[name]) < flat_w.numel() - 1:
        assert torch.equal(flat_w[-1:], keep_w[-1:])
    assert near(api.wpsgd_clip_grads(tensors, max_norm))
    for g, og in zip(grads, old_g):
        if factor == 1.0:
            assert torch.equal(g.double(), og)
        else:
            half = 2.0 ** -8 if g.dtype == torch.bfloat16 else 2.0 ** -22
            assert ((g.double() - factor * og).abs() <= half * (factor * og).abs() + 1e-40).all()
    assert all(flat[d][0] == keep_g[d][0] for d in flat)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_changes_nothing(bad):
    grads, weights, flat, flat_w = packed([100, 20000, 7], [torch.float32, torch.bfloat16], 3)
    grads[1][12345] = bad
    tensors = api.wpsgd_tensor_list(grads, weights)
    g, w = [t.clone() for t in grads], flat_w.clone()
    for call in (lambda: api.wpsgd_grad_norm(tensors), lambda: api.wpsgd_clipped_step(tensors, 0.1, 0.1, 1.0), lambda: api.wpsgd_clip_grads(tensors, 1.0)):
        norm = float(call())
        assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
        assert torch.equal(flat_w, w) and all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(grads, g))


def test_squares_that_fp32_cannot_hold():
    for v in (1e25, 1e-30):
        g = torch.full((1000,), v, device="cuda")
        w = torch.zeros(1000, device="cuda")
        tensors = api.wpsgd_tensor_list([g], [w])
        want = float(g[0]) * math.sqrt(1000)
        assert abs(float(api.wpsgd_grad_norm(tensors)) / want - 1) <= 2.0 ** -23
        api.wpsgd_clipped_step(tensors, 1.0, 0.0, want / 2)
        assert (w.double() / float(g[0]) + 0.5).abs().max() <= 2.0 ** -22
    g = torch.full((1000,), 3e38, device="cuda")      # finite in fp64, not as an fp32 norm: reported as inf, the step is still taken
    w = torch.zeros(1000, device="cuda")
    tensors = api.wpsgd_tensor_list([g], [w])
    assert float(api.wpsgd_clipped_step(tensors, 1.0, 0.0, 1.0)) == math.inf
    assert (w.double() * math.sqrt(1000) + 1).abs().max() <= 2.0 ** -20


def test_no_clipping_is_the_plain_step_and_zero_gradients_shrink():
    grads, weights, _, _ = packed([1000, 50], [torch.float32], 5)
    old = [w.double() for w in weights]
    tensors = api.wpsgd_tensor_list(grads, weights)
    api.wpsgd_clipped_step(tensors, 0.1, 0.5)
    for w, o, g in zip(weights, old, grads):
        assert ((w.double() - (0.95 * o - 0.1 * g.double())).abs() <= 2.0 ** -22 * (o.abs() + 0.1 * g.double().abs())).all()
    for g in grads:
        g.zero_()
    old = [w.double() for w in weights]
    assert float(api.wpsgd_clipped_step(tensors, 0.1, 0.5, 1.0)) == 0
    for w, o in zip(weights, old):
        assert ((w.double() - 0.95 * o).abs() <= 2.0 ** -22 * o.abs()).all()


def test_the_norm_is_the_derivative_of_nothing_but_its_own_square():
    """d norm / d g_i = g_i / norm: clipping to a little under the norm moves along it; checked by differences of the norm call"""
    g = torch.randn(50, dtype=torch.float32, generator=torch.Generator().manual_seed(1)).cuda()
    tensors = api.wpsgd_tensor_list([g])
    n0 = float(api.wpsgd_grad_norm(tensors))
    h = 2.0 ** -6
    for i in range(0, 50, 7):
        keep = float(g[i])
        g[i] = keep + h
        up = float(api.wpsgd_grad_norm(tensors))
        g[i] = keep - h
        down = float(api.wpsgd_grad_norm(tensors))
        g[i] = keep
        # third derivative of the norm <= 3 / norm^2; the norms are rounded to fp32
        assert abs((up - down) / (2 * h) - keep / n0) <= h * h / (2 * n0 * n0) + 2.0 ** -23 * n0 / h


def test_refusals():
    g, w = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    only = api.wpsgd_tensor_list([g])
    both = api.wpsgd_tensor_list([g], [w])
    for bad in (lambda: api.wpsgd_clipped_step(only, 0.1, 0.0, 1.0), lambda: api.wpsgd_clipped_step(both, 0.0, 0.0, 1.0),
                lambda: api.wpsgd_clipped_step(both, 2.0, 0.5, 1.0), lambda: api.wpsgd_clipped_step(both, 0.1, -1.0, 1.0),
                lambda: api.wpsgd_clipped_step(both, 0.1, 0.1, 0.0), lambda: api.wpsgd_clipped_step(both, 0.1, 0.1, math.nan),
                lambda: api.wpsgd_clip_grads(both, -1.0), lambda: api.wpsgd_clip_grads(both, math.nan)):
        with pytest.raises(api.WpsgdError) as e:
            bad()
        assert e.value.status == api.INVALID_ARG
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(api.WpsgdError) as e:
        api.wpsgd_grad_norm(both, workspace=small)
    assert e.value.status == api.WORKSPACE_TOO_SMALL
    for bad in (lambda: api.wpsgd_tensor_list([g.half()]), lambda: api.wpsgd_tensor_list([g], [w[:5]]), lambda: api.wpsgd_tensor_list([g], [w.bfloat16()]),
                lambda: api.wpsgd_tensor_list([torch.ones(4, 6, device="cuda").t()]), lambda: api.wpsgd_tensor_list([g.cpu()])):
        with pytest.raises(AssertionError):
            bad()
    torch.cuda.synchronize()
    assert (w == 1).all()
