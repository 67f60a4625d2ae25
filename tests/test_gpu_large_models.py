"""Norm, clipping and step of models that are cut into large chunks (over 8 Mi elements: 16384 to a chunk), and of small models around their chunks' ends (2048), against the
formulas in 64 bits."""
import math

import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

EDGES = [16383, 16384, 16385, 1, 0, 3, 2 * 16384, 2 * 16384 + 7]
SIZES = {
    "nine million": EDGES + [9_000_001],                         # 550 chunks: fewer than there are partial sums
    "just over": EDGES + [(8 << 20) + 1 - sum(EDGES)],
    "just under": EDGES + [(8 << 20) - sum(EDGES)],              # small chunks still
    "twenty million": [20_000_003] + EDGES,                      # more chunks than partial sums
    "seventy million": EDGES + [70_000_001, 5],                  # more chunks than workgroups of the step
    "many": [40_000 + i * 13 % 977 for i in range(300)],
    "small": [2047, 2048, 2049, 1, 0, 2 * 2048 + 5, 4095],
}


@pytest.mark.parametrize("dtypes", [[torch.float32], [torch.bfloat16], [torch.float32, torch.bfloat16]])
@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("clips", [True, False])
def test_norm_clip_and_step(name, dtypes, clips):
    sizes, total = SIZES[name], sum(SIZES[name]) + 2
    g = torch.Generator(device="cuda").manual_seed(len(name))
    flat = {d: (torch.randn(total, generator=g, device="cuda") * 0.1).to(d) for d in dtypes}
    flat_w = torch.randn(total, generator=g, device="cuda")
    ends = [1]
    for n in sizes:
        ends.append(ends[-1] + n)
    grads = [flat[dtypes[i % len(dtypes)]][a:b] for i, (a, b) in enumerate(zip(ends, ends[1:]))]
    weights = [flat_w[a:b] for a, b in zip(ends, ends[1:])]
    old_g, old_w = [t.clone() for t in grads], flat_w.clone()
    kept = {d: t.clone() for d, t in flat.items()}
    want = math.sqrt(math.fsum(float(t.double().square().sum()) for t in grads))
    max_norm = 0.3 * want if clips else 2 * want
    factor, eta, lam = min(1.0, max_norm / want), 0.25, 0.02
    tensors = api.wpsgd_tensor_list(grads, weights)
    near = lambda v: abs(float(v) - want) <= 2.0 ** -24 * want * (1 + 1e-6)  # noqa: E731  (fp64 sums, rounded once)
    assert near(api.wpsgd_grad_norm(tensors)) and near(api.wpsgd_clipped_step(tensors, eta, lam, max_norm))
    for w, a, og in zip(weights, ends, old_g):
        ow = old_w[a:a + len(w)].double()
        ideal = (1 - eta * lam) * ow - eta * factor * og.double()
        assert bool(((w.double() - ideal).abs() <= 2.0 ** -24 * ideal.abs() + 1e-12 * (ow.abs() + og.double().abs()) + 2.0 ** -150).all())
    assert float(flat_w[0]) == float(old_w[0]) and float(flat_w[-1]) == float(old_w[-1]) and all(torch.equal(flat[d], kept[d]) for d in flat)
    assert near(api.wpsgd_clip_grads(tensors, max_norm))
    for t, og in zip(grads, old_g):
        if factor == 1.0:
            assert torch.equal(t, og)
        else:
            ideal = factor * og.double()
            half = 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24
            assert bool(((t.double() - ideal).abs() <= (half * (1 + 1e-4) + 1e-12) * ideal.abs() + 2.0 ** -140).all())
    assert all(float(flat[d][0]) == float(kept[d][0]) and float(flat[d][-1]) == float(kept[d][-1]) for d in flat)


def test_the_same_bits_twice():
    flat = torch.randn(20_000_003, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    tensors = api.wpsgd_tensor_list([flat])
    first = api.wpsgd_grad_norm(tensors)
    assert all(torch.equal(first, api.wpsgd_grad_norm(tensors)) for _ in range(5))


def test_one_value_that_is_not_finite_stops_a_large_step():
    g, w = torch.ones(10_000_000, device="cuda"), torch.ones(10_000_000, device="cuda")
    g[9_999_999] = math.nan
    tensors = api.wpsgd_tensor_list([g], [w])
    assert math.isnan(float(api.wpsgd_clipped_step(tensors, 0.1, 0.1, 1.0))) and bool((w == 1).all())
    g[9_999_999] = math.inf
    assert float(api.wpsgd_clip_grads(tensors, 1.0)) == math.inf and bool((w == 1).all()) and bool((g[:-1] == 1).all())
