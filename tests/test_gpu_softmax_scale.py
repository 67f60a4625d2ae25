"""A scale that fp32 cannot hold, beside row weights that bring its product back: the gradient's factor is scale * weight."""
import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [9, 3000, 140000])
@pytest.mark.parametrize("scale,weight", [(2.0 ** 140, 2.0 ** -120), (2.0 ** -170, 2.0 ** 100), (-(2.0 ** 200), 2.0 ** -149), (2.0 ** -200, 1.0)])
def test_the_product_of_scale_and_weight(c, dtype, scale, weight):
    g = torch.Generator().manual_seed(c)
    z = torch.randn(2, c, generator=g).to(dtype).cuda()
    z[1, 3:6] = -float("inf")
    labels = torch.randint(0, 3, (2,), generator=g).cuda()
    plain = api.wpsgd_softmax_loss(z, labels)
    w = torch.full((2,), weight, device="cuda")
    loss, grad = api.wpsgd_softmax_loss(z, labels, scale=scale, row_weights=w)
    factor = scale * weight
    # the factor is a power of two, so that only what turns subnormal is rounded
    want = plain[1].double() * factor
    assert bool(((grad.double() - want).abs() <= (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149)).all())
    assert torch.equal(loss, plain[0] * weight)
