"""Gradients of classes far below the largest, in fp32: each keeps its own last places."""
import math

import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", [40, 257, 1000, 4099, 9000, 20000, 65537, 131075])
def test_small_classes_keep_their_places(c):
    """Scores on a grid of 1/16, so that differences from the largest are exact.  A class's gradient over the largest one's is e^(z - m): two units in the last place for the
    exponential, and a rounded product on either side, 2^-22 + 2^-23 together; subnormal values are off by 2^-148 (half a spacing for the exponential, half for the product, and the
    largest's own)."""
    g = torch.Generator().manual_seed(c)
    z = -torch.randint(1, 103 * 16, (3, c), generator=g).double() / 16
    z[:, 1] = 0.0
    z[1] += 7.0
    z[2] -= 1000.0
    labels = torch.zeros(3, dtype=torch.int64)
    loss, grad = api.wpsgd_softmax_loss(z.float().cuda(), labels.cuda())
    p = grad.double().cpu()
    ratio = torch.exp(z - z.max(1, keepdim=True).values)
    largest = p[:, 1:2]
    want = ratio * largest
    off = (p - want).abs()[:, 1:]
    assert (off <= ((2.0 ** -22 + 2.0 ** -23) * want + 2.0 ** -148)[:, 1:]).all()
    assert (p > 0)[:, 1:][want[:, 1:] > 2.0 ** -148].all()
    # the sum itself: at most 2^12 additions by one thread and a tree
    assert ((1 / largest[:, 0] - ratio.sum(1)).abs() <= 2.0 ** -12 * ratio.sum(1)).all()
    assert ((loss.double().cpu() - (torch.logsumexp(z, 1) - z[:, 0])).abs() <= 2.0 ** -11 + 2.0 ** -21 * z.abs().amax(1)).all()


def test_differences_of_the_largest_and_a_masked_class():
    z = torch.full((2, 300), -math.inf)
    z[:, 7] = 3.0
    z[0, 200] = torch.finfo(torch.float32).min
    z[1, 200] = 3.0 - 103.0
    _, grad = api.wpsgd_softmax_loss(z.cuda(), torch.tensor([7, 7], device="cuda"))
    grad = grad.double().cpu()
    assert not grad[0].any() and abs(float(grad[1, 200]) - math.exp(-103.0)) <= 2.0 ** -149 and int((grad[1] != 0).sum()) == 1
