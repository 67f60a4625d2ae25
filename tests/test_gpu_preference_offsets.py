"""Offsets that are wrong for one pair of the preference loss and right for others: only the first shows it."""
import math

import pytest
import torch

from paper_1708_04801_amd import api
from test_gpu_preference_loss import Case, ends_of

pytestmark = pytest.mark.gpu

GOOD = ends_of(3, 3, 2, 2, 4, 1)                      # 0 3 6 8 10 14 15, and two rows behind
# offsets, and the pairs whose own three are still right
BAD = [([0, 3, 6, 8, 10, 14, 2], [0, 1]), ([0, 3, 6, 8, 10, 14, 1 << 40], [0, 1]), ([0, 3, 6, 8, 10, 14, -1], [0, 1]), ([0, 3, 6, 8, 10, 18, 15], [0, 1]),
       ([22, 3, 6, 8, 10, 14, 15], [1, 2]), ([7, 3, 6, 8, 10, 14, 15], [1, 2]), ([-(1 << 62), 3, 6, 8, 10, 14, 15], [1, 2]), ([0, 3, 6, 1, 10, 14, 15], [0, 2]),
       ([0, 3, 99, 8, 10, 14, 15], [2]), ([9, 3, 6, 8, 10, 14, 5], [1])]


def pairs_of(k, offsets, **more):
    return api.wpsgd_preference_loss(k.z.clone(), k.labels.cuda(), torch.tensor(offsets).cuda(), ref_log=k.ref.cuda(), row_weights=k.w.float().cuda(),
                                     pair_weights=k.pw.float().cuda(), beta=k.beta, scale=k.scale, **more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [50, 3000, 70000])
def test_the_other_pairs_are_what_they_are(c, dtype):
    k = Case(GOOD, c, dtype, c, behind=2)
    want = k.run()
    for offsets, sound in BAD:
        for grad in (False, True):
            loss, margin, _ = pairs_of(k, offsets, grad=grad)
            lost = [p for p in range(3) if p not in sound]
            assert torch.equal(loss[sound], want[0][sound]) and torch.equal(margin[sound], want[1][sound]), offsets
            assert torch.isnan(loss[lost]).all() and torch.isnan(margin[lost]).all(), offsets


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [50, 900, 3000])
def test_the_other_pairs_where_the_gradient_takes_the_scores_place(c, dtype):
    """also where wrong offsets put a row into two pairs, or between them and behind them at once"""
    k = Case(GOOD, c, dtype, c, behind=2)
    want = k.run()
    cases = [(o, s, want[0][s], want[1][s]) for o, s in BAD]
    for offsets, sound in (([0, 6, 8, 8, 2, 4, 8], [0, 2]), ([3, 8, 15, 15, 0, 2, 4], [0, 2]), ([4, 6, 9, 1, 1, 1, 8], [0, 2])):
        alone = [pairs_of(k, [v] * (2 * p) + offsets[2 * p:2 * p + 3] + [offsets[2 * p + 2]] * (4 - 2 * p)) for p in sound for v in offsets[2 * p:2 * p + 1]]
        cases.append((offsets, sound, torch.stack([a[0][p] for a, p in zip(alone, sound)]), torch.stack([a[1][p] for a, p in zip(alone, sound)])))
    for offsets, sound, losses, margins in cases:
        for _ in range(3):
            z = k.z.clone()
            loss, margin, _ = api.wpsgd_preference_loss(z, k.labels.cuda(), torch.tensor(offsets).cuda(), ref_log=k.ref.cuda(), row_weights=k.w.float().cuda(),
                                                        pair_weights=k.pw.float().cuda(), beta=k.beta, scale=k.scale, grad=z)
            lost = [p for p in range(3) if p not in sound]
            assert torch.equal(loss[sound], losses) and torch.equal(margin[sound], margins), offsets
            assert torch.isnan(loss[lost]).all() and torch.isnan(margin[lost]).all(), offsets


@pytest.mark.parametrize("pairs", [1, 8, 511, 512, 513, 3000])
def test_few_rows_and_many_pairs(pairs):
    """up to 512 pairs in one launch, and more: the same results, whether the gradient takes the scores' place or not"""
    k = Case(ends_of(2, 1, 1, 3), 70, "f32", pairs, weighted=False)
    ends = torch.zeros(2 * pairs + 1, dtype=torch.int64)
    if pairs == 1:
        ends[:] = torch.tensor([0, 3, 7])
    else:
        ends[-4:] = torch.tensor(k.ends[1:])
    k.ends, k.pw = ends.tolist(), torch.ones(pairs)
    got = k.run()
    k.check(got)
    inside = k.run(grad=k.z)
    assert all(torch.equal(a, b) for a, b in zip(got, inside))
    assert (api.wpsgd_preference_loss_workspace(7, 70, pairs, torch.float32) == 0) == (pairs <= 512)
