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
