"""min_p just above, at and just below weights that occur, where top_k ends among the classes of that weight: by lists compared each with each, longer
lists, and rows without a list."""
import numpy as np
import pytest
import torch

import class_reference as ref
from paper_1708_04801_amd import api
from test_gpu_draw_classes import T_ONE, check, whole_scores

pytestmark = pytest.mark.gpu


def beside(v, step):
    """the fp32 number next to v on that side, or v"""
    v = np.float32(v)
    return float(v if step == 0 else np.nextafter(v, np.float32(step * 2)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,low", [(700, 24), (6000, 24), (6000, 6), (20000, 24), (131072, 24), (131072, 8)])
def test_ties_of_the_last_class_of_top_k_have_to_reach_min_p(c, low, dtype):
    z = whole_scores(2, c, dtype, c + low, low=low)
    u = torch.rand(2, generator=torch.Generator().manual_seed(c)).cuda()
    for i in range(2):
        one = z[i:i + 1]
        scores = one[0].float().cpu().numpy()
        top = scores.max()
        for s in sorted({int(v) for v in top - scores if 0 < v <= 24})[:14]:
            over, up_to = int((scores > top - s).sum()), int((scores >= top - s).sum())
            top_k = (over + up_to + 1) // 2                      # among the classes of that score, or its only one
            for step in (-1, 0, 1):
                min_p = beside(2.0 ** -s, step)
                check(one, u[i:i + 1], dict(top_k=top_k, min_p=min_p))
                check(one, u[i:i + 1], dict(top_k=top_k, min_p=min_p, top_p=0.8))
            check(one, u[i:i + 1], dict(min_p=beside(2.0 ** -s, 1)))


@pytest.mark.parametrize("c,top_k", [(1000, 100), (1000, 200), (1000, 500), (20000, 200), (20000, 900), (20000, 3000)])
def test_scores_a_step_below_the_largest_do_not_reach_all_of_its_weight(c, top_k):
    """ten scores of 1 and the rest one step of fp32 below: their weight 2^(-2^-24 log2 e) = 1 - 2^-24 is under a min_p of 1 (temperature 1/4: 1 - 2^-22)"""
    z = torch.full((1, c), float(np.nextafter(np.float32(1), np.float32(0))))
    at = torch.randperm(c, generator=torch.Generator().manual_seed(c))[:10]
    z[0, at] = 1.0
    for u in (0.0, 0.35, 0.999):
        drawn, probs = api.wpsgd_draw_classes(z.cuda(), torch.tensor([u], device="cuda"), temperature=0.25, top_k=top_k, min_p=1.0)
        assert int(drawn) == int(at.sort().values[int(u * 10)]) and abs(float(probs) - 0.1) < 1e-7


@pytest.mark.parametrize("reach", [40, 200, 900, 3000])
def test_what_top_k_leaves_does_not_say_which_path_a_row_takes(reach):
    """the classes that min_p leaves are the same whatever top_k is over their number"""
    c = 30000
    at = torch.randperm(c, generator=torch.Generator().manual_seed(reach))
    z = torch.full((1, c), -6.0)
    z[0, at[:reach]] = 0.0
    z[0, at[reach:2 * reach]] = -1.0
    u = torch.tensor([0.7])
    want = ref.draw(z[0].tolist(), float(u[0]), 1.0, 0, 1.0, beside(0.5, 1))
    assert want[2] == reach << 31
    for top_k in [k for k in (50, 128, 129, 250, 300, 1000, 1024, 1025, 2000, 10000, 29999) if k >= reach]:
        drawn, probs = api.wpsgd_draw_classes(z.bfloat16().cuda(), u.cuda(), temperature=T_ONE, top_k=top_k, min_p=beside(0.5, 1))
        assert int(drawn) == want[0] and float(probs) == float(np.float32(want[1] / want[2]))
