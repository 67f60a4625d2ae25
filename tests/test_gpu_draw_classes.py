"""Classes drawn from scores, against the definition.  With temperature log2(e), rounded as the library rounds it, and whole-numbered scores every
weight is an exact power of two, and the drawn classes have to be the definition's."""
import math

import numpy as np
import pytest
import torch

import class_reference as ref
from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
T_ONE = float(np.float32(1.4426950408889634))        # the scores' unit is then one power of two
INF = math.inf

RULES = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=64), dict(top_k=1500), dict(top_p=0.5), dict(top_p=0.9), dict(top_p=0.0), dict(top_p=0.999999),
         dict(min_p=0.25), dict(min_p=1.0), dict(min_p=2.0 ** -9), dict(top_k=30, top_p=0.75), dict(top_k=5, min_p=0.125, top_p=0.6), dict(top_p=0.99, min_p=2.0 ** -14),
         dict(temperature=0.0), dict(top_k=-3, top_p=1.5)]


def whole_scores(n, c, dtype, seed, low=24, pad=0):
    """whole numbers from -low to 0, large ones rare, ties everywhere"""
    rng = np.random.default_rng(seed)
    z = -np.minimum(rng.geometric(0.05, size=(n, c + pad)), low)[:, ::-1] + np.where(rng.random((n, c + pad)) < 3.0 / c, 10, 0)
    return torch.from_numpy(z.copy()).to(DTYPES[dtype]).cuda()[:, :c]


def check(z, u, rule):
    n = z.shape[0]
    settings = dict(dict(temperature=T_ONE, top_k=0, top_p=1.0, min_p=0.0), **rule)
    drawn, probs = api.wpsgd_draw_classes(z, u, **settings)
    rows = z.float().cpu().tolist()
    for i in range(n):
        one = {k: (float(v[i]) if isinstance(v, torch.Tensor) else v) for k, v in settings.items()}
        want, q, total = ref.draw(rows[i], float(u[i]), None if one["temperature"] == 0 else T_ONE / one["temperature"], int(one["top_k"]),
                                  float(np.float32(one["top_p"])), float(np.float32(one["min_p"])))
        assert int(drawn[i]) == want, (i, one, int(drawn[i]), want)
        assert float(probs[i]) == float(np.float32(q / total)), (i, one)
    return drawn, probs


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,pad", [(3, 1, 0), (5, 2, 0), (6, 63, 0), (8, 100, 1), (5, 1000, 0), (4, 4097, 3), (3, 10007, 0)])
def test_draws_are_the_definitions(n, c, pad, dtype):
    z = whole_scores(n, c, dtype, c, pad=pad)
    g = torch.Generator().manual_seed(c)
    for rule in RULES:
        check(z, torch.rand(n, generator=g).cuda(), rule)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [33000, 131072, 140001, 1 << 18])
def test_long_rows(c, dtype):
    z = whole_scores(2, c, dtype, c)
    g = torch.Generator().manual_seed(c)
    for rule in RULES:
        check(z, torch.rand(2, generator=g).cuda(), rule)


@pytest.mark.parametrize("c", [5, 900, 20000, 131072])
def test_equal_scores_and_the_ends_of_u(c):
    """all classes tie: the first ones by index are kept, and u walks them evenly"""
    z = torch.full((7, c), -3.5, device="cuda")
    below = float(np.nextafter(np.float32(1), np.float32(0)))
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 0.9, below, 1e-30], device="cuda")
    for rule in (dict(), dict(top_k=4), dict(top_p=0.5), dict(top_p=0.3, top_k=max(1, c // 2)), dict(min_p=1.0), dict(temperature=0.0)):
        drawn, _ = check(z, u, rule)
        if rule.get("temperature") == 0.0:
            assert not drawn.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [9, 700, 33000])
def test_masked_rows(c, dtype):
    z = whole_scores(12, c, dtype, c + 1)
    lowest = torch.finfo(DTYPES[dtype]).min
    z[0] = -INF                                       # nothing to draw
    z[1] = math.nan
    z[2] = -INF
    z[2, c - 1] = lowest                              # one class, with the lowest score there is
    z[3, ::2] = -INF
    z[4, 1::2] = math.nan
    z[5] = lowest
    z[6, :] = -INF
    z[6, [0, c // 2, c - 1]] = torch.tensor([-1.0, 0.0, -1.0], device="cuda", dtype=z.dtype)
    z[7, 3] = INF                                     # the only class with weight
    z[8, [2, 5]] = INF                                # two of them
    z[9, 0] = -0.0
    z[9, 1:] = 0.0
    z[10, : c // 2] = lowest
    z[11, 1:] = math.nan
    g = torch.Generator().manual_seed(c)
    for rule in RULES:
        drawn, probs = check(z, torch.rand(12, generator=g).cuda(), rule)
        assert drawn[0] == drawn[1] == -1 and not probs[:2].any() and drawn[2] == c - 1 and drawn[7] == 3 and drawn[11] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,low", [(3000, 2), (30000, 1), (60000, 3)])
def test_scores_with_hardly_a_difference(c, low, dtype):
    """thousands of ties at the end of the run: more than a list holds"""
    z = whole_scores(3, c, dtype, c + low, low=low)
    g = torch.Generator().manual_seed(c)
    for rule in RULES + [dict(top_k=c - 1), dict(top_k=c // 2, top_p=0.7), dict(top_k=1024), dict(top_k=1025, top_p=0.3, min_p=0.5)]:
        check(z, torch.rand(3, generator=g).cuda(), rule)


def test_settings_of_each_row_its_own():
    n, c = 40, 3001
    z = whole_scores(n, c, "bf16", 7)
    g = torch.Generator().manual_seed(2)
    pick = lambda v, dt: torch.tensor(v, dtype=dt)[torch.randint(0, len(v), (n,), generator=g)].cuda()  # noqa: E731
    check(z, torch.rand(n, generator=g).cuda(), dict(temperature=pick([0.0, T_ONE, T_ONE, 2 * T_ONE], torch.float32), top_k=pick([0, 1, 40, 5000, -1], torch.int32),
                                                     top_p=pick([1.0, 0.9, 0.5, 0.01], torch.float32), min_p=pick([0.0, 0.0, 0.0625], torch.float32)))


@pytest.mark.parametrize("c,spread", [(50, 1.0), (1000, 3.0), (32000, 2.0), (131072, 1.0), (131072, 5.0)])
def test_draws_from_any_scores_lie_where_u_says(c, spread):
    """Weights in 64 bits.  A weight is off by at most (3 |z| ln 2 + 2) 2^-24 < 5e-6 of itself (|z| <= 32 powers of two) and 2^-32 of the largest: every sum by
    eps.  The drawn class's interval of the kept classes' sums has to reach to within 2 eps of u, and a class within eps of the end of the run may be kept or not."""
    n = 32
    g = torch.Generator().manual_seed(c)
    z = torch.randn(n, c, generator=g) * spread
    u = torch.rand(n, generator=g)
    for temperature, top_k, top_p in ((1.0, 0, 1.0), (0.7, 0, 0.9), (1.3, 200, 1.0), (1.0, 40, 0.8)):
        drawn, probs = api.wpsgd_draw_classes(z.cuda(), u.cuda(), temperature=temperature, top_k=top_k, top_p=top_p)
        for i in range(n):
            x = z[i].double()
            w = torch.exp((x - x.max()) / temperature)
            order = torch.sort(z[i], descending=True, stable=True).indices
            if top_k:
                order = order[:top_k]
            at = int(drawn[i])
            eps = 1e-5 + c * 2.0 ** -32
            total = float(w[order].sum())
            if top_p < 1:
                front = w[order].cumsum(0) - w[order]
                sure, maybe = order[front < (top_p - eps) * total], order[front < (top_p + eps) * total]
            else:
                sure = maybe = order
            assert at in maybe.tolist()
            # between the sums over the fewest and the most classes that may be kept
            lo = float(w[sure[sure < at]].sum()) / float(w[maybe].sum())
            hi = float(w[maybe[maybe <= at]].sum()) / float(w[sure].sum())
            assert lo - 2 * eps <= float(u[i]) <= hi + 2 * eps
            assert float(w[at]) / float(w[maybe].sum()) * (1 - 2 * eps) <= float(probs[i]) + 2.0 ** -31 and \
                float(probs[i]) <= float(w[at]) / float(w[sure].sum()) * (1 + 2 * eps) + 2.0 ** -31


def test_a_row_gets_the_same_answer_in_any_company():
    z = torch.randn(90, 40000, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    u = torch.rand(90, generator=torch.Generator().manual_seed(4)).cuda()
    rule = dict(temperature=0.9, top_k=300, top_p=0.93, min_p=0.01)
    drawn, probs = api.wpsgd_draw_classes(z, u, **rule)
    for lo, hi in ((0, 1), (17, 18), (40, 60), (89, 90)):
        d, p = api.wpsgd_draw_classes(z[lo:hi], u[lo:hi], **rule)
        assert torch.equal(d, drawn[lo:hi]) and torch.equal(p, probs[lo:hi])


def test_frequencies_follow_the_weights():
    c, n = 6, 20000
    z = torch.tensor([0.0, -1.0, -2.0, 0.0, -INF, -4.0]).repeat(n, 1).cuda()
    u = torch.rand(n, generator=torch.Generator().manual_seed(6)).cuda()
    drawn, _ = api.wpsgd_draw_classes(z, u, temperature=T_ONE)
    got = torch.bincount(drawn, minlength=c).double().cpu() / n
    w = 2.0 ** z[0].double().cpu()
    assert ((got - w / w.sum()).abs() <= 5 * math.sqrt(0.25 / n)).all() and got[4] == 0


def test_rows_behind_the_32_bit_offset():
    n, c = 20000, 131072
    z = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    z[-1, 77777] = 20.0
    drawn, _ = api.wpsgd_draw_classes(z, torch.full((n,), 0.5, device="cuda"), top_k=5)
    assert drawn[-1] == 77777 and (drawn[:-1] == 2).all()


def test_refusals():
    z, u = torch.zeros(3, 8, device="cuda"), torch.zeros(3, device="cuda")
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=math.nan), dict(min_p=1.5), dict(min_p=math.nan)):
        with pytest.raises(api.WpsgdError) as e:
            api.wpsgd_draw_classes(z, u, **bad)
        assert e.value.status == api.INVALID_ARG
    for bad in (lambda: api.wpsgd_draw_classes(z, u[:2]), lambda: api.wpsgd_draw_classes(z, u.double()), lambda: api.wpsgd_draw_classes(z.half(), u),
                lambda: api.wpsgd_draw_classes(z, u, top_k=torch.zeros(3, dtype=torch.int64, device="cuda")), lambda: api.wpsgd_draw_classes(z.cpu(), u),
                lambda: api.wpsgd_draw_classes(z, u, top_p=torch.zeros(2, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    drawn, _ = api.wpsgd_draw_classes(z[:0], u[:0])
    assert drawn.numel() == 0
    with pytest.raises(api.WpsgdError) as e:
        api.wpsgd_draw_classes(torch.zeros(1, (1 << 18) + 1, device="cuda"), u[:1])
    assert e.value.status == api.UNSUPPORTED
    # settings of rows cannot be refused: a temperature that is no positive number is 0, a min_p over 1 is 1
    drawn, _ = api.wpsgd_draw_classes(z, u + 0.9, temperature=torch.tensor([-1.0, math.nan, 1.0], device="cuda"),
                                      min_p=torch.tensor([0.0, 0.0, 7.0], device="cuda"))
    assert drawn.tolist() == [0, 0, 7]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [61, 64, 65, 128, 129, 255, 257, 8192, 8193])
def test_lists_about_as_long_as_those_compared_each_with_each(c, dtype):
    """few classes, so that all of them are listed, and the row lengths on both sides of the number of threads' change"""
    z = whole_scores(5, c, dtype, 3 * c)
    g = torch.Generator().manual_seed(c)
    for rule in (dict(top_k=50), dict(top_k=60, top_p=0.9), dict(top_k=120, top_p=0.6, min_p=0.125), dict(top_k=254), dict(top_k=40, min_p=0.5), dict(top_p=0.8)):
        check(z, torch.rand(5, generator=g).cuda(), rule)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,low", [(5000, 1), (8000, 2)])
def test_middling_rows_with_hardly_a_difference(c, low, dtype):
    """lists without room for what reaches the top_k-th score"""
    z = whole_scores(4, c, dtype, c + low, low=low)
    g = torch.Generator().manual_seed(low)
    for rule in (dict(top_k=50), dict(top_k=200, top_p=0.9), dict(top_k=2500), dict(top_p=0.5), dict(top_p=0.97), dict(min_p=0.5)):
        check(z, torch.rand(4, generator=g).cuda(), rule)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [6000, 15000, 26246, 131072])
def test_many_kept_of_rows_in_which_few_threads_have_scores(c, dtype):
    """top_k near the number of threads: scores in a corner of the row, in few places all over it, and everywhere"""
    z = whole_scores(4, c, dtype, c)
    z[0, 1500:] = -INF
    z[1, :c - 1200] = -INF
    keep = torch.zeros(c, dtype=torch.bool, device="cuda")
    keep[::37] = True
    z[2, ~keep] = -INF
    g = torch.Generator().manual_seed(c)
    for rule in (dict(top_k=250), dict(top_k=1000), dict(top_k=1024, top_p=0.9), dict(top_k=1000, min_p=0.125, top_p=0.5)):
        check(z, torch.rand(4, generator=g).cuda(), rule)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [700, 8192, 30000, 131072])
def test_min_p_that_keeps_few_or_seems_to(c, dtype):
    """rows whose kept classes have room in a list, and rows of equal scores, of which a sample sees next to nothing"""
    z = whole_scores(4, c, dtype, c + 1)
    z[2] = -2.0
    z[3] = -5.0
    z[3, ::2] = -4.0
    g = torch.Generator().manual_seed(c)
    for rule in (dict(min_p=2.0 ** -6, top_p=0.9), dict(min_p=0.25, top_p=0.5), dict(min_p=2.0 ** -20, top_p=0.95), dict(top_k=2000, top_p=0.7), dict(min_p=1.0, top_p=0.99)):
        check(z, torch.rand(4, generator=g).cuda(), rule)
