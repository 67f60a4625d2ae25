"""The calls that the cases of training on answers make, on inputs as they make them: small vocabularies with classes masked, where a row that does not count may have its first class
masked, against the definitions in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

import answer_reference as ref
from conftest import ROOT

pytestmark = pytest.mark.gpu

# Off by: a score less the row's largest, a place of the exponential and eight additions of them in fp32 (the sums over them are in fp64), 2^-24 each of what they are: the first of
# at most 32 here.  Under 2^-18 of a probability, and as much of a log of a row's sum.
EXP = 2.0 ** -18


@pytest.fixture(scope="module")
def cases():
    spec = importlib.util.spec_from_file_location("more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.own = True
    return module


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,kl", [(62, 3, 0.02), (92, 5, 0.2), (200, 4, 0.0), (300, 17, 0.2)])
def test_policy(cases, rows, classes, kl, storage):
    met = 0
    for seed in range(6):
        s = cases.prepare(dict(op="policy", rows=rows, classes=classes, storage=storage, masked=True, kl=kl), seed)
        loss, log_p, grad = (t.double().cpu() for t in cases.run(s))
        z, d, w, A = s["Z"].double().cpu(), s["drawn"].cpu(), s["weights"].cpu(), s["advantage"].cpu()
        old, rf = s["old"].cpu(), s["ref"].cpu() if kl else None
        want, logs, want_grad, factor = ref.policy_loss(z, d, old.tolist(), rf.tolist() if kl else None, A, w, s["low"], s["high"], kl, s["scale"])
        out = d < 0
        met += int((out & (z[:, 0] == -math.inf)).sum())
        assert not loss[out].any() and not log_p[out].any() and not grad[out].any()
        ratio = torch.exp(logs - old.double())
        # a ratio this near to a border may be on either side of it (the loss hardly moves, the factor may be 0 or whole)
        near = ((ratio - (1 - s["low"])).abs() <= 2 * EXP * ratio) | ((ratio - (1 + s["high"])).abs() <= 2 * EXP * ratio)
        back = torch.exp(rf.double() - logs) if kl else torch.zeros(rows, dtype=torch.float64)
        move = 1.01 * EXP * w.double() * (A.double().abs() * ratio + kl * (1 + back)) * ~out
        assert ((log_p - logs).abs() <= EXP + 2.0 ** -24 * logs.abs())[~out].all()
        assert ((loss - want).abs() <= move + 2.0 ** -24 * want.abs()).all()
        share = torch.softmax(z, 1)
        share[torch.arange(rows), d.clamp(min=0)] += 1
        rounded = 2.0 ** -8 if storage == "bf16" else 2.0 ** -22
        size = (s["scale"] * move + (EXP + 2.0 ** -22) * factor.abs())[:, None] * share + rounded * want_grad.abs() + 1e-37
        assert ((grad - want_grad).abs() <= size)[~near].all()
    assert met > 0                                    # of rows that do not count and have class 0 masked


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("pairs,length,classes", [(6, 9, 3), (10, 12, 4), (32, 40, 3)])
def test_preference(cases, pairs, length, classes, storage):
    met = 0
    for seed in range(6):
        s = cases.prepare(dict(op="preference", pairs=pairs, length=length, classes=classes, storage=storage, kind="logistic", masked=True), seed)
        loss, margin, grad = (t.double().cpu() for t in cases.run(s))
        z, labels, ends = s["Z"].double().cpu(), s["labels"].cpu(), s["offsets"].tolist()
        n, w = len(z), s["pair_weights"].cpu()
        out = labels < 0
        met += int((out & (z[:, 0] == -math.inf)).sum())
        want, want_margin, want_grad, slopes = ref.preference_loss(z, labels, ends, s["ref"].tolist(), torch.ones(n), w, False, s["beta"], s["smoothing"], s["scale"])
        off = s["beta"] * EXP * torch.tensor([b - a for a, b in zip(ends[:-2:2], ends[2::2])], dtype=torch.float64)
        assert ((margin - want_margin).abs() <= off + 2.0 ** -24 * want_margin.abs()).all() and ((loss - want).abs() <= w * off + 2.0 ** -24 * want.abs()).all()
        share = torch.softmax(z, 1)
        share[torch.arange(n), labels.clamp(min=0)] += 1
        bound = (2.0 ** -8 if storage == "bf16" else 2.0 ** -22) * want_grad.abs() + 1e-37
        for p in range(pairs):
            a, b = ends[2 * p], ends[2 * p + 2]
            bound[a:b] += s["scale"] * s["beta"] * float(w[p]) * (float(off[p]) / 4 + EXP + 2.0 ** -22) * share[a:b]
        assert ((grad - want_grad).abs() <= bound).all() and not grad[out].any() and not grad[ends[-1]:].any()
    assert met > 0
