"""Training on answers, dropout and four bits as a program calls them: one behind the other, on other streams, in HIP graphs, in the example."""
import importlib.util
import os

import pytest
import torch

from conftest import ROOT
from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu


class Round:
    """a batch's way through all of them, with its inputs made beforehand"""

    def __init__(self, n=48, classes=300, d=200, seed=0, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        self.x = torch.randn(500, d, generator=g).to(dtype).cuda()
        self.W = (torch.randn(classes, d, generator=g) * 0.1).cuda()
        self.rows = torch.randint(0, 500, (n,), generator=g).cuda()
        self.u = torch.rand(n, generator=g).cuda()
        self.advantage = torch.randn(n, generator=g).cuda()
        self.ends = torch.tensor([0, 5, 11, 20, n - 4], dtype=torch.int64).cuda()
        self.more = torch.zeros(1, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()

    def __call__(self, stream=None):
        n, d = len(self.rows), self.x.shape[1]
        X, W = api.Matrix(500, d, dense=self.x), api.Matrix(self.W.shape[0], d, dense=self.W)
        x = api.wpsgd_dropout(X, 0.2, 5, chain=1, step=2, rows=self.rows, more_steps=self.more, stream=stream)
        D = api.Matrix(n, d, dense=x)
        W4 = api.wpsgd_quantize_nibbles(W, group=64, stream=stream)
        Z = api.wpsgd_nibble_matmul(D, W4, dtype=torch.float32, stream=stream)
        drawn, _ = api.wpsgd_draw_classes(Z, self.u, top_k=30, stream=stream)
        first, _ = api.wpsgd_softmax_loss(Z, drawn, grad=False, stream=stream)
        loss, log_prob, G = api.wpsgd_policy_loss(Z, drawn, self.advantage, old_log=first, ref_log=first, kl=0.1, scale=0.5, stream=stream)
        pair, margin, P = api.wpsgd_preference_loss(Z, drawn, self.ends, ref_log=first, beta=0.2, stream=stream)
        wide = api.wpsgd_preference_loss(Z.repeat(1, 4) if stream is None else self.wide, drawn, self.ends, stream=stream)       # (more classes than one launch takes)
        dx = api.wpsgd_dropout(D, 0.2, 5, chain=1, step=2, more_steps=self.more, out=x, stream=stream)
        self.keep = (W4, Z, first, P)
        return x, drawn, loss, log_prob, G, pair, margin, P, *wide, dx


def result(out):
    torch.cuda.synchronize()
    return [t.clone() for t in out]


def same(a, b):
    return all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip(a, b))


def test_another_stream_gives_the_same_bits():
    r = Round()
    want = result(r())
    r.wide = r.keep[1].repeat(1, 4)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        out = r()
    stream.synchronize()
    assert same(want, result(out))
    out = r(stream=stream)                            # named, while another stream is current
    stream.synchronize()
    assert same(want, result(out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_graph_of_all_of_them_replays(dtype):
    r = Round(seed=1, dtype=dtype)
    r()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r()
    for step in (0, 3, 1, 3):                         # the mask goes on from replay to replay
        r.more.fill_(step)
        want = result(r())                            # eager work of the program's own between the replays
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert same(want, result(out))


def test_results_for_a_named_stream_are_not_memory_that_the_current_one_still_writes():
    """work that waits on the current stream writes to blocks that have been given back; calls that name another stream run meanwhile"""
    r = Round(seed=2)
    want = result(r())
    r.wide = r.keep[1].repeat(1, 4)
    sizes = {t.numel() * t.element_size() for t in want} | {r.keep[0].codes.numel(), 2 * r.keep[0].scales.numel(), 4 * r.keep[1].numel(), 1024}
    r.keep = None
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    torch.cuda._sleep(100_000_000)                    # some tens of milliseconds
    held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sorted(sizes) for _ in range(8)]
    for t in held:
        t.fill_(0x5A)
    del held, t
    out = r(stream=stream)
    stream.synchronize()
    assert same(want, result(out))


def test_gradients_of_scores_through_all_of_them_match_differences():
    """the class vectors' gradient of the policy loss, through scores in 8-bit blocks, against differences of the loss along it: a step of h against the gradient lowers the
    loss by h times its squared norm"""
    n, classes, d = 64, 200, 256
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n, d, generator=g, device="cuda")
    W = torch.randn(classes, d, generator=g, device="cuda") * 0.05
    D = api.Matrix(n, d, dense=x)
    x8, xt8 = api.wpsgd_quantize(D), api.wpsgd_quantize(D, transpose=True)
    old = torch.empty(n, device="cuda")
    advantage = torch.randn(n, generator=g, device="cuda")
    ends = torch.arange(0, n + 1, 4, device="cuda")
    u = torch.rand(n, generator=g, device="cuda")

    def scores(weights):                              # (the products' own rounding stays out of the differences: rows in 8 bits, class vectors in fp32)
        values = x8.codes.float().view(n, -1, 128) * torch.exp2(x8.exps[:, :d // 128].float() - 127)[..., None]
        return values.view(n, d) @ weights.t()

    Z = scores(W)
    drawn, _ = api.wpsgd_draw_classes(Z, u)
    old = -api.wpsgd_softmax_loss(Z, drawn, grad=False)[0]
    calls = [lambda z: api.wpsgd_policy_loss(z, drawn, advantage, old_log=old - 0.01, ref_log=old, kl=0.2, scale=1.0 / n),
             lambda z: api.wpsgd_preference_loss(z, drawn, ends, ref_log=old, beta=0.5, scale=1.0 / n)]
    for call in calls:
        loss, _, G = call(Z)
        dW = api.wpsgd_block_matmul(api.wpsgd_quantize(api.Matrix(n, classes, dense=G), transpose=True), xt8, dtype=torch.float32)
        exact = G.t() @ (x8.codes.float().view(n, -1, 128) * torch.exp2(x8.exps[:, :d // 128].float() - 127)[..., None]).view(n, d)
        assert float((dW - exact).norm() / exact.norm()) < 2.0 ** -3          # both operands of the product in 8 bits: 2^-4 of an element each
        h = 1e-3
        up, down = (float(call(scores(W + s * h * exact))[0].double().sum()) / n for s in (1, -1))
        # the quotient leaves out h^2 / 6 of third derivatives, which along 1e-3 of the gradient are far under 1e-3 of the slope, and the losses' own 2^-20
        slope = float(exact.double().square().sum())
        assert abs((up - down) / (2 * h) - slope) <= 1e-2 * slope + 2.0 ** -20 / h


def test_the_example_tunes_and_serves():
    spec = importlib.util.spec_from_file_location("many_class_workers", os.path.join(ROOT, "examples", "many_class_workers.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    m, d, classes, heads = 1024, 256, 100, 2
    x, labels = example.data_set(m, d, classes, heads)
    X = api.Matrix(m, d, dense=x)
    row = (torch.randn(heads * classes * d, generator=torch.Generator().manual_seed(1)) * 0.01).cuda()
    before = row.clone()
    right, margins = example.tune(row, X, labels, classes, d, heads, steps=3, batch=64)
    assert right.shape == margins.shape == (3,) and bool(torch.isfinite(row).all()) and not torch.equal(row, before)
    assert bool(((right >= 0) & (right <= 1)).all()) and float(margins[0].abs()) < 10
    model = example.Heads(row, classes, d, heads)
    rows, u = torch.arange(5, device="cuda"), torch.rand(5, generator=torch.Generator().manual_seed(2)).cuda()
    answers = example.serve(model.four_bits(), X, rows, u, top_k=10)
    assert answers.shape == (5, heads) and bool(((answers >= 0) & (answers < classes)).all())
