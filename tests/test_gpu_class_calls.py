"""The many-class operators as a program calls them: on other streams, in a HIP graph, one behind the other."""
import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu


class Step:
    """one worker's step with all its buffers made beforehand"""

    def __init__(self, n=70, classes=300, d=200, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.x = torch.randn(500, d, generator=g).bfloat16().cuda()
        self.rows = torch.randint(0, 500, (n,), generator=g).cuda()
        self.labels = torch.randint(0, classes, (n,), generator=g).cuda()
        self.W0 = (torch.randn(classes, d, generator=g) * 0.1).cuda()
        self.W = self.W0.clone()
        self.u = torch.rand(n, generator=g).cuda()
        self.dW = torch.empty_like(self.W)
        self.tensors = api.wpsgd_tensor_list([self.dW.view(-1)], [self.W.view(-1)])
        torch.cuda.synchronize()

    def __call__(self, stream=None):
        X = api.Matrix(500, self.x.shape[1], dense=self.x)
        W = api.Matrix(self.W.shape[0], self.W.shape[1], dense=self.W)
        x, w = api.wpsgd_quantize(X, rows=self.rows, stream=stream), api.wpsgd_quantize(W, stream=stream)
        Z = api.wpsgd_block_matmul(x, w, stream=stream)
        drawn, probs = api.wpsgd_draw_classes(Z, self.u, top_k=20, top_p=0.9, stream=stream)
        loss, G = api.wpsgd_softmax_loss(Z, self.labels, scale=1.0 / len(self.rows), stream=stream)
        g = api.wpsgd_quantize(api.Matrix(G.shape[0], G.shape[1], dense=G), transpose=True, stream=stream)
        xt = api.wpsgd_quantize(X, rows=self.rows, transpose=True, stream=stream)
        api.wpsgd_block_matmul(g, xt, out=self.dW, stream=stream)
        norm = api.wpsgd_clipped_step(self.tensors, 0.5, 1e-3, 0.05, stream=stream)
        self.keep = (x, w, Z, G, g, xt)
        return drawn, probs, loss, norm

    def result(self, out):
        torch.cuda.synchronize()
        return [t.clone() for t in out] + [self.W.clone()]


def test_another_stream_gives_the_same_bits():
    s = Step()
    want = s.result(s())
    s.W.copy_(s.W0)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        out = s()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, s.result(out)))
    s.W.copy_(s.W0)
    torch.cuda.synchronize()
    out = s(stream=stream)                            # named, while another stream is current
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, s.result(out)))


def test_a_graph_of_the_whole_step_replays():
    s = Step(seed=1)
    s()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    s.W.copy_(s.W0)
    with torch.cuda.graph(graph):
        out = s()
    for _ in range(4):
        s.W.copy_(s.W0)
        torch.cuda.synchronize()
        want = s.result(s())                          # eager work of the program's own between the replays
        s.W.copy_(s.W0)
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, s.result(out)))


def test_steps_bring_the_loss_down():
    """the whole batch's loss is convex and a step of length 0.025 against its gradient lowers it, each time"""
    s = Step(seed=2)
    losses = [float(s()[2].double().mean()) for _ in range(30)]
    assert all(b < a for a, b in zip(losses, losses[1:]))


def test_the_workers_example():
    """unequal workers learn, and the loss of their weighted average is under the weighted average of their losses, as the loss is convex (8-bit
    rows and class vectors give and take 1 % of it)"""
    import importlib.util
    import math
    import os

    from conftest import ROOT
    spec = importlib.util.spec_from_file_location("many_class_workers", os.path.join(ROOT, "examples", "many_class_workers.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    start, workers, average, answers, labels = example.train(m=4096, d=256, classes=300, heads=2, steps=(30, 30, 20, 10), batch=256)
    assert abs(start - math.log(300)) < 1e-4                      # zero class vectors: every class alike
    a = api.wpsgd_weights([30, 30, 20, 10], 2.0, 1e-4)
    assert all(v < start for v in workers) and average < 1.01 * sum(x * v for x, v in zip(a, workers)) and average < start
    assert answers.shape == labels.shape == (2048, 2) and bool(((answers >= 0) & (answers < 300)).all())
    assert float((answers == labels).double().mean()) > 1 / 300 + 5 * math.sqrt(1 / 300 / answers.numel())      # more often than by chance


def test_results_for_a_named_stream_are_not_memory_that_the_current_one_still_writes():
    """work that waits on the current stream writes to blocks that have been given back; calls that name another stream run meanwhile"""
    s = Step(seed=2)
    want = s.result(s())
    sizes = {t.numel() * t.element_size() for t in want} | {8192, 256, 512} | {t.codes.numel() for t in s.keep if isinstance(t, api.BlockMatrix)} | \
        {t.exps.numel() for t in s.keep if isinstance(t, api.BlockMatrix)} | {t.numel() * t.element_size() for t in s.keep if isinstance(t, torch.Tensor)}
    s.W.copy_(s.W0)
    s.keep = None
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    torch.cuda._sleep(100_000_000)                    # some tens of milliseconds
    held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sorted(sizes) for _ in range(8)]
    for t in held:
        t.fill_(0x5A)
    del held, t
    out = s(stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, s.result(out)))
