"""Which device the calls for training on answers, dropout and four bits are made on, with the stand-ins of the many-class calls: tensors of GPU 1 while GPU 0 is the current one, and
operands that lie on different ones."""
import pytest
import torch

from paper_1708_04801_amd import api
from test_class_devices import Standin, seen  # noqa: F401  (the fixture)

F, B, I, U8 = torch.float32, torch.bfloat16, torch.int64, torch.uint8


def calls_of(index):
    def on(odd, name):
        return 1 - index if odd == name else index

    def vector(n, dtype, odd, name):
        return Standin((n,), dtype, on(odd, name))

    def policy(stream=None, odd=None):
        v = {name: vector(4, F, odd, name) for name in ("old_log", "ref_log", "row_weights", "loss", "log_prob")}
        api.wpsgd_policy_loss(Standin((4, 9), F, index), vector(4, I, odd, "drawn"), vector(4, F, odd, "advantage"), grad=Standin((4, 9), F, on(odd, "grad")), stream=stream, **v)

    def preference(stream=None, odd=None):
        v = {name: vector(4, F, odd, name) for name in ("ref_log", "row_weights")}
        v.update({name: vector(2, F, odd, name) for name in ("pair_weights", "loss", "margin")})
        api.wpsgd_preference_loss(Standin((4, 9), F, index), vector(4, I, odd, "labels"), vector(5, I, odd, "offsets"), grad=Standin((4, 9), F, on(odd, "grad")),
                                  workspace=Standin((8192,), U8, on(odd, "workspace")), stream=stream, **v)

    def dropout(stream=None, odd=None):
        api.wpsgd_dropout(api.Matrix(6, 200, dense=Standin((6, 200), F, index)), 0.5, 1, rows=vector(3, I, odd, "rows"), more_steps=vector(1, I, odd, "more_steps"),
                          out=Standin((3, 200), F, on(odd, "out")), stream=stream)

    def quantize(stream=None, odd=None):
        api.wpsgd_quantize_nibbles(api.Matrix(6, 200, dense=Standin((6, 200), F, index)), group=64, rows=vector(3, I, odd, "rows"),
                                   codes=Standin((3, 128), U8, on(odd, "codes")), scales=Standin((3, 8), B, on(odd, "scales")), stream=stream)

    def matmul(stream=None, odd=None):
        w = api.NibbleMatrix(5, 200, 64, Standin((5, 128), U8, on(odd, "codes")), Standin((5, 8), B, on(odd, "scales")))
        api.wpsgd_nibble_matmul(api.Matrix(6, 200, dense=Standin((6, 200), F, index)), w, rows=vector(3, I, odd, "rows"), out=Standin((3, 5), F, on(odd, "out")), stream=stream)

    return {"wpsgd_policy_loss": (policy, ["drawn", "advantage", "old_log", "ref_log", "row_weights", "loss", "log_prob", "grad"]),
            "wpsgd_preference_loss": (preference, ["labels", "offsets", "ref_log", "row_weights", "pair_weights", "loss", "margin", "grad", "workspace"]),
            "wpsgd_dropout": (dropout, ["rows", "more_steps", "out"]), "wpsgd_quantize_nibbles": (quantize, ["rows", "codes", "scales"]),
            "wpsgd_nibble_matmul": (matmul, ["codes", "scales", "rows", "out"])}


NAMES = list(calls_of(0))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("index", [0, 1])
def test_work_is_queued_on_the_operands_device(seen, name, index):  # noqa: F811
    calls_of(index)[name][0]()
    calls_of(index)[name][0](stream=77)
    assert seen == [(name, index, 1000 + index), (name, index, 77)]
    assert torch.cuda.current_device() == 0


@pytest.mark.parametrize("name,odd", [(n, o) for n in NAMES for o in calls_of(0)[n][1]])
def test_operands_of_two_devices_are_refused(seen, name, odd):  # noqa: F811
    for index in (0, 1):
        with pytest.raises(AssertionError):
            calls_of(index)[name][0](odd=odd)
    assert seen == []


@pytest.mark.parametrize("name", NAMES)
def test_streams_of_another_device_are_refused(seen, name):  # noqa: F811
    stream = type("S", (), {"cuda_stream": 5, "device_index": 0})()
    with pytest.raises(AssertionError):
        calls_of(1)[name][0](stream=stream)
    assert seen == []
