"""Which device the many-class calls are made on, with stand-ins for tensors, streams and the library, as on a machine with several GPUs: tensors of GPU 1 while GPU 0 is the
current one, and operands that lie on different ones."""
import contextlib

import pytest
import torch

from paper_1708_04801_amd import api


class Standin:
    """what the binding asks of a contiguous GPU tensor"""
    made = 0

    def __init__(self, shape, dtype, index):
        self.shape = torch.Size(shape if isinstance(shape, (tuple, list, torch.Size)) else (shape,))
        self.dtype, self.device, self.is_cuda = dtype, torch.device("cuda", index), True
        Standin.made += 1
        self.at = Standin.made << 20

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [1] * len(self.shape)
        for j in range(len(s) - 2, -1, -1):
            s[j] = s[j + 1] * max(1, self.shape[j + 1])
        return tuple(s) if i is None else s[i]

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device.index

    def data_ptr(self):
        return self.at

    def new_empty(self, shape, dtype=None):
        return Standin(shape, dtype or self.dtype, self.device.index)


@pytest.fixture
def seen(monkeypatch):
    """(name, current device, stream) of each call that queues work; the current device is 0"""
    now, calls = [0], []

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        yield
        now[0] = before

    class Library:
        def __getattr__(self, name):
            if name.endswith(("_workspace", "_bytes")):
                return lambda *a: 4096
            return lambda *a: calls.append((name, now[0], a[-1])) or api.OK

    monkeypatch.setattr(api, "load", lambda: Library())
    monkeypatch.setattr(torch, "Tensor", Standin)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(api, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda i=None: type("S", (), {"cuda_stream": 1000 + (now[0] if i is None else torch.device("cuda", i).index if isinstance(i, int) else i.index)})())
    monkeypatch.setattr(api, "_raw_stream", lambda index: 1000 + index, raising=False)
    if hasattr(torch._C, "_cuda_getCurrentRawStream"):
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index)
    return calls


F, B, I, C, U8 = torch.float32, torch.bfloat16, torch.int64, torch.float8_e4m3fn, torch.uint8


def block(index, rows=6, other=None):
    return api.BlockMatrix(rows, 200, Standin((rows, 256), C, index), Standin((rows, 4), U8, index if other is None else other))


def calls_of(index):
    """every call that queues work, its operands on GPU `index`; each takes the name of an operand that shall be on another"""
    def on(odd, name):
        return 1 - index if odd == name else index

    def quantize(stream=None, odd=None):
        x = api.Matrix(6, 200, dense=Standin((6, 200), F, index))
        api.wpsgd_quantize(x, rows=Standin((3,), I, on(odd, "rows")), codes=Standin((3, 256), C, on(odd, "codes")), exps=Standin((3, 4), U8, on(odd, "exps")), stream=stream)

    def matmul(stream=None, odd=None):
        b = block(index, 5)
        if odd == "B":
            b = block(1 - index, 5)
        elif odd == "exps":
            b = block(index, 5, 1 - index)
        api.wpsgd_block_matmul(block(index), b, out=Standin((6, 5), F, on(odd, "out")), workspace=Standin((4096,), U8, on(odd, "workspace")), stream=stream)

    def loss(stream=None, odd=None):
        api.wpsgd_softmax_loss(Standin((4, 9), F, index), Standin((4,), I, on(odd, "labels")), row_weights=Standin((4,), F, on(odd, "weights")),
                               loss=Standin((4,), F, on(odd, "loss")), grad=Standin((4, 9), F, on(odd, "grad")), stream=stream)

    def listed(stream=None, odd=None):
        return api.wpsgd_tensor_list([Standin((8,), F, index), Standin((8,), F, on(odd, "grad"))], [Standin((8,), F, index), Standin((8,), F, on(odd, "weight"))], stream=stream)

    def step(name, *args):
        def call(stream=None, odd=None):
            t = api.TensorList([], [], Standin((256,), U8, index), api._CTensorList())
            getattr(api, name)(t, *args, norm=Standin((1,), F, on(odd, "norm")), workspace=Standin((8192,), U8, on(odd, "workspace")), stream=stream)
        return call

    def draw(stream=None, odd=None):
        api.wpsgd_draw_classes(Standin((4, 9), B, index), Standin((4,), F, on(odd, "u")), top_p=Standin((4,), F, on(odd, "top_p")),
                               drawn=Standin((4,), I, on(odd, "drawn")), probs=Standin((4,), F, on(odd, "probs")), stream=stream)

    return {"wpsgd_quantize": (quantize, ["rows", "codes", "exps"]), "wpsgd_block_matmul": (matmul, ["B", "exps", "out", "workspace"]),
            "wpsgd_softmax_loss": (loss, ["labels", "weights", "loss", "grad"]), "wpsgd_tensor_list_make": (listed, ["grad", "weight"]),
            "wpsgd_grad_norm": (step("wpsgd_grad_norm"), ["norm", "workspace"]), "wpsgd_clip_grads": (step("wpsgd_clip_grads", 1.0), ["norm", "workspace"]),
            "wpsgd_clipped_step": (step("wpsgd_clipped_step", 0.1, 0.0, 1.0), ["norm", "workspace"]), "wpsgd_draw_classes": (draw, ["u", "top_p", "drawn", "probs"])}


NAMES = list(calls_of(0))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("index", [0, 1])
def test_work_is_queued_on_the_operands_device(seen, name, index):
    calls_of(index)[name][0]()
    calls_of(index)[name][0](stream=77)
    assert seen == [(name, index, 1000 + index), (name, index, 77)]
    assert torch.cuda.current_device() == 0


@pytest.mark.parametrize("name,odd", [(n, o) for n in NAMES for o in calls_of(0)[n][1]])
def test_operands_of_two_devices_are_refused(seen, name, odd):
    for index in (0, 1):
        with pytest.raises(AssertionError):
            calls_of(index)[name][0](odd=odd)
    assert seen == []


@pytest.mark.parametrize("name", NAMES)
def test_streams_of_another_device_are_refused(seen, name):
    stream = type("S", (), {"cuda_stream": 5, "device_index": 0})()
    with pytest.raises(AssertionError):
        calls_of(1)[name][0](stream=stream)
    assert seen == []
