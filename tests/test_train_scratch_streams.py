"""The binding's training scratch and the streams that use it."""
import pytest

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, ptr):
        self.cuda_stream = ptr


class Buffer:
    def __init__(self):
        self.streams = []

    def data_ptr(self):
        return 256

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)


def test_the_scratch_is_recorded_once_for_every_stream_that_uses_it(monkeypatch):
    """No device: the layer's training calls with a stand-in for the library and for torch's streams."""
    from paper_2408_05646_b200 import binding as B
    default, under, seen = Stream(7), [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            under.append(self.stream)

        def __exit__(self, *a):
            under.pop()

    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    monkeypatch.setattr(B, "lib", Lib())
    monkeypatch.setattr(B, "_call_on", lambda *a: 0)
    monkeypatch.setattr(B, "device_alloc", lambda n, device: seen.append(under[-1]) or Buffer())
    monkeypatch.setattr(B.torch.cuda, "stream", On)
    monkeypatch.setattr(B.torch.cuda, "current_stream", lambda device=None: default)
    monkeypatch.setattr(B.torch._C, "_cuda_getCurrentRawStream", lambda index: default.cuda_stream, raising=False)
    lay = object.__new__(B.EigenAttnLayer)
    lay.handle, lay.B, lay.H, lay.device, lay.torch_dtype = None, 1, 1, torch.device("cuda:0"), torch.float32
    lay.offs_k = lay.offs_v = [0, 8]
    monkeypatch.setattr(lay, "_packed", lambda *a: 256, raising=False)
    monkeypatch.setattr(lay, "_new_out", lambda *a, **k: None, raising=False)
    x, a, b = torch.zeros(1, 4, 8), Stream(1), Stream(2)
    lay.train_forward(x, x, x)                               # (nothing attached: the library's to refuse)
    first = lay.train_attach(4, stream=a)
    assert seen == [a]
    lay.train_forward(x, x, x, stream=a)
    lay.train_backward(x, stream=a)
    lay.train_backward(x, stream=b)
    lay.train_forward(x, x, x)
    lay.train_forward(x, x, x, stream=b)
    assert first.streams == [1, 2, 7]
    second = lay.train_attach(4)
    assert seen == [a, None]
    lay.train_backward(x, stream=b)
    assert second.streams == [2] and first.streams == [1, 2, 7]
    lay.train_detach()
    lay.train_forward(x, x, x, stream=b)
    assert second.streams == [2]
