"""The 4-bit floating-point calls of the binding run on the device of their matrix, whatever device is current, and take
no tensor of another device.  No GPU: tensors that only say where they are, and a library that records its calls."""
import contextlib

import pytest
import torch

from paper_2309_15531_b200 import binding as B


class Tensor:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, dev, *shape, dtype=torch.bfloat16):
        self.dev, self.shape, self.dtype, self.device = dev, shape, dtype, torch.device("cuda", dev)
        self._version = 0

    def get_device(self):
        return self.dev

    def dim(self):
        return len(self.shape)

    def stride(self, k=None):
        s = [1] * len(self.shape)
        for i in range(len(s) - 2, -1, -1):
            s[i] = s[i + 1] * self.shape[i + 1]
        return tuple(s) if k is None else s[k]

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def data_ptr(self):
        return 4096 * (self.dev + 1)

    def is_contiguous(self):
        return True

    def is_inference(self):
        return False


@pytest.fixture
def calls(monkeypatch):
    """(entry point, stream, current device) of every call; device 0 is current, device d's stream is 100 + d."""
    made, current = [], [0]

    class Library:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, args[-1], current[0]))
                return 0
            return call

        def adadim_fp4_scale_bytes(self, *args):
            return 512

        def adadim_workspace_bytes(self, *args):
            return 256

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d
        yield
        current[0] = before

    real = torch.empty, torch.zeros
    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(B, "_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda t: None)

    def made_on(real):
        def f(*shape, dtype=torch.float32, device=None):
            shape = shape[0] if len(shape) == 1 and isinstance(shape[0], (tuple, list)) else shape
            return Tensor(torch.device(device).index or 0, *shape, dtype=dtype)
        return f

    monkeypatch.setattr(torch, "empty", made_on(real[0]))
    monkeypatch.setattr(torch, "zeros", made_on(real[1]))
    return made


def _i32(dev, n):
    return Tensor(dev, n, dtype=torch.int32)


def _f32(dev):
    return Tensor(dev, 1, dtype=torch.float32)


def _everything(dev, **other):
    """One call of each entry point with everything on `dev`, except what `other` names."""
    at = lambda name: other.get(name, dev)
    W = B.Fp4Tensor(32, 64, B.NVFP4, device=f"cuda:{at('W')}")
    Ws = B.Fp4Tensor(32, 64, B.NVFP4, experts=2, device=f"cuda:{at('W')}")
    x = Tensor(dev, 4, 64)
    q, qg = B.Fp4Tensor(4, 64, B.NVFP4, device=f"cuda:{at('q')}"), B.Fp4Tensor(4, 64, B.NVFP4, groups=2, device=f"cuda:{at('q')}")
    y, ws, st = Tensor(at("y"), 4, 32), Tensor(at("workspace"), 1024, dtype=torch.uint8), _i32(at("status"), 1)
    off, idx, amax = _i32(at("offsets"), 3), _i32(at("row_index"), 4), _f32(at("amax"))
    return {
        "absmax": lambda: B.absmax(x, amax),
        "quantize": lambda: B.quantize_fp4(x, B.NVFP4, amax=amax, q=q, values=Tensor(at("values"), 4, 64)),
        "quantize_groups": lambda: B.quantize_fp4(x, B.NVFP4, amax=amax, q=qg, row_index=idx, offsets=off),
        "linear": lambda: B.fp4_linear(x, W, x_amax=amax, y=y, workspace=ws, status=st),
        "matmul": lambda: B.fp4_linear(q, W, y=y, status=st),
        "linear_grouped": lambda: B.fp4_linear_grouped(x, off, Ws, row_index=idx, x_amax=amax, y=y, workspace=ws, status=st),
        "matmul_grouped": lambda: B.fp4_linear_grouped(qg, off, Ws, y=y, status=st),
    }


ENTRIES = ["absmax", "quantize", "quantize_groups", "linear", "matmul", "linear_grouped", "matmul_grouped"]


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("entry", ENTRIES)
def test_a_call_runs_on_the_device_of_its_matrix(calls, entry, dev):
    _everything(dev)[entry]()
    assert len(calls) == 1 and calls[0][1:] == (100 + dev, dev)


@pytest.mark.parametrize("entry,name", [
    ("absmax", "amax"), ("quantize", "amax"), ("quantize", "q"), ("quantize", "values"), ("quantize_groups", "row_index"),
    ("quantize_groups", "offsets"), ("linear", "W"), ("linear", "y"), ("linear", "workspace"), ("linear", "status"),
    ("linear", "amax"), ("matmul", "W"), ("matmul", "y"), ("matmul", "status"), ("linear_grouped", "W"),
    ("linear_grouped", "y"), ("linear_grouped", "workspace"), ("linear_grouped", "status"), ("linear_grouped", "offsets"),
    ("linear_grouped", "row_index"), ("linear_grouped", "amax"), ("matmul_grouped", "W"), ("matmul_grouped", "y"),
    ("matmul_grouped", "status"), ("matmul_grouped", "offsets")])
def test_a_tensor_of_another_device_is_refused(calls, entry, name):
    with pytest.raises((AssertionError, ValueError)):
        _everything(0, **{name: 1})[entry]()
    assert calls == []
