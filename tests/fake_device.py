"""Stand-ins for device tensors, streams and the library, for tests of the binding without a GPU."""
import contextlib

import torch


class Tensor:
    """What the binding asks of a tensor; `under`: the stream whose allocations were current when it was made."""

    def __init__(self, shape, dtype=torch.float32, device="cuda", stride=None, under=None):
        self.shape = (shape,) if isinstance(shape, int) else tuple(shape)
        self.dtype, self.under = dtype, under
        self.device = torch.device(device)
        self.is_cuda = self.device.type == "cuda"
        self._stride = tuple(stride) if stride is not None else tuple(
            torch.Size(self.shape[k + 1:]).numel() for k in range(len(self.shape)))
        self._dense, self.used_on = stride is None, []

    def numel(self):
        return torch.Size(self.shape).numel()

    def dim(self):
        return len(self.shape)

    def stride(self, k=None):
        return self._stride if k is None else self._stride[k]

    def is_contiguous(self):
        return self._dense

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        self.used_on.append(stream)

    def __iter__(self):
        return iter([Tensor(self.shape[1:], self.dtype, self.device, under=self.under) for _ in range(self.shape[0])])


class Stream:
    cuda_stream = 0x5EED


class Library:
    """Accepts every call, and keeps them; sizes of workspaces are 512 bytes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 512 if name.endswith("_workspace_bytes") else 0
        return call


class Machine:
    """Puts the stand-ins into the modules that are given; made: every tensor that was allocated since."""

    def __init__(self, monkeypatch, *modules):
        self.lib, self.made, streams = Library(), [], []

        @contextlib.contextmanager
        def current(stream):
            streams.append(stream)
            yield
            streams.pop()

        def empty(shape, dtype=None, device=None):
            t = Tensor(shape, dtype or torch.float32, device or "cpu", under=streams[-1] if streams else None)
            self.made.append(t)
            return t
        for m in modules:
            monkeypatch.setattr(m, "lib", self.lib)
        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(torch.cuda, "stream", current)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda: streams[-1] if streams else "current")
