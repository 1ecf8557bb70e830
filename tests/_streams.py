"""A stand-in for the GPU and its caching allocator: tensors in host memory that
say they are on cuda:0 and keep which stream was current when they were
allocated and which streams they were recorded for, and library calls that only
note their arguments."""
import struct

import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib


class Stream:
    def __init__(self, raw, device=0):
        self.cuda_stream, self.device = raw, torch.device("cuda", device)


class Gpu:
    def __init__(self, monkeypatch, calls):
        """``calls``: the library's functions that launch, by what stands in
        for each of them (called with the call's arguments)."""
        self.current = self.first = Stream(0x100)
        self.side = Stream(0x200)
        self.made = []  # tensors allocated, in order (kept, so that no address comes twice)
        real, gpu = _lib.lib(), self

        class Library:
            def __getattr__(self, name):
                return calls.get(name) or getattr(real, name)

        class On:
            def __init__(self, stream):
                self.stream = stream

            def __enter__(self):
                self.before, gpu.current = gpu.current, self.stream

            def __exit__(self, *a):
                gpu.current = self.before

        library, empty = Library(), torch.empty
        monkeypatch.setattr(_lib, "lib", lambda: library)
        monkeypatch.setattr(_lib, "native_rows", lambda: None)
        monkeypatch.setattr(pa, "_copy_blocks", lambda *a: None)
        monkeypatch.setattr(torch.cuda, "stream", On)
        monkeypatch.setattr(torch.cuda, "set_stream", lambda s: setattr(gpu, "current", s))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: gpu.current)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: gpu.current.cuda_stream)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
        monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw) if device is None else self.tensor(empty(*a, **kw)))
        monkeypatch.setattr(torch, "empty_like", lambda t: t.new_empty(t.shape))

    def tensor(self, t):
        x = torch.Tensor._make_subclass(Tensor, t)
        x.gpu, x.allocated, x.recorded = self, self.current, []
        self.made.append(x)
        return x

    def holder(self, address):
        """The allocated tensor that an address lies in."""
        at = [t for t in self.made if t.data_ptr() <= address < t.data_ptr() + max(1, t.numel() * t.element_size())]
        assert len(at) == 1, (hex(address), len(at))
        return at[0]


class Tensor(torch.Tensor):
    __torch_function__ = torch._C._disabled_torch_function_impl
    device = property(lambda self: torch.device("cuda", 0))
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0

    def new_empty(self, *size, dtype=None):
        shape = size[0] if len(size) == 1 and not isinstance(size[0], int) else size
        return self.gpu.tensor(torch.zeros(tuple(shape), dtype=dtype or self.dtype))

    def record_stream(self, stream):
        self.recorded.append(stream)


def addresses(packed):
    """The 8-byte words of a packed argument struct."""
    return struct.unpack(f"={len(packed) // 8}Q", packed)
