"""The cache's front end on the CPU: real sizes and layouts, calls that would
launch are only noted.  For tests of what the front end lets through."""
import torch

from paper_2508_01744_amd import _lib as L
from paper_2508_01744_amd import kv

LAUNCHING = ("reset", "plan", "commit", "append", "attend", "export")


class Lib:
    def __init__(self, real):
        self.real, self.calls, self.args = real, [], []

    def __getattr__(self, name):
        if not name.startswith("agft_kv_"):
            return getattr(self.real, name)
        if name[8:] not in LAUNCHING:
            return getattr(self.real, name)

        def note(*args):
            self.calls.append(name[8:])
            self.args.append(args)
            return L.AGFT_OK
        return note


class Device:
    """Stands for the CPU where a torch.device is asked for its index."""
    type, index = "cpu", -1

    def __eq__(self, other):
        return other is self or str(other) == "cpu"

    def __str__(self):
        return "cpu"


def install(monkeypatch):
    """The front end's objects go to the CPU; returns the library that notes calls."""
    lib = Lib(L.lib())

    def empty(self, *shape, dtype):
        n = dtype.itemsize
        for s in shape:
            n *= s
        raw = torch.zeros(n + 256, dtype=torch.uint8)
        at = -raw.data_ptr() % 256
        return raw[at:at + n].view(dtype).view(shape)
    monkeypatch.setattr(L, "lib", lambda: lib)
    monkeypatch.setattr(kv, "_device", lambda device: Device())
    monkeypatch.setattr(kv._OnStream, "_empty", empty)
    monkeypatch.setattr(kv, "_current_raw_stream", lambda index: 0)
    monkeypatch.setattr(kv, "_current_device", lambda: Device.index, raising=False)
    return lib
