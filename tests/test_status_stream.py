"""On which stream, and with which device current, a scratch's status is read: the device and its streams are made up.  CPU only."""
import types

import torch

from paper_2608_15531_b200 import binding as fq


class Scratch:
    is_cuda = True

    def __init__(self, index):
        self.device = torch.device("cuda", index)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000 * (1 + self.device.index)


class Cuda:
    """Two devices, the first one current; each has a current stream of its own."""

    def __init__(self, monkeypatch):
        self.now, self.read = 0, []
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0x50 + self.index(device)))
        monkeypatch.setattr(torch.cuda, "device", self.guard)
        monkeypatch.setattr(fq, "lib", lambda: types.SimpleNamespace(fq_check_status=self.check))

    def index(self, device):
        return self.now if device is None else torch.device(device).index if not isinstance(device, int) else device

    def guard(self, device):
        cuda, want = self, self.index(device)

        class Guard:
            def __enter__(self):
                self.before, cuda.now = cuda.now, want

            def __exit__(self, *a):
                cuda.now = self.before
        return Guard()

    def check(self, workspace, stream):
        self.read.append((workspace.value, stream.value, self.now))
        return fq.FQ_OK


def test_the_status_is_read_behind_the_calls_of_the_scratch_s_own_device(monkeypatch):
    """The FP4 calls run on their tensors' device, on its current stream, whichever device is current."""
    cuda = Cuda(monkeypatch)
    fq.fq_check_status(Scratch(0))
    fq.fq_check_status(Scratch(1))
    fq.fq_check_status(Scratch(1), stream=types.SimpleNamespace(cuda_stream=0x77))
    assert cuda.read == [(0x1000, 0x50, 0), (0x2000, 0x51, 1), (0x2000, 0x77, 1)]
    assert cuda.now == 0


def test_no_workspace_is_the_library_s_to_refuse(monkeypatch):
    cuda = Cuda(monkeypatch)
    fq.fq_check_status(None)
    assert cuda.read == [(None, 0x50, 0)]
