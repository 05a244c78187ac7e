"""What the GPU tests of the operators around the training step share."""
import numpy as np
import torch

DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step of the storage type, relative to the value
U = 2.0 ** -24                                     # half a step of fp32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(seed, *shape):
    return torch.randn(shape, generator=gen(seed))


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def np32(t):
    return t.detach().float().cpu().numpy()


class Guarded:
    """A device tensor between two runs of a known byte; check() says whether anything outside it was written."""

    def __init__(self, shape, dtype, fill=None):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.slab = torch.full((256 + n + (-n % 16) + 256,), 0xA5, dtype=torch.uint8, device=DEV)
        self.n = n
        self.t = self.slab[256:256 + n].view(dtype).view(shape)
        if fill is not None:
            self.t.copy_(fill)

    def check(self):
        assert torch.all(self.slab[:256] == 0xA5) and torch.all(self.slab[256 + self.n:] == 0xA5), "written outside the tensor"


def replayed(call, outputs, rounds=3):
    """call() captured into a graph and replayed; the outputs after each replay."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    seen = []
    for _ in range(rounds):
        for t in outputs:
            t.fill_(1)
        torch.cuda.synchronize()
        torch.ones(1000, device=DEV).sum().item()      # the program's own work between replays
        g.replay()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in outputs])
    return seen
