"""What runner.LmBatch hands to the library, on any stream (CPU only: the calls
are replaced by ones that record their arguments)."""
import numpy as np
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import LmBatch
from test_abi import _ensure_built


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


class _Context:
    def __init__(self, device):
        self.torch_device = torch.device(device)


def _batch(device, **kw):
    rng = np.random.Generator(np.random.PCG64(1))
    wl = W.make_workload("lm", [W.chain(int(n)) for n in (3, 7, 5)], N=1, D=4, H=64, C=9, rng=rng,
                         inputs="all", labels="all")
    table = torch.zeros(6, wl.D, device=device)
    b = LmBatch(wl, table, np.arange(wl.n_x) % 6, _Context(device), **kw)
    b.sched = object()
    return b


@pytest.fixture
def calls(monkeypatch):
    """Every binding call that would reach the GPU, as (name, arguments)."""
    _ensure_built()
    seen = []
    for name in ("embed", "embed_grad", "forward", "backward", "infer", "vocab_grad", "vocab_loss"):
        monkeypatch.setattr(B, name, lambda *a, _n=name: seen.append((_n, a)))
    for name in ("workspace_bytes", "infer_workspace_bytes"):
        monkeypatch.setattr(B, name, lambda *a: 64)
    return seen


def test_outputs_of_its_calls_stay_its_own(calls):
    """The calls only enqueue, on the context's stream: a tensor that a call
    writes must outlive it, or torch's allocator gives its memory to the current
    stream's next tensor while the kernel that writes it still waits."""
    b = _batch("cpu")
    b.alloc()
    for _ in range(2):
        b.forward()
        b.backward()
        b.infer()
    held = [t for v in vars(b).values() for t in (v.values() if isinstance(v, dict) else [v])]
    for name, args in calls:
        for a in args:
            if isinstance(a, torch.Tensor):
                assert any(a is t for t in held), name


class _DeviceWork(TorchDispatchMode):
    """The operations that read a tensor of the batch's device."""

    def __init__(self, device):
        super().__init__()
        self.device, self.seen = torch.device(device), []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if any(isinstance(a, torch.Tensor) and a.device == self.device for a in args):
            self.seen.append(str(func))
        return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("head_dtype", [torch.float32, torch.bfloat16])
def test_it_is_made_without_work_on_torch_s_stream(calls, head_dtype):
    """Copies from the host are complete when they return; a kernel on torch's
    current stream is not, and the context's stream does not wait for it."""
    word = np.zeros((15, 2), dtype=np.int32)
    with _DeviceWork("meta") as work:
        b = _batch("meta", head_dtype=head_dtype,
                   teacher=(word, word.astype(np.float32), 0.5, 2.0))
        b.alloc()
    assert b.Ws.dtype == head_dtype and b.Ws.shape == (64, 9)
    assert not [f for f in work.seen if not f.startswith("aten.empty_like")]
