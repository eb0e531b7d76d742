"""Rules on logits whose arrays are NULL or not read: which calls the library takes,
and that they change nothing (what it refuses is in test_gpu_next_refused)."""
import ctypes as ct

import pytest
import torch

from paper_1712_04048_amd import binding as B
from test_gpu_rules import _float32_by_default, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

N, C = 3, 700


@pytest.mark.parametrize("kind", ["nothing", "penalties, L = 0", "past alone", "words, K = 0", "M alone", "biases, K = 0"])
def test_steps_left_out(ctx, kind):
    z = torch.randn(N, C, generator=torch.Generator().manual_seed(1)).cuda()
    out = torch.full_like(z, float("nan"))
    two = torch.full((N,), 2.0, device="cuda")
    far = torch.full((N, 4), 1 << 30, dtype=torch.int32, device="cuda")   # words out of range, were they read
    kw = {"nothing": {},
          "penalties, L = 0": dict(repeat=two.data_ptr(), presence=two.data_ptr(), frequency=two.data_ptr()),
          "past alone": dict(past=far.data_ptr(), L=4),
          "words, K = 0": dict(extra_word=far.data_ptr()),
          "M alone": dict(M=5),
          "biases, K = 0": dict(extra=two.data_ptr())}[kind]
    torch.cuda.synchronize()
    r = B.cavs_rules(**{**dict(z_type=0, out_type=0, n=N, C=C), **kw})
    assert B.lib().cavs_adjust_logits(ctx._h, ct.byref(r), z.data_ptr(), out.data_ptr(), None, None, None, 0) == B.OK
    ctx.sync()   # would say that a word was out of range
    assert torch.equal(out, z)
