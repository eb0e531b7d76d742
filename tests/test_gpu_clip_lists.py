"""Clipping of lists of gradients on the GPU: which norms clip, and which stores they
take."""
import math

import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B
from test_gpu_clip import _call, _float32_by_default, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("v,scale", [(3e38, 1.0), (1e30, 1e30), (1e30, -1e30), (3e38, 3e38)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_norm_beyond_fp32_clips(ctx, v, scale, dtype):
    """Written as infinity, by the gradients or by scale; an infinite gradient beside
    them, whose norm reads the same, leaves them unclipped."""
    x = (v * (1 - torch.rand(5000, generator=torch.Generator().manual_seed(1)) / 2)).to(dtype).cuda()
    y = torch.empty_like(x)
    want, _, [(w, b)] = R.clip([x], scale, 2.0, [dtype])
    assert want > torch.finfo(F32).max
    assert float(_call(ctx, [x], 2.0, [y], scale)) == math.inf
    assert R.outside(y, w, b) <= 1.0
    if scale == 1.0:
        bad = torch.full((3,), math.inf, dtype=dtype, device="cuda")
        assert float(_call(ctx, [x, bad], 2.0, [y, bad.clone()], scale)) == math.inf
        assert torch.equal(y, x)
