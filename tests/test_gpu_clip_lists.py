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


FAR, NEAR = "k_clip_scale<far>", "k_clip_scale"


@pytest.mark.parametrize("sizes,out,want", [
    ([10] * 4000, True, [NEAR]),               # 4000 chunks of ten elements
    ([10] * 4097, True, [NEAR] * 2),           # a second table
    ([1 << 22] * 2, True, [FAR]), ([(1 << 23) - 4, 3], True, [NEAR]), ([1 << 23], True, [FAR]),
    ([1 << 23] + [1000] * 7, False, [NEAR]),   # the largest one is only counted
])
def test_stores_go_past_the_caches_by_what_is_written(ctx, sizes, out, want):
    src = torch.randn(sum(sizes), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    grads = list(src.split(sizes))
    dst = torch.full((sum(sizes),), float("nan"), dtype=BF16, device="cuda")
    outs = list(dst.split(sizes))
    if not out:
        outs[0] = None
    norm, ws = torch.empty(1, device="cuda"), torch.empty(B.clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.timing(True)
    B.clip_grads(ctx, B.GradList(grads, outs), 1.0, norm, ws)
    names = [r[0] for r in ctx.timing_read()]
    ctx.timing(False)
    assert [n for n in names if n.startswith(NEAR)] == want
    true, nb, [(w, b)] = R.clip([src], 1.0, 1.0, [BF16])
    skip = 0 if out else sizes[0]
    assert abs(float(norm) - true) <= nb and R.outside(dst[skip:], w[skip:], b[skip:]) <= 1.0
    assert torch.isnan(dst[:skip]).all()
