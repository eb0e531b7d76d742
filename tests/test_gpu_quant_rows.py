"""How exactly the 4-bit product takes its rows, on the GPU: each word has one weight
that is not 0, so that y is x as the product takes it, times that weight.  And the
largest weights."""
import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B
from test_gpu_quant import _float32_by_default, _packed, ctx  # noqa: F401
from test_quant_rows import bound

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [7, 16, 40, 300])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_one_weight_a_word(ctx, n, group, dtype):
    """Within the header's bound for x, and u of y for the sum of the two halves (the
    scale is a power of two, the code -8); bf16 values from 2^-31 of their largest on
    come out as they are."""
    H = 256
    g = torch.Generator().manual_seed(n + group)
    weight = torch.exp2(torch.randint(-9, 10, (H,), generator=g).double())
    q = _packed(ctx, torch.diag(weight).float().cuda(), group, False)
    x = torch.randn(n, H, generator=g) * torch.exp2(-45 * torch.rand(n, H, generator=g))
    x[:, 5::128] = 8 + 7 * torch.rand(n, 2, generator=g)        # each block's largest
    x[0, :128] = 1 + torch.rand(128, generator=g)               # a block of one binade
    x[1, 3], x[1, 9] = 16384 + 4 + 2.0 ** -9, 16384 * (2 - 2.0 ** -20)
    x[2] *= 2.0 ** -100
    x = x.to(dtype)
    y = torch.full((n, H), float("nan"), device="cuda")
    B.quant_product(ctx, q, x.cuda(), y)
    ctx.sync()
    got, x = y.cpu().double() / weight, x.double()
    for i in range(n):
        for at in (0, 128):
            row, mine = x[i, at:at + 128], got[i, at:at + 128]
            top = float(row.abs().max())
            room = torch.from_numpy(bound(row.numpy(), top, dtype)) + R.U * mine.abs()
            assert ((mine - row).abs() <= room).all(), (i, at)
            if dtype == BF16:
                kept = row.abs() >= 2.0 ** -31 * top
                assert torch.equal(mine[kept], row[kept]), (i, at)


@pytest.mark.parametrize("shift", [False, True])
def test_weights_at_the_end_of_fp32(ctx, shift):
    """Below 2^127 they stay finite; the largest floats come out as s and m say, which
    are infinities."""
    big = torch.finfo(F32).max
    under = 2.0 ** 127 * (1 - 2.0 ** -24)
    W = torch.zeros(32, 5)
    W[:, 0], W[:, 1], W[:, 2] = under, big, torch.linspace(0.9 * under, under, 32)
    W[::2, 3], W[1::2, 3] = under, -under
    W[:, 4] = (torch.linspace(-1, 1, 32).double() * big).float()
    W = W.cuda()
    q = _packed(ctx, W, 32, shift)
    want = R.weights(*R.quantise(W, 32, shift), 32).float()
    back = torch.zeros_like(W)
    B.quant_unpack(ctx, q, back)
    ctx.sync()
    assert torch.equal(back, want)
    assert torch.isfinite(back[:, [0, 2, 3]]).all() and torch.isinf(back[:, 1]).all()
