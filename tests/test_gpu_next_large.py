"""Rows, weights and gradients past 2^31 and 2^32 elements; the largest sizes."""
import math

import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)
    torch.cuda.empty_cache()


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _fill(shape, seed):
    return torch.empty(shape, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(seed))


def test_weights_past_2_32(ctx):
    """W [2^15, 2^17 + 5]: the largest H; columns at both ends and in the middle."""
    H, C = 1 << 15, (1 << 17) + 5
    W = _fill((H, C), 1)
    q = B.QuantWeights(torch.empty(B.quant_bytes(H, C, 64, True), dtype=torch.uint8, device="cuda"), H, C, 64, True)
    B.quant_pack(ctx, q, W)
    x = torch.tanh(_fill((3, H), 2))
    y = torch.full((3, C), float("nan"), device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    for at in (0, 65530, C - 40):
        part = W[:, at:at + 40]
        w, b = R.product(x, *R.quantise(part, 64, True), 64, None, False)
        assert R.outside(y[:, at:at + 40], w, b) <= 1.0
    back = W.zero_()
    B.quant_unpack(ctx, q, back)
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    w = x.double() @ back[:, C - 300:].double()
    # the weights rounded to bf16 once more
    bound = (2 * H + 16) * R.U * (x.double().abs() @ back[:, C - 300:].double().abs()) + R.BF * (
        x.double().abs() @ back[:, C - 300:].double().abs())
    assert R.outside(y[:, C - 300:], w, bound) <= 1.0


@pytest.mark.parametrize("H", [64, 2000])
def test_the_most_rows(ctx, H):
    """2^20 rows, in groups of 32 and of 16; the first, the last and those between."""
    n, C = 1 << 20, 21
    x = _fill((n, H), 4)
    W = torch.randn(H, C, generator=torch.Generator("cuda").manual_seed(5), device="cuda")
    q = B.QuantWeights(torch.empty(B.quant_bytes(H, C, 64), dtype=torch.uint8, device="cuda"), H, C, 64)
    B.quant_pack(ctx, q, W)
    y = torch.full((n, C), float("nan"), device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    assert not torch.isnan(y).any()
    for at in (0, (1 << 19) - 40, n - 80):
        w, b = R.product(x[at:at + 80], *R.quantise(W, 64, False), 64, None, False)
        assert R.outside(y[at:at + 80], w, b) <= 1.0


def test_logits_past_2_32(ctx):
    """4100 rows of 2^20 words: scored and adjusted, rows on both sides looked at."""
    H, C, n = 32, 1 << 20, 4100
    g = torch.Generator("cuda").manual_seed(3)
    W = torch.randn(H, C, generator=g, device="cuda")
    x = torch.randn(n, H, generator=g, device="cuda")
    q = B.QuantWeights(torch.empty(B.quant_bytes(H, C, 32), dtype=torch.uint8, device="cuda"), H, C, 32)
    B.quant_pack(ctx, q, W)
    z = torch.full((n, C), float("nan"), dtype=BF16, device="cuda")
    B.quant_product(ctx, q, x, z)
    past = torch.randint(0, C, (n, 7), generator=g, device="cuda").int()
    rules = dict(past=past, frequency=torch.full((n,), 0.5, device="cuda"))
    best = torch.empty(n, dtype=torch.int32, device="cuda")
    lse = torch.empty(n, device="cuda")
    ws = torch.empty(B.adjust_workspace_bytes(n, C), dtype=torch.uint8, device="cuda")
    ctx.sync()
    rows = [0, 2047, 2048, 4095, 4096, n - 1]
    w, b = R.product(x[rows], *R.quantise(W, 32, False), 32, None, True)
    assert R.outside(z[rows], w, b) <= 1.0
    before = z[rows].clone()
    B.adjust_logits(ctx, B.LogitRules(**rules), z, z, best, lse, ws)
    ctx.sync()
    v, vb = R.rules(before, **{k: t[rows] for k, t in rules.items()})
    assert R.outside(z[rows], v, vb + R.BF * v.abs()) <= 1.0
    top = v.amax(1)
    assert (top - v.gather(1, best[rows].long()[:, None])[:, 0] <= 2 * vb.amax(1)).all()
    # ln sum exp over 2^20 words: 512 segments' parts, 16 in a lane of the join
    want, lb = R.lse(v, vb)
    assert R.outside(lse[rows], want, lb) <= 1.0


@pytest.mark.parametrize("n", [1 << 32, (1 << 32) - 5])
def test_gradients_of_2_32_elements(ctx, n):
    g = torch.full((n,), 2.0 ** -10, dtype=BF16, device="cuda")
    g[-1] = 3.0
    norm = torch.empty(1, device="cuda")
    ws = torch.empty(B.clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    B.clip_grads(ctx, B.GradList([g]), 1.0, norm, ws)
    ctx.sync()
    want = math.sqrt((n - 1) * 2.0 ** -20 + 9.0)
    assert abs(float(norm) - want) <= 2 * R.U * want
    assert float(g[-1]) == pytest.approx(3.0 / want, rel=R.BF)
    first = float(g[0])
    assert first == pytest.approx(2.0 ** -10 / want, rel=R.BF)
    assert int((g[:-1] != first).sum()) == 0
