"""The head in 4 bits on the GPU against its 64-bit form, its data against the
header's words."""
import math

import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
FORMS = [(128, False), (64, False), (32, False), (128, True), (64, True), (32, True)]


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _weights(g, H, C, dtype):
    W = torch.randn(H, C, generator=g) * (0.01 + torch.rand(C, generator=g))
    return W.to(dtype).cuda()


def _packed(ctx, W, group, shift):
    H, C = W.shape
    data = torch.full((B.quant_bytes(H, C, group, shift),), 0xa5, dtype=torch.uint8, device="cuda")
    q = B.QuantWeights(data, H, C, group, shift)
    B.quant_pack(ctx, q, W)
    return q


@pytest.mark.parametrize("group,shift", FORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,C", [(1, 1), (7, 3), (128, 16), (129, 17), (64, 100), (300, 85), (512, 1000),
                                 (96, 63), (160, 65), (1000, 33)])
def test_codes_and_scales(ctx, H, C, dtype, group, shift):
    """Bit for bit, each place where the header puts it, zeros past the ends."""
    W = _weights(torch.Generator().manual_seed(H * C + group), H, C, dtype)
    q = _packed(ctx, W, group, shift)
    ctx.sync()
    code, s, m = R.from_data(q.data, H, C, group, shift)
    want = [t.cpu() for t in R.quantise(W, group, shift)]
    groups = want[1].shape[0]
    assert torch.equal(code[:H, :C], want[0])
    assert torch.equal(s[:groups, :C], want[1]) and torch.equal(m[:groups, :C], want[2])
    assert not code[H:].any() and not code[:, C:].any() and not s[:, C:].any() and not m[:, C:].any()
    assert not s[groups:].any() and not m[groups:].any()
    for out in (F32, BF16):
        back = torch.full((H, C), float("nan"), dtype=out, device="cuda")
        B.quant_unpack(ctx, q, back)
        ctx.sync()
        assert torch.equal(back.cpu(), R.weights(*want, group).float().to(out))


@pytest.mark.parametrize("shift", [False, True])
def test_weights_half_way_between_two_codes(ctx, shift):
    """Weights that are whole and half steps of a scale that is a power of two, and
    their neighbours: the even code where it is half way."""
    step = torch.arange(-16, 15, dtype=torch.float64) / 2
    w = torch.cat([step, step * (1 + 2.0 ** -23), step * (1 - 2.0 ** -24), step + 2.0 ** -20])
    W = torch.zeros(128, 5)
    W[:w.numel(), :] = w.float()[:, None] * torch.tensor([1.0, 2.0 ** -20, 2.0 ** 30, -1.0, 0.5])
    W[w.numel(), :] = -8 * torch.tensor([1.0, 2.0 ** -20, 2.0 ** 30, -1.0, 0.5])
    W = W.cuda()
    q = _packed(ctx, W, 128, shift)
    ctx.sync()
    code, s, m = R.from_data(q.data, 128, 5, 128, shift)
    want = [t.cpu() for t in R.quantise(W, 128, shift)]
    assert torch.equal(s[:, :5], want[1]) and torch.equal(code[:, :5], want[0]) and torch.equal(m[:, :5], want[2])


def test_odd_groups_of_weights(ctx):
    """Zeros, one value, the smallest and largest floats, infinities and NaN."""
    big, tiny = torch.finfo(F32).max, 2.0 ** -149
    cols = [0.0, 3.0, -3.0, big, -big, tiny, 2.0 ** -126, 1e-42, 1e30, 2.0 ** -130]
    for shift in (False, True):
        W = torch.randn(64, len(cols) + 3, generator=torch.Generator().manual_seed(1))
        for c, v in enumerate(cols):
            W[:, c] = v
            W[::3, c] = -v / 3
        W[5, len(cols)], W[40, len(cols) + 1], W[9, len(cols) + 2] = math.inf, math.nan, -math.inf
        W = W.cuda()
        for group in (32, 64, 128):
            q = _packed(ctx, W, group, shift)
            ctx.sync()
            code, s, m = R.from_data(q.data, *W.shape, group, shift)
            want = [t.cpu() for t in R.quantise(W, group, shift)]
            n, C = want[1].shape
            assert torch.equal(torch.isnan(s[:n, :C]), torch.isnan(want[1]))
            assert torch.equal(s[:n, :C].nan_to_num(7.0), want[1].nan_to_num(7.0))
            assert torch.equal(m[:n, :C], want[2]) and torch.equal(code[:64, :C], want[0])


@pytest.mark.parametrize("group,shift", FORMS)
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,H,C", [(1, 1, 1), (1, 64, 100), (2, 128, 16), (3, 129, 17), (1, 512, 1000), (16, 300, 333),
                                   (17, 256, 85), (33, 200, 50), (64, 512, 777), (65, 70, 40), (5, 1100, 65)])
def test_product(ctx, n, H, C, types, group, shift):
    g = torch.Generator().manual_seed(n * H + C)
    W = _weights(g, H, C, types[0])
    x = torch.tanh(1.5 * torch.randn(n, H, generator=g)).to(types[0]).cuda()
    bias = torch.randn(C, generator=g).cuda() if (n + C) % 2 else None
    q = _packed(ctx, W, group, shift)
    want, bound = R.product(x, *R.quantise(W, group, shift), group, bias, types[1] == BF16)
    got = []
    for _ in range(2):
        y = torch.full((n, C), float("nan"), dtype=types[1], device="cuda")
        B.quant_product(ctx, q, x, y, bias=bias)
        ctx.sync()
        got.append(y)
    assert R.outside(got[0], want, bound) <= 1.0
    assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,H,C", [(16, 4096, 300), (64, 2100, 100), (64, 4096, 64), (20, 9000, 33), (200, 700, 2000),
                                   (1, 32768, 40), (1, 2048, 40000), (7, 1024, 33333), (64, 640, 33000)])
def test_long_products(ctx, n, H, C, dtype):
    """Rows that take several turns through LDS, words for every workgroup and more."""
    g = torch.Generator(device="cuda").manual_seed(n + H + C)
    W = (torch.randn(H, C, generator=g, device="cuda") / math.sqrt(H)).to(dtype)
    x = torch.randn(n, H, generator=g, device="cuda").to(dtype)
    for group, shift in ((128, False), (32, True)):
        q = _packed(ctx, W, group, shift)
        y = torch.full((n, C), float("nan"), device="cuda")
        B.quant_product(ctx, q, x, y)
        ctx.sync()
        want, bound = R.product(x, *R.quantise(W, group, shift), group, None, False)
        assert R.outside(y, want, bound) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_very_different_magnitudes(ctx, dtype):
    """Large and small values in one block, whole rows near both ends of the type."""
    g = torch.Generator().manual_seed(4)
    W = _weights(g, 256, 40, F32)
    W[::2] = 0.0   # words read only every other place
    x = torch.randn(6, 256, generator=g)
    x[0, ::2] *= 2.0 ** 30
    x[1] *= torch.exp2(torch.randint(-40, 40, (256,), generator=g).float())
    x[2] *= 2.0 ** 100
    x[3] *= 2.0 ** -110
    x[4] = 0.0
    x[5, :128] = 0.0
    x = x.to(dtype).cuda()
    W = W.cuda()
    q = _packed(ctx, W, 64, False)
    y = torch.empty(6, 40, device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    want, bound = R.product(x, *R.quantise(W, 64, False), 64, None, False)
    assert R.outside(y, want, bound) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [False, True])
def test_the_largest_and_smallest_values_of_x(ctx, dtype, shift):
    """Just below 2^115, all codes -8 and of one sign, so that a group's sum is the
    largest there is; and 2^-112."""
    W = torch.full((256, 20), 0.125)
    W[::2, 10:] = -0.125
    x = torch.full((2, 256), 2.0 ** 115 * (1 - 2.0 ** -8))
    x[1] = 2.0 ** -112
    x, W = x.to(dtype).cuda(), W.cuda()
    q = _packed(ctx, W, 128, shift)
    y = torch.empty(2, 20, device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    want, bound = R.product(x, *R.quantise(W, 128, shift), 128, None, False)
    assert R.outside(y, want, bound) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [3, 40])
def test_rows_that_are_not_finite_stay_alone(ctx, dtype, n):
    g = torch.Generator().manual_seed(5)
    W = _weights(g, 200, 70, dtype)
    x = torch.randn(n, 200, generator=g)
    want, bound = R.product(x.to(dtype), *[t.cpu() for t in R.quantise(W, 128, True)], 128, None, False)
    x[0, 3], x[2, 150] = math.inf, math.nan
    q = _packed(ctx, W, 128, True)
    y = torch.empty(n, 70, device="cuda")
    B.quant_product(ctx, q, x.to(dtype).cuda(), y)
    ctx.sync()
    assert not torch.isfinite(y[0]).any() and torch.isnan(y[2]).all()
    rest = [i for i in range(n) if i not in (0, 2)]
    assert R.outside(y[rest].cpu(), want[rest], bound[rest]) <= 1.0


def test_a_word_without_finite_weights_stays_alone(ctx):
    g = torch.Generator().manual_seed(6)
    W = _weights(g, 200, 70, F32)
    x = torch.randn(4, 200, generator=g).cuda()
    W[3, 11] = math.nan
    q = _packed(ctx, W, 128, False)
    y = torch.empty(4, 70, device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    want, bound = R.product(x, *R.quantise(W, 128, False), 128, None, False)
    assert torch.isnan(y[:, 11]).all()
    assert R.outside(y, want, bound) <= 1.0


def test_tensors_inside_an_allocation(ctx):
    """x, y, W and bias that begin at any element; what lies beside y stays."""
    g = torch.Generator().manual_seed(7)
    for t in (F32, BF16):
        for off in (1, 2, 3):
            W = torch.empty(100 * 37 + off, dtype=t, device="cuda")[off:].view(100, 37)
            W.copy_(_weights(g, 100, 37, t))
            x = torch.empty(5 * 100 + off, dtype=t, device="cuda")[off:].view(5, 100)
            x.copy_(torch.randn(5, 100, generator=g))
            bias = torch.randn(37 + off, generator=g).cuda()[off:]
            room = torch.full((5 * 37 + off + 9,), 3.0, dtype=t, device="cuda")
            y = room[off:off + 5 * 37].view(5, 37)
            q = _packed(ctx, W, 64, True)
            B.quant_product(ctx, q, x, y, bias=bias)
            ctx.sync()
            want, bound = R.product(x, *R.quantise(W, 64, True), 64, bias, t == BF16)
            assert R.outside(y, want, bound) <= 1.0
            assert (room[:off] == 3.0).all() and (room[off + 5 * 37:] == 3.0).all()
            back = torch.full((100 * 37 + off + 9,), 3.0, dtype=t, device="cuda")
            B.quant_unpack(ctx, q, back[off:off + 3700].view(100, 37))
            ctx.sync()
            assert (back[:off] == 3.0).all() and (back[off + 3700:] == 3.0).all()


def test_no_rows(ctx):
    q = _packed(ctx, torch.randn(64, 20, device="cuda"), 64, False)
    B.quant_product(ctx, q, torch.empty(0, 64, device="cuda"), torch.empty(0, 20, device="cuda"))
    ctx.sync()


def test_many_rows(ctx):
    """More rows than the call is made for, each computed as it is alone."""
    g = torch.Generator(device="cuda").manual_seed(8)
    W = torch.randn(64, 48, generator=g, device="cuda")
    x = torch.randn(70000, 64, generator=g, device="cuda")
    q = _packed(ctx, W, 64, False)
    y = torch.full((70000, 48), float("nan"), device="cuda")
    B.quant_product(ctx, q, x, y)
    ctx.sync()
    want, bound = R.product(x, *R.quantise(W, 64, False), 64, None, False)
    assert R.outside(y, want, bound) <= 1.0
