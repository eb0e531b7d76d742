"""The vocabulary head's gradients at sizes past 2^32 of something: words that
are cleared, terms of a sum."""
import math

import pytest
import torch

import lm_ref as R
from paper_1712_04048_amd import binding as B
from test_gpu_vocab import check, grad, loss, make, reference

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


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


def test_no_row_clears_every_gradient(ctx):
    """16 GB of dW_s: 2^32 words and some, more than a launch has threads."""
    H, C = 1 << 15, (1 << 18) + 6
    assert H * C * 2 // 4 > 2 ** 32
    W, dW = (torch.empty(H, C, dtype=BF16, device="cuda") for _ in range(2))
    dW.fill_(3.0)
    bs, dbs = torch.zeros(C, device="cuda"), torch.full((C,), 3.0, device="cuda")
    head = B.VocabHead(h=torch.empty(0, H, device="cuda"), Ws=W, bs=bs,
                       label=torch.empty(0, dtype=torch.int32, device="cuda"))
    loss = torch.full((1,), 3.0, device="cuda")
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    B.vocab_grad(ctx, head, loss, None, torch.empty_like(head.h), dW, dbs, none)
    ctx.sync()
    assert float(loss) == 0.0 and int(torch.count_nonzero(dbs)) == 0
    assert sum(int(torch.count_nonzero(part)) for part in dW.split(1 << 12)) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [70, 2100])
def test_weight_gradient_of_a_million_rows(ctx, dtype, C):
    """dW_s and dbs summed over 2^20 rows of 2^31 states, exactly but for their last
    roundings, z kept (70 words) and formed again for two pieces (2 100).

    W_s = 0 and 64 words that the bias does not mask: p = 1/64 and dz = 1/64 or
    -63/64, which bf16 holds; states of +-1 by the row's word.  Every partial sum is
    a multiple of 1/64 below 2^18, so fp32 adds them exactly in any order.  Then
    comes unit / rows (a rounding), its product (another) and the store."""
    n, H = 1 << 20, 2112
    assert n * H > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(C)
    words = (torch.arange(64, device="cuda") * ((C - 1) // 63)).int()
    bs = torch.full((C,), -math.inf, device="cuda")
    bs[words.long()] = 0.0
    kind = torch.randint(0, 64, (n,), generator=g, device="cuda")
    sign = (torch.randint(0, 2, (64, H), generator=g, device="cuda") * 2 - 1).to(dtype)
    h = sign[kind]
    y = words[kind]
    y[: n // 2: 3] = -1
    head = B.VocabHead(h=h, Ws=torch.zeros(H, C, dtype=dtype, device="cuda"), bs=bs, label=y)
    loss, dh = torch.empty(1, device="cuda"), torch.empty_like(h)
    dW, dbs = torch.empty_like(head.Ws), torch.empty_like(bs)
    ws = torch.empty(B.vocab_workspace_bytes(head, True), dtype=torch.uint8, device="cuda")
    B.vocab_grad(ctx, head, loss, None, dh, dW, dbs, ws)
    ctx.sync()
    on = y >= 0
    live = int(on.sum())

    def sums(rows):
        """sum of h_i dz_i and of dz_i over some rows, [H, 64] and [64]"""
        count = torch.bincount(kind[rows], minlength=64).double()
        own = count[:, None] * sign.double()     # by word, the states of its rows
        return own.sum(0)[:, None] / 64 - own.t(), count.sum() / 64 - count

    total, db = sums(on)
    assert float(torch.bincount(kind[on]).max()) + live / 64 < 2 ** 18
    rounding = 3 * R.U + (R.BF if dtype == BF16 else 0.0)

    def spread(t):
        out = torch.zeros(*t.shape[:-1], C, dtype=torch.float64, device="cuda")
        out[..., words.long()] = t / live
        return out

    want, bound = spread(total), spread(total).abs() * rounding
    assert R.outside(dW, want, bound) <= 1.0
    assert R.outside(dbs, spread(db), spread(db).abs() * 3 * R.U) <= 1.0
    assert int(torch.count_nonzero(dh)) == 0
    assert abs(float(loss) - math.log(64)) <= 8 * R.U * math.log(64)
    # rows that were left out would be seen: one in fp32, in bf16 some hundredth of them
    part = 1 if dtype == F32 else 1 << 14
    for at in (1, n // 2, n - part):
        left = on.clone()
        left[at: at + part] = False
        assert R.outside(spread(sums(left)[0]), want, bound) > 1.0
    assert R.outside(torch.zeros_like(dW), want, bound) > 1.0


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("n,C,K", [(1, 3, 0), (70, 300, 4), (300, 2001, 0), (600, 33000, 3)])
def test_largest_width_of_the_states(ctx, types, n, C, K):
    """H = 2^15, on tiles of every size."""
    head = make(n, n, C, 1 << 15, types, pad=0.1 if n > 1 else 0.0, K=K, alpha=0.5, temp=2.0 if K else 1.0)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
    alone = loss(ctx, head)
    ctx.sync()
    assert torch.equal(alone["loss"], got["loss"])


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_many_pieces(ctx, types):
    """Seven (fp32) and four pieces of the vocabulary, the halves of dz in turn, the last
    one narrower."""
    head = make(7, 40000, 12301, 64, types, pad=0.1)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
