"""The vocabulary head's gradients at sizes past 2^32 of something: words that
are cleared, terms of a sum."""
import pytest
import torch

from paper_1712_04048_amd import binding as B

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
