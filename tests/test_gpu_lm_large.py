"""Rows past 2^31 elements: the vocabulary head's states and gradients, the
embedding's table."""
import pytest
import torch

import lm_ref as R
from paper_1712_04048_amd import binding as B

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def test_head_rows(ctx):
    n, H, C = 1 << 20, 2112, 70
    assert n * H > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(0)
    h = torch.empty(n, H, dtype=BF16, device="cuda")
    h.normal_(generator=g)
    W = (torch.randn(H, C, generator=g, device="cuda", dtype=torch.float32) / 46).to(BF16)
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    y[: n // 2: 3] = -1
    head = B.VocabHead(h=h, Ws=W, label=y)
    f = dict(dtype=torch.float32, device="cuda")
    loss, row, dh, dW = torch.empty(1, **f), torch.empty(n, **f), torch.empty_like(h), torch.empty_like(W)
    ws = torch.empty(B.vocab_workspace_bytes(head, True), dtype=torch.uint8, device="cuda")
    B.vocab_grad(ctx, head, loss, row, dh, dW, None, ws)
    ctx.sync()
    live = int((y >= 0).sum())
    at = torch.cat([torch.arange(40), torch.arange(n - 300, n)]).cuda()
    want, bound = R.head(h[at], W, None, y[at])
    assert R.outside(row[at], want["row_loss"], bound["row_loss"]) <= 1.0
    # of the mean over every row the gradient is the sample's, rescaled
    part = int((y[at] >= 0).sum()) / live
    assert R.outside(dh[at], want["dh"] * part, bound["dh"] * part + R.BF * want["dh"].abs() * part) <= 1.0
    assert float(dh[: n // 2: 3].abs().max()) == 0.0
    mean = float(row.double().sum() / live)
    assert abs(float(loss) - mean) <= 2 * R.U * abs(mean)
    # dW_s over half a million rows: the sum of blocks' references
    total, lim = torch.zeros(H, C, dtype=torch.float64, device="cuda"), torch.zeros(H, C, dtype=torch.float64, device="cuda")
    for part_rows in torch.arange(n, device="cuda").split(1 << 16):
        k = int((y[part_rows] >= 0).sum())
        w, b = R.head(h[part_rows], W, None, y[part_rows])
        total += w["dWs"] * k / live
        # the blocks' bounds, and the additions over every row in place of a block's
        lim += (b["dWs"] + 2 * n * R.U * 4 * w["dWs"].abs()) * k / live
    scale = float(h.float().abs().mean()) * 2.0   # sum of |h| |dz| per row and word, at most
    lim += 2 * n * R.U * scale / C + R.BF * total.abs()
    assert R.outside(dW, total, lim) <= 1.0


def test_table(ctx):
    C, D = 1_100_000, 2048
    assert C * D > 2 ** 31
    E = torch.zeros(C, D, dtype=BF16, device="cuda")
    word = torch.tensor([0, C - 1, C - 2, 5, C - 1], dtype=torch.int32, device="cuda")
    E[word.long()] = torch.randn(5, D, device="cuda", dtype=torch.float32).to(BF16)
    X = torch.empty(5, D, dtype=BF16, device="cuda")
    emb = B.Embedding(E, 2.0)
    B.embed(ctx, emb, word, X)
    ctx.sync()
    assert torch.equal(X, E[word.long()] * 2)
    dE = torch.full_like(E, 3.0)
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, 5), dtype=torch.uint8, device="cuda")
    B.embed_grad(ctx, emb, word, X, dE, ws)
    ctx.sync()
    seen = torch.zeros(C, dtype=torch.bool, device="cuda")
    seen[word.long()] = True
    assert torch.equal(dE[0], X[0] * 2) and torch.equal(dE[C - 2], X[2] * 2)
    assert torch.equal(dE[C - 1], ((X[1].float() + X[4].float()) * 2).to(BF16))
    assert int((dE != 0).any(1).sum()) == int(seen.sum())


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_loss_of_more_tiles_than_a_launch_has_threads(ctx, dtype):
    n, H, C = 1 << 20, 64, (1 << 18) + 300
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(n, H, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    W = (torch.randn(H, C, generator=g, device="cuda", dtype=torch.float32) / 8).to(dtype)
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    head = B.VocabHead(h=h, Ws=W, label=y)
    loss, row = (torch.empty(k, dtype=torch.float32, device="cuda") for k in (1, n))
    ws = torch.empty(B.vocab_workspace_bytes(head, False), dtype=torch.uint8, device="cuda")
    B.vocab_loss(ctx, head, loss, row, ws)
    ctx.sync()
    at = torch.cat([torch.arange(100), torch.arange(n - 100, n)]).cuda()
    want, bound = R.head(h[at], W, None, y[at])
    assert R.outside(row[at], want["row_loss"], bound["row_loss"]) <= 1.0
    mean = float(row.double().mean())
    assert abs(float(loss) - mean) <= 2 * R.U * abs(mean)


def test_table_of_more_blocks_than_a_launch_has_threads(ctx):
    """Rows of an odd length, so a block of 64 values to a wavefront."""
    C, D = (1 << 21) + 5, 16383
    word = torch.tensor([0, C - 1, C - 2, 5, C - 1], dtype=torch.int32, device="cuda")
    dX = torch.randn(5, D, device="cuda", dtype=torch.float32).to(BF16)
    dE = torch.full((C, D), 3.0, dtype=BF16, device="cuda")
    emb = B.Embedding(dE, 1.0)   # its size and type; the table itself is not read
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, 5), dtype=torch.uint8, device="cuda")
    B.embed_grad(ctx, emb, word, dX, dE, ws)
    ctx.sync()
    assert torch.equal(dE[0], dX[0]) and torch.equal(dE[5], dX[3]) and torch.equal(dE[C - 2], dX[2])
    assert torch.equal(dE[C - 1], (dX[1].float() + dX[4].float()).to(BF16))
    assert sum(int((part != 0).any(1).sum()) for part in dE.split(1 << 16)) == 4
