"""The embedding and its gradient on the GPU against their 64-bit forms."""
import pytest
import torch

import lm_ref as R
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


def _words(g, n, C, kind):
    if kind == "one":
        return torch.full((n,), C // 2, dtype=torch.int32)
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int32)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    w = (u * C).long() if kind == "even" else (C ** u - 1).long()
    w = torch.where(torch.rand(n, generator=g) < 0.05, -1, w.clamp(max=C - 1))
    return w.int()


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,C,D", [(1, 1, 1), (5, 3, 3), (17, 40, 64), (300, 7, 300), (1000, 5000, 85),
                                   (64, 100, 1028), (2, 3, 8)])
def test_rows(ctx, types, n, C, D):
    """scale E rounded once: a fp32 product, so equal bit for bit to torch's."""
    g = torch.Generator().manual_seed(n * C + D)
    E = torch.randn(C, D, generator=g).to(types[0]).cuda()
    word = _words(g, n, C, "skew").cuda()
    X = torch.full((n, D), float("nan"), dtype=types[1], device="cuda")
    B.embed(ctx, B.Embedding(E, 3.3), word, X)
    ctx.sync()
    s = torch.tensor(3.3, dtype=F32)
    want = torch.where((word >= 0)[:, None], E.float()[word.clamp(min=0).long()] * s.cuda(), 0.0)
    assert torch.equal(X, want.to(types[1]))


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,C,D,kind", [
    (1, 1, 1, "even"), (3, 5, 7, "even"), (32, 4, 64, "one"), (33, 4, 64, "one"), (65, 1, 12, "one"),
    (64, 2000, 8, "none"), (5000, 9, 40, "one"), (4867, 2000, 300, "skew"), (2000, 513, 85, "skew"),
    (3000, 33000, 16, "even"), (20000, 300, 520, "skew"), (100, 130, 1024, "even")])
def test_table_gradient(ctx, types, n, C, D, kind):
    g = torch.Generator().manual_seed(n + C + D)
    word = _words(g, n, C, kind).cuda()
    dX = torch.randn(n, D, generator=g).to(types[1]).cuda()
    emb = B.Embedding(torch.empty(C, D, dtype=types[0], device="cuda"), 0.7)
    ws = torch.full((B.embed_grad_workspace_bytes(emb, n),), 255, dtype=torch.uint8, device="cuda")
    got = []
    for _ in range(2):
        dE = torch.full((C, D), float("nan"), dtype=types[0], device="cuda")
        B.embed_grad(ctx, emb, word, dX, dE, ws)
        ctx.sync()
        got.append(dE)
    scale = float(torch.tensor(0.7, dtype=F32))
    want, bound = R.embed_grad(word, dX, C, scale, types[0] == BF16)
    assert R.outside(got[0], want, bound) <= 1.0
    assert torch.equal(got[0], got[1])


def test_unaligned_tables_and_rows(ctx):
    """Tensors that begin inside an allocation, at any element."""
    g = torch.Generator().manual_seed(0)
    word = _words(g, 70, 9, "even").cuda()
    for t in (F32, BF16):
        for off in (1, 2, 3, 4):
            E = torch.randn(9 * 16 + off, generator=g).to(t).cuda()[off:].view(9, 16)
            X = torch.zeros(70 * 16 + off, dtype=t, device="cuda")[off:].view(70, 16)
            B.embed(ctx, B.Embedding(E), word, X)
            ctx.sync()
            assert torch.equal(X, R.embed(E, word, 1.0).to(t))
            dE = torch.zeros(9 * 16 + off, dtype=t, device="cuda")[off:].view(9, 16)
            emb = B.Embedding(E)
            ws = torch.empty(B.embed_grad_workspace_bytes(emb, 70), dtype=torch.uint8, device="cuda")
            B.embed_grad(ctx, emb, word, X, dE, ws)
            ctx.sync()
            want, bound = R.embed_grad(word, X, 9, 1.0, t == BF16)
            assert R.outside(dE, want, bound) <= 1.0


def test_no_words(ctx):
    emb = B.Embedding(torch.randn(6, 10, device="cuda"))
    word = torch.empty(0, dtype=torch.int32, device="cuda")
    X = torch.empty(0, 10, device="cuda")
    B.embed(ctx, emb, word, X)
    dE = torch.full((6, 10), 5.0, device="cuda")
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, 0), dtype=torch.uint8, device="cuda")
    B.embed_grad(ctx, emb, word, X, dE, ws)
    ctx.sync()
    assert float(dE.abs().max()) == 0.0


def test_words_out_of_range_are_reported_and_read_nothing(ctx):
    emb = B.Embedding(torch.randn(6, 8, device="cuda"))
    for bad in (6, -2, 2 ** 31 - 1, -2 ** 31):
        word = torch.tensor([1, bad, 5], dtype=torch.int32, device="cuda")
        X = torch.empty(3, 8, device="cuda")
        B.embed(ctx, emb, word, X)
        with pytest.raises(B.CavsError) as e:
            ctx.sync()
        assert e.value.status == B.ERR_RANGE
        ctx.sync()   # the report clears it
        assert torch.equal(X, emb.E[[1, 0, 5]] * torch.tensor([1.0, 0.0, 1.0], device="cuda")[:, None])
        dE = torch.empty(6, 8, device="cuda")
        ws = torch.empty(B.embed_grad_workspace_bytes(emb, 3), dtype=torch.uint8, device="cuda")
        B.embed_grad(ctx, emb, word, torch.ones(3, 8, device="cuda"), dE, ws)
        with pytest.raises(B.CavsError) as e:
            ctx.sync()
        assert e.value.status == B.ERR_RANGE
        assert dE.sum(1).tolist() == [0, 8, 0, 0, 0, 8]


def test_nonfinite_rows_stay_in_their_word(ctx):
    emb = B.Embedding(torch.zeros(40, 8, device="cuda"))
    word = torch.arange(40, dtype=torch.int32, device="cuda").repeat(3)
    dX = torch.ones(120, 8, device="cuda")
    dX[5], dX[47] = float("nan"), float("inf")
    dE = torch.empty(40, 8, device="cuda")
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, 120), dtype=torch.uint8, device="cuda")
    B.embed_grad(ctx, emb, word, dX, dE, ws)
    ctx.sync()
    want = torch.full((40, 8), 3.0, device="cuda")
    want[5], want[7] = float("nan"), float("inf")
    assert torch.equal(dE.nan_to_num(7.0), want.nan_to_num(7.0))


def test_refusals(ctx):
    emb = B.Embedding(torch.zeros(5, 8, device="cuda"))
    word = torch.zeros(4, dtype=torch.int32, device="cuda")
    X, dE = torch.zeros(4, 8, device="cuda"), torch.zeros(5, 8, device="cuda")
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, 4), dtype=torch.uint8, device="cuda")
    calls = [
        (lambda: B.embed(ctx, emb, word.long(), X), B.ERR_ARG),
        (lambda: B.embed(ctx, emb, word, X[:3]), B.ERR_ARG),
        (lambda: B.embed(ctx, emb, word.cpu(), X), B.ERR_ARG),
        (lambda: B.embed(ctx, B.Embedding(emb.E.cpu()), word, X), B.ERR_ARG),
        (lambda: B.embed_grad(ctx, emb, word, X, dE[:4], ws), B.ERR_ARG),
        (lambda: B.embed_grad(ctx, emb, word, X, dE.bfloat16(), ws), B.ERR_ARG),
        (lambda: B.embed_grad(ctx, emb, word, X, dE, ws[:-1]), B.ERR_WORKSPACE),
        (lambda: B.embed_grad(ctx, emb, word, X, dE, ws.float()), B.ERR_ARG),
    ]
    for call, status in calls:
        with pytest.raises(B.CavsError) as e:
            call()
        assert e.value.status == status


def test_replays_of_a_captured_gradient(ctx):
    """Captured on its own stream, replayed with other words between eager calls."""
    g = torch.Generator().manual_seed(1)
    C, D, n = 300, 64, 1500
    emb = B.Embedding(torch.randn(C, D, generator=g).cuda(), 2.0)
    word = _words(g, n, C, "skew").cuda()
    X, dX = torch.empty(n, D, device="cuda"), torch.randn(n, D, generator=g).cuda()
    dE = torch.empty(C, D, device="cuda")
    ws = torch.empty(B.embed_grad_workspace_bytes(emb, n), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    own = B.Context(0, s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        B.embed(own, emb, word, X)
        B.embed_grad(own, emb, word, dX, dE, ws)
    ws2, dE2, X2 = torch.empty_like(ws), torch.empty_like(dE), torch.empty_like(X)
    for _ in range(3):
        word.copy_(_words(g, n, C, "skew"))
        torch.cuda.synchronize()
        graph.replay()
        B.embed(ctx, emb, word, X2)
        B.embed_grad(ctx, emb, word, dX, dE2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(X, X2) and torch.equal(dE, dE2)
    own.sync()
    own.close()
