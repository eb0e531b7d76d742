"""The vocabulary head on the GPU against its 64-bit form: cross entropy and
distillation, losses and every gradient, within the bounds of lm_ref."""
import math

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


def make(seed, n, C, H, types=(F32, F32), pad=0.0, K=0, alpha=0.0, temp=1.0, bias=True, mask=0.0,
         sure=3.0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(H, C, generator=g) / math.sqrt(H)).to(types[1])
    y = torch.randint(0, C, (n,), generator=g)
    x = torch.tanh(torch.randn(n, H, generator=g) + sure * torch.rand(n, 1, generator=g) * W[:, y].t().float())
    b = 0.3 * torch.randn(C, generator=g) if bias else None
    if mask:
        off = torch.rand(C, generator=g) < mask
        off[y] = False
        b[off] = -math.inf
    if pad:
        y[torch.rand(n, generator=g) < pad] = -1
    kw = {}
    if K:
        fine = torch.arange(C) if not mask else torch.nonzero(torch.isfinite(b)).flatten()
        word = fine[torch.randint(0, fine.numel(), (n, K), generator=g)]   # repeats among them
        gone = torch.rand(n, K, generator=g) < 0.1
        gone[::7] = True
        word[gone] = -1
        logit = 3 * torch.randn(n, K, generator=g)
        logit[::5, -1] = -math.inf
        kw = dict(top_word=word.int().cuda(), top_logit=logit.cuda(), alpha=alpha, temp=temp)
    return B.VocabHead(h=x.to(types[0]).cuda(), Ws=W.cuda(), bs=b.cuda() if bias else None,
                       label=y.int().cuda(), **kw)


def outputs(head, fill=float("nan")):
    n, H, C = head.h.shape[0], head.h.shape[1], head.Ws.shape[1]
    o = dict(loss=torch.full((1,), fill, device="cuda"), row_loss=torch.full((n,), fill, device="cuda"),
             dh=torch.full((n, H), fill, dtype=head.h.dtype, device="cuda"),
             dWs=torch.full((H, C), fill, dtype=head.Ws.dtype, device="cuda"))
    if head.bs is not None:
        o["dbs"] = torch.full((C,), fill, device="cuda")
    return o


def workspace(head, train):
    """Of ones' bits: a value read before it is written is a NaN."""
    return torch.full((max(1, B.vocab_workspace_bytes(head, train)),), 255, dtype=torch.uint8, device="cuda")


def grad(ctx, head, ws=None, o=None):
    o = o or outputs(head)
    ws = workspace(head, True) if ws is None else ws
    B.vocab_grad(ctx, head, o["loss"], o["row_loss"], o["dh"], o["dWs"], o.get("dbs"), ws)
    return o


def loss(ctx, head):
    o = {k: v for k, v in outputs(head).items() if k in ("loss", "row_loss")}
    B.vocab_loss(ctx, head, o["loss"], o["row_loss"], workspace(head, False))
    return o


def reference(head, **kw):
    return R.head(head.h, head.Ws, head.bs, head.label, head.top_word, head.top_logit, head.alpha,
                  head.temp, **kw)


def check(got, want, bound):
    far = {k: R.outside(got[k], want[k], bound[k]) for k in got}
    assert all(v <= 1.0 for v in far.values()), far


# one row and word to many; few rows, few words, tiles of either size, odd ends
SHAPES = [(1, 1, 64), (1, 17, 64), (3, 100, 128), (64, 1000, 64), (65, 255, 320), (257, 513, 64),
          (300, 2049, 192), (1000, 4100, 128), (17, 20001, 256), (640, 64, 512),
          (40000, 33, 64), (130, 40003, 64), (64, 129, 1088), (2100, 4097, 64)]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("n,C,H", SHAPES)
def test_cross_entropy(ctx, types, n, C, H):
    head = make(n + C, n, C, H, types, pad=0.2 if n > 4 else 0.0, bias=n % 2 == 1)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
    alone = loss(ctx, head)
    ctx.sync()
    check(alone, want, bound)
    assert torch.equal(alone["row_loss"], got["row_loss"]) and torch.equal(alone["loss"], got["loss"])


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,C,H,K,alpha,T", [
    (1, 5, 64, 1, 1.0, 1.0), (40, 300, 64, 3, 0.5, 1.0), (100, 1001, 128, 16, 0.7, 2.0),
    (257, 513, 64, 64, 1.0, 4.0), (30, 90, 64, 100, 0.3, 1.0), (20, 5000, 192, 256, 0.9, 0.5),
    (300, 2049, 64, 9, 0.0, 3.0)])
def test_distillation(ctx, types, n, C, H, K, alpha, T):
    head = make(n + C + K, n, C, H, types, pad=0.2 if n > 4 else 0.0, K=K, alpha=alpha, temp=T,
                mask=0.1 if C > 50 else 0.0)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
    alone = loss(ctx, head)
    ctx.sync()
    assert torch.equal(alone["row_loss"], got["row_loss"]) and torch.equal(alone["loss"], got["loss"])


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_teacher_alone_needs_no_labels(ctx, types):
    head = make(3, 50, 700, 64, types, K=8, alpha=1.0, temp=2.0)
    with_labels = grad(ctx, head)
    head.label = None
    without = grad(ctx, head)
    ctx.sync()
    want, bound = reference(head)
    check(without, want, bound)
    for k in without:
        assert torch.equal(with_labels[k], without[k]), k


@pytest.mark.parametrize("types,n,C,H,K", [
    # more than 256 MB of dL/dz: two pieces, the last one narrower
    ((F32, F32), 8300, 8801, 64, 0), ((BF16, BF16), 16500, 8801, 64, 0),
    ((F32, F32), 8300, 8801, 64, 3), ((BF16, BF16), 16500, 8801, 64, 3),
    # three, with few rows live
    ((BF16, BF16), 60000, 5800, 64, 0),
    # one piece whose z is formed twice (bf16), and kept (H = 1024)
    ((BF16, BF16), 5000, 7100, 64, 0), ((BF16, BF16), 5000, 7100, 64, 5),
    ((BF16, BF16), 300, 5003, 1024, 5), ((BF16, BF16), 3000, 12000, 1024, 0)])
def test_pieces_of_the_vocabulary(ctx, types, n, C, H, K):
    head = make(5, n, C, H, types, pad=0.95 if n == 60000 else 0.1, K=K, alpha=0.4, temp=2.0)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_no_scored_row_and_no_row(ctx, types):
    head = make(1, 70, 130, 64, types)
    head.label.fill_(-1)
    got = grad(ctx, head)
    ctx.sync()
    assert all(float(v.float().abs().max()) == 0.0 for v in got.values())
    empty = B.VocabHead(h=head.h[:0], Ws=head.Ws, bs=head.bs, label=head.label[:0])
    got = grad(ctx, empty)
    ctx.sync()
    assert all(float(v.float().abs().max()) == 0.0 for v in got.values() if v.numel())
    o = loss(ctx, empty)
    ctx.sync()
    assert float(o["loss"]) == 0.0


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_masked_words(ctx, types):
    """-inf and the type's lowest value in the bias; a label among the masked
    words has an infinite loss and the gradient of its formula."""
    head = make(2, 90, 600, 64, types, mask=0.5)
    head.bs[::3] = torch.finfo(F32).min
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
    head = make(2, 90, 600, 64, types)
    head.bs[int(head.label[7])] = -math.inf
    same = head.label == head.label[7]
    got = grad(ctx, head)
    ctx.sync()
    assert torch.isinf(got["loss"]).all() and torch.equal(torch.isinf(got["row_loss"]), same)
    want, bound = reference(head)
    for k in ("dh", "dWs", "dbs"):
        assert R.outside(got[k], want[k], bound[k]) <= 1.0, k


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("n", [5, 200])
def test_a_word_masked_by_its_weights(ctx, types, n):
    """-inf times a positive state: the word is out of every row's softmax, and
    what the next row of W_s holds behind the last word stays out too."""
    head = make(12, n, 70, 64, types)
    head.h[:, 1] = head.h[:, 1].abs() + 0.1
    head.h[:, 0] = -head.h[:, 0].abs() - 0.1
    head.label[head.label == 0] = 1
    masked = B.VocabHead(h=head.h, Ws=head.Ws.clone(), bs=head.bs.clone(), label=head.label)
    masked.bs[0] = -math.inf
    want, bound = reference(masked)
    head.Ws[1, 0] = -math.inf
    got = loss(ctx, head)
    ctx.sync()
    check(got, want, bound)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,temp", [(40, 1 / 64), (300, 0.25), (40, 64.0), (300, 16.0)])
def test_temperatures(ctx, types, n, temp):
    head = make(13, n, 700, 128, types, K=9, alpha=0.5, temp=temp)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_nan_stays_in_its_row(ctx, types):
    # In fp32 the NaN's tile is formed again on the fp32 instruction: its other
    # rows' sums round in another order, each within the bounds of its terms.
    head = make(4, 300, 400, 64, types)
    clean = grad(ctx, head)
    ctx.sync()
    want, bound = reference(head)
    head.h[11, 5] = float("nan")
    got = grad(ctx, head)
    ctx.sync()
    bad = torch.arange(300, device="cuda") == 11
    assert torch.equal(torch.isnan(got["row_loss"]), bad)
    assert torch.equal(torch.isnan(got["dh"]).any(1), bad)
    assert R.outside(got["dh"][~bad], want["dh"][~bad], bound["dh"][~bad]) <= 1.0
    if types[1] == BF16:
        assert torch.equal(got["dh"][~bad], clean["dh"][~bad])
    assert torch.isnan(got["loss"]).all() and torch.isnan(got["dWs"]).all()
    head.label[11] = -1   # a row that is not scored is not read
    got = grad(ctx, head)
    ctx.sync()
    assert not any(torch.isnan(v).any() for v in got.values())


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("n", [2, 15, 16, 17])
@pytest.mark.parametrize("C,H,K", [(1000, 64, 0), (9001, 192, 5), (130, 320, 40)])
def test_rows_of_one_group(ctx, types, n, C, H, K):
    """The kernels for at most 16 rows, and the first row past them."""
    head = make(n + C, n, C, H, types, pad=0.3, K=K, alpha=0.5 if K else 0.0, temp=2.0 if K else 1.0)
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)
    got = loss(ctx, head)
    ctx.sync()
    check(got, want, bound)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,C,H", [(3, 600001, 64), (64, 450000, 64), (1, (1 << 20), 128), (65, 420000, 64)])
def test_few_rows_of_many_words_stay_in_their_workspace(ctx, types, n, C, H):
    head = make(31, n, C, H, types, bias=False)
    need = B.vocab_workspace_bytes(head, True)
    ws = torch.full((need + (1 << 28),), 255, dtype=torch.uint8, device="cuda")
    got = grad(ctx, head, ws=ws[:need])
    ctx.sync()
    assert bool((ws[need:] == 255).all())
    want, bound = reference(head)
    check(got, want, bound)


def test_large_logits(ctx):
    """Scores of thousands: only the largest words of a row count."""
    head = make(6, 100, 700, 64)
    head.Ws *= 2000.0
    want, bound = reference(head)
    got = grad(ctx, head)
    ctx.sync()
    check(got, want, bound)


def test_labels_out_of_range_are_reported(ctx):
    head = make(7, 20, 60, 64, K=4, alpha=0.5)
    plain = grad(ctx, head)
    ctx.sync()
    for what, bad in (("label", 60), ("label", -2), ("top_word", 60), ("top_word", -5)):
        h = make(7, 20, 60, 64, K=4, alpha=0.5)
        keep = make(7, 20, 60, 64, K=4, alpha=0.5)
        t, k = getattr(h, what), getattr(keep, what)
        at = (3,) if what == "label" else (3, 1)
        t[at], k[at] = bad, -1
        got = grad(ctx, h)
        with pytest.raises(B.CavsError) as e:
            ctx.sync()
        assert e.value.status == B.ERR_RANGE
        want = grad(ctx, keep)
        ctx.sync()
        for name in got:
            assert torch.equal(got[name], want[name]), (what, bad, name)
    again = grad(ctx, head)
    ctx.sync()
    assert all(torch.equal(again[k], plain[k]) for k in plain)


def test_refusals(ctx):
    head = make(1, 8, 30, 64, K=2, alpha=0.5)
    o, ws = outputs(head), workspace(head, True)
    args = lambda **kw: [dict(o, **kw)[k] for k in ("loss", "row_loss", "dh", "dWs", "dbs")]

    def run(h=head, w=ws, **kw):
        return lambda: B.vocab_grad(ctx, h, *args(**kw), w)

    def changed(**kw):
        return B.VocabHead(**{**vars(head), **kw})

    cases = [
        (run(w=ws[:-256]), B.ERR_WORKSPACE), (run(w=ws[1:]), B.ERR_WORKSPACE), (run(dbs=None), B.ERR_ARG),
        (run(h=changed(bs=None)), B.ERR_ARG), (run(dh=o["dh"].bfloat16()), B.ERR_ARG),
        (run(dWs=o["dWs"].t()), B.ERR_ARG), (run(loss=None), B.ERR_ARG),
        (run(h=changed(alpha=-0.1)), B.ERR_ARG), (run(h=changed(temp=0.0)), B.ERR_ARG),
        (run(h=changed(label=None)), B.ERR_ARG), (run(h=changed(h=head.h.cpu())), B.ERR_ARG),
        (run(h=B.VocabHead(h=head.h[:, :32].contiguous(), Ws=head.Ws[:32].contiguous(), bs=head.bs,
                           label=head.label), dh=o["dh"][:, :32].contiguous(),
             dWs=o["dWs"][:32].contiguous()), B.ERR_UNSUPPORTED),
        (run(h=changed(Ws=torch.empty(64 * 30 + 1, device="cuda")[1:].view(64, 30))), B.ERR_ARG),
        (run(dh=torch.empty(8 * 64 + 1, device="cuda")[1:].view(8, 64)), B.ERR_ARG),
    ]
    for k, (call, status) in enumerate(cases):
        with pytest.raises(B.CavsError) as e:
            call()
        assert e.value.status == status, (k, e.value)
    padded = torch.empty(ws.numel() + 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.CavsError) as e:
        run(w=padded[1:])()
    assert e.value.status == B.ERR_ARG
    run()()
    ctx.sync()


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_difference_quotients(ctx, types):
    """The gradient along a direction d against (L(x + e d) - L(x - e d)) / 2e.

    Along h, L's third derivative is at most 2 max|dz|^3 with dz = d W, so the
    quotient is off by e^2 / 3 max|dz|^3; each loss by its bound, over e."""
    head = make(8, 60, 500, 64, types, K=6, alpha=0.5, temp=1.0)
    head.h, dtype = head.h.float(), types[0]
    g = torch.Generator().manual_seed(1)
    d = torch.randn(60, 64, generator=g).cuda()
    # a step that bf16 takes exactly: 2^-8 around multiples of 2^-6 inside (-1, 1)
    h0 = ((head.h * 64).round() / 64).clamp(-63 / 64, 63 / 64)
    step = 2.0 ** -8 * d.sign()
    vals, bounds = [], []
    for s in (1, -1):
        head.h = (h0 + s * step).to(dtype)
        assert torch.equal(head.h.double(), h0.double() + s * step.double())
        o = loss(ctx, head)
        ctx.sync()
        vals.append(float(o["loss"]))
        bounds.append(float(reference(head, grad=False)[1]["loss"]))
    head.h = h0.to(dtype)
    o = grad(ctx, head)
    ctx.sync()
    got = float((o["dh"].double() * step.double()).sum())
    bound = float((reference(head)[1]["dh"] * step.abs().double()).sum())
    big = float((step.double() @ head.Ws.double()).abs().max())
    assert abs((vals[0] - vals[1]) / 2 - got) <= big ** 3 / 3 + sum(bounds) / 2 + bound


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
def test_replays_of_a_captured_step(ctx, types):
    head = make(9, 500, 1300, 128, types, K=5, alpha=0.4, temp=2.0, pad=0.1)
    s = torch.cuda.Stream()
    own = B.Context(0, s)
    o, ws = outputs(head), workspace(head, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        grad(own, head, ws, o)
    for k in range(3):
        other = make(20 + k, 500, 1300, 128, types, K=5, alpha=0.4, temp=2.0, pad=0.3 * k)
        for name in ("h", "Ws", "bs", "label", "top_word", "top_logit"):
            getattr(head, name).copy_(getattr(other, name))
        torch.cuda.synchronize()
        graph.replay()
        want = grad(ctx, other)
        torch.cuda.synchronize()
        for name in o:
            assert torch.equal(o[name], want[name]), (k, name)
    own.sync()
    own.close()


def test_two_contexts_on_two_streams(ctx):
    """Two heads at once, each with its context, stream and workspace."""
    heads = [make(30 + k, 700, 3000, 128, t, pad=0.1) for k, t in enumerate([(F32, F32), (BF16, BF16)])]
    alone = []
    for h in heads:
        alone.append(grad(ctx, h))
        ctx.sync()
    streams = [torch.cuda.Stream() for _ in heads]
    own = [B.Context(0, s) for s in streams]
    outs, wss = [outputs(h) for h in heads], [workspace(h, True) for h in heads]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, h, o, w in zip(own, heads, outs, wss):
            grad(c, h, w, o)
    for c in own:
        c.sync()
        c.close()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a[k], o[k]) for k in a)


def test_one_workspace_for_batches_of_a_size(ctx):
    """Rows that a batch before left scored do not show in the next one."""
    full = make(40, 400, 900, 64)
    ws = workspace(full, True)
    grad(ctx, full, ws)
    part = make(41, 400, 900, 64, pad=0.9)
    got = grad(ctx, part, ws)
    ctx.sync()
    fresh = grad(ctx, part)
    ctx.sync()
    assert all(torch.equal(got[k], fresh[k]) for k in got)
