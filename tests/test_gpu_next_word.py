"""The operators together, as a program uses them: a training step that ends with
clipping, the next words of a batch; streams, captured graphs, two contexts."""
import math

import numpy as np
import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import LmBatch

pytestmark = pytest.mark.gpu

KEYS = ["dWx", "dU", "db", "dWs", "dbs", "dE"]


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _model(seed=3, C=999):
    rng = np.random.Generator(np.random.PCG64(seed))
    lengths = rng.integers(5, 30, size=9)
    wl = W.make_workload("lm", [W.chain(int(n)) for n in lengths], N=1, D=20, H=128, C=C, rng=rng,
                         inputs="all", labels="all")
    table = torch.from_numpy(rng.standard_normal((50, wl.D)).astype(np.float32)).cuda()
    words = rng.integers(-1, 50, wl.n_x).astype(np.int32)
    return wl, table, words, torch.from_numpy(np.cumsum(lengths).astype(np.int32) - 1).cuda()


@pytest.mark.parametrize("head_dtype", [torch.float32, torch.bfloat16])
def test_a_training_step_that_clips(ctx, head_dtype):
    wl, table, words, _ = _model()
    plain = LmBatch(wl, table, words, ctx, head_dtype=head_dtype)
    plain.run()
    grads = [plain.grads[k] for k in KEYS]
    want, nb, outs = R.clip(grads, 1.0, 0.01, [g.dtype for g in grads])
    assert want > 0.01
    b = LmBatch(wl, table, words, ctx, head_dtype=head_dtype, max_norm=0.01)
    got = b.run()
    assert abs(float(b.norm) - want) <= nb
    for k, (w, bound) in zip(KEYS, outs):
        assert R.outside(b.grads[k], w, bound) <= 1.0, k
    assert torch.equal(b.grads["dX"], plain.grads["dX"]) and got["loss"] == float(plain.loss)
    # a limit that is not reached changes nothing
    free = LmBatch(wl, table, words, ctx, head_dtype=head_dtype, max_norm=1e6)
    free.run()
    assert all(torch.equal(free.grads[k], plain.grads[k]) for k in KEYS)


@pytest.mark.parametrize("group,shift", [(128, False), (32, True)])
def test_next_words(ctx, group, shift):
    wl, table, words, last = _model()
    b = LmBatch(wl, table, words, ctx)
    b.schedule()
    b.alloc()
    b.quantise(group, shift)
    n, C = last.shape[0], wl.C
    g = torch.Generator().manual_seed(1)
    past = torch.randint(-1, C, (n, 20), generator=g).int().cuda()
    mask = torch.randint(-2 ** 31, 2 ** 31, (2, -(-C // 32)), generator=g).int().cuda()
    state = (torch.arange(n) % 3 - 1).int().cuda()
    rules = dict(past=past, repeat=torch.full((n,), 1.3, device="cuda"), mask=mask, mask_row=state,
                 temp=torch.full((n,), 0.7, device="cuda"))
    for use in ({}, rules):
        best = b.next_words(last, B.LogitRules(**use))
        ctx.sync()
        x = b.h[last.long()]
        z, zb = R.product(x, *R.quantise(b.Ws, group, shift), group, b.bs, False)
        # the rules are steps of slope up to 1.3 / 0.7 of what the product is off by
        v, vb = R.rules(z, **use)
        vb = vb + torch.where(torch.isfinite(v), 1.3 / 0.7 * zb, 0.0)
        assert R.outside(b.logits, v, vb) <= 1.0
        short = v.amax(1) - v.gather(1, best.long()[:, None])[:, 0]
        assert (short <= 2 * vb.amax(1)).all()
        w, wb = R.lse(v, vb)
        assert R.outside(b.lse, w, wb) <= 1.0


def _step(c, s):
    B.embed(c, s["emb"], s["word"], s["x"])
    B.quant_product(c, s["q"], s["x"], s["z"], bias=s["b"])
    B.adjust_logits(c, s["rules"], s["z"], s["z"], s["best"], s["lse"], s["ws"])
    B.clip_grads(c, s["grads"], 1.0, s["norm"], s["wc"])


def _state(c, seed, n=5, H=256, C=20000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    s = dict(emb=B.Embedding(randn(40, H)), word=torch.randint(0, 40, (n,), generator=g, device="cuda").int(),
             x=torch.empty(n, H, device="cuda"), z=torch.empty(n, C, device="cuda"), b=randn(C),
             best=torch.empty(n, dtype=torch.int32, device="cuda"), lse=torch.empty(n, device="cuda"))
    s["q"] = B.QuantWeights(torch.empty(B.quant_bytes(H, C), dtype=torch.uint8, device="cuda"), H, C)
    s["W"] = randn(H, C) / 16
    torch.cuda.synchronize()   # made on torch's stream, read on the context's
    B.quant_pack(c, s["q"], s["W"])
    s["rules"] = B.LogitRules(past=torch.randint(-1, C, (n, 50), generator=g, device="cuda").int(),
                              frequency=torch.rand(n, generator=g, device="cuda"))
    s["ws"] = torch.empty(B.adjust_workspace_bytes(n, C), dtype=torch.uint8, device="cuda")
    s["src"] = [randn(3000, 100), randn(77)]
    s["out"] = [torch.empty_like(x) for x in s["src"]]
    s["grads"] = B.GradList(s["src"], s["out"])
    s["norm"] = torch.empty(1, device="cuda")
    s["wc"] = torch.empty(B.clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    c.sync()
    torch.cuda.synchronize()
    return s


def _outputs(s):
    return [s[k].clone() for k in ("x", "z", "best", "lse", "norm")] + [o.clone() for o in s["out"]]


@pytest.mark.parametrize("n,H,C", [(5, 256, 20000), (16, 2048, 5000), (1, 64, 300)])
def test_captured_and_replayed(ctx, n, H, C):
    """Replays on changed inputs, with eager work between them, equal eager calls."""
    stream = torch.cuda.Stream()
    c = B.Context(0, stream)
    s = _state(c, 1, n, H, C)
    _step(c, s)
    c.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _step(c, s)
    g = torch.Generator(device="cuda").manual_seed(5)
    for k in range(4):
        s["word"].copy_(torch.randint(0, 40, s["word"].shape, generator=g, device="cuda"))
        s["src"][0].mul_(0.9 + 0.1 * k)
        s["rules"].past.copy_(torch.randint(-1, C, s["rules"].past.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = _outputs(s)
        for o in [s["x"], s["z"], s["lse"], s["norm"]] + s["out"]:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        _step(c, s)
        c.sync()
        assert all(torch.equal(a, b) for a, b in zip(got, _outputs(s))), k
        torch.randn(1000, 1000, device="cuda").sum()
    c.close()


def test_two_contexts_at_once(ctx):
    """Steps of two contexts on two streams, beside each other: the same as alone."""
    cs = [B.Context(0, torch.cuda.Stream()) for _ in range(2)]
    ss = [_state(c, 10 + k) for k, c in enumerate(cs)]
    want = []
    for c, s in zip(cs, ss):
        _step(c, s)
        c.sync()
        want.append(_outputs(s))
        for o in [s["x"], s["z"], s["lse"], s["norm"]] + s["out"]:
            o.fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s in zip(cs, ss):
            _step(c, s)
    for c in cs:
        c.sync()
    for s, w in zip(ss, want):
        assert all(torch.equal(a, b) for a, b in zip(_outputs(s), w))
    for c in cs:
        c.close()


def test_timing_names_the_kernels(ctx):
    s = _state(ctx, 2)
    ctx.timing(True)
    _step(ctx, s)
    names = [r[0] for r in ctx.timing_read()]
    ctx.timing(False)
    assert [n.split("<")[0] for n in names] == ["k_embed", "k_quant_product", "k_rules", "k_rules_join", "k_clip_norm",
                                                "k_clip_scale"]
