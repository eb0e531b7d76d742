"""Next words after the head has changed, on the GPU: as those of a model that has
the new head from the start."""
import numpy as np
import pytest
import torch

from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd.runner import LmBatch
from test_gpu_next_word import _float32_by_default, _model, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def _made(c, wl, table, words):
    b = LmBatch(wl, table, words, c)
    b.schedule()
    b.alloc()
    return b


def _words(b, last):
    best = b.next_words(last)
    b.ctx.sync()
    return best.clone(), b.logits.clone(), b.lse.clone()


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("group,shift", [(128, False), (32, True)])
def test_a_changed_head(ctx, group, shift):
    """Changed in place, then by a step of a fused optimiser, whose changes torch does
    not count, after the step's gradients."""
    wl, table, words, last = _model()
    b = _made(ctx, wl, table, words)
    b.quantise(group, shift)
    before = _words(b, last)

    def fresh():
        new = _made(ctx, wl, table, words)
        new.Ws.copy_(b.Ws)
        torch.cuda.synchronize()
        new.quantise(group, shift)
        return _words(new, last)

    b.Ws.mul_(-0.5)
    torch.cuda.synchronize()
    after = _words(b, last)
    assert not torch.equal(before[1], after[1]) and _same(after, fresh())
    p = torch.nn.Parameter(b.Ws)
    p.grad = b.grads["dWs"]
    opt = torch.optim.Adam([p], lr=0.1, fused=True)
    b.forward()
    b.backward()
    ctx.sync()
    opt.step()
    torch.cuda.synchronize()
    stepped = _words(b, last)
    assert not torch.equal(after[1], stepped[1]) and _same(stepped, fresh())


def test_a_captured_call_finds_the_head_of_the_same_form(ctx):
    """quantise() between replays writes where the captured call reads."""
    wl, table, words, last = _model(5, 700)
    stream = torch.cuda.Stream()
    c = B.Context(0, stream)
    b = _made(c, wl, table, words)
    torch.cuda.synchronize()
    b.next_words(last)
    c.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.next_words(last)
    for k in range(4):
        b.Ws.mul_(-0.9)
        torch.cuda.synchronize()
        b.quantise()
        c.sync()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (b.best, b.logits, b.lse)]
        b.logits.fill_(float("nan"))
        torch.cuda.synchronize()
        assert _same(got, _words(b, last)), k
        torch.randn(1000, 1000, device="cuda").sum()
    c.close()
