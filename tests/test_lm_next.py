"""What runner.LmBatch hands to the library for a clipped step and for next words
(CPU only: the calls are replaced by ones that record their arguments)."""
import numpy as np
import pytest
import torch

from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import LmBatch
from test_abi import _ensure_built


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


class _Context:
    torch_device = torch.device("cpu")

    def __init__(self):
        self.synced = 0

    def sync(self):
        self.synced += 1


@pytest.fixture
def made(monkeypatch):
    _ensure_built()
    seen = []
    for name in ("embed", "embed_grad", "forward", "backward", "infer", "vocab_grad", "clip_grads", "quant_pack",
                 "quant_product", "adjust_logits"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **kw: seen.append((_n, a, kw)))
    for name in ("workspace_bytes", "infer_workspace_bytes"):
        monkeypatch.setattr(B, name, lambda *a: 64)
    rng = np.random.Generator(np.random.PCG64(1))
    wl = W.make_workload("lm", [W.chain(int(n)) for n in (3, 7, 5)], N=1, D=4, H=64, C=9, rng=rng,
                         inputs="all", labels="all")

    def make(**kw):
        b = LmBatch(wl, torch.zeros(6, wl.D), np.arange(wl.n_x) % 6, _Context(), **kw)
        b.sched = object()
        b.alloc()
        return b, seen
    return make


def test_a_step_clips_last_and_every_parameter_s_gradient(made):
    b, seen = made(max_norm=2.5)
    b.forward()
    b.backward()
    name, args, _ = seen[-1]
    assert name == "clip_grads" and args[1] is b.clip and args[2] == 2.5 and args[3] is b.norm
    held = {id(g) for g in b.clip.grads}
    assert held == {id(g) for k, g in b.grads.items() if k != "dX"} and len(held) == 6
    assert b.clip.out is b.clip.grads


def test_a_step_without_a_limit_does_not_clip(made):
    b, seen = made()
    b.forward()
    b.backward()
    assert "clip_grads" not in [s[0] for s in seen] and not hasattr(b, "clip")


def test_next_words(made):
    b, seen = made()
    last = torch.tensor([2, 9, 14], dtype=torch.int32)
    rules = B.LogitRules(temp=torch.ones(3))
    best = b.next_words(last, rules)
    assert [s[0] for s in seen] == ["quant_pack", "embed", "infer", "embed", "quant_product", "adjust_logits"]
    rows, product, adjust = seen[3][1], seen[4], seen[5][1]
    assert rows[1].E is b.h and rows[2] is last and rows[3] is b.rows
    assert product[1][1] is b.quant and product[1][2] is b.rows and product[2]["bias"] is b.bs
    assert adjust[1] is rules and adjust[2] is b.logits and adjust[3] is b.logits and adjust[4] is best
    # its own again, as long as there are as many; others only after a wait
    waits = b.ctx.synced
    assert b.next_words(last) is best and b.ctx.synced == waits and seen[-1][1][1] is b.rules
    assert [s[0] for s in seen].count("quant_pack") == 1
    assert b.next_words(last[:1].clone()) is not best and b.ctx.synced == waits + 1


def test_a_head_is_quantised_again_after_a_wait(made):
    b, seen = made()
    b.quantise(64)
    waits, first = b.ctx.synced, b.quant
    b.quantise(32, True)
    assert b.ctx.synced == waits + 1 and b.quant is not first and (b.quant.group, b.quant.shift) == (32, True)
