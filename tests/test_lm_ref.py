"""The 64-bit forms that the GPU tests compare with, pinned by library routines,
automatic differentiation and differences (CPU)."""
import math

import pytest
import torch

import lm_ref as R

F = torch.nn.functional


@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def _case(seed, n=7, C=23, H=64, K=5):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn(n, H, generator=g, dtype=torch.float64)
    W = torch.randn(H, C, generator=g, dtype=torch.float64) * 0.2
    b = torch.randn(C, generator=g, dtype=torch.float64)
    y = torch.randint(-1, C, (n,), generator=g)
    y[0] = 3
    word = torch.stack([torch.randperm(C, generator=g)[:K] for _ in range(n)])
    word[1, 2:] = -1
    word[2] = -1
    word[3, 1] = word[3, 0]
    return h, W, b, y, word, torch.randn(n, K, generator=g, dtype=torch.float64)


def test_cross_entropy_is_the_library_s():
    h, W, b, y, _, _ = _case(0)
    leaves = [t.clone().requires_grad_() for t in (h, W, b)]
    loss = F.cross_entropy(leaves[0] @ leaves[1] + leaves[2], y, ignore_index=-1)
    loss.backward()
    out, _ = R.head(h, W, b, y)
    assert abs(float(out["loss"] - loss)) < 1e-12
    for k, t in zip(("dh", "dWs", "dbs"), leaves):
        assert torch.allclose(out[k], t.grad, atol=1e-13, rtol=1e-10), k


@pytest.mark.parametrize("alpha,T", [(1.0, 1.0), (0.4, 1.0), (0.7, 2.5)])
def test_distillation_is_the_divergence_and_its_gradient(alpha, T):
    h, W, b, y, word, logit = _case(1)
    leaves = [t.clone().requires_grad_() for t in (h, W, b)]
    z = leaves[0] @ leaves[1] + leaves[2]
    q, _ = R.teacher(word, logit, T)
    dense = torch.zeros_like(z).scatter_add(1, word.clamp(min=0), q).detach()
    rows = y >= 0
    # kl_div's sum q ln q merges a word that is listed twice; the loss keeps its entries apart
    kl = F.kl_div(F.log_softmax(z / T, 1), dense, reduction="none").sum(1)
    kl = kl + (torch.special.xlogy(q, q).sum(1) - torch.special.xlogy(dense, dense).sum(1))
    ce = F.cross_entropy(z, y.clamp(min=0), reduction="none")
    value = (1 - alpha) * ce + alpha * T * T * kl
    loss = value[rows].mean()
    loss.backward()
    out, _ = R.head(h, W, b, y, word, logit, alpha, T)
    assert abs(float(out["loss"] - loss)) < 1e-12
    for k, t in zip(("dh", "dWs", "dbs"), leaves):
        assert torch.allclose(out[k], t.grad, atol=1e-13, rtol=1e-10), k


def test_gradients_by_differences():
    h, W, b, y, word, logit = _case(2)
    args = dict(label=y, top_word=word, top_logit=logit, alpha=0.6, temp=2.0)
    out, _ = R.head(h, W, b, **args)
    g = torch.Generator().manual_seed(9)
    for k, name in ((0, "dh"), (1, "dWs"), (2, "dbs")):
        t = [h, W, b]
        d = torch.randn(t[k].shape, generator=g, dtype=torch.float64)
        e = 1e-5

        def loss(sign):
            s = list(t)
            s[k] = t[k] + sign * e * d
            return float(R.head(*s, **args, grad=False)[0]["loss"])

        assert abs((loss(1) - loss(-1)) / (2 * e) - float((out[name] * d).sum())) < 1e-8, name


def test_embedding_gradient_is_the_library_s():
    g = torch.Generator().manual_seed(3)
    E = torch.randn(11, 6, generator=g, dtype=torch.float64)
    word = torch.randint(-1, 11, (40,), generator=g)
    dX = torch.randn(40, 6, generator=g, dtype=torch.float64)
    leaf = E.clone().requires_grad_()
    X = torch.where((word >= 0)[:, None], F.embedding(word.clamp(min=0), leaf) * 1.5, 0.0)
    X.backward(dX)
    assert torch.equal(R.embed(E, word, 1.5), X.detach())
    dE, bound = R.embed_grad(word, dX, 11, 1.5, False)
    assert torch.allclose(dE, leaf.grad, atol=1e-13)
    assert R.outside(leaf.grad, dE, bound) <= 1.0


def test_bounds_reject_a_planted_mistake():
    """A gradient that forgets one row's label, or one word of the sum, is outside."""
    h, W, b, y, _, _ = _case(4, n=40, C=200)
    h, W, b = h.float(), W.float(), b.float()
    out, bound = R.head(h, W, b, y)
    wrong, _ = R.head(h, W, b, torch.where(torch.arange(40) == 0, 4, y))
    for k in out:
        assert R.outside(out[k], out[k], bound[k]) == 0.0
        assert R.outside(wrong[k], out[k], bound[k]) > 10.0, k


def test_rows_and_words_that_are_not_there():
    h, W, b, _, word, logit = _case(5)
    none = torch.full((7,), -1)
    out, _ = R.head(h, W, b, none)
    assert all(float(v.abs().max()) == 0.0 for v in out.values())
    q, some = R.teacher(torch.full_like(word, -1), logit, 1.0)
    assert not some.any() and float(q.abs().max()) == 0.0
    low = torch.full_like(logit, -math.inf)
    q, some = R.teacher(word, low, 1.0)
    assert not some.any() and float(q.abs().max()) == 0.0
