"""Words that the weights mask: W_s holds -inf where every state has the other
sign, so that the word is out of each row's softmax.  A state of 0 there has the
score NaN, which must not leave rows that take no part in the gradient."""
import math

import pytest
import torch

import lm_ref as R
from paper_1712_04048_amd import binding as B
from test_gpu_vocab import BF16, F32, check, grad, make

pytestmark = pytest.mark.gpu


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


def masked(head, words):
    """(the head with `words` masked by row 1 of W_s, the same masked by the bias)"""
    head.h[:, 1] = head.h[:, 1].abs() + 0.1
    for w in words:
        if head.label is not None:
            head.label[head.label == w] = 1
        if head.top_word is not None:
            head.top_word[head.top_word == w] = -1
    by_bias = B.VocabHead(**{**vars(head), "bs": head.bs.clone(), "Ws": head.Ws.clone()})
    by_bias.bs[words] = -math.inf
    head.Ws[1, words] = -math.inf
    return head, by_bias


def compare(got, by_bias):
    """dL/dh of the masking row is dz W = 0 times -inf, a NaN by its formula."""
    want, bound = R.head(by_bias.h, by_bias.Ws, by_bias.bs, by_bias.label, by_bias.top_word,
                         by_bias.top_logit, by_bias.alpha, by_bias.temp)
    for o in (got, want, bound):
        o["dh"] = torch.cat([o["dh"][:, :1], o["dh"][:, 2:]], 1)
    check(got, want, bound)


# z kept and formed twice, in one piece of the vocabulary and in two
ROUTES = [((F32, F32), 40, 90), ((BF16, BF16), 40, 90), ((F32, F32), 300, 700), ((BF16, BF16), 300, 700),
          ((BF16, BF16), 3000, 8401), ((F32, BF16), 3000, 8400), ((F32, F32), 8300, 8801),
          ((BF16, BF16), 16500, 8801)]


@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("types,n,C", ROUTES)
def test_gradients_of_a_word_masked_by_its_weights(ctx, types, n, C, K):
    """With one live row in the last group, the others of its tile are not live."""
    head = make(n + K, n, C, 64, types, pad=0.1, K=K, alpha=0.4 if K else 0.0, temp=2.0 if K else 1.0)
    head, by_bias = masked(head, [0, C // 2, C - 1])
    live = torch.nonzero(head.label >= 0).flatten()
    head.label[live[1:1 + (live.numel() - 1) % 64]] = -1
    assert int((head.label >= 0).sum()) % 64 == 1
    got = grad(ctx, head)
    ctx.sync()
    compare(got, by_bias)


@pytest.mark.parametrize("types,n,C", ROUTES[2:7])
def test_a_row_without_a_teacher_s_word_has_no_gradient(ctx, types, n, C):
    """With the teacher alone its term is 0, whatever its scores are."""
    head = make(n, n, C, 64, types, K=8, alpha=1.0, temp=2.0)
    head.label = None
    head, by_bias = masked(head, [0, C - 1])
    none = (head.top_word < 0).all(1)
    assert int(none.sum()) >= n // 7
    head.h[none, 1] = 0.0   # scores of 0 times -inf
    got = grad(ctx, head)
    ctx.sync()
    compare(got, by_bias)
