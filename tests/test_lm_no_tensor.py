"""What is no tensor is refused with the binding's own error (CPU only)."""
import pytest
import torch

from paper_1712_04048_amd import binding as B
from test_abi import _ensure_built


class _Context:
    torch_device = torch.device("cpu")
    _h = None

    def check(self, status):
        raise AssertionError("the library was called")


@pytest.fixture
def made():
    _ensure_built()
    f = dict(dtype=torch.float32)
    emb = B.Embedding(torch.zeros(5, 8, **f))
    head = B.VocabHead(h=torch.zeros(4, 64, **f), Ws=torch.zeros(64, 10, **f),
                       label=torch.zeros(4, dtype=torch.int32))
    return dict(emb=emb, head=head, word=torch.zeros(4, dtype=torch.int32), X=torch.zeros(4, 8, **f),
                loss=torch.zeros(1, **f), ws=torch.zeros(16, dtype=torch.uint8))


@pytest.mark.parametrize("what", [None, 3, [0, 1]])
def test_arguments_that_are_no_tensors(made, what):
    emb, head, word, X, loss, ws = (made[k] for k in ("emb", "head", "word", "X", "loss", "ws"))
    c = _Context()

    def changed(**kw):
        return B.VocabHead(**{**vars(head), **kw})

    calls = [
        lambda: B.embed(c, emb, what, X), lambda: B.embed(c, emb, word, what),
        lambda: B.embed(c, B.Embedding(what), word, X),
        lambda: B.embed_grad(c, emb, what, X, emb.E, ws), lambda: B.embed_grad(c, emb, word, what, emb.E, ws),
        lambda: B.embed_grad(c, emb, word, X, what, ws), lambda: B.embed_grad(c, emb, word, X, emb.E, what),
        lambda: B.vocab_loss(c, changed(h=what), loss, None, ws),
        lambda: B.vocab_loss(c, changed(Ws=what), loss, None, ws),
        lambda: B.vocab_loss(c, changed(top_word=what, top_logit=loss), loss, None, ws),
        lambda: B.vocab_loss(c, head, what, None, ws), lambda: B.vocab_loss(c, head, loss, None, what),
        lambda: B.vocab_grad(c, head, loss, None, what, head.Ws, None, ws),
        lambda: B.vocab_grad(c, head, loss, None, head.h, what, None, ws),
        lambda: B.vocab_grad(c, head, loss, None, head.h, head.Ws, None, what),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(B.CavsError) as e:
            call()
        assert e.value.status == B.ERR_ARG, k
