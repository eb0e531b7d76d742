"""What the embedding and the vocabulary head refuse before a GPU is reached:
the binding's checks of tensors, and workspace queries of arguments that the
calls refuse (CPU only)."""
import ctypes as ct
import os
import subprocess
import tempfile

import pytest
import torch

from paper_1712_04048_amd import binding as B
from test_abi import HEADER, _ensure_built

@pytest.fixture(autouse=True)
def _float32_by_default():
    """Other modules leave torch's default type changed."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


PROBE = r"""
#include <stddef.h>
#include <stdio.h>
#include "cavs.h"
#define F(S, m) printf(#S "." #m " %zu\n", offsetof(S, m));
int main(void) {
  printf("cavs_embedding %zu\ncavs_vocab %zu\n", sizeof(cavs_embedding), sizeof(cavs_vocab));
  F(cavs_embedding, D) F(cavs_embedding, E) F(cavs_embedding, scale)
  F(cavs_vocab, C) F(cavs_vocab, h) F(cavs_vocab, bs) F(cavs_vocab, label) F(cavs_vocab, K)
  F(cavs_vocab, top_word) F(cavs_vocab, top_logit) F(cavs_vocab, alpha) F(cavs_vocab, temp)
  printf("types.f32 %d\ntypes.bf16 %d\n", CAVS_T_F32, CAVS_T_BF16);
  return 0;
}
"""


def test_struct_layouts_match_header():
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "probe.c"), os.path.join(d, "probe")
        open(src, "w").write(PROBE)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.dirname(HEADER), src, "-o", exe])
        out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    vals = {k: int(v) for k, v in (line.split() for line in out.strip().splitlines())}
    assert (vals.pop("types.f32"), vals.pop("types.bf16")) == (B.T_F32, B.T_BF16)
    for key, v in vals.items():
        cls = getattr(B, key.split(".")[0])
        assert (getattr(cls, key.split(".")[1]).offset if "." in key else ct.sizeof(cls)) == v, key


def _head(n=4, H=64, C=10, **kw):
    d = dict(h=torch.zeros(n, H), Ws=torch.zeros(H, C), bs=torch.zeros(C),
             label=torch.zeros(n, dtype=torch.int32))
    d.update(kw)
    return B.VocabHead(**d)


TEACHER = dict(top_word=torch.zeros(4, 3, dtype=torch.int32),
               top_logit=torch.zeros(4, 3, dtype=torch.float32), alpha=0.5)


@pytest.mark.parametrize("kw", [
    dict(h=torch.zeros(4, 32)), dict(h=torch.zeros(4, 64, dtype=torch.float16)),
    dict(h=torch.zeros(64)), dict(h=torch.zeros(64, 4).t()), dict(Ws=torch.zeros(10, 64).t()),
    dict(bs=torch.zeros(9)), dict(bs=torch.zeros(10, dtype=torch.bfloat16)),
    dict(label=torch.zeros(4, dtype=torch.int64)), dict(label=torch.zeros(5, dtype=torch.int32)),
    dict(top_word=torch.zeros(4, 3, dtype=torch.int32)), dict(top_logit=torch.zeros(4, 3)),
    dict(TEACHER, top_logit=torch.zeros(4, 2)), dict(TEACHER, top_logit=torch.zeros(4, 3).bfloat16()),
    dict(TEACHER, top_word=torch.zeros(4, 3, dtype=torch.int64)),
])
def test_head_tensors_are_checked(kw):
    with pytest.raises(B.CavsError) as e:
        _head(**kw).raw()
    assert e.value.status == B.ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(h=torch.zeros(4, 96), Ws=torch.zeros(96, 10)), dict(label=None),
    dict(TEACHER, alpha=1.5), dict(TEACHER, alpha=float("nan")), dict(TEACHER, temp=0.0),
    dict(TEACHER, temp=float("inf")), dict(TEACHER, label=None),
    dict(TEACHER, top_word=torch.zeros(4, 257, dtype=torch.int32), top_logit=torch.zeros(4, 257)),
])
def test_refused_heads_have_no_workspace(kw):
    _ensure_built()
    assert B.vocab_workspace_bytes(_head(), True) > 0
    assert B.vocab_workspace_bytes(_head(**kw), True) == 0
    assert B.vocab_workspace_bytes(_head(**kw), False) == 0


@pytest.mark.parametrize("temp,ok", [(1 / 64, True), (64.0, True), (0.015, False), (64.1, False), (-1.0, False),
                                     (float("nan"), False)])
def test_temperatures(temp, ok):
    _ensure_built()
    assert (B.vocab_workspace_bytes(_head(**dict(TEACHER, temp=temp)), True) > 0) == ok


def test_head_workspace_does_not_hold_the_logits():
    _ensure_built()

    def need(n, C, train, t):
        h = B.VocabHead(h=torch.empty(n, 64, dtype=t), Ws=torch.empty(64, C, dtype=t),
                        label=torch.empty(n, dtype=torch.int32))
        return B.vocab_workspace_bytes(h, train)

    for t, size in ((torch.float32, 4), (torch.bfloat16, 2)):
        logits = 4 * 65536 * 100000
        assert need(65536, 100000, False, t) < logits / 20
        assert need(65536, 100000, True, t) < logits / 10
        # of one size, what the vocabulary adds is its statistics alone
        a, b = need(65536, 50000, True, t), need(65536, 100000, True, t)
        assert b - a < 4 * 65536 * 50000 / 25, (a, b)


def test_embedding_tensors_are_checked():
    _ensure_built()
    E = torch.zeros(5, 8)
    assert B.embed_grad_workspace_bytes(B.Embedding(E), 10) > 0
    assert B.embed_grad_workspace_bytes(B.Embedding(E), 0) > 0
    assert B.embed_grad_workspace_bytes(B.Embedding(E), -1) == 0
    assert B.embed_grad_workspace_bytes(B.Embedding(torch.zeros(5, 0)), 4) == 0
    assert B.embed_grad_workspace_bytes(B.Embedding(torch.zeros(0, 8)), 4) == 0
    for bad in (torch.zeros(5), torch.zeros(8, 5).t(), torch.zeros(5, 8, dtype=torch.float64)):
        with pytest.raises(B.CavsError):
            B.Embedding(bad).raw(torch.float32)
    with pytest.raises(B.CavsError):
        B.Embedding(E).raw(torch.float16)


def test_sizes_past_the_kernels_are_refused():
    """Through the C ABI, whose queries read no memory."""
    _ensure_built()
    L = B.lib()

    def vocab(**kw):
        d = dict(h_type=0, w_type=0, n=10, H=64, C=100, label=16)
        d.update(kw)
        return L.cavs_vocab_workspace_bytes(ct.byref(B.cavs_vocab(**d)), 1)

    assert vocab() > 0 and vocab(n=1 << 20, C=1 << 20) > 0 and vocab(H=1 << 15) > 0
    for kw in (dict(n=(1 << 20) + 1), dict(C=(1 << 20) + 1), dict(H=(1 << 15) + 64), dict(H=0), dict(C=0),
               dict(n=-1), dict(K=-1), dict(h_type=2), dict(w_type=-1),
               dict(K=3, alpha=0.5, temp=1e-40)):
        assert vocab(**kw) == 0, kw

    def grad(n=10, **kw):
        d = dict(e_type=0, x_type=0, n_words=10, D=8)
        d.update(kw)
        return L.cavs_embed_grad_workspace_bytes(ct.byref(B.cavs_embedding(**d)), n)

    assert grad() > 0 and grad(n=1 << 22, n_words=1 << 22) > 0 and grad(D=1 << 14) > 0
    for kw in (dict(n=(1 << 22) + 1), dict(n_words=(1 << 22) + 1), dict(D=(1 << 14) + 1), dict(e_type=2),
               dict(x_type=-1)):
        assert grad(**kw) == 0, kw
    assert L.cavs_vocab_workspace_bytes(None, 0) == 0 and L.cavs_embed_grad_workspace_bytes(None, 1) == 0
