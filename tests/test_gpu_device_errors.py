"""Errors that kernels record are each reported once, whatever order and number
they come in."""
import pytest
import torch

from paper_1712_04048_amd import binding as B
from paper_1712_04048_amd import workloads as W
from paper_1712_04048_amd.runner import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("word_first", [False, True])
@pytest.mark.parametrize("read", ["sync", "timing_read"])
def test_a_wait_that_gave_up_does_not_hide_a_word_out_of_range(monkeypatch, word_first, read):
    ctx = B.Context(0)
    try:
        b = Batch(W.config_varlstm(2, K=12), ctx)
        b.schedule()
        b.alloc()
        E = torch.ones(4, 8, dtype=torch.float32, device="cuda")
        X = torch.empty(2, 8, dtype=torch.float32, device="cuda")
        word = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        monkeypatch.setenv("CAVS_XCD_LOOP", "1")
        monkeypatch.setenv("CAVS_PERSIST_SPIN", "-1")
        if word_first:
            B.embed(ctx, B.Embedding(E), word, X)
        b.forward()
        if not word_first:
            B.embed(ctx, B.Embedding(E), word, X)
        seen = []
        for _ in range(3):
            try:
                getattr(ctx, read)()
                seen.append(None)
            except B.CavsError as e:
                seen.append(e.status)
        assert seen == [B.ERR_HIP, B.ERR_RANGE, None]
    finally:
        torch.cuda.synchronize()
        ctx.close()
