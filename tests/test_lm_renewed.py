"""When runner.LmBatch rounds its head to 4 bits again (CPU only: the calls are
replaced by ones that record their arguments)."""
import torch

from paper_1712_04048_amd import binding as B
from test_lm_next import _float32_by_default, made  # noqa: F401

LAST = torch.tensor([2, 9, 14], dtype=torch.int32)


def _packs(seen):
    return [s[1] for s in seen if s[0] == "quant_pack"]


def test_a_changed_head_is_rounded_again_where_it_is(made):
    """After weights that torch has changed, and after a step's gradients, whatever
    changes the weights then: into the same memory, in the same form, without a wait."""
    b, seen = made()
    b.quantise(64, True)
    b.next_words(LAST)
    first, waits = b.quant, b.ctx.synced

    def renewed(times):
        b.next_words(LAST)
        b.next_words(LAST)
        packs = _packs(seen)
        assert len(packs) == times and packs[-1][2] is b.Ws
        assert packs[-1][1].data is first.data and (b.quant.group, b.quant.shift) == (64, True)
        assert b.ctx.synced == waits

    renewed(1)
    b.Ws.add_(1.0)
    renewed(2)
    with torch.no_grad():
        b.Ws.view(-1)[3] = 7.0
    renewed(3)
    b.forward()
    renewed(3)
    b.backward()
    renewed(4)
    b.Ws = b.Ws.clone()
    renewed(5)
    b.quantise(64, True)
    renewed(6)


def test_a_head_whose_changes_torch_does_not_count(made):
    """Weights made in inference mode have no count of their changes: a step's
    gradients and quantise() renew them."""
    b, seen = made()
    with torch.inference_mode():
        b.Ws = b.Ws.clone()
    b.next_words(LAST)
    b.next_words(LAST)
    assert len(_packs(seen)) == 1
    b.backward()
    b.next_words(LAST)
    assert len(_packs(seen)) == 2


def test_a_head_of_the_program_s_own_stays(made):
    """Packed weights that the program has put there (from a file, say) are not written."""
    b, seen = made()
    b.quantise(64)
    own = B.QuantWeights(torch.full_like(b.quant.data, 9), 64, 9, 64)
    for b.quant in (own, own):
        b.backward()
        b.Ws.add_(1.0)
        b.next_words(LAST)
    assert len(_packs(seen)) == 1 and b.quant is own
    b.quantise(64)
    assert len(_packs(seen)) == 2 and b.quant is not own and _packs(seen)[-1][1].data is not own.data
    b.next_words(LAST)
    assert len(_packs(seen)) == 2


def test_a_form_that_is_refused_leaves_the_head(made, monkeypatch):
    b, seen = made()
    b.quantise(64)
    first = b.quant

    def refuse(*a):
        raise B.CavsError(B.ERR_ARG, "refused")
    with monkeypatch.context() as m:
        m.setattr(B, "quant_pack", refuse)
        for form in ((48, False), (64, True)):
            try:
                b.quantise(*form)
            except B.CavsError:
                pass
            else:
                raise AssertionError(form)
            assert b.quant is first
    b.next_words(LAST)
    assert len(_packs(seen)) == 1


def test_what_is_returned_lasts_until_the_next_call(made):
    """As next_words says: one buffer for all calls of as many rows."""
    b, seen = made()
    first = b.next_words(LAST)
    held = (b.logits, b.lse)
    assert b.next_words(LAST) is first and (b.logits, b.lse) == held


def test_the_gradients_that_are_written_are_clipped(made):
    """Those that the program has put into ``grads`` after alloc() too; none that it left out."""
    b, seen = made(max_norm=1.0)
    b.backward()
    listed = b.clip
    b.backward()
    assert b.clip is listed
    b.grads["dWs"] = torch.empty_like(b.grads["dWs"])
    b.grads["dU"] = None
    b.backward()
    name, args, _ = seen[-1]
    assert name == "clip_grads" and args[1] is b.clip and len(args[1].grads) == 5
    assert {id(g) for g in args[1].grads} == {id(g) for k, g in b.grads.items() if k not in ("dX", "dU")}
