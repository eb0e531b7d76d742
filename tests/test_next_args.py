"""What the head in 4 bits, the rules on logits and the clipping of gradients refuse
before a GPU is reached: the binding's checks of tensors, and size queries of
arguments that the calls refuse (CPU only).  The plain forms that the GPU tests
compare with, against torch's own."""
import ctypes as ct
import math
import os
import subprocess
import tempfile

import pytest
import torch

import next_ref as R
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
  printf("cavs_grad %zu\ncavs_quant %zu\ncavs_rules %zu\n", sizeof(cavs_grad), sizeof(cavs_quant), sizeof(cavs_rules));
  F(cavs_grad, out) F(cavs_grad, n) F(cavs_grad, g_type) F(cavs_grad, out_type)
  F(cavs_quant, C) F(cavs_quant, group) F(cavs_quant, shift) F(cavs_quant, data)
  F(cavs_rules, out_type) F(cavs_rules, C) F(cavs_rules, L) F(cavs_rules, past) F(cavs_rules, repeat)
  F(cavs_rules, presence) F(cavs_rules, frequency) F(cavs_rules, bias) F(cavs_rules, K) F(cavs_rules, extra_word)
  F(cavs_rules, extra) F(cavs_rules, M) F(cavs_rules, mask) F(cavs_rules, mask_row) F(cavs_rules, temp)
  return 0;
}
"""


def test_struct_layouts_match_header():
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "probe.c"), os.path.join(d, "probe")
        open(src, "w").write(PROBE)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.dirname(HEADER), src, "-o", exe])
        out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    for line in out.strip().splitlines():
        key, v = line.split()
        cls = getattr(B, key.split(".")[0])
        assert (getattr(cls, key.split(".")[1]).offset if "." in key else ct.sizeof(cls)) == int(v), key


class _Context:
    torch_device = torch.device("cpu")
    _h = None

    def check(self, status):
        raise AssertionError("the library was called")


def _refused(call):
    with pytest.raises(B.CavsError) as e:
        call()
    assert e.value.status == B.ERR_ARG


@pytest.mark.parametrize("H,C", [(1, 1), (128, 16), (129, 17), (300, 85), (32768, 1 << 20)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shift", [False, True])
def test_bytes_of_packed_weights(H, C, group, shift):
    """As the header lays them out; what the binding expects of a tensor, without the call."""
    _ensure_built()
    blocks = -(-C // 16) * -(-H // 128)
    want = blocks * 1024 + blocks * 16 * (128 // group) * (4 if shift else 2)
    assert B.quant_bytes(H, C, group, shift) == want
    if want < 1 << 20:
        B.QuantWeights(torch.zeros(want, dtype=torch.uint8), H, C, group, shift).raw()
        _refused(lambda: B.QuantWeights(torch.zeros(want + 1, dtype=torch.uint8), H, C, group, shift).raw())


def test_sizes_that_are_refused_have_no_bytes():
    _ensure_built()
    for kw in (dict(H=0), dict(C=0), dict(H=-1), dict(group=16), dict(group=96), dict(group=0), dict(H=32769),
               dict(C=(1 << 20) + 1)):
        assert B.quant_bytes(**{**dict(H=64, C=64), **kw}) == 0, kw
    q = B.cavs_quant(64, 64, 64, 2, None)
    assert B.lib().cavs_quant_bytes(ct.byref(q)) == 0 and B.lib().cavs_quant_bytes(None) == 0
    for n, C, ok in ((1, 1, True), (0, 5, True), (1 << 20, 1 << 20, True), (-1, 5, False), (5, 0, False),
                     ((1 << 20) + 1, 5, False), (5, (1 << 20) + 1, False)):
        assert (B.adjust_workspace_bytes(n, C) > 0) == ok, (n, C)
    assert B.clip_workspace_bytes() > 0


BAD = [None, 3, [0, 1]]


@pytest.mark.parametrize("what", BAD)
def test_arguments_that_are_no_tensors(what):
    _ensure_built()
    c, f = _Context(), dict(dtype=torch.float32)
    q = B.QuantWeights(torch.zeros(B.quant_bytes(64, 10), dtype=torch.uint8), 64, 10)
    x, y, ws = torch.zeros(2, 64, **f), torch.zeros(2, 10, **f), torch.zeros(1 << 18, dtype=torch.uint8)
    W, n1 = torch.zeros(64, 10, **f), torch.zeros(1, **f)
    i = torch.zeros(2, dtype=torch.int32)
    calls = [
        lambda: B.quant_pack(c, B.QuantWeights(what, 64, 10), W), lambda: B.quant_pack(c, q, what),
        lambda: B.quant_unpack(c, q, what), lambda: B.quant_product(c, q, what, y),
        lambda: B.quant_product(c, q, x, what),
        lambda: B.adjust_logits(c, B.LogitRules(), what, y, i, None, ws),
        lambda: B.adjust_logits(c, B.LogitRules(), y, y, i, None, what),
        lambda: B.clip_grads(c, what, 1.0, n1, ws), lambda: B.clip_grads(c, B.GradList([x]), 1.0, what, ws),
        lambda: B.clip_grads(c, B.GradList([x]), 1.0, n1, what), lambda: B.GradList([x, what]),
    ]
    if what is not None:   # None leaves these out
        calls += [lambda: B.quant_product(c, q, x, y, bias=what),
                  lambda: B.adjust_logits(c, B.LogitRules(), y, what, i, None, ws),
                  lambda: B.adjust_logits(c, B.LogitRules(), y, y, what, None, ws),
                  lambda: B.adjust_logits(c, B.LogitRules(), y, y, i, what, ws), lambda: B.GradList([x], [what])]
        calls += [lambda k=k: B.LogitRules(**{**dict(past=torch.zeros(2, 3, dtype=torch.int32)), k: what}).raw(2, 10, 0, 0)
                  for k in ("bias", "past", "repeat", "presence", "frequency", "extra_word", "extra", "mask", "mask_row",
                            "temp")]
    for call in calls:
        _refused(call)


F, I = torch.zeros, lambda *s: torch.zeros(*s, dtype=torch.int32)


@pytest.mark.parametrize("kw", [
    dict(bias=F(9)), dict(bias=F(10).bfloat16()), dict(past=I(3, 4)), dict(past=I(2)), dict(past=F(2, 4)),
    dict(past=I(4, 2).t()), dict(repeat=F(2)), dict(presence=F(2)), dict(frequency=F(2)),
    dict(past=I(2, 4), repeat=F(3)), dict(past=I(2, 4), repeat=F(2, 1)), dict(past=I(2, 4), frequency=F(2).double()),
    dict(extra_word=I(2, 3)), dict(extra=F(2, 3)), dict(extra_word=I(2, 3), extra=F(2, 4)),
    dict(extra_word=I(2, 3).long(), extra=F(2, 3)), dict(mask=I(2)), dict(mask=I(2, 2)), dict(mask=F(2, 1)),
    dict(mask=I(2, 1), mask_row=I(3)), dict(mask=I(2, 1), mask_row=F(2)), dict(temp=F(1)), dict(temp=F(2).bfloat16()),
])
def test_rules_tensors_are_checked(kw):
    _refused(lambda: B.LogitRules(**kw).raw(2, 10, 0, 0))


@pytest.mark.parametrize("kw", [
    dict(x=F(2, 63)), dict(x=F(64)), dict(x=F(2, 64).half()), dict(x=F(64, 2).t()), dict(y=F(2, 11)), dict(y=F(3, 10)),
    dict(y=F(2, 10).double()), dict(bias=F(9)), dict(bias=F(10).bfloat16()),
])
def test_product_tensors_are_checked(kw):
    _ensure_built()
    q = B.QuantWeights(torch.zeros(B.quant_bytes(64, 10), dtype=torch.uint8), 64, 10)
    a = {**dict(x=F(2, 64), y=F(2, 10), bias=None), **kw}
    _refused(lambda: B.quant_product(_Context(), q, a["x"], a["y"], bias=a["bias"]))


def test_gradient_lists_are_checked():
    g = [F(3, 4), F(5).bfloat16()]
    assert [r.n for r in B.GradList(g).raw] == [12, 5]
    for bad in ([F(3, 4)], [F(4, 3), F(5)], [F(3, 4), F(5).half()], [F(4, 3).t(), F(5)], [F(3, 4), F(6)]):
        _refused(lambda: B.GradList(g, bad))
    _refused(lambda: B.GradList([F(4, 3).t()]))
    _refused(lambda: B.GradList([g[0], g[1], g[0]]))
    _refused(lambda: B.GradList(g[:1] * 2, [g[0], g[0]]))
    B.GradList(g[:1] * 2, [g[0], None])
    _refused(lambda: B.GradList([I(3)]))
    _refused(lambda: B.GradList([F(3), torch.zeros(3, device="meta")]))


# --- the plain forms ----------------------------------------------------------


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shift", [False, True])
def test_rounding_is_to_the_nearest_of_sixteen(group, shift):
    """No level of the group is closer to a weight than its own, but where its range ends."""
    g = torch.Generator().manual_seed(group)
    W = torch.randn(150, 9, generator=g)
    q, s, m = R.quantise(W, group, shift)
    What = R.weights(q, s, m, group)
    rep = lambda a: a.repeat_interleave(group, 0)[:150]
    levels = rep(s)[..., None] * torch.arange(-8, 8, dtype=torch.float64) + rep(m)[..., None]
    best = (levels - W.double()[..., None]).abs().amin(-1)
    assert ((What - W.double()).abs() <= best + 1e-15).all()
    # within half a step of it inside the range, a step (the scale's rounding) outside
    assert ((What - W.double()).abs() <= rep(s).abs() * 1.1).all()


def test_norm_and_clipping_are_torch_s():
    g = torch.Generator().manual_seed(1)
    p = [torch.nn.Parameter(torch.zeros(s, dtype=torch.float64)) for s in ((3, 4), (7,))]
    for x in p:
        x.grad = torch.randn(x.shape, generator=g, dtype=torch.float64)
    norm, _, out = R.clip([x.grad for x in p], 1.0, 0.5, [torch.float32] * 2)
    total = torch.nn.utils.clip_grad_norm_(p, 0.5)
    assert abs(norm - float(total)) < 1e-12
    for x, (w, _) in zip(p, out):
        assert (x.grad - w).abs().max() < 3e-6   # torch adds 1e-6 to the norm


def test_rules_in_a_small_case_by_hand():
    z = torch.tensor([[2.0, -1.0, 0.5, 3.0]])
    v, _ = R.rules(z, past=torch.tensor([[0, 1, 1, -1]], dtype=torch.int32), repeat=torch.tensor([2.0]),
                   presence=torch.tensor([0.25]), frequency=torch.tensor([0.5]), bias=torch.tensor([0.0, 0.0, 1.0, 0.0]),
                   extra_word=torch.tensor([[2, 2]], dtype=torch.int32), extra=torch.tensor([[1.0, 2.0]]),
                   mask=torch.tensor([[0b0111]], dtype=torch.int32), temp=torch.tensor([0.5]))
    assert v.tolist() == [[2 * (1 - 0.25 - 0.5), 2 * (-2 - 0.25 - 1.0), 2 * 4.5, -math.inf]]
    want, _ = R.lse(v, torch.zeros_like(v))
    assert abs(float(want) - math.log(sum(math.exp(x) for x in v[0].tolist()))) < 1e-12


def test_packed_weights_are_read_by_the_header_s_words():
    """A layout written by hand: word 17, row 141 of 200 x 20, in groups of 64 with shifts."""
    H, C, group = 200, 20, 64
    data = torch.zeros(B.quant_bytes(H, C, group, True), dtype=torch.uint8)
    block = 1 * 2 + 1                                  # word 17: tile 1 of 2; row 141: block 1 of 2
    k = 141 - 128                                      # 13: dword 0, lane group 1, i = 5: nibble 6
    data[block * 1024 + (16 * 1 + 1) * 16 + 3] = 0x0b   # nibble 6 is byte 3, low half
    at = 4 * 1024 + 2 * (((block * 16 + 1) * 2 + 0) * 2)
    data[at:at + 4] = torch.tensor([1.5, -2.0], dtype=torch.bfloat16).view(torch.uint8)
    q, s, m = R.from_data(data, H, C, group, True)
    assert q[141, 17] == 3 and (q == -8).sum() == q.numel() - 1 and k == 13
    assert s[2, 17] == 1.5 and m[2, 17] == -2.0
