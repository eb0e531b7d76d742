"""The rules on logits on the GPU against their 64-bit form."""
import math

import pytest
import torch

import next_ref as R
from paper_1712_04048_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


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


def _call(ctx, rules, z, out_type=F32, inplace=False, pick=True):
    n, C = z.shape
    nan = float("nan")
    out = z if inplace else torch.full((n, C), nan, dtype=out_type, device="cuda")
    best = torch.full((n,), -77, dtype=torch.int32, device="cuda") if pick else None
    lse = torch.full((n,), nan, device="cuda") if pick else None
    ws = torch.full((max(1, B.adjust_workspace_bytes(n, C)),), 255, dtype=torch.uint8, device="cuda")
    B.adjust_logits(ctx, B.LogitRules(**rules), z, out, best, lse, ws)
    ctx.sync()
    return out, best, lse


def _check(ctx, z, rules, out_type=F32):
    want, bound = R.rules(z, **rules)
    out, best, lse = _call(ctx, rules, z, out_type)
    store = (R.BF if out_type == BF16 else 0.0) * torch.where(torch.isfinite(want), want, 0.0).abs()
    assert R.outside(out, want, bound + store) <= 1.0
    # the best word's v is the largest, but for the bounds of the two
    top = want.amax(1)
    none = top == -math.inf
    assert torch.equal(best < 0, none)
    at = best.clamp(min=0).long()[:, None]
    short = top - want.gather(1, at)[:, 0]
    assert (short[~none] <= (2 * bound.amax(1))[~none]).all()
    w, b = R.lse(want, bound)
    assert R.outside(lse, w, b) <= 1.0
    # none of it changes from run to run, nor with what is asked for
    again = _call(ctx, rules, z, out_type)
    assert torch.equal(again[0], out) and torch.equal(again[1], best) and torch.equal(again[2], lse)
    assert torch.equal(_call(ctx, rules, z, out_type, pick=False)[0], out)
    if z.dtype == out_type:
        kept = z.clone()
        o, p, q = _call(ctx, rules, kept, inplace=True)
        assert torch.equal(o, out) and torch.equal(p, best) and torch.equal(q, lse)


def _rules(g, n, C, kinds, L=30, K=5, M=3):
    r = lambda *s: torch.rand(*s, generator=g)
    words = lambda *s: torch.randint(-1, C, s, generator=g).int()
    d = {}
    if set(kinds) & set("rpf"):
        d["past"] = torch.where(r(n, L) < 0.3, words(n, 1), words(n, L))
    if "r" in kinds:
        d["repeat"] = 0.5 + r(n)
    if "p" in kinds:
        d["presence"] = r(n) - 0.3
    if "f" in kinds:
        d["frequency"] = r(n) - 0.3
    if "b" in kinds:
        d["bias"] = torch.randn(C, generator=g)
        d["bias"][::7] = -math.inf
    if "e" in kinds:
        d["extra_word"], d["extra"] = words(n, K), 3 * torch.randn(n, K, generator=g)
    if "m" in kinds:
        d["mask"] = torch.randint(-2 ** 31, 2 ** 31, (M, -(-C // 32)), generator=g).int()
        d["mask"][0] = 0
        d["mask_row"] = torch.randint(-1, M, (n,), generator=g).int()
    if "t" in kinds:
        d["temp"] = 0.2 + r(n)
    return {k: v.cuda() for k, v in d.items()}


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("kinds", ["", "r", "p", "f", "b", "e", "m", "t", "rpf", "rpfbemt"])
@pytest.mark.parametrize("n,C", [(1, 1), (3, 7), (2, 33), (5, 4096), (4, 4097), (3, 10000), (2, 16384), (2, 16385),
                                 (7, 50001)])
def test_rules(ctx, n, C, kinds, types):
    g = torch.Generator().manual_seed(n * C + len(kinds))
    z = (3 * torch.randn(n, C, generator=g)).to(types[0]).cuda()
    _check(ctx, z, _rules(g, n, C, kinds), types[1])


@pytest.mark.parametrize("L", [1, 2, 255, 257, 5000])
def test_pasts_of_any_length(ctx, L):
    g = torch.Generator().manual_seed(L)
    z = torch.randn(4, 9000, generator=g).cuda()
    rules = _rules(g, 4, 9000, "rpf", L=L)
    rules["past"][1] = -1              # nothing said so far
    rules["past"][2] = 8999            # one word, L times
    _check(ctx, z, rules)


def test_an_empty_past(ctx):
    g = torch.Generator().manual_seed(9)
    z = torch.randn(3, 100, generator=g).cuda()
    e = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    rules = dict(past=e, repeat=torch.full((3,), 2.0, device="cuda"), extra_word=e, extra=torch.empty(3, 0, device="cuda"))
    assert torch.equal(_call(ctx, rules, z)[0], z)


@pytest.mark.parametrize("K", [1, 300, 1024])
def test_words_listed_more_than_once_add_up(ctx, K):
    g = torch.Generator().manual_seed(K)
    z = torch.randn(3, 6000, generator=g).cuda()
    rules = _rules(g, 3, 6000, "e", K=K)
    rules["extra_word"][0, :] = 5999
    rules["extra_word"][1] %= 40
    _check(ctx, z, rules)


def test_one_mask_for_all_and_one_for_each(ctx):
    g = torch.Generator().manual_seed(11)
    z = torch.randn(5, 1000, generator=g).cuda()
    for M in (1, 5):
        mask = torch.randint(-2 ** 31, 2 ** 31, (M, 32), generator=g).int().cuda()
        _check(ctx, z, dict(mask=mask))


def test_first_of_the_largest(ctx):
    """Equal values at the ends of a thread's, a wavefront's and a workgroup's words."""
    for C, places in ((20000, (8, 7, 19999)), (20000, (4096, 4095 + 1)), (70001, (70000, 65536)), (512, (511, 504, 8)),
                      (100000, (99999, 0)), (9000, (8191, 8000))):
        z = torch.full((2, C), -1.0, device="cuda")
        z[0, list(places)] = 2.0
        out, best, _ = _call(ctx, {}, z)
        assert best.tolist() == [min(places), 0]


def test_rows_with_nothing_left(ctx):
    """Every word masked, every logit -inf, masked infinities and NaN."""
    C = 5000
    z = torch.zeros(6, C, device="cuda")
    z[1] = -math.inf
    z[2, 17], z[3, 4999], z[4, 4500] = math.nan, math.nan, math.inf
    z[5, 1] = math.inf
    mask = torch.full((6, -(-C // 32)), -1, dtype=torch.int32, device="cuda")
    mask[0] = 0
    mask[2, 0] = -1 & ~(1 << 17)
    out, best, lse = _call(ctx, dict(mask=mask), z)
    assert best.tolist() == [-1, -1, 0, 0, 4500, 1]
    assert lse[0] == -math.inf and lse[1] == -math.inf and torch.isnan(lse[3])
    assert lse[4] == math.inf and lse[5] == math.inf
    assert abs(float(lse[2]) - math.log(C - 1)) < 64 * R.U + 5 * R.U * math.log(C)
    assert (out[0] == -math.inf).all() and out[2, 17] == -math.inf and torch.isnan(out[3, 4999])
    z[:] = math.nan
    out, best, lse = _call(ctx, {}, z)
    assert (best == -1).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("field", ["past", "extra_word", "mask_row"])
@pytest.mark.parametrize("bad", [9000, -2, 2 ** 31 - 1, -2 ** 31])
def test_words_out_of_range_count_as_none(ctx, field, bad):
    g = torch.Generator().manual_seed(12)
    z = torch.randn(4, 9000, generator=g).cuda()
    rules = _rules(g, 4, 9000, "rpfem")
    if rules[field].dim() == 2:
        rules[field][2, 3] = bad
    else:
        rules[field][2] = bad
    with pytest.raises(B.CavsError) as e:
        _call(ctx, rules, z)
    assert e.value.status == B.ERR_RANGE
    fine = dict(rules)
    fine[field] = torch.where(rules[field] == bad, -1, rules[field])
    out = torch.empty_like(z)
    ws = torch.empty(B.adjust_workspace_bytes(4, 9000), dtype=torch.uint8, device="cuda")
    B.adjust_logits(ctx, B.LogitRules(**rules), z, out, None, None, ws)
    with pytest.raises(B.CavsError):
        ctx.sync()
    assert torch.equal(out, _call(ctx, fine, z)[0])


def test_only_what_is_asked_for(ctx):
    g = torch.Generator().manual_seed(13)
    z = torch.randn(3, 40000, generator=g).cuda()
    ws = torch.empty(B.adjust_workspace_bytes(3, 40000), dtype=torch.uint8, device="cuda")
    kept = z.clone()
    _, best, lse = _call(ctx, {}, z)
    b, l = torch.empty_like(best), torch.empty_like(lse)
    B.adjust_logits(ctx, B.LogitRules(), z, None, b, None, ws)
    B.adjust_logits(ctx, B.LogitRules(), z, None, None, l, ws)
    ctx.sync()
    assert torch.equal(b, best) and torch.equal(l, lse) and torch.equal(z, kept)


def test_logits_inside_an_allocation(ctx):
    g = torch.Generator().manual_seed(14)
    for t in (F32, BF16):
        for off in (1, 2, 3, 5):
            z = torch.empty(3 * 777 + off, dtype=t, device="cuda")[off:].view(3, 777)
            z.copy_(torch.randn(3, 777, generator=g))
            bias = torch.randn(777 + off, generator=g).cuda()[off:]
            room = torch.full((3 * 777 + off + 9,), 3.0, dtype=t, device="cuda")
            out = room[off:off + 3 * 777].view(3, 777)
            ws = torch.empty(B.adjust_workspace_bytes(3, 777), dtype=torch.uint8, device="cuda")
            B.adjust_logits(ctx, B.LogitRules(bias=bias), z, out, None, None, ws)
            ctx.sync()
            assert torch.equal(out, (z.float() + bias).to(t))
            assert (room[:off] == 3.0).all() and (room[off + 3 * 777:] == 3.0).all()


def test_no_rows(ctx):
    z = torch.empty(0, 50, device="cuda")
    _call(ctx, {}, z)


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_many_logits_at_odd_places(ctx, types):
    """Enough of them that they are written past the caches: the same bits as row by row."""
    g = torch.Generator(device="cuda").manual_seed(15)
    n, C, off = 41, 420001, 1
    src = torch.randn(n * C + off, generator=g, device="cuda").to(types[0])
    z = src[off:].view(n, C)
    room = torch.full((n * C + off + 8,), 9.0, dtype=types[1], device="cuda")
    out = room[off:off + n * C].view(n, C)
    cpu = torch.Generator().manual_seed(15)
    rules = _rules(cpu, n, C, "rpfbemt")
    ws = torch.empty(B.adjust_workspace_bytes(n, C), dtype=torch.uint8, device="cuda")
    best, lse = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    B.adjust_logits(ctx, B.LogitRules(**rules), z, out, best, lse, ws)
    ctx.sync()
    assert (room[:off] == 9.0).all() and (room[off + n * C:] == 9.0).all()
    for i in (0, 1, 20, n - 1):
        one = {k: v if k in ("bias", "mask") else v[i:i + 1] for k, v in rules.items()}
        o, b, l = _call(ctx, one, z[i:i + 1].contiguous(), types[1])
        assert torch.equal(o[0], out[i]) and torch.equal(b[0], best[i])
        assert abs(float(l) - float(lse[i])) <= 128 * R.U * (1 + abs(float(l)))   # other pieces, other sums
