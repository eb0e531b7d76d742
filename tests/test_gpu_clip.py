"""The gradients' norm and clipping on the GPU against their 64-bit form."""
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


def _call(ctx, grads, limit, out=None, scale=1.0):
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = torch.full((B.clip_workspace_bytes(),), 255, dtype=torch.uint8, device="cuda")
    B.clip_grads(ctx, B.GradList(grads, out), limit, norm, ws, scale=scale)
    ctx.sync()
    return norm


SIZES = {
    "one": [1], "few": [7, 0, 8, 1, 9], "odd": [8191, 8192, 8193, 3, 100001], "large": [3000001, 5],
    "many": [(37 * k) % 501 for k in range(500)], "same": [4096] * 121, "set": [10] * 160, "sets": [5000] * 321,
}
THOUSANDS = [(k % 7) * (k % 3) for k in range(4000)] + [4099, 1] * 1500 + [0] * 50 + [20000]


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("limit,scale", [(1.0, 1.0), (math.inf, 0.125), (1e9, 1.0), (0.5, -3.0), (0.0, 1.0)])
def test_clipped(ctx, sizes, types, limit, scale):
    g = torch.Generator(device="cuda").manual_seed(len(sizes))
    grads = [(10.0 ** (k % 5 - 3) * torch.randn(n, generator=g, device="cuda")).to(types[0])
             for k, n in enumerate(SIZES[sizes])]
    kept = [x.clone() for x in grads]
    want, nb, outs = R.clip(grads, scale, limit, [types[1]] * len(grads))
    for _ in range(2):
        out = [torch.full(x.shape, float("nan"), dtype=types[1], device="cuda") for x in grads]
        norm = _call(ctx, grads, limit, out, scale)
        assert abs(float(norm) - want) <= nb
        for o, (w, b) in zip(out, outs):
            assert R.outside(o, w, b) <= 1.0
        assert all(torch.equal(x, y) for x, y in zip(grads, kept))
    if types[0] == types[1]:
        again = _call(ctx, grads, limit, scale=scale)
        assert torch.equal(again, norm) and all(torch.equal(x, y) for x, y in zip(grads, out))


def test_more_gradients_than_a_table_holds(ctx):
    flat = torch.randn(sum(THOUSANDS), generator=torch.Generator().manual_seed(2)).cuda()
    grads, kept = list(flat.split(THOUSANDS)), flat.clone()
    out = torch.full_like(flat, float("nan"))
    norm = _call(ctx, grads, 2.0, list(out.split(THOUSANDS)))
    want, nb, [(w, b)] = R.clip([kept], 1.0, 2.0, [F32])
    assert abs(float(norm) - want) <= nb and R.outside(out, w, b) <= 1.0 and torch.equal(flat, kept)
    assert torch.equal(_call(ctx, grads, 2.0), norm) and torch.equal(flat, out)


def test_shapes_types_and_places_together(ctx):
    """A list of both types, some in place, some written elsewhere, some only counted,
    beginning at any element of an allocation; what lies beside them stays."""
    g = torch.Generator().manual_seed(3)
    grads, out, room = [], [], []
    for k in range(40):
        t = (F32, BF16)[k % 2]
        n = [1, 17, 333, 9000, 40000][k % 5]
        r = torch.full((n + 16,), 9.0, dtype=t, device="cuda")
        x = r[k % 8:k % 8 + n]
        x.copy_(torch.randn(n, generator=g))
        grads.append(x)
        room.append((r, k % 8, n))
        if k % 3 == 0:
            out.append(x)
        elif k % 3 == 1:
            out.append(None)
        else:
            r = torch.full((n + 16,), 9.0, dtype=(BF16, F32)[k % 4 // 2], device="cuda")
            room.append((r, k % 5, n))
            out.append(r[k % 5:k % 5 + n])
    kept = [x.clone() for x in grads]
    want, nb, outs = R.clip(grads, 1.0, 2.0, [F32 if o is None else o.dtype for o in out])
    norm = _call(ctx, grads, 2.0, out)
    assert abs(float(norm) - want) <= nb
    for x, y, o, (w, b) in zip(grads, kept, out, outs):
        if o is None or o is not x:
            assert torch.equal(x, y)
        if o is not None:
            assert R.outside(o, w, b) <= 1.0
    for r, off, n in room:
        assert (r[:off] == 9.0).all() and (r[off + n:] == 9.0).all()


def test_nothing_to_clip(ctx):
    assert float(_call(ctx, [], 1.0)) == 0.0
    z = torch.zeros(1000, device="cuda")
    assert float(_call(ctx, [z], 1.0)) == 0.0 and not z.any()
    assert float(_call(ctx, [torch.empty(0, device="cuda")], 0.0)) == 0.0


def test_squares_beyond_fp32(ctx):
    """Gradients whose squares fp32 cannot hold, at both ends."""
    for v in (1e30, 3e38, 1e-30, 2.0 ** -149):
        x = torch.full((5000,), v, device="cuda")
        y = torch.empty_like(x)
        norm = _call(ctx, [x], 1.0, [y])
        true = float(x[0].double()) * math.sqrt(5000)
        if true < torch.finfo(F32).max:
            assert abs(float(norm) - true) <= 2 * R.U * true + 2.0 ** -149
        else:
            assert float(norm) == math.inf   # as a float; it still clips
        f = min(1.0, 1.0 / true)
        assert (y.double() - x.double() * f).abs().max() <= 3 * R.U * float(x[0]) * f + 2.0 ** -149


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_clips_nothing(ctx, bad):
    x, y = torch.randn(3000, device="cuda"), torch.randn(50000, device="cuda")
    y[49999] = bad
    kept = [x.clone(), y.clone()]
    norm = _call(ctx, [x, y], 1.0)
    assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
    assert torch.equal(x, kept[0]) and torch.equal(y[:49999], kept[1][:49999])
    out = [torch.empty_like(x), torch.empty_like(y)]
    _call(ctx, [x, y], 1.0, out, scale=2.0)
    assert torch.equal(out[0], 2 * x)


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (BF16, F32)])
def test_many_elements_at_odd_places(ctx, types):
    """Enough of them that they are written past the caches, from any element on."""
    g = torch.Generator(device="cuda").manual_seed(9)
    n = [5000001, 17, 4000003]
    for off in (0, 1, 3):
        src = torch.randn(sum(n) + off, generator=g, device="cuda").to(types[0])
        room = torch.full((sum(n) + off + 8,), 9.0, dtype=types[1], device="cuda")
        grads, out = list(src[off:].split(n)), list(room[off:off + sum(n)].split(n))
        want, nb, outs = R.clip(grads, 1.0, 2.0, [types[1]] * 3)
        norm = _call(ctx, grads, 2.0, out)
        assert abs(float(norm) - want) <= nb
        for o, (w, b) in zip(out, outs):
            assert R.outside(o, w, b) <= 1.0
        assert (room[:off] == 9.0).all() and (room[off + sum(n):] == 9.0).all()
