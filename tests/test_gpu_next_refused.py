"""Calls that the library refuses on the host: the status, nothing enqueued, and the
context as good as before."""
import ctypes as ct
import math

import pytest
import torch

from paper_1712_04048_amd import binding as B

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


@pytest.fixture(scope="module")
def p():
    """An address inside 1 MB of zeros, aligned to 256 bytes."""
    t = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    yield t.data_ptr()
    torch.cuda.synchronize()
    assert not t.any()   # nothing was written


def _quant(p, **kw):
    return B.cavs_quant(**{**dict(H=64, C=20, group=32, shift=0, data=p), **kw})


@pytest.mark.parametrize("status,kw", [
    (B.ERR_ARG, dict(H=0)), (B.ERR_ARG, dict(C=-1)), (B.ERR_ARG, dict(group=48)), (B.ERR_ARG, dict(shift=2)),
    (B.ERR_UNSUPPORTED, dict(H=40000)), (B.ERR_UNSUPPORTED, dict(C=1 << 21)), (B.ERR_ARG, dict(data=None)),
    (B.ERR_ARG, dict(data=8))])
def test_packed_weights(ctx, p, status, kw):
    L = B.lib()
    if kw.get("data") == 8:
        kw = dict(data=p + 8)
    q = _quant(p, **kw)
    if "data" not in kw:
        assert L.cavs_quant_pack(ctx._h, ct.byref(q), 0, p, p) == status
    assert L.cavs_quant_unpack(ctx._h, ct.byref(q), 0, p) == status
    assert L.cavs_quant_product(ctx._h, ct.byref(q), 0, p, 1, None, 0, p + 4096) == status
    assert L.cavs_last_error(ctx._h) != b""


def test_products(ctx, p):
    L, q = B.lib(), _quant(p)

    def call(x_type=0, x=p, n=1, bias=None, y_type=0, y=p + 4096, raw=q):
        return L.cavs_quant_product(ctx._h, ct.byref(raw) if raw is not None else None, x_type, x, n, bias, y_type, y)

    assert call(n=0) == B.OK
    for kw in (dict(x_type=2), dict(y_type=-1), dict(x=None), dict(y=None), dict(x=p + 2), dict(y=p + 1, y_type=1),
               dict(n=-1), dict(bias=p + 2), dict(raw=None)):
        assert call(**kw) == B.ERR_ARG, kw
    assert call(n=(1 << 20) + 1) == B.ERR_UNSUPPORTED
    for kw in (dict(W=None), dict(t=3), dict(W=p + 2), dict(data=None), dict(data=p + 8)):
        a = {**dict(t=0, W=p, data=p), **kw}
        assert L.cavs_quant_pack(ctx._h, ct.byref(q), a["t"], a["W"], a["data"]) == B.ERR_ARG, kw
    assert L.cavs_quant_pack(None, ct.byref(q), 0, p, p) == B.ERR_ARG
    ctx.sync()


def test_rules(ctx, p):
    L = B.lib()

    def call(z=p, out=p + (1 << 18), best=None, lse=None, ws=p + (1 << 19), n_ws=1 << 18, rules=True, **kw):
        r = B.cavs_rules(**{**dict(z_type=0, out_type=0, n=2, C=100), **kw})
        return L.cavs_adjust_logits(ctx._h, ct.byref(r) if rules else None, z, out, best, lse, ws, n_ws)

    assert call(n=0, z=None) == B.OK
    for kw in (dict(rules=False), dict(z_type=2), dict(out_type=-1), dict(n=-1), dict(C=0), dict(L=-1), dict(K=-1),
               dict(M=-1), dict(z=None), dict(out=None), dict(z=p + 2), dict(out=p + 2), dict(out=p, out_type=1),
               dict(L=3, repeat=p), dict(L=3, presence=p), dict(L=3, frequency=p), dict(K=2), dict(K=2, extra=p),
               dict(K=2, extra_word=p), dict(mask=p), dict(mask=p, M=3), dict(mask_row=p), dict(mask=p, mask_row=p),
               dict(C=5000, best=p, ws=p + 8)):
        assert call(**kw) == B.ERR_ARG, kw
    for kw in (dict(n=(1 << 20) + 1), dict(C=(1 << 20) + 1), dict(L=(1 << 20) + 1), dict(K=1025)):
        assert call(**kw) == B.ERR_UNSUPPORTED, kw
    for kw in (dict(ws=None), dict(n_ws=0), dict(n_ws=B.adjust_workspace_bytes(2, 5000) - 1)):
        assert call(C=5000, best=p, **kw) == B.ERR_WORKSPACE, kw
    ctx.sync()


def test_gradients(ctx, p):
    L, need = B.lib(), B.clip_workspace_bytes()
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(count=1, scale=1.0, limit=1.0, norm=p, at=ws.data_ptr(), n_ws=need, listed=True, **kw):
        g = B.cavs_grad(**{**dict(g=p, out=p, n=4, g_type=0, out_type=0), **kw})
        return L.cavs_clip_grads(ctx._h, ct.byref(g) if listed else None, count, scale, limit, norm, at, n_ws)

    for kw in (dict(count=-1), dict(listed=False), dict(scale=math.inf), dict(scale=math.nan), dict(limit=-1.0),
               dict(limit=math.nan), dict(norm=None), dict(g=None), dict(n=-1), dict(g_type=2), dict(out_type=-1),
               dict(g=p + 2), dict(out=p + 2), dict(out_type=1), dict(at=ws.data_ptr() + 4)):
        assert call(**kw) == B.ERR_ARG, kw
    assert call(n=(1 << 32) + 1) == B.ERR_UNSUPPORTED
    for kw in (dict(at=None), dict(n_ws=need - 1)):
        assert call(**kw) == B.ERR_WORKSPACE, kw
    ctx.sync()
