"""Plain 64-bit forms of the embedding and the vocabulary head, with bounds on
how far 32-bit sums may be from them.

u = 2^-24 is fp32's half step; a rounding to bf16 is off by at most 2^-8 of the
value (torch.finfo(torch.bfloat16).eps / 2).

* A product summed over n terms in fp32, in any order, the split products' six
  terms each included: at most (2 n + 16) u of the sum of the terms' magnitudes.
* exp(x) of a rounded x: x carries two roundings (the difference, the change of
  base), the instruction one step: relative (2 |x| + 4) 2u.
* Positive sums over the vocabulary: a term passes the additions of its slot of
  64 (fp32) or 128 (bf16) words, 16 or 32 in a lane and two between lanes, then
  one for each slot of its lane of the join, which takes every 64th, and 64 for
  the lanes.  It is multiplied by an exponential (9 u each, their exponents add up
  to the term's own) where the slot is joined from wavefronts, where it joins the
  lane's sum, wherever the largest z grows between groups of eight slots, and
  with the lanes'.  600 u covers all of that up to 900 000 words, and 2^20 where
  the largest z grows in no more than 25 of a lane's 32 groups (test_lm_bounds).
"""
import math

import torch

U = 2.0 ** -24
BF = 2.0 ** -8


def round_to(x, bf):
    return x.bfloat16().double() if bf else x.double()


def embed(E, word, scale):
    X = torch.zeros(word.numel(), E.shape[1], dtype=torch.float64, device=E.device)
    at = torch.nonzero(word >= 0).flatten()
    X[at] = E.double()[word[at].long()] * scale
    return X


def embed_grad(word, dX, n_words, scale, out_bf):
    """dE and its bound."""
    def total(rows):
        out = torch.zeros(n_words, dX.shape[1], dtype=torch.float64, device=dX.device)
        at = word >= 0
        return out.index_add_(0, word[at].long(), rows[at])

    dE = total(dX.double()) * scale
    count = torch.bincount(word[word >= 0].long(), minlength=n_words)[:, None]
    bound = (count + 1) * U * total(dX.double().abs()) * abs(scale)
    return dE, bound + (BF if out_bf else U) * dE.abs()


def teacher(top_word, top_logit, T):
    """q [n, K] and whether a row has a teacher's word."""
    there = (top_word >= 0) & (top_logit != -math.inf)
    t = torch.where(there, top_logit.double() / T, -math.inf)
    some = there.any(1)
    q = torch.zeros_like(t)
    if some.any():
        q[some] = torch.softmax(t[some], 1)
    return q, some


def head(h, Ws, bs=None, label=None, top_word=None, top_logit=None, alpha=0.0, temp=1.0,
         grad=True):
    """Outputs by name and bounds by the same names."""
    wbf, hbf = Ws.dtype == torch.bfloat16, h.dtype == torch.bfloat16
    dev, n, H, C = h.device, h.shape[0], h.shape[1], Ws.shape[1]
    K = 0 if top_word is None else top_word.shape[1]
    if not K:
        alpha, temp = 0.0, 1.0
    x, W = round_to(h, wbf), Ws.double()
    rows = torch.arange(n, device=dev) if label is None else torch.nonzero(label >= 0).flatten()
    nl = rows.numel()
    count = max(1, nl)
    x = x[rows]
    z = x @ W
    ez = (2 * H + 16) * U * (x.abs() @ W.abs()) + U * z.abs()
    if bs is not None:
        z = z + bs.double()
        ez = ez + U * torch.where(torch.isfinite(z), z, 0.0).abs()
    row_loss = torch.zeros(n, dtype=torch.float64, device=dev)
    row_bound = torch.zeros_like(row_loss)
    out, bound = {}, {}
    m = z.amax(1, keepdim=True) if nl else z.sum(1, keepdim=True)
    fin = lambda v: torch.where(torch.isfinite(v), v, 0.0)
    far = fin(z - m).abs()

    def soft(T):
        e = torch.exp((z - m) / T)
        s = e.sum(1, keepdim=True)
        p = e / s
        rel = (2 * far / T + 4) * 2 * U + ez / T     # of exp((z - m) / T), m's own error apart
        rel_s = (p * rel).sum(1, keepdim=True) + 600 * U
        lse = s.log() + m / T
        return p, p * (rel + rel_s + 8 * U), lse, rel_s

    value, vb = torch.zeros(nl, dtype=torch.float64, device=dev), torch.zeros(nl, dtype=torch.float64, device=dev)
    dz, edz = torch.zeros_like(z), torch.zeros_like(z)
    if alpha < 1.0:
        p, ep, lse, rs = soft(1.0)
        y = label[rows].long()[:, None]
        zy = z.gather(1, y)
        value += (1 - alpha) * (lse - zy)[:, 0]
        vb += (1 - alpha) * (rs + ez.gather(1, y) + 4 * U * (fin(zy).abs() + fin(m).abs() + fin(lse).abs()))[:, 0]
        dz += (1 - alpha) * p.scatter_add(1, y, torch.full_like(zy, -1.0))
        edz += (1 - alpha) * (ep + 2 * U * p.scatter_add(1, y, torch.ones_like(zy)))
    if K and alpha > 0.0:
        T = temp
        q, some = teacher(top_word[rows], top_logit[rows], T)
        there = q > 0
        t = torch.where(there, top_logit[rows].double() / T, 0.0)
        p, ep, lse, rs = soft(T)
        at = top_word[rows].long().clamp(min=0)
        zt = torch.where(there, z.gather(1, at), 0.0)
        terms = torch.special.xlogy(q, q) + torch.where(there, q * (lse - zt / T), 0.0)
        value += alpha * T * T * terms.sum(1) * some
        eq = q * ((2 * t.abs().amax(1, keepdim=True) + K + 16) * 4 * U)
        parts = q * ((q.clamp(min=1e-300).log()).abs() + (fin(zt).abs() + fin(m).abs()) / T + fin(lse).abs())
        vb += alpha * T * T * ((2 * K + 16) * U * parts.sum(1) + (q * ez.gather(1, at)).sum(1) / T + rs[:, 0]
                               + (eq * (parts / q.clamp(min=1e-300))).sum(1)) * some
        dz += alpha * T * (p * some[:, None]).scatter_add(1, at, -q)
        edz += alpha * T * (ep + 2 * U * p).scatter_add(1, at, eq + (K + 4) * U * q) * some[:, None]
    row_loss[rows], row_bound[rows] = value, vb + 4 * U * fin(value).abs()
    out["row_loss"], bound["row_loss"] = row_loss, row_bound
    out["loss"] = (row_loss.sum() / count).reshape(1)
    bound["loss"] = (row_bound.sum() / count + 4 * U * fin(row_loss).abs().sum() / count).reshape(1)
    if not grad:
        return out, bound
    dz, edz = dz / count, edz / count
    edz = edz + 4 * U * dz.abs()
    if bs is not None:
        out["dbs"] = dz.sum(0)
        bound["dbs"] = edz.sum(0) + (nl + 16) * U * dz.abs().sum(0)
    if wbf:
        edz = edz + BF * (dz.abs() + edz)
    dh = torch.zeros(n, H, dtype=torch.float64, device=dev)
    bh = torch.zeros_like(dh)
    dh[rows] = dz @ W.t()
    bh[rows] = edz @ W.t().abs() + (2 * C + 16) * U * ((dz.abs() + edz) @ W.t().abs())
    out["dh"], bound["dh"] = dh, bh + (BF if hbf else U) * (dh.abs() + bh)
    dW = x.t() @ dz
    bW = x.t().abs() @ edz + (2 * nl + 16) * U * (x.t().abs() @ (dz.abs() + edz))
    out["dWs"], bound["dWs"] = dW, bW + (BF if wbf else U) * (dW.abs() + bW)
    return out, bound


def outside(got, want, bound):
    """The largest |got - want| / bound (inf where one is not finite and the other is)."""
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    # a denormal's worth of slack where the bound itself is 0
    over = (got - want).abs() / (bound + 1e-38)
    over = torch.where(torch.isnan(over), math.inf, over)
    over = torch.where(same, 0.0, over)
    return float(over.max()) if over.numel() else 0.0
