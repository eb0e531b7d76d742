"""Plain 64-bit forms of the head in 4 bits, of the rules on logits and of the
gradients' norm and clipping, with bounds on how far 32-bit sums may be from them.

u = 2^-24 is fp32's half step; a rounding to bf16 is off by at most 2^-8 of the
value (torch.finfo(torch.bfloat16).eps / 2).

* The 4-bit product: x, scaled so that its block's largest value is at least 2^14, is
  a half, or the sum of two, 2^-23 of it (2 u) away at most, or half of a half's smallest
  step (2^-24): 2^-39 of the block's largest value.  A product of a half and a code is exact;
  of H terms each passes at most H additions in fp32 and two multiplications (the group's
  scale; the powers of two are exact), and with a shift the same again, of |m x|:
  (2 H + 16) u of the sum of the terms' magnitudes, as for any fp32 product.
* Rules: each step is one rounding of a value no larger than the magnitudes'
  sum; nine steps and K additions of a word's extras at most.
* ln sum exp: v's bound, as ln sum exp moves no more than its largest argument;
  exp of a rounded x: (2 |x| + 4) 2 u of each term, averaged by the terms; 16 terms
  of a thread, 6 additions in a wavefront, up to 16 parts in a lane of the join and 6
  additions there, each part scaled once (9 u): 64 u; the logarithm 4 u of its value,
  the last sum u.
* Norm and clipping: sums in 64 bits (2^-53 times the number of terms at most,
  2^-23 of the value at 2^30 of them, far less than that in pairs: u covers it) and one
  rounding; the factor's rounding, the product's, and that to bf16.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
BF = 2.0 ** -8


def quantise(W, group, shift):
    """Codes [H, C] in -8 .. 7, scales and shifts [groups, C], 64 bits."""
    W = W.double()
    q, S, M = [], [], []
    for w in W.split(group):
        lo, hi = w.amin(0), w.amax(0)
        if shift:
            s = ((hi - lo) / 15).float().bfloat16().double()
            m = ((hi + lo + s) / 2).float().bfloat16().double()
        else:
            s = (-torch.where(hi > -lo, hi, lo) / 8).float().bfloat16().double()
            m = torch.zeros_like(s)
        bad = ~torch.isfinite(w).all(0)
        s[bad], m[bad] = math.nan, 0.0
        t = torch.round((w - m) / s).clamp(-8, 7)
        q.append(torch.where((s == 0) | bad, 0.0, t))
        S.append(s)
        M.append(m)
    return torch.cat(q), torch.stack(S), torch.stack(M)


def weights(q, s, m, group):
    H = q.shape[0]
    rep = lambda a: a.repeat_interleave(group, 0)[:H]
    return rep(s) * q + rep(m)


def from_data(data, H, C, group, shift):
    """Codes, scales and shifts read from packed weights by the header's words."""
    raw = data.cpu().numpy()
    T, KB, sub = -(-C // 16), -(-H // 128), 128 // group
    code = raw[:T * KB * 1024]
    k, c = np.meshgrid(np.arange(KB * 128), np.arange(T * 16), indexing="ij")
    i = k % 8
    p = np.where(i % 2 == 0, i // 2, 4 + i // 2)
    at = ((c // 16) * KB + k // 128) * 1024 + (16 * (k // 8 % 4) + c % 16) * 16 + (k // 32 % 4) * 4 + p // 2
    q = (code[at] >> (4 * (p % 2))) & 15
    rest = torch.from_numpy(raw[T * KB * 1024:].copy()).view(torch.bfloat16).double()
    rest = rest.view(T, KB, 16, sub, 2 if shift else 1).permute(1, 3, 0, 2, 4).reshape(KB * sub, T * 16, -1)
    return (torch.from_numpy(q.astype(np.float64)) - 8, rest[..., 0],
            rest[..., 1] if shift else torch.zeros_like(rest[..., 0]))


def product(x, q, s, m, group, bias, out_bf):
    """y and its bound."""
    H = x.shape[1]
    W, x = weights(q, s, m, group), x.double()
    y = x @ W
    rep = lambda a: a.repeat_interleave(group, 0)[:H]
    big = (rep(s) * q).abs() + rep(m).abs()
    bound = (2 * H + 16) * U * (x.abs() @ big)
    top = torch.cat([b.abs().amax(1, keepdim=True).expand_as(b) for b in x.split(128, 1)], 1)
    bound += 2.0 ** -39 * (top @ big)
    if bias is not None:
        y = y + bias.double()
        bound = bound + U * y.abs()
    return y, bound + (BF if out_bf else U) * y.abs()


def rules(z, bias=None, past=None, repeat=None, presence=None, frequency=None, extra_word=None, extra=None,
          mask=None, mask_row=None, temp=None):
    """v [n, C], its bound before it is stored, and a lambda for lse's bound."""
    n, C = z.shape
    v = z.double().clone()
    mag = v.abs()
    K = 0
    col = lambda a: a.double()[:, None]
    if past is not None:
        k = torch.zeros(n, C + 1, dtype=torch.float64, device=z.device)
        ok = (past >= 0) & (past < C)
        k.scatter_add_(1, torch.where(ok, past.long(), C), torch.ones_like(past, dtype=torch.float64))
        k = k[:, :C]
        said = k > 0
        if repeat is not None:
            r = col(repeat)
            v = torch.where(said, torch.where(v > 0, v / r, v * r), v)
            mag = torch.maximum(mag, v.abs())
        if presence is not None:
            v = torch.where(said, v - col(presence), v)
            mag = mag + col(presence).abs()
        if frequency is not None:
            v = v - col(frequency) * k
            mag = mag + col(frequency).abs() * k
    if bias is not None:
        v = v + bias.double()
        mag = mag + torch.where(torch.isfinite(bias), bias, 0.0).double().abs()
    if extra_word is not None:
        K = extra_word.shape[1]
        row, at = torch.nonzero((extra_word >= 0) & (extra_word < C), as_tuple=True)
        w = extra_word[row, at].long()
        add = torch.zeros_like(v)
        add.index_put_((row, w), extra[row, at].double(), accumulate=True)
        v = v + add
        mag.index_put_((row, w), extra[row, at].double().abs(), accumulate=True)
    if mask is not None:
        M = mask.shape[0]
        state = (mask_row.long() if mask_row is not None else
                 torch.zeros(n, dtype=torch.long, device=z.device) if M == 1 else torch.arange(n, device=z.device))
        c = torch.arange(C, device=z.device)
        allowed = (mask.long()[:, c // 32] >> (c % 32)) & 1 == 1
        free = (state < 0) | (state >= M)
        v = torch.where(allowed[torch.where(free, 0, state)] | free[:, None], v, -math.inf)
    if temp is not None:
        v, mag = v / col(temp), mag / col(temp)
    bound = (9 + K) * U * mag
    return v, torch.where(torch.isfinite(v), bound, 0.0)


def lse(v, bound):
    want = torch.logsumexp(v, 1)
    x = (v - want[:, None])
    p = torch.where(torch.isfinite(v), torch.exp(x), 0.0)
    top = v.amax(1, keepdim=True)
    far = torch.where(p > 0, (v - top).abs(), 0.0)
    return want, bound.amax(1) + ((2 * far + 4) * 2 * U * p).sum(1) + 64 * U + 5 * U * want.abs() + \
        4 * U * torch.log(torch.exp(want[:, None] - top)).abs()[:, 0]


def clip(grads, scale, limit, types):
    """The norm, its bound, and each output with its bound."""
    norm = abs(scale) * math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    f = scale * (limit / norm if norm > limit and math.isfinite(norm) else 1.0)
    out = []
    for g, t in zip(grads, types):
        o = g.double() * f
        out.append((o, (3 * U + (BF if t == torch.bfloat16 else 0.0)) * o.abs() + 2.0 ** -149 * (1 + (
            2.0 ** 15 if t == torch.bfloat16 else 0))))
    return norm, 2 * U * norm, out


def outside(got, want, bound):
    """The largest share of its bound that an element is off by; 0 / 0 is 0."""
    got = got.double().to(want.device)
    fine = torch.isfinite(want)
    if not torch.equal(torch.isnan(got), torch.isnan(want)):
        return math.inf
    if not torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]):
        return math.inf
    d = (got - want).abs()[fine]
    b = bound.to(want.device).expand_as(want)[fine]
    return float(torch.where(d == 0, 0.0, d / b).max()) if d.numel() else 0.0
