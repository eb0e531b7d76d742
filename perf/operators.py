"""The operators at the two ends of a language model over this library's
recurrent cells: the embedding that makes the pulled rows and gives its table's
gradient, and the vocabulary head (softmax cross entropy, distillation from a
teacher's top logits) that takes the pushed states and returns their gradient.

Where ``own`` is false, ``run`` computes them from elementary torch operations
in 32 bits; where it is true it makes the calls that a user of the binding
makes.  ``exact`` gives the outputs from the operators' definitions in 64 bits.
"""
import functools
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# A case: op embed (X = scale * table rows), embed_grad (the table's gradient),
# loss (the head's mean and per-row losses), grad (those and every gradient).
#   n words or rows, C words of the vocabulary, D / H columns, type of the
#   tables, rows and their gradients
#   zipf  exponent of the word frequencies: 1.0 is text, 0 spreads them evenly
#   pad   share of the rows that carry no label (padding of a batch's sentences)
#   K     teacher's words per row (0: no teacher), alpha its weight, temp the
#         temperature
#   bias  the head has a bias; some of its words are masked with -inf


def _embed(op, n, C, D, dtype, zipf=1.0, scale=1.0, name=None):
    c = dict(op=op, n=n, C=C, D=D, type=dtype, zipf=zipf, scale=scale)
    return dict(c, name=name) if name else c


def _head(op, n, C, H, dtype, pad=0.0, K=0, alpha=0.0, temp=1.0, bias=True, name=None):
    c = dict(op=op, n=n, C=C, H=H, type=dtype, pad=pad, K=K, alpha=alpha, temp=temp, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decoding step of a small batch: launch and latency.
        _embed("embed", 8, 32000, 512, "bf16", scale=22.627417, name="embed_step"),
        # The words of a training batch of long sentences.
        _embed("embed", 32768, 50001, 1024, "bf16", scale=32.0, name="embed_batch"),
        # The leaves of a batch of parsed sentences, 300-wide word vectors.
        _embed("embed_grad", 4867, 20000, 300, "f32", name="embed_grad_trees"),
        # The same training batch: the most frequent word is thousands of rows.
        _embed("embed_grad", 32768, 50001, 1024, "bf16", scale=32.0, name="embed_grad_batch"),
        # Scoring the next words of a few sentences: the weights are read once for 4 rows.
        _head("loss", 4, 50001, 1024, "bf16", name="ce_score"),
        # Perplexity of the language model that the library's benchmark trains.
        _head("loss", 2275, 10000, 512, "f32", name="ce_eval_lm"),
        # Its training step: fp32, 10 000 words, a loss at every step of 64 sentences.
        _head("grad", 2275, 10000, 512, "f32", name="ce_train_lm"),
        # An ordinary training step in bf16: an odd vocabulary, an eighth of the rows padding.
        _head("grad", 8192, 50001, 1024, "bf16", pad=0.125, name="ce_train_bf16"),
        # The largest: a wide model and a multilingual vocabulary.
        _head("grad", 8192, 128000, 2048, "bf16", bias=False, name="ce_train_large"),
        # A teacher's distribution over a validation set, no gradient.
        _head("loss", 1000, 32000, 512, "f32", K=16, alpha=1.0, temp=2.0, name="distill_eval"),
        # A small fp32 student: label and teacher mixed.
        _head("grad", 777, 10000, 512, "f32", pad=0.1, K=16, alpha=0.5, name="distill_train_lm"),
        # A bf16 student with 64 words a row and a temperature.
        _head("grad", 4096, 32000, 1024, "bf16", pad=0.05, K=64, alpha=0.7, temp=2.0,
              name="distill_train_bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["embed", "embed_grad", "ce", "ce", "distill", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    C = _log(rng, 100, 130000)
    if kind.startswith("embed"):
        return _embed(kind, _log(rng, 1, 65536), C, _log(rng, 64, 2048), dtype,
                      zipf=rng.choice([0.0, 0.7, 1.0]), scale=rng.choice([1.0, 8.0, 27.712813]))
    H = 64 * _log(rng, 1, 32)
    op = rng.choice(["loss", "grad"])
    n = _log(rng, 1, 8192)
    # fp32 and small vocabularies take the ordinary share of the work; no case
    # costs more than the largest listed one
    top = (8192 * 128000 * 2048) // (12 if dtype == "f32" else 1)
    n = max(1, min(n, top // (C * H)))
    pad = rng.choice([0.0, 0.0, 0.3, 0.9])
    bias = rng.random() < 0.7
    if kind == "ce":
        return _head(op, n, C, H, dtype, pad=pad, bias=bias)
    return _head(op, n, C, H, dtype, pad=pad, K=_log(rng, 1, min(100, C)),
                 alpha=round(rng.uniform(0.1, 1.0), 2), temp=rng.choice([1.0, 2.0, 4.0]), bias=bias)


def _words(g, n, C, zipf):
    """Words by rank frequency 1 / rank^zipf, ranks spread over the ids."""
    if zipf == 0.0:
        return torch.randint(0, C, (n,), generator=g, device=DEV, dtype=torch.int64)
    w = torch.arange(1, C + 1, device=DEV, dtype=torch.float64).pow(-zipf).cumsum(0)
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * w[-1]
    rank = torch.searchsorted(w, u).clamp_(max=C - 1)
    return torch.randperm(C, generator=g, device=DEV)[rank]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[case["type"]]
    n, C = case["n"], case["C"]
    s = dict(case=case)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if case["op"] in ("embed", "embed_grad"):
        D = case["D"]
        s["word"] = _words(g, n, C, case["zipf"]).int()
        if n > 16:   # a few padded places
            s["word"][torch.randint(0, n, (max(1, n // 64),), generator=g, device=DEV)] = -1
        s["E"] = (0.05 * randn(C, D)).to(t)
        if case["op"] == "embed":
            s["out"] = torch.empty(n, D, dtype=t, device=DEV)
        else:
            s["dX"] = (0.01 * randn(n, D)).to(t)
            s["out"] = torch.empty(C, D, dtype=t, device=DEV)
        if own:
            B, ctx = _library()
            s["emb"] = B.Embedding(E=s["E"], scale=case["scale"])
            if case["op"] == "embed_grad":
                s["ws"] = _bytes(B.embed_grad_workspace_bytes(s["emb"], n))
        return s

    H, K = case["H"], case["K"]
    s["W"] = (1.0 / math.sqrt(H) * randn(H, C)).to(t)
    s["b"] = 0.1 * randn(C) if case["bias"] else None
    label = _words(g, n, C, 1.0)
    # states of a cell, in (-1, 1): part of the way to their label's column,
    # some rows sure of it and some not
    toward = s["W"][:, label].t().float()
    sure = 6.0 * torch.rand(n, 1, generator=g, device=DEV)
    s["h"] = torch.tanh(0.7 * randn(n, H) + sure * toward).to(t)
    if case["bias"] and C > 64:   # words that may not come, none of them a label
        off = torch.randint(0, C, (C // 64,), generator=g, device=DEV)
        keep = s["b"][label].clone()
        s["b"][off] = -math.inf
        s["b"][label] = keep
    if case["pad"] > 0.0:
        label[torch.rand(n, generator=g, device=DEV) < case["pad"]] = -1
    s["label"] = label.int()
    if K:
        # a teacher's best words: the label among them as a rule, no masked word
        fine = torch.nonzero(torch.isfinite(s["b"])).flatten() if case["bias"] else None
        at = torch.rand(n, K, generator=g, device=DEV).pow_(3)
        N = fine.numel() if fine is not None else C
        # K different places: a stride from a random start, wrapped
        step = max(1, N // max(1, K))
        first = (at[:, :1] * N).long()
        place = (first + step * torch.arange(K, device=DEV)) % N
        top = fine[place] if fine is not None else place
        if K > 1:
            hit = (label >= 0) & ~(top == label[:, None]).any(1)
            top[:, 0] = torch.where(hit, label, top[:, 0])
        logit = (3.0 * randn(n, K)).sort(1, descending=True).values + 2.0
        short = torch.randint(1, K + 1, (n, 1), generator=g, device=DEV)
        some = torch.rand(n, 1, generator=g, device=DEV) < 0.25   # rows that came with fewer words
        top[some & (torch.arange(K, device=DEV) >= short)] = -1
        s["top_word"], s["top_logit"] = top.int().contiguous(), logit.contiguous()
    else:
        s["top_word"] = s["top_logit"] = None
    s["loss"] = torch.empty(1, device=DEV)
    s["row_loss"] = torch.empty(n, device=DEV)
    if case["op"] == "grad":
        s["dh"] = torch.empty(n, H, dtype=t, device=DEV)
        s["dW"] = torch.empty(H, C, dtype=t, device=DEV)
        s["db"] = torch.empty(C, device=DEV) if case["bias"] else None
    if own:
        B, ctx = _library()
        s["head"] = B.VocabHead(h=s["h"], Ws=s["W"], bs=s["b"], label=s["label"],
                                top_word=s["top_word"], top_logit=s["top_logit"],
                                alpha=case["alpha"], temp=case["temp"])
        s["ws"] = _bytes(B.vocab_workspace_bytes(s["head"], case["op"] == "grad"))
    return s


@functools.lru_cache(maxsize=None)
def _library():
    """The binding and a context on the current stream, kept by the program."""
    from paper_1712_04048_amd import binding as B
    return B, B.Context(0)


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "embed":
        return _plain_embed(s["word"], s["E"], c["scale"])
    if c["op"] == "embed_grad":
        return _plain_embed_grad(s["word"], s["dX"], c["scale"], s["E"])
    return _plain_head(s, c["op"] == "grad")


def _run_own(s):
    B, ctx = _library()
    c = s["case"]
    if c["op"] == "embed":
        B.embed(ctx, s["emb"], s["word"], s["out"])
        return s["out"]
    if c["op"] == "embed_grad":
        B.embed_grad(ctx, s["emb"], s["word"], s["dX"], s["out"], s["ws"])
        return s["out"]
    if c["op"] == "loss":
        B.vocab_loss(ctx, s["head"], s["loss"], s["row_loss"], s["ws"])
        return dict(loss=s["loss"], row_loss=s["row_loss"])
    B.vocab_grad(ctx, s["head"], s["loss"], s["row_loss"], s["dh"], s["dW"], s["db"], s["ws"])
    return dict(loss=s["loss"], row_loss=s["row_loss"], dh=s["dh"], dW=s["dW"],
                **({"db": s["db"]} if s["db"] is not None else {}))


# --- plain forms --------------------------------------------------------------


def _plain_embed(word, E, scale):
    w = word.long()
    rows = E[w.clamp(min=0)].float() * scale
    return torch.where((w >= 0)[:, None], rows, 0.0).to(E.dtype)


def _plain_embed_grad(word, dX, scale, E):
    w = word.long()
    seen = (w >= 0)[:, None]
    dE = torch.zeros(E.shape, device=E.device)
    dE.index_add_(0, w.clamp(min=0), torch.where(seen, dX.float(), 0.0))
    return (dE * scale).to(E.dtype)


def _plain_head(s, train):
    c, h, W = s["case"], s["h"].float(), s["W"].float()
    alpha, T = (c["alpha"], c["temp"]) if c["K"] else (0.0, 1.0)
    label = s["label"].long()
    seen = label >= 0
    row = torch.arange(label.numel(), device=DEV)
    count = seen.sum().clamp(min=1).double()
    z = h @ W
    if s["b"] is not None:
        z += s["b"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = label.clamp(min=0)
    value = (1.0 - alpha) * (total.log() + top - z.gather(1, at[:, None]))[:, 0]
    if c["K"]:
        word = s["top_word"].long()
        there = word >= 0
        t = torch.where(there, s["top_logit"] / T, -math.inf)
        best = t.amax(1, keepdim=True)
        some = torch.isfinite(best)
        q = torch.where(there & some, torch.exp(t - torch.where(some, best, 0.0)), 0.0)
        q = q / q.sum(1, keepdim=True).clamp(min=1e-30)
        eT = torch.exp((z - top) / T)
        totalT = eT.sum(1, keepdim=True)
        at_top = z.gather(1, word.clamp(min=0))
        terms = q * (torch.where(q > 0, q, 1.0).log() + (totalT.log() + (top - at_top) / T))
        value = value + alpha * T * T * torch.where(q > 0, terms, 0.0).sum(1)
    value = torch.where(seen, value, 0.0)
    out = dict(loss=(value.double().sum() / count).float().reshape(1), row_loss=value)
    if not train:
        return out
    scale = torch.where(seen, 1.0, 0.0)[:, None] / count.float()
    dz = e.mul_((1.0 - alpha) / total)
    dz[row, at] -= 1.0 - alpha
    if c["K"]:
        dz += eT.mul_(alpha * T * some / totalT)
        dz.scatter_add_(1, word.clamp(min=0), -alpha * T * q)
    dz *= scale
    out["dh"] = (dz @ W.t()).to(s["h"].dtype)
    out["dW"] = (h.t() @ dz).to(s["W"].dtype)
    if s["b"] is not None:
        out["db"] = dz.sum(0)
    return out


# --- what one pass cannot do without ------------------------------------------


def work(case):
    size = 4 if case["type"] == "f32" else 2
    n, C = case["n"], case["C"]
    if case["op"] == "embed":
        return {"bytes": 4 * n + 2 * n * case["D"] * size, "flops": n * case["D"]}
    if case["op"] == "embed_grad":
        return {"bytes": 4 * n + (n + C) * case["D"] * size, "flops": n * case["D"]}
    H, K = case["H"], case["K"]
    seen = n * (1.0 - case["pad"])   # rows without a label need no work
    read = (seen * H + H * C) * size + 4 * n + 8 * seen * K + (4 * C if case["bias"] else 0)
    if case["op"] == "loss":
        return {"bytes": read + 4 * n, "flops": 2.0 * seen * C * H}
    return {"bytes": read + 4 * n + (n * H + H * C) * size + (4 * C if case["bias"] else 0),
            "flops": 6.0 * seen * C * H}


# --- the definitions in 64 bits -----------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        E, w = s["E"].double(), s["word"].long()
        X = torch.zeros(w.numel(), E.shape[1], dtype=torch.float64, device=DEV)
        at = torch.nonzero(w >= 0).flatten()
        X[at] = torch.nn.functional.embedding(w[at], E) * float(case["scale"])
        return X
    if case["op"] == "embed_grad":
        w = s["word"].long()
        at = torch.nonzero(w >= 0).flatten()
        at = at[torch.argsort(w[at], stable=True)]
        word, counts = torch.unique_consecutive(w[at], return_counts=True)
        # each word's sum as a difference of the running sums over sorted rows
        run_ = torch.cumsum(s["dX"][at].double(), 0)
        end = torch.cumsum(counts, 0) - 1
        total = run_[end]
        total[1:] -= run_[end[:-1]]
        dE = torch.zeros(s["E"].shape, dtype=torch.float64, device=DEV)
        dE[word] = total * float(case["scale"])
        return dE
    # The head by automatic differentiation, labelled rows alone, a block at a time.
    F = torch.nn.functional
    n, C, K = case["n"], case["C"], case["K"]
    alpha, T = (case["alpha"], case["temp"]) if K else (0.0, 1.0)
    grad = case["op"] == "grad"
    rows = torch.nonzero(s["label"] >= 0).flatten()
    count = max(1, rows.numel())
    W = s["W"].double().requires_grad_(grad)
    b = s["b"].double().requires_grad_(grad) if s["b"] is not None else None
    row_loss = torch.zeros(n, dtype=torch.float64, device=DEV)
    dh = torch.zeros(s["h"].shape, dtype=torch.float64, device=DEV)
    for part in rows.split(max(1, (1 << 28) // C)):
        h = s["h"][part].double().requires_grad_(grad)
        z = h @ W if b is None else F.linear(h, W.t(), b)
        value = (1.0 - alpha) * F.cross_entropy(z, s["label"][part].long(), reduction="none")
        if K:
            word, logit = s["top_word"][part].long(), s["top_logit"][part].double()
            q = torch.softmax(torch.where(word >= 0, logit / T, -math.inf), 1)
            q = torch.nan_to_num(q)   # rows without a word
            log_p = torch.log_softmax(z / T, 1).gather(1, word.clamp(min=0))
            log_p = torch.where(q > 0, log_p, 0.0)
            value = value + alpha * T * T * (torch.special.xlogy(q, q) - q * log_p).sum(1)
        row_loss[part] = value.detach()
        if grad:
            (value.sum() / count).backward()
            dh[part] = h.grad
    out = dict(loss=(row_loss.sum() / count).reshape(1), row_loss=row_loss)
    if grad:
        out.update(dh=dh, dW=W.grad if W.grad is not None else torch.zeros_like(W).detach())
        if b is not None:
            out["db"] = b.grad if b.grad is not None else torch.zeros_like(b).detach()
    return out
