"""More operators around a language model of this library's cells: the head in
4 bits that scores the next words of a few sentences (its weights' rounding and
its product), the rules that decide which word may come next (penalties, biases,
grammar masks, temperature), and the gradient's norm and clipping that end a
training step.

Where ``own`` is false, ``run`` computes them from elementary torch operations
in 32 bits (64 where a rounding to whole numbers or a long sum needs them); where
it is true it makes the calls that a user of the binding makes.  ``exact`` gives
the outputs from the operators' definitions in 64 bits.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}

# A case: op pack (weights to 4 bits and back: what the rounding leaves of them),
# product (y = x What + bias), rules (logits to what the next word is drawn from),
# clip (norm of all gradients, and the clipped ones).
#   n rows, H rows and C words of the head, type of weights / rows / logits /
#   gradients and out of what is written
#   group  weights that share a scale, shift whether they share a shift as well
#   L words so far, K words with a bias of their own, per row; masks a table's rows
#   past, dense, temp  whether there are penalties, a bias of every word, a temperature
#   shapes of the gradients ("512x2048 2048"), clip: whether they are clipped


def _pack(H, C, dtype, group, shift, name=None):
    c = dict(op="pack", H=H, C=C, type=dtype, group=group, shift=shift)
    return dict(c, name=name) if name else c


def _product(n, H, C, dtype, out, group, shift, bias=True, name=None):
    c = dict(op="product", n=n, H=H, C=C, type=dtype, out=out, group=group, shift=shift, bias=bias)
    return dict(c, name=name) if name else c


def _rules(n, C, dtype, out, L=0, past="", K=0, dense=False, masks=0, temp=False, pick=True, name=None):
    c = dict(op="rules", n=n, C=C, type=dtype, out=out, L=L, past=past, K=K, dense=dense, masks=masks,
             temp=temp, pick=pick)
    return dict(c, name=name) if name else c


def _clip(shapes, dtype, out, clip=True, scale=1.0, name=None):
    c = dict(op="clip", shapes=shapes, type=dtype, out=out, clip=clip, scale=scale)
    return dict(c, name=name) if name else c


def _many(rng, count, total):
    """`count` sizes that add up to about `total`, from one element on."""
    part = [math.exp(rng.uniform(0.0, 5.0)) for _ in range(count)]
    return " ".join(str(max(1, int(total * p / sum(part)))) for p in part)


def listed():
    return [
        # The benchmark language model's head, once after its training.
        _pack(512, 10000, "f32", 128, False, name="pack_lm"),
        # A wider bf16 head of an odd vocabulary, small groups with a shift.
        _pack(1024, 50001, "bf16", 64, True, name="pack_wide"),
        # The next word of one sentence: launch and latency.
        _product(1, 512, 10000, "bf16", "bf16", 128, False, name="head_one"),
        # The next words of the benchmark's batch of 64 sentences, its fp32 states.
        _product(64, 512, 10000, "f32", "f32", 128, False, name="head_batch"),
        # Four sentences, an odd vocabulary, groups with a shift.
        _product(4, 1024, 50001, "bf16", "f32", 64, True, name="head_few"),
        # The largest: sixteen beams of a wide model and a multilingual vocabulary.
        _product(16, 2048, 128000, "bf16", "f32", 128, False, bias=False, name="head_large"),
        # One sentence: what it has said so far, and a temperature.
        _rules(1, 10000, "f32", "f32", L=40, past="r", temp=True, name="rules_one"),
        # A batch with long histories, every penalty, biases of some words and of all.
        _rules(64, 50001, "f32", "f32", L=512, past="rpf", K=16, dense=True, temp=True,
               name="rules_batch"),
        # Structured output: each sentence in a state of a grammar, one of them without a way on.
        _rules(256, 128000, "bf16", "bf16", L=100, past="pf", masks=24, name="rules_grammar"),
        # The gradients of the benchmark language model, in fp32.
        _clip("512x2048 512x2048 2048 512x10000 10000 10000x512", "f32", "f32", name="clip_lm"),
        # Many small tensors of odd sizes, bf16 gradients to fp32 ones for an optimiser.
        _clip(_many(random.Random(1), 300, 2000000), "bf16", "f32", scale=0.125, name="clip_many"),
        # A wide bf16 model with a large table and head.
        _clip("50001x1024 1024x4096 1024x4096 4096 1024x50001 50001", "bf16", "bf16", name="clip_large"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["pack", "product", "product", "rules", "rules", "clip", "clip"])
    dtype, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    group, shift = rng.choice([32, 64, 128]), rng.random() < 0.5
    C = _log(rng, 100, 130000)
    if kind == "pack":
        most = 1024 * 50001 // (C * SIZE[dtype] // 2)
        return _pack(min(_log(rng, 64, 4096), most), C, dtype, group, shift)
    if kind == "product":
        H = _log(rng, 64, 4096)
        C = min(C, 2048 * 128000 // H)
        n = min(_log(rng, 1, 64), max(1, 16 * 2048 * 128000 // (H * C)))
        return _product(n, H, C, dtype, out, group, shift, bias=rng.random() < 0.7)
    if kind == "rules":
        n = min(_log(rng, 1, 512), 256 * 128000 // (2 * C))
        past = "".join(k for k in "rpf" if rng.random() < 0.6)
        return _rules(n, C, dtype, out, L=_log(rng, 1, 4096) if past else 0, past=past,
                      K=rng.choice([0, 0, 1, _log(rng, 1, 64)]), dense=rng.random() < 0.4,
                      masks=rng.choice([0, 0, 1, _log(rng, 1, 64)]), temp=rng.random() < 0.6,
                      pick=rng.random() < 0.8)
    count = _log(rng, 1, 300)
    return _clip(_many(rng, count, _log(rng, 1000, 50000000)), dtype, out, clip=rng.random() < 0.8,
                 scale=rng.choice([1.0, 0.125, 3.0]))


def _shapes(case):
    return [tuple(int(k) for k in s.split("x")) for s in case["shapes"].split()]


def _zipf(g, shape, C):
    """Words by rank frequency 1 / rank, ranks spread over the ids."""
    u = torch.rand(*shape, generator=g, device=DEV, dtype=torch.float64)
    rank = (torch.exp(u * math.log(C + 1.0)) - 1.0).long().clamp_(max=C - 1)
    return torch.randperm(C, generator=g, device=DEV)[rank]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = TYPES[case["type"]]
    to = TYPES[case["out"]] if "out" in case else t
    s = dict(case=case)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(*shape, generator=g, device=DEV)

    if case["op"] in ("pack", "product"):
        H, C = case["H"], case["C"]
        # columns of words that came often are longer
        W = (1.0 / math.sqrt(H) * randn(H, C) * uniform(0.5, 2.0, C)).to(t)
        if case["op"] == "pack":
            s["W"], s["out"] = W, torch.empty_like(W)
        else:
            n = case["n"]
            s["x"] = torch.tanh(1.2 * randn(n, H)).to(t)   # states of a cell
            s["b"] = 0.1 * randn(C) if case["bias"] else None
            s["y"] = torch.empty(n, C, dtype=to, device=DEV)
        if own:
            B, ctx = _library()
            s["q"] = B.QuantWeights(_bytes(B.quant_bytes(H, C, case["group"], case["shift"])), H, C,
                                    group=case["group"], shift=case["shift"])
            if case["op"] == "product":
                B.quant_pack(ctx, s["q"], W)
        elif case["op"] == "product":
            s["code"], s["scale"], s["shift"] = _plain_pack(W, case["group"], case["shift"])
        return s

    if case["op"] == "rules":
        n, C, L, K, M = case["n"], case["C"], case["L"], case["K"], case["masks"]
        z = 2.0 * randn(n, C)
        if C > 32:   # a few likely words a row
            z.scatter_add_(1, torch.randint(0, C, (n, 8), generator=g, device=DEV), uniform(4.0, 10.0, n, 8))
        s["z"] = z.to(t)
        del z
        s["past"] = s["repeat"] = s["presence"] = s["frequency"] = None
        if L:
            # text so far, many of its words likely to come again; rows of other
            # lengths are filled up with -1
            past = _zipf(g, (n, L), C)
            likely = s["z"].float().topk(min(4, C), 1).indices
            again = torch.randint(0, likely.shape[1], (n, L), generator=g, device=DEV)
            past = torch.where(uniform(0.0, 1.0, n, L) < 0.05, likely.gather(1, again), past)
            length = torch.randint(0, L + 1, (n, 1), generator=g, device=DEV)
            length[0] = L
            s["past"] = torch.where(torch.arange(L, device=DEV) < length, past, -1).int().contiguous()
            if "r" in case["past"]:
                s["repeat"] = uniform(1.0, 1.5, n)
            if "p" in case["past"]:
                s["presence"] = uniform(0.0, 1.0, n)
            if "f" in case["past"]:
                s["frequency"] = uniform(0.0, 0.5, n)
        s["bias"] = 0.5 * randn(C) if case["dense"] else None
        s["word"] = s["extra"] = None
        if K:
            s["word"] = torch.randint(-1, C, (n, K), generator=g, device=DEV).int()
            s["extra"] = 4.0 * randn(n, K)
        s["mask"] = s["mask_row"] = None
        if M:
            # states that allow a share of the words, from a few to all but a few;
            # the first allows none
            share = uniform(-9.0, 3.0, M, 1).sigmoid()
            bits = uniform(0.0, 1.0, M, C) < share
            bits[0] = False
            s["mask"] = _pack_bits(bits)
            s["mask_row"] = torch.randint(-1, M, (n,), generator=g, device=DEV).int()
            s["mask_row"][n // 2] = 0
        s["temp"] = uniform(0.5, 1.5, n) if case["temp"] else None
        s["out"] = torch.empty(n, C, dtype=to, device=DEV)
        s["best"] = torch.empty(n, dtype=torch.int32, device=DEV) if case["pick"] else None
        s["lse"] = torch.empty(n, device=DEV) if case["pick"] else None
        if own:
            B, ctx = _library()
            s["rules"] = B.LogitRules(
                bias=s["bias"], past=s["past"], repeat=s["repeat"], presence=s["presence"],
                frequency=s["frequency"], extra_word=s["word"], extra=s["extra"], mask=s["mask"],
                mask_row=s["mask_row"], temp=s["temp"])
            s["ws"] = _bytes(B.adjust_workspace_bytes(n, C))
        return s

    # gradients of very different magnitudes, one tensor to the next
    s["g"] = [(10.0 ** float(k % 5 - 3) * randn(*shape)).to(t) for k, shape in enumerate(_shapes(case))]
    if len(s["g"]) > 16:   # one after the other in a buffer that an optimiser takes whole
        s["flat"] = torch.empty(sum(x.numel() for x in s["g"]), dtype=to, device=DEV)
        s["out"] = [o.view(x.shape) for o, x in zip(s["flat"].split([x.numel() for x in s["g"]]), s["g"])]
    else:
        s["out"] = [torch.empty(x.shape, dtype=to, device=DEV) for x in s["g"]]
    s["norm"] = torch.empty(1, device=DEV)
    # a norm that is mostly above the limit, as it is in training
    s["limit"] = 1.0 if case["clip"] else math.inf
    if own:
        B, ctx = _library()
        s["grads"] = B.GradList(s["g"], s["out"])
        s["ws"] = _bytes(B.clip_workspace_bytes())
    return s


@functools.lru_cache(maxsize=None)
def _library():
    """The binding and a context on the current stream, kept by the program."""
    from paper_1712_04048_amd import binding as B
    return B, B.Context(0)


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def _pack_bits(bits):
    """[M, C] truth values as int32 [M, ceil(C / 32)], word c in bit c % 32."""
    M, C = bits.shape
    full = torch.zeros(M, -(-C // 32) * 32, dtype=torch.int64, device=DEV)
    full[:, :C] = bits
    v = (full.view(M, -1, 32) << torch.arange(32, device=DEV)).sum(2)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).int()


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    return dict(pack=_plain_round, product=_plain_product, rules=_plain_rules, clip=_plain_clip)[op](s)


def _run_own(s):
    B, ctx = _library()
    c = s["case"]
    if c["op"] == "pack":
        B.quant_pack(ctx, s["q"], s["W"])
        B.quant_unpack(ctx, s["q"], s["out"])
        return s["out"]
    if c["op"] == "product":
        B.quant_product(ctx, s["q"], s["x"], s["y"], bias=s["b"])
        return s["y"]
    if c["op"] == "rules":
        B.adjust_logits(ctx, s["rules"], s["z"], s["out"], s["best"], s["lse"], s["ws"])
        return dict(out=s["out"], **(dict(best=s["best"], lse=s["lse"]) if c["pick"] else {}))
    B.clip_grads(ctx, s["grads"], s["limit"], s["norm"], s["ws"], scale=c["scale"])
    return dict(norm=s["norm"], out=s.get("flat", s["out"]))


# --- plain forms --------------------------------------------------------------


def _plain_pack(W, G, shift):
    """Codes [H, C] (0 .. 15), scales and shifts [groups, C] (bf16)."""
    H, C = W.shape
    code, scales, shifts = [], [], []
    for part in W.split(max(1, (1 << 26) // H), 1):
        P = -(-H // G) * G
        w = torch.cat([part, part[-1:].expand(P - H, -1)]).view(P // G, G, -1)
        lo, hi = w.amin(1).double(), w.amax(1).double()
        if shift:
            s = ((hi - lo) / 15.0).float().bfloat16()
            m = (0.5 * (lo + hi) + 0.5 * s.double()).float().bfloat16()
        else:
            s = (-0.125 * torch.where(hi > -lo, hi, lo)).float().bfloat16()
            m = torch.zeros_like(s)
        sd, md = s.double()[:, None], m.double()[:, None]
        q = torch.round((w.double() - md) / torch.where(sd == 0, 1.0, sd)).clamp_(-8, 7)
        q = torch.where(sd == 0, 0.0, q)
        code.append((q + 8).to(torch.uint8).view(P, -1)[:H])
        scales.append(s)
        shifts.append(m)
    return (torch.cat(code, 1).contiguous(), torch.cat(scales, 1).contiguous(),
            torch.cat(shifts, 1).contiguous() if shift else None)


def _plain_weights(code, scale, shift, G):
    H = code.shape[0]
    W = (code.float() - 8.0) * scale.float().repeat_interleave(G, 0)[:H]
    return W if shift is None else W + shift.float().repeat_interleave(G, 0)[:H]


def _plain_round(s):
    c = s["case"]
    return _plain_weights(*_plain_pack(s["W"], c["group"], c["shift"]), c["group"]).to(s["W"].dtype)


def _plain_product(s):
    y = s["x"].float() @ _plain_weights(s["code"], s["scale"], s["shift"], s["case"]["group"])
    if s["b"] is not None:
        y += s["b"]
    return y.to(s["y"].dtype)


def _plain_rules(s):
    c = s["case"]
    n, C = c["n"], c["C"]
    v = s["z"].float()
    if s["past"] is not None:
        word = s["past"].long()
        count = torch.zeros(n, C + 1, device=DEV)
        count.scatter_add_(1, torch.where(word < 0, C, word), torch.ones(1, device=DEV).expand(n, c["L"]))
        count = count[:, :C]
        said = count > 0
        if s["repeat"] is not None:
            r = s["repeat"][:, None]
            v = torch.where(said, torch.where(v > 0, v / r, v * r), v)
        if s["presence"] is not None:
            v = torch.where(said, v - s["presence"][:, None], v)
        if s["frequency"] is not None:
            v = v - s["frequency"][:, None] * count
    if s["bias"] is not None:
        v = v + s["bias"]
    if s["word"] is not None:
        word = s["word"].long()
        extra = torch.zeros(n, C + 1, device=DEV)
        row = torch.arange(n, device=DEV)
        for k in range(c["K"]):   # a word listed twice: in the list's order
            extra[row, torch.where(word[:, k] < 0, C, word[:, k])] += s["extra"][:, k]
        v = v + extra[:, :C]
    if s["mask"] is not None:
        shift = torch.arange(32, device=DEV, dtype=torch.int32)
        allowed = ((s["mask"][:, :, None] >> shift) & 1).bool().view(s["mask"].shape[0], -1)[:, :C]
        state = s["mask_row"].long()
        ok = allowed[state.clamp(min=0)] | (state < 0)[:, None]
        v = torch.where(ok, v, -math.inf)
    if s["temp"] is not None:
        v = v / s["temp"][:, None]
    out = dict(out=v.to(s["out"].dtype))
    if c["pick"]:
        top = v.amax(1, keepdim=True)
        none = top == -math.inf
        place = torch.where(v == top, torch.arange(C, device=DEV), C).amin(1)
        out["best"] = torch.where(none[:, 0], -1, place).int()
        total = torch.exp(v - torch.where(none, 0.0, top)).sum(1)
        out["lse"] = total.log() + top[:, 0]
    return out


def _plain_clip(s):
    c = s["case"]
    total = sum((x.double() ** 2).sum() for x in s["g"])
    norm = abs(c["scale"]) * total.sqrt()
    coef = (c["scale"] * (s["limit"] / norm).clamp(max=1.0)).float()
    for x, o in zip(s["g"], s["out"]):
        o.copy_(x.float() * coef)
    return dict(norm=norm.float().reshape(1), out=s.get("flat", s["out"]))


# --- what one pass cannot do without ------------------------------------------


def work(case):
    size = SIZE[case["type"]]
    if case["op"] in ("pack", "product"):
        H, C = case["H"], case["C"]
        packed = 0.5 * H * C + 2 * -(-H // case["group"]) * C * (2 if case["shift"] else 1)
        if case["op"] == "pack":
            return {"bytes": 2 * H * C * size + 2 * packed, "flops": 4.0 * H * C}
        n = case["n"]
        return {"bytes": packed + n * H * size + n * C * SIZE[case["out"]] + (4 * C if case["bias"] else 0),
                "flops": 2.0 * n * H * C}
    if case["op"] == "rules":
        n, C = case["n"], case["C"]
        used = min(case["masks"], n)
        row = 4 * case["L"] + 8 * case["K"] + 4 * len(case["past"]) + (4 if case["masks"] else 0) + \
            (4 if case["temp"] else 0) + (8 if case["pick"] else 0)
        return {"bytes": n * C * (size + SIZE[case["out"]]) + n * row + (4 * C if case["dense"] else 0) +
                used * C / 8, "flops": 4.0 * n * C}
    count = sum(math.prod(shape) for shape in _shapes(case))
    return {"bytes": count * (size + SIZE[case["out"]]) + 4, "flops": 3.0 * count}


# --- the definitions in 64 bits -----------------------------------------------


def _exact_weights(W, G, shift):
    """What 4 bits leave of W, group after group, in 64 bits."""
    H = W.shape[0]
    What = torch.empty(W.shape, dtype=torch.float64, device=DEV)
    levels = torch.arange(-8, 8, dtype=torch.float64, device=DEV)
    for at in range(0, H, G):
        w = W[at:at + G].double()
        lo, hi = w.min(0).values, w.max(0).values
        if shift:
            s = ((hi - lo) / 15.0).float().bfloat16().double()
            m = ((lo + hi + s) / 2.0).float().bfloat16().double()
        else:
            s = (torch.where(hi + lo > 0, hi, lo) / -8.0).float().bfloat16().double()
            m = torch.zeros_like(s)
        # the even neighbour where a weight is half way
        q = torch.zeros_like(w)
        some = s != 0
        q[:, some] = ((w - m)[:, some] / s[some]).round()
        q = torch.minimum(torch.maximum(q, levels[0]), levels[-1])
        What[at:at + G] = torch.addcmul(m, q, s)
    return What


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pack":
        return _exact_weights(s["W"], case["group"], case["shift"])
    if case["op"] == "product":
        # the weights as prepare made them, before they were rounded
        g = torch.Generator(device=DEV).manual_seed(seed)
        H, C = case["H"], case["C"]
        W = 1.0 / math.sqrt(H) * torch.randn(H, C, generator=g, device=DEV)
        W = (W * (0.5 + 1.5 * torch.rand(C, generator=g, device=DEV))).to(TYPES[case["type"]])
        y = []
        for part in W.split(max(1, (1 << 26) // H), 1):
            y.append(s["x"].double() @ _exact_weights(part, case["group"], case["shift"]))
        y = torch.cat(y, 1)
        return y if s["b"] is None else y + s["b"].double()
    if case["op"] == "rules":
        n, C = case["n"], case["C"]
        v = s["z"].double()
        if case["L"]:
            row, at = torch.nonzero(s["past"] >= 0, as_tuple=True)
            flat, times = torch.unique(row * C + s["past"][row, at].long(), return_counts=True)
            row, word = flat // C, flat % C
            x = v[row, word]
            if s["repeat"] is not None:
                r = s["repeat"].double()[row]
                x = torch.where(x > 0, x / r, x * r)
            if s["presence"] is not None:
                x = x - s["presence"].double()[row]
            if s["frequency"] is not None:
                x = x - s["frequency"].double()[row] * times
            v[row, word] = x
        if s["bias"] is not None:
            v += s["bias"].double()
        if case["K"]:
            row, at = torch.nonzero(s["word"] >= 0, as_tuple=True)
            v.index_put_((row, s["word"][row, at].long()), s["extra"][row, at].double(), accumulate=True)
        if case["masks"]:
            c = torch.arange(C, device=DEV)
            for i, state in enumerate(s["mask_row"].tolist()):
                if state >= 0:
                    word = s["mask"][state].long()[c // 32]
                    v[i, (word >> (c % 32)) % 2 == 0] = -math.inf
        if s["temp"] is not None:
            v /= s["temp"].double()[:, None]
        out = dict(out=v)
        if case["pick"]:
            top, place = v.max(1)
            first = torch.nonzero(v == top[:, None])   # row after row, words ascending
            place = place.scatter_reduce(0, first[:, 0], first[:, 1], "amin", include_self=False)
            out["best"] = torch.where(top == -math.inf, -1, place).int()
            out["lse"] = torch.logsumexp(v, 1)
        return out
    norm = abs(case["scale"]) * torch.stack([torch.linalg.vector_norm(x.double()) for x in s["g"]]).norm()
    coef = case["scale"] * (1.0 if s["limit"] == math.inf else torch.clamp(s["limit"] / norm, max=1.0))
    out = [x.double() * coef for x in s["g"]]
    return dict(norm=norm.reshape(1), out=torch.cat([x.flatten() for x in out]) if "flat" in s else out)
