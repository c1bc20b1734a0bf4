"""Operators of a transformer block's training step, and the clipping of its gradients, as cases that can be timed.

A case is one pass through one operator, as a training program calls it:

  op = "rotary"      head_norm_rotary: the root-mean-square norm of each query's and key's head and the rotation by
                     its position, in one pass; with "back" its backward pass, whose weight gradients are reduced
                     over all tokens and heads
  op = "attention"   packed_attention: attention of each token to those of its own sequence, causal or not, with
                     query heads that share key heads and sequences of different lengths behind one another; with
                     "back" its gradients as well
  op = "clip"        clip_gradients: the mean of the replicas' flat gradient buffers, the norm over all tensors, each
                     tensor's own, and the mean scaled to a largest norm

Ranges that the cases stand for: 1 to 32,768 tokens with 1 to 32 query heads of 32 to 128 elements, 1 to 16 of
which share a key head, in bf16 or fp32, positions up to a million; attention over 1 to 64 sequences of 0 to 16,384
tokens; 1 to 300 gradient tensors of 1 thousand to 355 million elements in all, 1 to 8 replicas.

With `own` false a pass is made of elementary torch operations in 32 bits, in 64 where 32 lose what matters.
"""
from __future__ import annotations

import math
import random

import torch

own = False

NORM_EPS, CLIP_EPS = 1e-6, 1e-6
BASE = 10000.0
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST_PAIRS = 32 * 128 * 16384 * 16385 // 2  # heads * dim * pairs of tokens of the largest attention


# ------------------------------------------------------------------------------------------------- the cases
def _rotary(name, tokens, heads, kv, dim, dtype, back, first=0, interleaved=False, pad=0):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "dtype": dtype,
            "back": back, "first": first, "interleaved": interleaved, "pad": pad}


def _attention(name, lengths, heads, kv, dim, dtype, back, causal=True):
    return {"name": name, "op": "attention", "lengths": lengths, "heads": heads, "kv": kv, "dim": dim, "dtype": dtype,
            "back": back, "causal": causal}


def _clip(name, n, tensors, g, clips=True):
    return {"name": name, "op": "clip", "n": n, "tensors": tensors, "g": g, "clips": clips}


def listed():
    return [
        # a few tokens of an fp32 run, with neighbouring elements as pairs, far into a text: the call is what counts
        _rotary("rotary_small", 61, 6, 3, 80, "f32", False, first=100003, interleaved=True, pad=5),
        # queries and keys of a GPT-medium-sized block (16 heads of 64) over 8 sequences of 1024 tokens
        _rotary("rotary_forward", 8192, 16, 16, 64, "bf16", False),
        # the backward pass of a larger block: 32 heads of 128 over 8 key heads, 16384 tokens
        _rotary("rotary_backward", 16384, 32, 8, 128, "bf16", True),
        # one short sequence: latency
        _attention("attention_small", "96", 4, 2, 64, "bf16", False),
        # evaluation of a GPT-medium-sized block over 8 sequences of 1024 tokens
        _attention("attention_forward", "1024*8", 16, 16, 64, "bf16", False),
        # its training step: the same with its gradients
        _attention("attention_train", "1024*8", 16, 16, 64, "bf16", True),
        # a training step on one long text, 32 heads of 128 over 8 key heads
        _attention("attention_long", "16384", 32, 8, 128, "bf16", True),
        # documents packed behind one another, of all lengths from none to thousands
        _attention("attention_packed", "1,0,317,1500,63,64,65,2,1031,0,128,129,5,700,411,2048", 12, 4, 80, "bf16", True),
        # an fp32 run of an encoder, not causal
        _attention("attention_f32", "513,700", 6, 6, 64, "f32", True, causal=False),
        # the smallest parameter set of this repository, 4 replicas
        _clip("clip_small", 65536, 1, 4),
        # a ResNet-50's parameters
        _clip("clip_resnet50", 25557032, 161, 4),
        # a GPT-medium's parameters
        _clip("clip_gpt_medium", 354823168, 292, 4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.4)))))))


def _heads(rng):
    share = rng.choice([1, 1, 2, 4, 8, 16])
    kv = rng.randint(1, max(1, 32 // share))
    return kv * share, kv


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "clip"])
    if op == "clip":
        n = _log(rng, 1000, 354823168)
        return {"op": op, "n": n, "tensors": min(n, _log(rng, 1, 300)), "g": rng.choice([1, 2, 3, 4, 4, 8]) if n < 150e6 else
                rng.choice([1, 2, 4]), "clips": rng.random() < 0.8}
    heads, kv = _heads(rng)
    dim, dtype = 8 * rng.randint(4, 16), rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "rotary":
        tokens = min(_log(rng, 1, 32768), 16384 * 40 * 128 // ((heads + kv) * dim * (2 if dtype == "f32" else 1)))
        return {"op": op, "tokens": max(1, tokens), "heads": heads, "kv": kv, "dim": dim, "dtype": dtype,
                "back": rng.random() < 0.6, "first": rng.choice([0, 0, _log(rng, 1, 900000)]),
                "interleaved": rng.random() < 0.3, "pad": rng.choice([0, 0, 8, 13])}
    total, count = _log(rng, 1, 16384), _log(rng, 1, 64)
    cuts = sorted(rng.randint(0, total) for _ in range(count - 1))
    lengths = [b - a for a, b in zip([0] + cuts, cuts + [total])]
    if rng.random() < 0.3:  # a batch of equal ones
        lengths = [max(1, total // count)] * count
    causal, back = rng.random() < 0.8, rng.random() < 0.6
    most = LARGEST_PAIRS // (16 if dtype == "f32" else 1)
    while heads * dim * sum(k * (k + 1) // 2 if causal else k * k for k in lengths) > most:
        lengths = [(k + 1) // 2 for k in lengths]
    return {"op": op, "lengths": ",".join(map(str, lengths)), "heads": heads, "kv": kv, "dim": dim, "dtype": dtype, "back": back,
            "causal": causal}


# ------------------------------------------------------------------------------------------------- the inputs
def _lengths(text):
    out = []
    for part in text.split(","):
        k, _, times = part.partition("*")
        out += [int(k)] * int(times or 1)
    return out


def _tensors(n, count):
    """(start, elements) of `count` tensors that fill n elements: as in networks, half of them are vectors and the
    rest of very different sizes."""
    rng = random.Random(n * 1009 + count)
    share = [rng.uniform(0.2, 1.0) ** 4 + 1e-3 if i % 2 == 0 else 1e-5 for i in range(count)]
    total, at, out = sum(share), 0, []
    for i, s in enumerate(share):
        k = n - at if i == count - 1 else max(1, min(int(n * s / total), n - at - (count - 1 - i)))
        out.append((at, k))
        at += k
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev) * scale

    op = case["op"]
    s = {"case": dict(case)}
    if op == "clip":
        n, g = case["n"], case["g"]
        s["tensors"] = _tensors(n, case["tensors"])
        common = normal(n, scale=1e-3)
        s["grads"] = [normal(n, scale=1e-3).add_(common) for _ in range(g)]
        s["out"] = torch.empty(n, device=dev)
        s["max_norm"] = 1e-3 * math.sqrt(n) * (0.5 if case["clips"] else 4.0)
        return s
    heads, kv, dim, t = case["heads"], case["kv"], case["dim"], TYPES[case["dtype"]]
    if op == "rotary":
        n = case["tokens"]
        # what a projection to queries, keys and values leaves: one row a token
        wide = normal(n, (heads + 2 * kv) * dim + case["pad"])
        wide *= 0.3 + torch.rand(n, 1, generator=gen, device=dev) * 2
        wide = wide.to(t)
        s["q"] = wide[:, :heads * dim].view(n, heads, dim)
        s["k"] = wide[:, heads * dim:(heads + kv) * dim].view(n, kv, dim)
        s["positions"] = torch.arange(n, device=dev) % 8192 + case["first"]
        s["frequencies"] = BASE ** (torch.arange(0, dim, 2, dtype=torch.float64, device=dev) / -dim)
        s["q_weight"], s["k_weight"] = 1 + normal(dim, scale=0.1), 1 + normal(dim, scale=0.1)
        if case["back"]:
            s["dq"], s["dk"] = normal(n, heads, dim, scale=1e-2).to(t), normal(n, kv, dim, scale=1e-2).to(t)
        return s
    lengths = _lengths(case["lengths"])
    n = sum(lengths)
    # the heads of queries and keys have norm sqrt(dim), and a query knows something of the key before its own token
    k = normal(n, kv, dim)
    before = torch.roll(k, 1, 0).repeat_interleave(heads // kv, 1)
    wide = torch.empty(n, (heads + 2 * kv) * dim, dtype=t, device=dev)
    s["q"], s["k"], s["v"] = (wide[:, a * dim:b * dim].view(n, b - a, dim)
                              for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    s["q"].copy_(normal(n, heads, dim, scale=0.8) + 0.6 * before * torch.rand(n, heads, 1, generator=gen, device=dev))
    s["k"].copy_(k)
    s["v"].copy_(normal(n, kv, dim))
    ends = [0]
    for length in lengths:
        ends.append(ends[-1] + length)
    s["lengths"] = lengths
    s["offsets"] = torch.tensor(ends, dtype=torch.int64, device=dev)
    if case["back"]:
        s["dout"] = normal(n, heads, dim, scale=1e-2).to(t)
    return s


# ------------------------------------------------------------------------------------------------- the plain forms
def _pairs(x, interleaved):
    """The two elements of every pair."""
    if interleaved:
        return x[..., 0::2], x[..., 1::2]
    half = x.shape[-1] // 2
    return x[..., :half], x[..., half:]


def _joined(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _plain_rotary(s):
    inter = s["case"]["interleaved"]
    angle = s["positions"].double()[:, None, None] * s["frequencies"]
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {}
    for name in ("q", "k"):
        x, weight = s[name].float(), s[name + "_weight"]
        rstd = (x.square().mean(-1, keepdim=True) + NORM_EPS).rsqrt()
        xhat = x * rstd
        if "dq" not in s:
            a, b = _pairs(xhat * weight, inter)
            out[name] = _joined(a * cos - b * sin, b * cos + a * sin, inter).to(s[name].dtype)
            continue
        a, b = _pairs(s["d" + name].float(), inter)
        dy = _joined(a * cos + b * sin, b * cos - a * sin, inter)
        g = dy * weight
        out["d" + name] = ((g - xhat * (g * xhat).mean(-1, keepdim=True)) * rstd).to(s[name].dtype)
        out["d" + name + "_weight"] = (dy * xhat).sum((0, 1), dtype=torch.float64).float()
    return out


def _plain_attention(s):
    case = s["case"]
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    scale, share, t = 1 / math.sqrt(dim), heads // kv, s["q"].dtype
    n = s["q"].shape[0]
    out = {"out": torch.empty(n, heads, dim, dtype=t, device=s["q"].device),
           "lse": torch.empty(heads, n, dtype=torch.float32, device=s["q"].device)}
    if "dout" in s:
        out["dq"] = torch.empty_like(out["out"])
        out["dk"], out["dv"] = (torch.empty(n, kv, dim, dtype=t, device=s["q"].device) for _ in range(2))
    at = 0
    for length in s["lengths"]:
        if length == 0:
            continue
        cut = slice(at, at + length)
        at += length
        mask = None
        if case["causal"]:
            mask = torch.ones(length, length, dtype=torch.bool, device=s["q"].device).triu_(1)
        # as many key heads at a time as keep the scores below a gigabyte
        each = max(1, min(kv, (1 << 28) // (length * length * share)))
        for h in range(0, kv, each):
            e = min(h + each, kv)
            q = s["q"][cut, h * share:e * share].float().transpose(0, 1).contiguous().view(e - h, share * length, dim)
            k, v = (s[x][cut, h:e].float().transpose(0, 1).contiguous() for x in "kv")
            z = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale).view(e - h, share, length, length)
            if mask is not None:
                z.masked_fill_(mask, -math.inf)
            top = z.amax(-1, keepdim=True)
            p = z.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            p = p.div_(total).view(e - h, share * length, length)
            o = torch.bmm(p, v).view(e - h, share, length, dim)
            out["lse"][h * share:e * share, cut] = (top + total.log()).view((e - h) * share, length)
            out["out"][cut, h * share:e * share] = o.view((e - h) * share, length, dim).transpose(0, 1).to(t)
            if "dout" not in s:
                continue
            do = s["dout"][cut, h * share:e * share].float().transpose(0, 1).contiguous().view(e - h, share * length, dim)
            out["dv"][cut, h:e] = torch.bmm(p.transpose(1, 2).contiguous(), do).transpose(0, 1).to(t)
            dp = torch.bmm(do, v.transpose(1, 2).contiguous())
            ds = dp.sub_((do * o.view_as(do)).sum(-1, keepdim=True)).mul_(p)
            dq = torch.bmm(ds, k).mul_(scale).view((e - h) * share, length, dim)
            out["dq"][cut, h * share:e * share] = dq.transpose(0, 1).to(t)
            out["dk"][cut, h:e] = torch.bmm(ds.transpose(1, 2).contiguous(), q).mul_(scale).transpose(0, 1).to(t)
    return out


def _plain_clip(s):
    mean, out = s["grads"][0], s["out"]
    if len(s["grads"]) > 1:
        mean = mean + s["grads"][1]
        for g in s["grads"][2:]:
            mean += g
        mean /= len(s["grads"])
    squares = torch.stack([mean[a:a + k].square().sum(dtype=torch.float64) for a, k in s["tensors"]])
    norm = squares.sum().sqrt()
    torch.mul(mean, (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0).float(), out=out)
    return {"out": out, "norm": norm.float(), "norms": squares.sqrt().float()}


# ------------------------------------------------------------------------------------------------- a pass
def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"rotary": _plain_rotary, "attention": _plain_attention, "clip": _plain_clip}[op](s)

    import paper_2104_05588_amd as daso

    if op == "rotary":
        how = {"eps": NORM_EPS, "interleaved": s["case"]["interleaved"]}
        if "dq" not in s:
            q, k = daso.head_norm_rotary(s["q"], s["k"], s["positions"], s["frequencies"], s["q_weight"], s["k_weight"], **how)
            return {"q": q, "k": k}
        dq, dk, dqw, dkw = daso.head_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["frequencies"],
                                                          s["q_weight"], s["k_weight"], **how)
        return {"dq": dq, "dq_weight": dqw, "dk": dk, "dk_weight": dkw}
    if op == "attention":
        how = {"offsets": s["offsets"], "causal": s["case"]["causal"]}
        out, lse = daso.packed_attention(s["q"], s["k"], s["v"], **how)
        if "dout" not in s:
            return {"out": out, "lse": lse}
        dq, dk, dv = daso.packed_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, **how)
        return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    norm, norms = daso.clip_gradients(s["grads"], s["max_norm"], s["tensors"], out=s["out"], eps=CLIP_EPS)
    return {"out": s["out"], "norm": norm, "norms": norms}


# ------------------------------------------------------------------------------------------------- what it takes
def work(case):
    op = case["op"]
    if op == "clip":
        return {"bytes": case["n"] * 4 * (case["g"] + 1) + 4 * case["tensors"] + 4, "flops": case["n"] * (case["g"] + 3)}
    heads, kv, dim, e = case["heads"], case["kv"], case["dim"], 2 if case["dtype"] == "bf16" else 4
    if op == "rotary":
        n = case["tokens"]
        elems = n * (heads + kv) * dim
        small = 8 * n + 4 * dim + 8 * dim
        if case["back"]:
            return {"bytes": 3 * elems * e + small + 8 * dim, "flops": 16 * elems}
        return {"bytes": 2 * elems * e + small, "flops": 9 * elems}
    lengths = _lengths(case["lengths"])
    n = sum(lengths)
    pairs = sum(k * (k + 1) // 2 if case["causal"] else k * k for k in lengths)
    row = dim * e
    if not case["back"]:
        return {"bytes": n * (2 * heads + 2 * kv) * row + 4 * n * heads, "flops": 4.0 * heads * dim * pairs}
    return {"bytes": n * (4 * heads + 4 * kv) * row + 4 * n * heads, "flops": 14.0 * heads * dim * pairs}


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        total = s["grads"][0].double()
        for g in s["grads"][1:]:
            total += g
        total /= case["g"]
        norms = torch.stack([torch.linalg.vector_norm(total[a:a + k]) for a, k in s["tensors"]])
        norm = torch.linalg.vector_norm(norms)
        if float(norm) + CLIP_EPS > s["max_norm"]:
            total *= s["max_norm"] / (float(norm) + CLIP_EPS)
        return {"out": total, "norm": norm, "norms": norms}
    if op == "rotary":
        dim = case["dim"]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           s["positions"].double()[:, None, None] * s["frequencies"])

        def as_complex(x):
            x = x.double()
            if case["interleaved"]:
                return torch.view_as_complex(x.reshape(*x.shape[:-1], dim // 2, 2).contiguous())
            return torch.complex(x[..., :dim // 2].contiguous(), x[..., dim // 2:].contiguous())

        def as_real(z):
            return torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat((z.real, z.imag), -1)

        out = {}
        for name in ("q", "k"):
            x, w = s[name].double(), s[name + "_weight"].double()
            size = ((x * x).mean(-1, keepdim=True) + NORM_EPS).sqrt()
            if not case["back"]:
                out[name] = as_real(as_complex(x / size * w) * turn)
                continue
            dy = as_real(as_complex(s["d" + name]) * turn.conj())
            # of x / size: (g - x (g . x) / (dim size^2)) / size
            g = dy * w
            out["d" + name] = (g - x * (g * x).sum(-1, keepdim=True) / (dim * size * size)) / size
            out["d" + name + "_weight"] = (dy * x / size).sum((0, 1))
        return out
    heads, kv, dim, lengths = case["heads"], case["kv"], case["dim"], s["lengths"]
    if heads * dim * sum(k * k for k in lengths) > 2 * LARGEST_PAIRS * 1.01:
        return None
    n, c = sum(lengths), 1 / math.sqrt(dim)
    f = dict(dtype=torch.float64, device="cuda")
    out = {"out": torch.empty(n, heads, dim, **f), "lse": torch.empty(heads, n, **f)}
    if case["back"]:
        out["dq"], out["dk"], out["dv"] = torch.empty(n, heads, dim, **f), torch.zeros(n, kv, dim, **f), torch.zeros(n, kv, dim, **f)
    for h in range(heads):
        of, at = h * kv // heads, 0
        for length in lengths:
            if length == 0:
                continue
            r = slice(at, at + length)
            at += length
            q, k, v = s["q"][r, h].double(), s["k"][r, of].double(), s["v"][r, of].double()
            z = torch.mm(q, k.T) * c
            if case["causal"]:
                z += torch.full_like(z, -math.inf).triu_(1)
            out["lse"][h, r] = torch.logsumexp(z, 1)
            z = torch.softmax(z, 1)
            o = torch.mm(z, v)
            out["out"][r, h] = o
            if case["back"]:
                do = s["dout"][r, h].double()
                out["dv"][r, of] += torch.mm(z.T, do)
                # the softmax's Jacobian: diag(p) - p p^T
                d = torch.mm(do, v.T)
                d = z * (d - (z * d).sum(1, keepdim=True))
                out["dq"][r, h] = torch.mm(d, k) * c
                out["dk"][r, of] += torch.mm(d.T, q) * c
    return out
