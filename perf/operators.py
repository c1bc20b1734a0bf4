"""Operators of a language model's training step around the synchronisation, as cases that can be timed.

A case is one pass through one operator, as a training program calls it:

  op = "norm"         layer_norm over rows (forward), and with "back" layer_norm_backward, whose weight
                      and bias gradients are reduced over all rows
  op = "loss"         linear_cross_entropy: the loss of an output projection over a large vocabulary, whose
                      logits are never kept; with "back" its gradients as well
  op = "orthogonal"   orthogonalize: Newton-Schulz products on a batch of matrices
  op = "muon"         muon_step: replica gradients averaged, momentum, orthogonalised update, parameters and
                      their bf16 form for the exchange, over the matrices of a flat parameter buffer

Ranges that the cases stand for: norms of 1 to 65,536 rows of 33 to 8192 elements in bf16 or fp32; losses of 1 to
8192 tokens over 100 to 50,257 classes with 32 to 2048 features in bf16 or fp32, up to half of the tokens
ignored; 1 to 24 matrices of 24 to 4096 rows and columns; steps over 1 to 150 matrices with 1 to 8 replicas.

With `own` false a pass is made of elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # the quintic that is in common use for this
NS_STEPS, NS_EPS = 5, 1e-7
LR, MU, DECAY = 0.02, 0.95, 0.01
IGNORE = -100
NORM_EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------- the cases
def _norm(name, rows, d, dtype, back, bias=True, pad=0):
    return {"name": name, "op": "norm", "rows": rows, "d": d, "dtype": dtype, "back": back, "bias": bias, "pad": pad}


def _loss(name, tokens, vocab, d, dtype, grad, back, ignored=0.0):
    return {"name": name, "op": "loss", "tokens": tokens, "vocab": vocab, "d": d, "dtype": dtype, "grad": grad,
            "back": back, "ignored": ignored}


def _orthogonal(name, batch, rows, cols, dtype):
    return {"name": name, "op": "orthogonal", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def _muon(name, shapes, g, nesterov=True):
    return {"name": name, "op": "muon", "shapes": shapes, "g": g, "nesterov": nesterov}


def listed():
    return [
        # a few rows of a small batch: the call itself is what counts
        _norm("norm_small", 64, 1024, "bf16", False),
        # one norm of a GPT-medium-sized block over 8 sequences of 1024 tokens, forward
        _norm("norm_forward", 8192, 1024, "bf16", False),
        # the same norm's backward pass over a larger batch
        _norm("norm_backward", 32768, 1024, "bf16", True),
        # an fp32 run with odd sizes, rows that lie in a wider buffer and no bias
        _norm("norm_backward_odd", 5003, 1601, "f32", True, bias=False, pad=7),
        # a classifier's head (1000 classes on 2048 features) over one batch
        _loss("loss_classifier", 256, 1000, 2048, "bf16", "bf16", True),
        # evaluation over GPT-medium's vocabulary: the loss alone
        _loss("loss_evaluate", 4096, 50257, 1024, "bf16", "bf16", False),
        # its training step; the weight's gradient goes into an fp32 gradient buffer, some tokens are padding
        _loss("loss_train", 8192, 50257, 1024, "bf16", "f32", True, ignored=0.1),
        # an fp32 run over a mid-sized vocabulary, odd in every size
        _loss("loss_train_f32", 1531, 10007, 515, "f32", "f32", True, ignored=0.3),
        # one small convolution's update (64 filters over 64 channels of 3x3)
        _orthogonal("orthogonal_small", 1, 64, 576, "bf16"),
        # one large square matrix
        _orthogonal("orthogonal_large", 1, 4096, 4096, "bf16"),
        # the 3x3 and 1x1 convolutions of a ResNet-50's last two stages as matrices, 4 replicas
        _muon("muon_convolutions", "256x2304*6,1024x256*6,256x1024*5,512x4608*3,2048x512*3,512x2048*2,2048x1024*1", 4),
        # every hidden matrix of a GPT-medium: 4 square ones and the two of the 4d-wide MLP in each of 24 blocks
        _muon("muon_gpt_medium", "1024x1024*96,4096x1024*24,1024x4096*24", 4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.4)))))))


def _size(rng, lo, hi, multiple):
    """A size of the range, over its logarithm: half the time a multiple of `multiple`, else any."""
    k = _log(rng, lo, hi)
    if rng.random() < 0.5:
        k = max(multiple, k // multiple * multiple)
    return max(lo, min(hi, k))


def draw(rng):
    op = rng.choice(["norm", "loss", "loss", "orthogonal", "muon"])
    if op == "norm":
        rows, d = _log(rng, 1, 65536), _size(rng, 33, 8192, 64)
        rows = max(1, min(rows, (32768 * 1024) // d))
        return {"op": op, "rows": rows, "d": d, "dtype": rng.choice(["bf16", "bf16", "f32"]), "back": rng.random() < 0.6,
                "bias": rng.random() < 0.7, "pad": rng.choice([0, 0, 8, 13])}
    if op == "loss":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        tokens, vocab, d = _log(rng, 1, 8192), _size(rng, 100, 50257, 64), _size(rng, 32, 2048, 64)
        most = 8192 * 50257 * 1024 // (4 if dtype == "f32" else 1)
        tokens = max(1, min(tokens, most // (vocab * d)))
        return {"op": op, "tokens": tokens, "vocab": vocab, "d": d, "dtype": dtype,
                "grad": "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]), "back": rng.random() < 0.75,
                "ignored": rng.choice([0.0, 0.1, 0.5])}
    if op == "orthogonal":
        rows, cols = _size(rng, 24, 4096, 32), _size(rng, 24, 4096, 32)
        batch = min(_log(rng, 1, 24), max(1, (4096 * 4096) // (rows * cols)))
        return {"op": op, "batch": batch, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    shapes = []
    for _ in range(rng.randint(1, 4)):
        rows, cols = _size(rng, 24, 2048, 32), _size(rng, 24, 2048, 32)
        shapes.append("%dx%d*%d" % (rows, cols, min(_log(rng, 1, 24), max(1, (8 << 20) // (rows * cols)))))
    return {"op": op, "shapes": ",".join(shapes), "g": rng.choice([1, 2, 4, 4, 8]), "nesterov": rng.random() < 0.75}


# ------------------------------------------------------------------------------------------------- the inputs
def _matrices(text):
    """[(rows, cols, count)] of "1024x256*6,..."; matrices lie end to end in the flat buffers, group by group."""
    out = []
    for part in text.split(","):
        shape, count = part.split("*")
        rows, cols = shape.split("x")
        out.append((int(rows), int(cols), int(count)))
    return out


def _gradients(gen, batch, rows, cols, rank=8):
    """Matrices as gradients of hidden layers are: a few strong directions over a dense remainder."""
    dev = gen.device
    x = torch.randn(batch, rows, cols, generator=gen, device=dev) * 1e-3
    r = min(rank, rows, cols)
    left = torch.randn(batch, rows, r, generator=gen, device=dev)
    right = torch.randn(batch, r, cols, generator=gen, device=dev)
    strength = 3e-3 / (1 + torch.arange(r, device=dev, dtype=torch.float32))
    return x.baddbmm_(left * strength, right)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev) * scale

    op = case["op"]
    s = {"case": dict(case)}
    if op == "norm":
        rows, d, t = case["rows"], case["d"], TYPES[case["dtype"]]
        wide = normal(rows, d + case["pad"])
        wide *= 0.5 + torch.rand(rows, 1, generator=gen, device=dev) * 2
        wide += normal(1, d + case["pad"], scale=0.3)
        s["x"] = wide.to(t)[:, :d]
        s["weight"] = 1 + normal(d, scale=0.1)
        s["bias"] = normal(d, scale=0.1) if case["bias"] else None
        if case["back"]:
            s["dy"] = normal(rows, d, scale=1e-2).to(t)
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = ((x - x.mean(1, keepdim=True)).square().mean(1) + NORM_EPS).rsqrt().float()
    elif op == "loss":
        n, v, d, t = case["tokens"], case["vocab"], case["d"], TYPES[case["dtype"]]
        s["weight"] = normal(v, d, scale=0.02).to(t)
        # words are as skewed as in text, and the features know something of the word that follows
        u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
        s["targets"] = torch.exp(u * math.log(v)).long().sub_(1).clamp_(0, v - 1)
        know = torch.rand(n, 1, generator=gen, device=dev) * 8
        s["hidden"] = (normal(n, d) + s["weight"][s["targets"]].float() * (know / (0.02 * math.sqrt(d)))).to(t)
        keep = torch.rand(n, generator=gen, device=dev) >= case["ignored"]
        s["targets"] = torch.where(keep, s["targets"], torch.full_like(s["targets"], IGNORE))
        if case["back"]:
            s["dloss"] = (0.5 + torch.rand(n, generator=gen, device=dev)) / max(n, 1)  # weighted tokens of a mean
            s["dweight"] = torch.empty(v, d, device=dev, dtype=TYPES[case["grad"]])
    elif op == "orthogonal":
        s["src"] = _gradients(gen, case["batch"], case["rows"], case["cols"]).to(TYPES[case["dtype"]])
    else:
        groups = _matrices(case["shapes"])
        total = sum(r * c * k for r, c, k in groups)
        s["params"] = normal(total, scale=0.02)
        s["momentum"] = torch.empty(total, device=dev)
        s["grads"] = [torch.empty(total, device=dev) for _ in range(case["g"])]
        s["wire"] = torch.empty(total, device=dev, dtype=torch.bfloat16)
        s["matrices"], at = [], 0
        for r, c, k in groups:
            common = _gradients(gen, k, r, c)
            s["momentum"][at:at + k * r * c] = (common + _gradients(gen, k, r, c)).flatten() * 8
            for g in s["grads"]:
                g[at:at + k * r * c] = common.flatten() + normal(k * r * c, scale=5e-4)
            s["matrices"] += [(at + i * r * c, r, c) for i in range(k)]
            at += k * r * c
    return s


# ------------------------------------------------------------------------------------------------- the plain forms
def _plain_norm(s):
    x, weight, bias = s["x"].float(), s["weight"], s["bias"]
    t, d = s["x"].dtype, s["x"].shape[1]
    if "dy" not in s:
        mean = x.mean(1)
        centred = x - mean[:, None]
        rstd = (centred.square().mean(1) + NORM_EPS).rsqrt()
        y = centred * rstd[:, None] * weight
        return {"y": (y if bias is None else y + bias).to(t), "mean": mean, "rstd": rstd}
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * weight
    dx = (g - g.sum(1, keepdim=True) / d - xhat * ((g * xhat).sum(1, keepdim=True) / d)) * rstd
    out = {"dx": dx.to(t), "dweight": (dy * xhat).sum(0)}
    if bias is not None:
        out["dbias"] = dy.sum(0)
    return out


def _plain_loss(s):
    hidden, weight, targets = s["hidden"].float(), s["weight"].float(), s["targets"]
    logits = hidden @ weight.t()
    top = logits.amax(1, keepdim=True)
    lse = (logits - top).exp_().sum(1).log() + top[:, 0]
    counted = targets != IGNORE
    at = torch.where(counted, targets, torch.zeros_like(targets))[:, None]
    loss = torch.where(counted, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    out = {"loss": loss, "lse": lse}
    if "dloss" in s:
        scale = torch.where(counted, s["dloss"], torch.zeros_like(lse))[:, None]
        p = logits.sub_(lse[:, None]).exp_()
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
        p *= scale
        out["dhidden"] = (p @ weight).to(s["hidden"].dtype)
        out["dweight"] = (p.t() @ hidden).to(s["dweight"].dtype)
    return out


def _plain_newton_schulz(u):
    """u: [batch, rows, cols] fp32."""
    a, b, c = COEFFICIENTS
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        poly = b * gram + c * torch.bmm(gram, gram)
        x = a * x + torch.bmm(poly, x)
    return x.transpose(1, 2) if tall else x


def _plain_muon(s):
    grads, params, m = s["grads"], s["params"], s["momentum"]
    mean = torch.stack(grads).sum(0) / len(grads) if len(grads) > 1 else grads[0]
    m.mul_(MU).add_(mean)
    u = mean + MU * m if s["case"]["nesterov"] else m
    at = 0
    for rows, cols, count in _matrices(s["case"]["shapes"]):
        n = rows * cols * count
        o = _plain_newton_schulz(u[at:at + n].view(count, rows, cols))
        x = params[at:at + n].view(count, rows, cols)
        x.mul_(1 - LR * DECAY).sub_(o, alpha=LR * math.sqrt(max(1.0, rows / cols)))
        at += n
    s["wire"].copy_(params)
    return {"params": params, "momentum": m, "wire": s["wire"]}


# ------------------------------------------------------------------------------------------------- a pass
def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        if op == "norm":
            return _plain_norm(s)
        if op == "loss":
            return _plain_loss(s)
        if op == "orthogonal":
            return _plain_newton_schulz(s["src"].float()).to(s["src"].dtype)
        return _plain_muon(s)

    import paper_2104_05588_amd as daso

    if op == "norm":
        if "dy" not in s:
            y, mean, rstd = daso.layer_norm(s["x"], s["weight"], s["bias"], eps=NORM_EPS)
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dweight, dbias = daso.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"],
                                                      bias=s["bias"] is not None)
        return {"dx": dx, "dweight": dweight} if dbias is None else {"dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "loss":
        loss, lse = daso.linear_cross_entropy(s["hidden"], s["weight"], s["targets"], ignore_index=IGNORE)
        out = {"loss": loss, "lse": lse}
        if "dloss" in s:
            out["dhidden"], out["dweight"] = daso.linear_cross_entropy_backward(
                s["dloss"], s["hidden"], s["weight"], s["targets"], lse, ignore_index=IGNORE, dweight=s["dweight"])
        return out
    if op == "orthogonal":
        return daso.orthogonalize(s["src"], steps=NS_STEPS, coefficients=COEFFICIENTS, eps=NS_EPS)
    daso.muon_step(s["grads"], s["params"], s["momentum"], s["matrices"], lr=LR, mu=MU, weight_decay=DECAY,
                   nesterov=s["case"]["nesterov"], steps=NS_STEPS, coefficients=COEFFICIENTS, eps=NS_EPS, wire=s["wire"])
    return {"params": s["params"], "momentum": s["momentum"], "wire": s["wire"]}


# ------------------------------------------------------------------------------------------------- what it takes
def _schulz_flops(rows, cols):
    """Two symmetric products, of which half is enough, and one full product a step."""
    m, n = min(rows, cols), max(rows, cols)
    return NS_STEPS * (m * m * n + m ** 3 + 2 * m * m * n)


def work(case):
    op = case["op"]
    if op == "norm":
        rows, d, e = case["rows"], case["d"], 2 if case["dtype"] == "bf16" else 4
        if case["back"]:
            return {"bytes": 3 * rows * d * e + 8 * rows + 4 * d * (3 if case["bias"] else 2), "flops": 12 * rows * d}
        return {"bytes": 2 * rows * d * e + 8 * rows + 4 * d * (2 if case["bias"] else 1), "flops": 8 * rows * d}
    if op == "loss":
        n, v, d, e = case["tokens"], case["vocab"], case["d"], 2 if case["dtype"] == "bf16" else 4
        if not case["back"]:
            return {"bytes": (n + v) * d * e + 16 * n, "flops": 2.0 * n * v * d}
        return {"bytes": (2 * n + v) * d * e + v * d * (2 if case["grad"] == "bf16" else 4) + 20 * n, "flops": 6.0 * n * v * d}
    if op == "orthogonal":
        k, e = case["batch"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * k * case["rows"] * case["cols"] * e, "flops": k * _schulz_flops(case["rows"], case["cols"])}
    groups = _matrices(case["shapes"])
    return {"bytes": sum(r * c * k for r, c, k in groups) * (4 * case["g"] + 18),
            "flops": sum(k * _schulz_flops(r, c) for r, c, k in groups)}


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        x, w = s["x"].double(), s["weight"].double()
        if not case["back"]:
            var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
            y = (x - mean) / (var + NORM_EPS).sqrt() * w
            if s["bias"] is not None:
                y = y + s["bias"].double()
            return {"y": y, "mean": mean[:, 0], "rstd": 1 / (var[:, 0] + NORM_EPS).sqrt()}
        # the Jacobian of the normalised row: rstd (I - 1 1'/d - xhat xhat'/d), with the statistics as given
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        xhat = (x - s["mean"].double()[:, None]) * r
        g = dy * w
        dx = r * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        out = {"dx": dx, "dweight": torch.einsum("ij,ij->j", dy, xhat)}
        if s["bias"] is not None:
            out["dbias"] = dy.sum(0)
        return out
    if op == "loss":
        h, w, t = s["hidden"].double(), s["weight"].double(), s["targets"]
        z = h @ w.T
        lse = torch.logsumexp(z, 1)
        live = (t != IGNORE).nonzero()[:, 0]
        loss = torch.zeros_like(lse)
        loss[live] = lse[live] - z[live, t[live]]
        out = {"loss": loss, "lse": lse}
        if case["back"]:
            dz = torch.zeros_like(z)
            dz[live] = torch.softmax(z[live], 1)
            dz[live, t[live]] -= 1
            dz *= s["dloss"].double()[:, None]
            out["dhidden"], out["dweight"] = dz @ w, dz.T @ h
        return out

    def polynomial(u):
        """The odd quintic of the singular values, step by step, from the definition."""
        k1, k3, k5 = COEFFICIENTS
        x = u / (torch.linalg.matrix_norm(u, keepdim=True) + NS_EPS)
        flip = x.shape[-2] > x.shape[-1]
        x = x.mT.contiguous() if flip else x
        for _ in range(NS_STEPS):
            cube = x @ x.mT @ x
            x = k1 * x + k3 * cube + k5 * (x @ x.mT @ cube)
        return x.mT if flip else x

    if op == "orthogonal":
        return polynomial(s["src"].double())
    g = sum(v.double() for v in s["grads"]) / case["g"]
    m = MU * s["momentum"].double() + g
    u = g + MU * m if case["nesterov"] else m
    x, at = s["params"].double(), 0
    for r, c, k in _matrices(case["shapes"]):
        cut = slice(at, at + r * c * k)
        x[cut] = (1 - LR * DECAY) * x[cut] - LR * max(1.0, r / c) ** 0.5 * polynomial(u[cut].view(k, r, c)).reshape(-1)
        at = cut.stop
    return {"params": x, "momentum": m, "wire": x}
