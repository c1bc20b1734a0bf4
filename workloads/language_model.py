"""A small language model trained by DASO's nodes, simulated on one GPU: the training operators
with the synchronisation, as a training program uses them together.

    python -m workloads.language_model --steps 60

Each node has one flat parameter buffer and g replicas.  A replica's forward pass reads the bf16 form
of the parameters (the node's `wire`, which the last step wrote) through layer_norm and
linear_cross_entropy; its backward pass writes fp32 gradients of the norms and of the output projection
straight into its flat gradient buffer.  Then the node averages its replicas and steps: FusedStep (SGD with momentum)
on the embedding, the output projection and the norms, MuonStep on the hidden matrices.  Every few batches the nodes exchange
`wire`, and a batch later global_merge takes the copies in.

    python -m workloads.language_model --heads 4 --kv-heads 2 --clip 1

gives each block causal attention in front of its two products (head_norm_rotary and packed_attention, each row of a batch
a sequence), and clips the replicas' mean gradient before the step (clip_gradients).

The tokens are drawn from a Markov chain whose entropy is the least loss that a model can reach."""
from __future__ import annotations

import argparse
import math
from typing import Dict, List, Optional, Tuple

import torch

import paper_2104_05588_amd as daso

ALIGN = 64  # elements: every tensor of the flat buffers starts on 128 bytes of the wire


class Layout:
    """Where the model's tensors lie in a flat buffer: first what SGD steps, then the hidden matrices."""

    def __init__(self, vocab: int, d: int, blocks: int, heads: int = 0, kv_heads: int = 0):
        self.vocab, self.d, self.blocks = vocab, d, blocks
        self.heads, self.kv_heads = heads, kv_heads or heads
        self.dim = d // heads if heads else 0  # of a head
        shapes = [("embedding", (vocab, d)), ("output", (vocab, d)), ("norm.weight", (d,)), ("norm.bias", (d,))]
        for b in range(blocks):
            shapes += [(f"{b}.norm.weight", (d,)), (f"{b}.norm.bias", (d,))]
            if heads:
                shapes += [(f"{b}.seen.norm.weight", (d,)), (f"{b}.seen.norm.bias", (d,)), (f"{b}.q.norm.weight", (self.dim,)),
                           (f"{b}.k.norm.weight", (self.dim,))]
        hidden = []
        for b in range(blocks):
            if heads:
                hidden += [(f"{b}.qkv", ((heads + 2 * self.kv_heads) * self.dim, d)), (f"{b}.join", (d, heads * self.dim))]
            hidden += [(f"{b}.up", (4 * d, d)), (f"{b}.down", (d, 4 * d))]
        self.spans: Dict[str, Tuple[int, Tuple[int, ...]]] = {}
        at = 0
        for name, shape in shapes + hidden:
            if hidden and name == hidden[0][0]:
                self.rest = at  # elements before the hidden matrices
            self.spans[name] = (at, shape)
            size = shape[0] * (shape[1] if len(shape) > 1 else 1)
            at += (size + ALIGN - 1) // ALIGN * ALIGN
        self.n = at
        if not blocks:
            self.rest = at
        self.matrices = [(self.spans[name][0], *shape) for name, shape in hidden]

    def view(self, flat: torch.Tensor, name: str) -> torch.Tensor:
        start, shape = self.spans[name]
        size = shape[0] * (shape[1] if len(shape) > 1 else 1)
        return flat[start:start + size].view(shape)

    def init(self, seed: int, device="cpu") -> torch.Tensor:
        gen = torch.Generator().manual_seed(seed)
        flat = torch.zeros(self.n)
        for name, (_, shape) in self.spans.items():
            v = self.view(flat, name)
            if name.endswith("norm.weight"):
                v.fill_(1.0)
            elif len(shape) == 2:
                v.copy_(torch.randn(shape, generator=gen) * (0.5 if name == "embedding" else shape[1] ** -0.5))
        return flat.to(device)


class Sequences:
    """Where a replica's tokens lie in their sequences: what its attention needs of a batch."""

    def __init__(self, lay: Layout, rows: int, length: int, device="cuda"):
        self.offsets = torch.arange(rows + 1, device=device) * length
        self.positions = torch.arange(length, device=device).repeat(rows)
        self.frequencies = daso.rotary_frequencies(lay.dim, device=device)


def _parts(lay: Layout, qkv: torch.Tensor):
    """The heads of queries, keys and values in the rows of their joint projection."""
    return qkv.view(-1, lay.heads + 2 * lay.kv_heads, lay.dim).split((lay.heads, lay.kv_heads, lay.kv_heads), 1)


def _attend(lay: Layout, b: int, w, f, x: torch.Tensor, at: Sequences):
    """x with what its tokens see, and what the way back needs."""
    y, mean, rstd = daso.layer_norm(x, f(f"{b}.seen.norm.weight"), f(f"{b}.seen.norm.bias"))
    q, k, v = _parts(lay, y @ w(f"{b}.qkv").t())
    tq, tk = daso.head_norm_rotary(q, k, at.positions, at.frequencies, f(f"{b}.q.norm.weight"), f(f"{b}.k.norm.weight"))
    out, lse = daso.packed_attention(tq, tk, v, at.offsets)
    return x + out.flatten(1) @ w(f"{b}.join").t(), (x, y, mean, rstd, q, k, v, tq, tk, out, lse)


def _attend_backward(lay: Layout, b: int, w, f, g, dx: torch.Tensor, kept: tuple, at: Sequences) -> torch.Tensor:
    x, y, mean, rstd, q, k, v, tq, tk, out, lse = kept
    g(f"{b}.join").copy_(dx.t() @ out.flatten(1))
    dqkv = torch.empty(len(x), (lay.heads + 2 * lay.kv_heads) * lay.dim, dtype=x.dtype, device=x.device)
    dq, dk, dv = _parts(lay, dqkv)
    daso.packed_attention_backward((dx @ w(f"{b}.join")).view_as(out), tq, tk, v, out, lse, at.offsets, dq=dq, dk=dk, dv=dv)
    daso.head_norm_rotary_backward(dq, dk, q, k, at.positions, at.frequencies, f(f"{b}.q.norm.weight"), f(f"{b}.k.norm.weight"),
                                   dq=dq, dk=dk, dq_weight=g(f"{b}.q.norm.weight"), dk_weight=g(f"{b}.k.norm.weight"))
    g(f"{b}.qkv").copy_(dqkv.t() @ y)
    dn, _, _ = daso.layer_norm_backward(dqkv @ w(f"{b}.qkv"), x, f(f"{b}.seen.norm.weight"), mean, rstd,
                                        dweight=g(f"{b}.seen.norm.weight"), dbias=g(f"{b}.seen.norm.bias"))
    return dx + dn


def gradients(lay: Layout, params: torch.Tensor, wire: torch.Tensor, tokens: torch.Tensor, targets: torch.Tensor,
              grad: torch.Tensor, at: Optional[Sequences] = None) -> torch.Tensor:
    """One replica's pass: the tokens' losses, and their mean's gradient into `grad` (all of it but the padding).  A model with
    heads needs `at`."""
    w, f, g = (lambda k: lay.view(wire, k)), (lambda k: lay.view(params, k)), (lambda k: lay.view(grad, k))
    x = w("embedding")[tokens]
    kept: List[tuple] = []
    for b in range(lay.blocks):
        seen = None
        if lay.heads:
            x, seen = _attend(lay, b, w, f, x, at)
        y, mean, rstd = daso.layer_norm(x, f(f"{b}.norm.weight"), f(f"{b}.norm.bias"))
        a = torch.relu(y @ w(f"{b}.up").t())
        kept.append((x, y, mean, rstd, a, seen))
        x = x + a @ w(f"{b}.down").t()
    h, mean, rstd = daso.layer_norm(x, f("norm.weight"), f("norm.bias"))
    loss, lse = daso.linear_cross_entropy(h, w("output"), targets)

    live = targets != -100
    dloss = live / live.sum().clamp(min=1)
    dh, _ = daso.linear_cross_entropy_backward(dloss, h, w("output"), targets, lse, dweight=g("output"))
    dx, _, _ = daso.layer_norm_backward(dh, x, f("norm.weight"), mean, rstd, dweight=g("norm.weight"), dbias=g("norm.bias"))
    for b in reversed(range(lay.blocks)):
        x, y, mean, rstd, a, seen = kept[b]
        g(f"{b}.down").copy_(dx.t() @ a)
        da = (dx @ w(f"{b}.down")) * (a > 0)
        g(f"{b}.up").copy_(da.t() @ y)
        dn, _, _ = daso.layer_norm_backward(da @ w(f"{b}.up"), x, f(f"{b}.norm.weight"), mean, rstd,
                                            dweight=g(f"{b}.norm.weight"), dbias=g(f"{b}.norm.bias"))
        dx = dx + dn
        if lay.heads:
            dx = _attend_backward(lay, b, w, f, g, dx, seen, at)
    g("embedding").zero_().index_add_(0, tokens, dx.float())
    return loss


class Node:
    """A node's buffers, and its step over g replica gradients, whose mean's norm is at most `clip` unless that is 0."""

    def __init__(self, lay: Layout, seed: int, g: int = 2, lr: float = 1.0, hidden_lr: float = 0.02, clip: float = 0.0):
        self.lay, self.clip = lay, clip
        self.params = lay.init(seed, "cuda")
        self.momentum = torch.zeros(lay.n, device="cuda")
        self.wire = torch.empty(lay.n, dtype=torch.bfloat16, device="cuda")
        self.grads = [torch.zeros(lay.n, device="cuda") for _ in range(g)]
        daso.pack_bf16(self.params, self.wire)
        k = lay.rest
        self._tensors = sorted((start, math.prod(shape)) for start, shape in lay.spans.values())
        stepped = self.grads[:1] if clip else self.grads  # clipping leaves the mean in the first replica's buffer
        self._rest = daso.FusedStep([t[:k] for t in stepped], self.params[:k], self.momentum[:k], [], [(0, k, 0)], lr=lr,
                                    mu=0.9, wire=self.wire[:k])
        self._hidden = daso.MuonStep(stepped, self.params, self.momentum, lay.matrices, lr=hidden_lr, wire=self.wire)

    def step(self, tokens: List[torch.Tensor], targets: List[torch.Tensor], at: Optional[Sequences] = None) -> torch.Tensor:
        """One batch, a part of it for each replica; the replicas' mean losses."""
        means = []
        for grad, x, t in zip(self.grads, tokens, targets):
            loss = gradients(self.lay, self.params, self.wire, x, t, grad, at)
            means.append(loss.sum() / (t != -100).sum().clamp(min=1))
        if self.clip:
            daso.clip_gradients(self.grads, self.clip, self._tensors)
        self._rest()
        self._hidden()
        return torch.stack(means)

    def merge(self, copies: List[torch.Tensor], S: int) -> None:
        """Takes in copies that were sent S batches ago."""
        daso.global_merge(self.params, copies, [(0, self.lay.n, S)], wire=self.wire)


class Chain:
    """Tokens of a Markov chain: `fan` likely successors for each token."""

    def __init__(self, vocab: int, seed: int, fan: int = 4):
        gen = torch.Generator().manual_seed(seed)
        p = torch.full((vocab, vocab), 0.05 / vocab)
        p.scatter_add_(1, torch.randint(vocab, (vocab, fan), generator=gen), torch.full((vocab, fan), 0.95 / fan))
        self.p = p
        q = torch.full((vocab,), 1.0 / vocab)
        for _ in range(50):
            q = q @ p
        self.entropy = float(-(q[:, None] * p * p.log()).sum())

    def sample(self, rows: int, length: int, gen: torch.Generator) -> torch.Tensor:
        p = self.p.to(gen.device)
        x = [torch.randint(p.shape[0], (rows,), generator=gen, device=gen.device)]
        for _ in range(length):
            x.append(torch.multinomial(p[x[-1]], 1, generator=gen)[:, 0])
        return torch.stack(x, 1)


def train(steps: int = 60, nodes: int = 2, g: int = 2, vocab: int = 1000, d: int = 256, blocks: int = 2, rows: int = 16,
          length: int = 64, every: int = 4, S: int = 1, seed: int = 0, heads: int = 0, kv_heads: int = 0, clip: float = 0.0,
          tell=None) -> Tuple[List[float], float, List[Node]]:
    """The mean loss of each batch, the chain's entropy and the nodes, which after the last batch hold one state."""
    lay, chain = Layout(vocab, d, blocks, heads, kv_heads), Chain(vocab, seed)
    at = Sequences(lay, rows, length) if heads else None
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    cluster = [Node(lay, seed, g, clip=clip) for _ in range(nodes)]
    sent: Dict[int, List[torch.Tensor]] = {}
    losses: List[float] = []
    for t in range(steps):
        means = []
        for node in cluster:
            parts = [chain.sample(rows, length, gen) for _ in range(g)]
            means.append(node.step([p[:, :-1].reshape(-1) for p in parts], [p[:, 1:].reshape(-1) for p in parts], at))
        if t - S in sent:
            copies = sent.pop(t - S)
            for node in cluster:
                node.merge(copies, S)
        if t % every == every - 1:
            sent[t] = [node.wire.clone() for node in cluster]
        losses.append(float(torch.stack(means).mean()))
        if tell:
            tell(t, losses[-1])
    copies = [node.wire.clone() for node in cluster]
    for node in cluster:  # a blocking average: the copies alone
        node.merge(copies, 0)
    return losses, chain.entropy, cluster


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--nodes", type=int, default=2)
    ap.add_argument("--replicas", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--features", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--heads", type=int, default=0, help="attention heads (0: no attention)")
    ap.add_argument("--kv-heads", type=int, default=0, help="heads of keys and values (0: as many)")
    ap.add_argument("--clip", type=float, default=0.0, help="largest norm of the averaged gradient (0: any)")
    a = ap.parse_args()

    def tell(t, loss):
        if t % 10 == 9 or t == 0:
            print(f"batch {t + 1:4d}  loss {loss:.4f}", flush=True)

    losses, entropy, _ = train(a.steps, a.nodes, a.replicas, a.vocab, a.features, a.blocks, heads=a.heads, kv_heads=a.kv_heads, clip=a.clip, tell=tell)
    print(f"loss {losses[0]:.4f} to {losses[-1]:.4f}; the chain's entropy is {entropy:.4f}")


if __name__ == "__main__":
    main()
