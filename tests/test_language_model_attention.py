"""The language model with attention and clipped gradients."""
import math

import numpy as np
import pytest
import torch

import paper_2104_05588_amd as daso
from workloads import language_model as LM


@pytest.mark.parametrize("vocab,d,blocks,heads,kv", [(100, 64, 2, 4, 2), (37, 48, 1, 2, 0)])
def test_layout_with_heads_holds_every_tensor_once(vocab, d, blocks, heads, kv):
    lay = LM.Layout(vocab, d, blocks, heads, kv)
    count = np.zeros(lay.n, np.int32)
    hidden = ("up", "down", "qkv", "join")
    for name, (start, shape) in lay.spans.items():
        count[start:start + int(np.prod(shape))] += 1
        assert (start >= lay.rest) == name.endswith(hidden)
    kv = kv or heads
    assert count.max() == 1
    assert count.sum() == 2 * vocab * d + 2 * d + blocks * (4 * d + 2 * d // heads + 8 * d * d + d * d * (2 * heads + 2 * kv) // heads)
    assert len(lay.matrices) == 4 * blocks
    plain = LM.Layout(vocab, d, blocks)
    assert not plain.heads and set(plain.spans) < set(lay.spans)


def plain_loss(lay, flat, tokens, targets, rows):
    """The model's mean loss in elementary operations."""
    w = lambda k: lay.view(flat, k)  # noqa: E731
    norm = lambda x, k: torch.nn.functional.layer_norm(x, (lay.d,), w(k + "norm.weight"), w(k + "norm.bias"))  # noqa: E731
    n, half, share = len(tokens), lay.dim // 2, lay.heads // lay.kv_heads
    length = n // rows
    angle = torch.arange(length).repeat(rows)[:, None, None] * daso.rotary_frequencies(lay.dim, device="cpu")
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1) | (torch.arange(n)[:, None] // length != torch.arange(n) // length)

    def turned(t, weight):
        t = t * (t.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight
        a, b = t[..., :half], t[..., half:]
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)

    x = w("embedding")[tokens]
    for b in range(lay.blocks):
        qkv = (norm(x, f"{b}.seen.") @ w(f"{b}.qkv").t()).view(n, -1, lay.dim)
        q, k, v = qkv.split((lay.heads, lay.kv_heads, lay.kv_heads), 1)
        q, k = turned(q, w(f"{b}.q.norm.weight")), turned(k, w(f"{b}.k.norm.weight"))
        seen = []
        for h in range(lay.heads):
            z = (q[:, h] @ k[:, h // share].t() / math.sqrt(lay.dim)).masked_fill(hidden, -math.inf)
            seen.append(z.softmax(1) @ v[:, h // share])
        x = x + torch.cat(seen, 1) @ w(f"{b}.join").t()
        x = x + torch.relu(norm(x, f"{b}.") @ w(f"{b}.up").t()) @ w(f"{b}.down").t()
    return torch.nn.functional.cross_entropy(norm(x, "") @ w("output").t(), targets, ignore_index=-100)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,d,blocks,heads,kv,rows,length", [(211, 64, 2, 4, 2, 3, 70), (300, 96, 1, 2, 2, 2, 129)])
def test_gradients_against_autograd(vocab, d, blocks, heads, kv, rows, length):
    """In bf16 against 64 bits: as without attention, 2 roundings a product, norm or sum of each block and pass, of which a block
    has 4 more here (two products, the rotation, the attention): 2^-9 * 16 * (3 blocks + 1)."""
    print(f"attention model's gradients {vocab} {d} {blocks} {heads} {kv} {rows} {length}", flush=True)
    lay = LM.Layout(vocab, d, blocks, heads, kv)
    flat = lay.init(5).bfloat16()
    gen = torch.Generator().manual_seed(6)
    n = rows * length
    tokens, targets = torch.randint(vocab, (n,), generator=gen), torch.randint(vocab, (n,), generator=gen)
    targets[::7] = -100
    exact = flat.double().requires_grad_()
    want_loss = plain_loss(lay, exact, tokens, targets, rows)
    want, = torch.autograd.grad(want_loss, exact)
    grad = torch.full((lay.n,), 7.0, device="cuda")
    loss = LM.gradients(lay, flat.float().cuda(), flat.cuda(), tokens.cuda(), targets.cuda(), grad, LM.Sequences(lay, rows, length))
    live = targets != -100
    tol = 2.0 ** -9 * 16 * (3 * blocks + 1)
    assert abs(float(loss.double().sum()) / int(live.sum()) - float(want_loss.detach())) <= tol * float(want_loss.detach())
    for name in lay.spans:
        g, e = lay.view(grad, name).double().cpu(), lay.view(want, name)
        assert float((g - e).norm()) <= tol * float(e.norm()), name


@pytest.mark.gpu
def test_training_with_attention_and_clipping_keeps_the_nodes_together():
    print("attention model's training", flush=True)
    losses, _, cluster = LM.train(steps=8, vocab=300, d=128, blocks=1, rows=4, length=48, heads=4, kv_heads=2, clip=0.5)
    assert all(np.isfinite(losses))
    for node in cluster[1:]:
        assert torch.equal(node.params, cluster[0].params) and torch.equal(node.wire, cluster[0].wire)
    # the gradient that the last step took is the replicas' mean, of a norm of no more than the clip
    node = cluster[0]
    norm, norms = daso.gradient_norm(node.grads[:1], node._tensors)
    assert float(norm) <= 0.5 * (1 + 2.0 ** -20) and norms.numel() == len(node.lay.spans)


@pytest.mark.gpu
def test_clipping_to_a_large_norm_steps_as_without():
    """The mean is the step's own: parameters of SGD's part have the same bits."""
    print("clip of a large norm", flush=True)
    lay = LM.Layout(50, 32, 1, 2, 1)
    gen = torch.Generator("cuda").manual_seed(1)
    tokens = [torch.randint(50, (2 * 33,), generator=gen, device="cuda") for _ in range(2)]
    nodes = [LM.Node(lay, 3, 2, clip=clip) for clip in (0.0, 1e9)]
    for node in nodes:
        node.step(tokens, tokens[::-1], LM.Sequences(lay, 2, 33))
    a, b = (node.params[:lay.rest] for node in nodes)
    assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,d,blocks,heads,kv,rows,length", [(211, 64, 2, 4, 2, 3, 70), (300, 96, 1, 2, 2, 2, 129)])
def test_gradients_of_an_fp32_model_against_autograd(vocab, d, blocks, heads, kv, rows, length):
    """A model whose matrices are fp32 throughout has no roundings that a missing or wrong term could hide behind: a product of at most 384
    terms is off by 384 * 2^-24 < 2^-15 of its terms, other steps by less; 16 of them a block and pass, as in bf16."""
    print(f"fp32 attention model's gradients {vocab} {d} {blocks} {heads} {kv} {rows} {length}", flush=True)
    lay = LM.Layout(vocab, d, blocks, heads, kv)
    flat = lay.init(5)
    gen = torch.Generator().manual_seed(6)
    n = rows * length
    tokens, targets = torch.randint(vocab, (n,), generator=gen), torch.randint(vocab, (n,), generator=gen)
    targets[::7] = -100
    exact = flat.double().requires_grad_()
    want_loss = plain_loss(lay, exact, tokens, targets, rows)
    want, = torch.autograd.grad(want_loss, exact)
    grad = torch.full((lay.n,), 7.0, device="cuda")
    loss = LM.gradients(lay, flat.cuda(), flat.cuda(), tokens.cuda(), targets.cuda(), grad, LM.Sequences(lay, rows, length))
    tol = 2.0 ** -15 * 16 * (3 * blocks + 1)
    assert abs(float(loss.double().sum()) / int((targets != -100).sum()) - float(want_loss.detach())) <= tol * float(want_loss.detach())
    for name in lay.spans:
        g, e = lay.view(grad, name).double().cpu(), lay.view(want, name)
        assert float((g - e).norm()) <= tol * float(e.norm()), name


@pytest.mark.gpu
def test_a_small_clip_is_the_steps_norm():
    """The replicas' mean gradient is longer than the clip, and the step takes it scaled to that."""
    print("a small clip", flush=True)
    lay, clip = LM.Layout(60, 64, 1, 4, 2), 1e-3
    gen = torch.Generator("cuda").manual_seed(2)
    tokens = [torch.randint(60, (3 * 40,), generator=gen, device="cuda") for _ in range(2)]
    at = LM.Sequences(lay, 3, 40)
    node = LM.Node(lay, 3, 2, clip=clip)
    before, want = node.params.clone(), torch.zeros(lay.n, dtype=torch.float64, device="cuda")
    for x, t in zip(tokens, tokens[::-1]):
        grad = torch.zeros(lay.n, device="cuda")
        LM.gradients(lay, node.params, node.wire, x, t, grad, at)
        want += grad.double() / 2
    long = float(want.norm())
    assert long > 10 * clip
    node.step(tokens, tokens[::-1], at)
    # the mean's, the factor's and the scaled value's roundings, of 2^-24 each; index_add's order may differ in the embedding
    got = node.grads[0].double()
    assert float((got - want * (clip / (long + 1e-6))).norm()) <= clip * 2.0 ** -16
    assert abs(float(got.norm()) - clip * long / (long + 1e-6)) <= clip * 2.0 ** -20
    # plain SGD of the first step: lr 1, momentum from zero
    k = lay.rest
    assert float((before[:k] - got[:k].float() - node.params[:k]).abs().max()) <= 2.0 ** -22 * float(before[:k].abs().max())
