"""The language model that runs the training operators with the synchronisation."""
import numpy as np
import pytest
import torch

import paper_2104_05588_amd as daso
from workloads import language_model as LM


@pytest.mark.parametrize("vocab,d,blocks", [(1000, 256, 2), (37, 33, 1), (50, 8, 0)])
def test_layout_holds_every_tensor_once(vocab, d, blocks):
    lay = LM.Layout(vocab, d, blocks)
    count = np.zeros(lay.n, np.int32)
    for name, (start, shape) in lay.spans.items():
        assert start % LM.ALIGN == 0
        count[start:start + int(np.prod(shape))] += 1
        assert (start >= lay.rest) == (name.endswith("up") or name.endswith("down"))
    assert count.max() == 1 and count.sum() == 2 * vocab * d + 2 * d + blocks * (2 * d + 8 * d * d)
    assert [(r, c) for _, r, c in lay.matrices] == [(4 * d, d), (d, 4 * d)] * blocks
    assert torch.equal(lay.init(3), lay.init(3)) and not torch.equal(lay.init(3), lay.init(4))


def test_chain_is_a_distribution_with_its_entropy():
    chain = LM.Chain(50, 1)
    assert torch.allclose(chain.p.sum(1), torch.ones(50), atol=1e-6)
    assert 0.5 * np.log(4) < chain.entropy < np.log(50)
    x = chain.sample(3, 7, torch.Generator().manual_seed(2))
    assert x.shape == (3, 8) and int(x.min()) >= 0 and int(x.max()) < 50


def plain_loss(lay, flat, tokens, targets):
    """The model's mean loss in elementary operations."""
    w = lambda k: lay.view(flat, k)  # noqa: E731
    norm = lambda x, k: torch.nn.functional.layer_norm(x, (lay.d,), w(k + "norm.weight"), w(k + "norm.bias"))  # noqa: E731
    x = w("embedding")[tokens]
    for b in range(lay.blocks):
        x = x + torch.relu(norm(x, f"{b}.") @ w(f"{b}.up").t()) @ w(f"{b}.down").t()
    return torch.nn.functional.cross_entropy(norm(x, "") @ w("output").t(), targets, ignore_index=-100)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,d,blocks,n", [(211, 64, 2, 300), (1000, 33, 1, 77)])
def test_gradients_against_autograd(vocab, d, blocks, n):
    """In bf16 against 64 bits: 2 roundings a product, norm or sum of each block and pass, of 2^-9 each, come to at most
    a share 2^-9 * 4 * (blocks + 1) * 2 of a gradient's norm where they add up, and relu's of values next to zero to as
    much again: 2^-9 * 16 * (blocks + 1)."""
    print(f"language model's gradients {vocab} {d} {blocks} {n}", flush=True)
    lay = LM.Layout(vocab, d, blocks)
    flat = lay.init(5).bfloat16()  # what the wire holds
    gen = torch.Generator().manual_seed(6)
    tokens, targets = torch.randint(vocab, (n,), generator=gen), torch.randint(vocab, (n,), generator=gen)
    targets[::7] = -100
    exact = flat.double().requires_grad_()
    want_loss = plain_loss(lay, exact, tokens, targets)
    want, = torch.autograd.grad(want_loss, exact)
    grad = torch.full((lay.n,), 7.0, device="cuda")
    loss = LM.gradients(lay, flat.float().cuda(), flat.cuda(), tokens.cuda(), targets.cuda(), grad)
    live = targets != -100
    assert not loss.cpu()[~live].any()
    tol = 2.0 ** -9 * 16 * (blocks + 1)
    assert abs(float(loss.double().sum()) / int(live.sum()) - float(want_loss)) <= tol * float(want_loss)
    for name in lay.spans:
        g, e = lay.view(grad, name).double().cpu(), lay.view(want, name)
        assert float((g - e).norm()) <= tol * float(e.norm()), name


@pytest.mark.gpu
def test_training_lowers_the_loss_and_keeps_the_nodes_together():
    print("language model's training", flush=True)
    losses, entropy, cluster = LM.train(steps=40, vocab=300, d=128, blocks=1)
    assert all(np.isfinite(losses))
    assert abs(losses[0] - np.log(300)) < 1.5
    assert losses[-1] < losses[0] - 0.5 * (losses[0] - entropy)  # half way to the least that can be reached
    for node in cluster[1:]:
        assert torch.equal(node.params, cluster[0].params) and torch.equal(node.wire, cluster[0].wire)
    want = torch.empty_like(cluster[0].wire)
    daso.pack_bf16(cluster[0].params, want)
    assert torch.equal(want, cluster[0].wire)
