"""The classifier over pixel sequences with dropout: its gradients against automatic differentiation of the formulas in 64 bits, under the
masks that the generator's definition gives for each layer's offset and the training step on the device."""
import pytest
import torch

import sequence_reference as ref
from paper_1912_05234_amd import inputs, pixels

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def plain(net, tokens, target, p, step):
    level, place, w, v, b = [x.double().cpu().requires_grad_() for x in net.parameters()]
    n, T = tokens.shape
    keep = [torch.from_numpy(ref.kept(n * T * 64, p, net.seed, offset + step)).view(n, T, 64) / (1.0 - p) for offset in (0, 1 << 40)]
    x = level[tokens.long()] * 8.0 * keep[0] + place[:T]
    q, k, u = (x @ w.t()).view(n, T, 3, 2, 32).permute(2, 0, 3, 1, 4)
    lag = torch.arange(T)[:, None] - torch.arange(T)
    weight = torch.where(lag >= 0, net.decay.double().cpu()[:, None, None] ** lag.clamp(min=0), 0.0)
    o = ((q @ k.transpose(2, 3)) * weight) @ u * net.scale
    h = o.transpose(1, 2).reshape(n, T, 64) * keep[1] + x
    z = h.mean(1) @ v.t() + b
    ((torch.nn.functional.softplus(z) - target.double() * z).sum() / n).backward()
    return torch.sigmoid(z), [x.grad for x in (level, place, w, v, b)]


@pytest.mark.parametrize("p,step", [(0.3, 0), (0.3, 5), (0.5, (1 << 33) + 1)])
def test_gradients_under_the_masks_of_a_step(p, step):
    images, labels = inputs.make_digits(3, 5)
    tokens, target = pixels.tokens_of(images), torch.eye(10)[torch.from_numpy(labels).long()]
    net = pixels.PixelClassifier(dropout=p)
    net.step.fill_(step)
    want_y, want = plain(net, tokens, target, p, step)
    y, saved = net.forward(tokens.to(DEV), p)
    # as without dropout: sums of up to 784 pixels and 64 columns in fp32, a few of them in a row, of magnitudes some times the results
    assert (y.double().cpu() - want_y).abs().max() <= 2.0 ** -12
    grads = net.gradient(saved, target.to(DEV), p)
    for g, w in zip(grads, want):
        assert g.shape == w.shape and (g.double().cpu() - w).abs().max() <= 2.0 ** -12 * w.abs().max()
    # and the bound tells masks apart: those of the next step do not pass
    other = plain(net, tokens, target, p, step + 1)[1]
    assert all((g.double().cpu() - w).abs().max() > 2.0 ** -12 * w.abs().max() for g, w in zip(grads[:4], other))


def test_training_reaches_what_the_documentation_says():
    """180 steps of 100 images: 99.8 % of a thousand held-out images as measured, 98 % at the least."""
    records = pixels.run(inputs.make_digits(6000, 1), inputs.make_digits(1000, 2), 3, report=lambda line: None)
    assert records[-1]["test_accuracy"] >= 0.98
