"""The classifier over pixel sequences: its gradients against automatic differentiation of the formulas in 64 bits, its form for
single pixels against the one for whole sequences, and training."""
import pytest
import torch

from paper_1912_05234_amd import inputs, pixels

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def plain(net, tokens, target, T):
    """Loss and gradients on the host in 64 bits, attention as a masked matrix of all pairs of pixels."""
    level, place, w, v, b = [p.double().cpu().requires_grad_() for p in net.parameters()]
    x = level[tokens.long()] * 8.0 + place[:T]
    q, k, u = (x @ w.t()).view(len(tokens), T, 3, 2, 32).permute(2, 0, 3, 1, 4)
    lag = torch.arange(T)[:, None] - torch.arange(T)
    weight = torch.where(lag >= 0, net.decay.double().cpu()[:, None, None] ** lag.clamp(min=0), 0.0)
    o = ((q @ k.transpose(2, 3)) * weight) @ u * net.scale
    h = o.transpose(1, 2).reshape(len(tokens), T, 64) + x
    z = h.mean(1) @ v.t() + b
    ((torch.nn.functional.softplus(z) - target.double() * z).sum() / len(z)).backward()
    return torch.sigmoid(z), [p.grad for p in (level, place, w, v, b)]


def test_gradients_of_the_whole_classifier():
    images, labels = inputs.make_digits(3, 5)
    tokens, target = pixels.tokens_of(images), torch.eye(10)[torch.from_numpy(labels).long()]
    net = pixels.PixelClassifier()
    want_y, want = plain(net, tokens, target, 784)
    y, saved = net.forward(tokens.to(DEV))
    # sums of up to 784 pixels and 64 columns in fp32, a few of them in a row: 2^-24 each, of magnitudes some times the results
    assert (y.double().cpu() - want_y).abs().max() <= 2.0 ** -12
    for g, w in zip(net.gradient(saved, target.to(DEV)), want):
        assert g.shape == w.shape and (g.double().cpu() - w).abs().max() <= 2.0 ** -12 * w.abs().max()


def test_pixels_one_by_one():
    images, _ = inputs.make_digits(5, 6)
    tokens = pixels.tokens_of(images).to(DEV)[:, :150].contiguous()
    net = pixels.PixelClassifier()
    streamed = net.stream(tokens)
    for t in (1, 2, 33, 150):
        whole, _ = net.forward(tokens[:, :t].contiguous())
        assert (streamed[:, t - 1] - whole).abs().max() <= 2.0 ** -12, t


def test_training_learns_the_digits():
    lines = []
    records = pixels.run(inputs.make_digits(3000, 1), inputs.make_digits(500, 2), 4, report=lines.append)
    assert len(lines) == 5 and records[-1]["train_loss"] < 0.8 * records[0]["train_loss"]
    assert records[-1]["test_accuracy"] > 0.5


def test_a_training_step_in_a_graph_draws_new_masks():
    images, labels = inputs.make_digits(10, 7)
    tokens, target = pixels.tokens_of(images).to(DEV), torch.eye(10, device=DEV)[torch.from_numpy(labels).long().to(DEV)]
    one, two = (pixels.PixelClassifier(dropout=0.3) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two.train_batch(tokens, target, 0.01)
    side.synchronize()
    one.train_batch(tokens, target, 0.01)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = two.train_batch(tokens, target, 0.01)
    seen = []
    for _ in range(3):
        want = one.train_batch(tokens, target, 0.01)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and all(torch.equal(a, b) for a, b in zip(one.parameters(), two.parameters()))
        seen.append(float(loss))
    assert len(set(seen)) == 3 and int(two.step) == 4
