"""The written-out gradients of block_reference against central differences, in 64 bits on the CPU."""
import pytest
import torch

import block_reference as ref


def differences(fn, x, error, h=1e-6):
    """d sum(error * fn(x)) / dx, element by element."""
    flat, out = x.reshape(-1), torch.zeros(x.numel(), dtype=x.dtype)
    for i in range(x.numel()):
        up, down = flat.clone(), flat.clone()
        up[i] += h
        down[i] -= h
        out[i] = sum(((a - b) * e).sum() for a, b, e in zip(fn(up.view_as(x)), fn(down.view_as(x)), error)) / (2 * h)
    return out.view_as(x)


def normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def close(a, b):
    assert (a - b).abs().max() <= 1e-7 * (1.0 + b.abs().max()), (a - b).abs().max()


@pytest.mark.parametrize("groups", [1, 3])
def test_norms(groups):
    x, res, gate, d_y, d_r, w = [normal(3, 12, seed=i) for i in range(5)] + [normal(12, seed=9)]
    (d_x, d_res, d_w), _ = ref.add_norm_gradient(d_y, res + 0.7 * x, w, d_r, 0.7, 1e-3, groups)
    close(d_x, differences(lambda v: ref.add_norm(v, w, res, 0.7, 1e-3, groups), x, (d_y, d_r)))
    close(d_res, differences(lambda v: ref.add_norm(x, w, v, 0.7, 1e-3, groups), res, (d_y, d_r)))
    close(d_w, differences(lambda v: ref.add_norm(x, v, res, 0.7, 1e-3, groups), w, (d_y, d_r)))
    (d_x, d_gate, d_w), _ = ref.norm_gate_gradient(d_y, x, w, gate, 0.7, 1e-3, groups)
    close(d_x, differences(lambda v: [ref.norm_gate(v, w, gate, res, 0.7, 1e-3, groups)], x, [d_y]))
    close(d_gate, differences(lambda v: [ref.norm_gate(x, w, v, res, 0.7, 1e-3, groups)], gate, [d_y]))
    close(d_w, differences(lambda v: [ref.norm_gate(x, v, gate, res, 0.7, 1e-3, groups)], w, [d_y]))


@pytest.mark.parametrize("active", [True, False])
def test_conv(active):
    x, w, b, first = normal(2, 5, 3), normal(3, 4, seed=1), normal(3, seed=2), normal(2, 3, 3, seed=3)
    d_y, d_last, n = normal(2, 5, 3, seed=4), normal(2, 3, 3, seed=5), [5, 1]
    grads = ref.conv_gradient(x, w, b, active, n, first, d_y, d_last)
    for got, (at, make) in zip(grads, [(x, lambda v: (v, w, b, first)), (w, lambda v: (x, v, b, first)), (b, lambda v: (x, w, v, first)), (first, lambda v: (x, w, b, v))]):
        def fn(v):
            x_, w_, b_, first_ = make(v)
            return ref.conv(x_, w_, b_, active, n, first_)[:2]
        close(got, differences(fn, at, (d_y, d_last)))


@pytest.mark.parametrize("soft", [True, False])
def test_scan(soft):
    x, dt, a, b, c = normal(2, 4, 6), normal(2, 4, 6, seed=1).abs(), -normal(6, 3, seed=2).abs(), normal(2, 4, 2, 3, seed=3), normal(2, 4, 2, 3, seed=4)
    skip, bias, first = normal(6, seed=5), normal(6, seed=6), normal(2, 6, 3, seed=7)
    d_y, d_last, n = normal(2, 4, 6, seed=8), normal(2, 6, 3, seed=9), [4, 1]
    args = [x, dt, a, b, c, skip, bias, first]
    run = lambda *v, **k: ref.scan(*v[:7], soft, n, v[7], **k)  # noqa: E731
    grads = run(*args, d_y=d_y, d_final=d_last)[1][0]
    for i, got in enumerate(grads):
        def fn(v):
            return run(*args[:i], v, *args[i + 1:])[0]
        close(got, differences(fn, args[i], (d_y, d_last)))
    y, state = run(*args)[0]  # the definition, one number at a time
    h = first[1, 4].clone()
    d = dt[1, 0, 4] + bias[4]
    d = torch.log1p(torch.exp(d)) if soft else d
    h = torch.exp(d * a[4]) * h + d * x[1, 0, 4] * b[1, 0, 1]
    assert torch.allclose(state[1, 4], h) and torch.allclose(y[1, 0, 4], (c[1, 0, 1] * h).sum() + skip[4] * x[1, 0, 4]) and (y[1, 1:] == 0.0).all()


def test_log_probs():
    logits, tokens = normal(3, 7), torch.tensor([[0, 0, 6], [3, -1, 9], [2, 2, 2]])
    logits[1, 4] = -float("inf")
    d, d_h = normal(3, 3, seed=1), normal(3, seed=2)
    want = differences(lambda v: ref.log_probs(v, tokens, 0.7, 0)[:2], torch.where(torch.isinf(logits), 0.0, logits), (d, d_h))
    got = ref.log_probs_gradient(torch.where(torch.isinf(logits), 0.0, logits), tokens, 0.7, d, d_h)
    close(got, want)
    masked = ref.log_probs_gradient(logits, tokens, 0.7, d, d_h)
    keep = [0, 1, 2, 3, 5, 6]  # an impossible token is as one that is not there
    close(masked[1:2, keep], ref.log_probs_gradient(logits[1:2, keep], tokens[1:2], 0.7, d[1:2], d_h[1:2]))
    assert masked[1, 4] == 0.0
    empty = torch.full((1, 4), -float("inf"), dtype=torch.float64)
    assert (ref.log_probs_gradient(empty, tokens[:1], 1.0, d[:1], d_h[:1]) == 0.0).all() and ref.log_probs(empty, tokens[:1], 1.0, 2)[1] == 0.0
