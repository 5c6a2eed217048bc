"""The operators around a block at the ends of what they take: offsets past 32 bits, more workgroups than one dimension of a grid has, the longest rows."""
import pytest
import torch

import block_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U


def filled(*shape, dtype=torch.bfloat16, seed=0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


def test_norms_past_32_bits():
    """2^31 elements and some: the last rows as by themselves, bit for bit."""
    N, D = (1 << 20) + 37, 2056
    x, w = filled(N, D), filled(D, dtype=torch.float32, seed=1)
    tail = slice(N - 50, N)
    y, r = binding.add_norm_fwd(x, w, residual=x, scale=0.5, groups=8)
    for a, b in zip((y[tail], r[tail]), binding.add_norm_fwd(x[tail], w, residual=x[tail], scale=0.5, groups=8)):
        assert torch.equal(a, b)
    del y, r
    d_x, d_gate, _ = binding.norm_gate_bwd(x, x, w, gate=x, groups=8)
    for a, b in zip((d_x[tail], d_gate[tail]), binding.norm_gate_bwd(x[tail], x[tail], w, gate=x[tail], groups=8)):
        assert torch.equal(a, b)


def test_log_probs_past_32_bits():
    N, V = 67201, 32003
    logits, tokens = filled(N, V), torch.randint(0, V, (N, 2), device=DEV)
    tail, d = slice(N - 30, N), torch.ones(N, 2, device=DEV)
    out, last = binding.log_probs_fwd(logits, tokens, top=3), binding.log_probs_fwd(logits[tail], tokens[tail].contiguous(), top=3)
    for a, b in zip(out, last):
        assert torch.equal(a[tail], b)
    grad = binding.log_probs_bwd(logits, tokens, out[2], d)
    assert torch.equal(grad[tail], binding.log_probs_bwd(logits[tail], tokens[tail].contiguous(), last[2], d[tail].contiguous()))


def test_the_longest_row():
    V = 1 << 24
    logits = filled(1, V, dtype=torch.float16)
    logits[0, V - 1], logits[0, 12345678] = 9.0, 9.0
    tokens = torch.tensor([[V - 1, V, 0]], device=DEV)
    lp, _, stats, top_lp, top = binding.log_probs_fwd(logits, tokens, top=64)
    want = torch.log_softmax(logits.double(), 1)
    order = logits.float().sort(dim=1, descending=True, stable=True).indices[:, :64]
    assert torch.equal(top.long(), order) and top[0, :2].tolist() == [12345678, V - 1] and lp[0, 1] == 0.0
    # (ln sum: 5000 roundings at most, in parts of 32768 and 512 of them joined; the mean of |z| is below 16)
    assert (top_lp.double() - want.gather(1, order)).abs().max() <= 5000 * U and (lp[0, 0].double() - want[0, V - 1]).abs() <= 5000 * U
    grad = binding.log_probs_bwd(logits, tokens, stats, torch.ones(1, 3, device=DEV))
    assert abs(float(grad[0, V - 1]) - 1.0) < 1e-2 and abs(float(grad[0, 0]) - 1.0) < 1e-2


def test_convolution_past_32_bits():
    T, D = (1 << 20) + 41, 2056
    x, w, b = filled(1, T, D), filled(D, 4, dtype=torch.float32, seed=1), filled(D, dtype=torch.float32, seed=2)
    y, state = binding.causal_conv_fwd(x, w, b, True, want_state=True)
    first = x[:, T - 103:T - 100].contiguous()
    last, last_state = binding.causal_conv_fwd(x[:, T - 100:], w, b, True, initial_state=first, want_state=True)
    assert torch.equal(y[:, T - 100:], last) and torch.equal(state, last_state) and torch.equal(state, x[:, T - 3:])
    del y
    d_x = binding.causal_conv_bwd(x, w, x, b, True)[0]
    assert torch.equal(d_x[:, T - 100:], binding.causal_conv_bwd(x[:, T - 100:], w, x[:, T - 100:], b, True, initial_state=first)[0])


def test_more_workgroups_of_the_convolution_than_one_dimension_of_a_grid_has():
    B, T = 72_000_001, 17
    x, w = filled(B, T, 1), torch.tensor([[0.5, -2.0]], device=DEV)
    d_x, d_w, _, _ = binding.causal_conv_bwd(x, w, x)
    v = x[-1000:, :, 0].float()
    want = -2.0 * v + 0.5 * torch.nn.functional.pad(v, (0, 1))[:, 1:]
    assert (d_x[-1000:, :, 0].float() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    squares = sum(x[i:i + 8_000_000, :, 0].double().pow(2).sum() for i in range(0, B, 8_000_000))
    # squares of one sign: 17 additions of a chunk, 32 of a workgroup, then 32 sums of a 32nd of all rows each, whose roundings have either sign
    assert (d_w[0, 1].double() - squares).abs() <= squares * U * (B * 2 / 32 / 32 + 100)


def test_more_workgroups_of_the_scan_than_one_dimension_of_a_grid_has():
    B = (1 << 22) + 5
    x, dt, b = (filled(B, 1, 1, dtype=torch.float32, seed=i) for i in (1, 2, 3))
    a, bc = torch.full((1, 1), -0.5, device=DEV), b.unsqueeze(3)
    first = filled(B, 1, 1, dtype=torch.float32, seed=4)
    y, state = binding.selective_scan_fwd(x, dt, a, bc, bc, softplus=False, initial_state=first, want_state=True)
    d, u = dt[:, 0].double(), (dt * x)[:, 0].double()
    h = torch.exp(-0.5 * d) * first[:, 0].double() + u * b[:, 0].double()
    bound = 64 * U * (torch.exp(-0.5 * d) * first[:, 0].double().abs() + (u * b[:, 0].double()).abs())
    assert ((state[:, 0].double() - h).abs() <= bound).all() and ((y[:, 0].double() - h * b[:, 0].double()).abs() <= bound * b[:, 0].double().abs() + 1e-30).all()
    grads = binding.selective_scan_bwd(x, dt, a, bc, bc, x, softplus=False, initial_state=first, want_d_state=True)
    g = (b * x)[:, 0].double()
    assert ((grads[0][:, 0].double() - d * g * b[:, 0].double()).abs() <= 64 * U * (d * g * b[:, 0].double()).abs() + 1e-30).all()
    assert ((grads[7][:, 0].double() - torch.exp(-0.5 * d) * g).abs() <= 64 * U * (torch.exp(-0.5 * d) * g).abs()).all()


def test_scan_past_32_bits():
    """The last tokens of 2^31 elements, whose state has forgotten what was 300 tokens before: as by themselves.  (A step of 0.69 and more at a = -1 leaves
    less than 2^-300 of it.)"""
    T, D = (1 << 17) + 9, 16400
    x, b = filled(1, T, D), filled(1, T, 1, 4, seed=1)
    dt = filled(1, T, D, seed=2).abs_()
    a = torch.full((D, 4), -1.0, device=DEV)
    y, state = binding.selective_scan_fwd(x, dt, a, b, b, want_state=True)
    cut = T - 600
    last, last_state = binding.selective_scan_fwd(x[:, cut:], dt[:, cut:], a, b[:, cut:], b[:, cut:], want_state=True)
    size = state.abs().max()
    assert (state - last_state).abs().max() <= 2000 * U * size
    assert (y[:, -200:].float() - last[:, -200:].float()).abs().max() <= 2.0 ** -7 * last.float().abs().max()
    del y
    d_x = binding.selective_scan_bwd(x, dt, a, b, b, x)[0]
    want = binding.selective_scan_bwd(x[:, cut:], dt[:, cut:], a, b[:, cut:], b[:, cut:], x[:, cut:])[0]
    assert (d_x[:, -200:].float() - want[:, -200:].float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
