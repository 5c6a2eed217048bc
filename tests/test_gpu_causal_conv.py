"""Short causal convolution against its definition in 64 bits.

Bounds, in roundings u of fp32.  p is a sum of K products onto a bias: (K + 2) u of its magnitudes P.  silu(p) = p s(p): the exponent is rounded
twice (|p| 2 u), exponential, sum and reciprocal are within 2 u each, one product: (2 |p| + 8) u of the result, and silu's slope is below 1.1.
silu' has a slope below 1/2; its own steps are (2 |p| + 12) u of s (1 + |p| (1 - s)).  Errors of inputs are K products of those of p, and the final state's error;
sums over tokens take at most 128 additions of a chunk, 32 of a workgroup, and with few of them 32 + 32 more."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U
# B, T, D, K, lengths, states, silu, bias, slices
CASES = [(1, 1, 1, 2, None, False, False, False, False), (2, 1, 9, 4, None, True, True, True, False), (3, 2, 8, 8, [2, 0, 1], True, True, True, True),
         (2, 9, 130, 3, [9, 4], False, True, True, False), (2, 37, 64, 4, None, True, True, False, True), (4, 64, 33, 5, [64, 3, 0, 50], True, False, True, True),
         (1, 300, 257, 4, None, False, True, True, False), (2, 129, 40, 6, [128, 129], True, True, True, False), (2, 17, 500, 7, None, True, True, True, True),
         (60, 20, 12, 4, None, False, True, True, False), (1, 5, 2100, 4, [5], True, True, True, False)]


def make(case, type_, seed=0):
    B, T, D, K, lengths, states, _, with_bias, slices = case
    gen = torch.Generator().manual_seed(seed + T + D)
    normal = lambda *shape, dtype=seq.TYPES[type_]: torch.randn(shape, generator=gen).to(dtype).to(DEV)  # noqa: E731
    x = normal(B, T, 2 * D + 1)[:, :, 1:D + 1] if slices else normal(B, T, D)
    d_y = normal(T, B, D).transpose(0, 1) if slices else normal(B, T, D)
    w, b = normal(D, K, dtype=torch.float32), normal(D, dtype=torch.float32) if with_bias else None
    n = None if lengths is None else torch.tensor([v if v < T else v + 7 for v in lengths], dtype=torch.int32, device=DEV)  # above T counts as T
    if n is not None and 0 in lengths:
        n[lengths.index(0)] = -3  # below 0 as 0
    first, d_last = (normal(B, K - 1, D), normal(B, K - 1, D)) if states else (None, None)
    for i, v in enumerate(lengths or []):  # what is not read may be anything
        x[i, v:], d_y[i, v:] = float("nan"), float("nan")
    return x, w, b, d_y, n, first, d_last


def wide(*tensors):
    return [None if t is None else t.double().cpu() for t in tensors]


def near(got, want, slack, what):
    seq.near(got, want.numpy(), slack.numpy(), got.dtype, what)


@pytest.mark.parametrize("type_", list(seq.TYPES))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_sequences(case, type_):
    (B, T, D, K, lengths, states, silu, _, _), (x, w, b, d_y, n, first, d_last) = case, make(case, type_)
    x64, w64, b64, d64, first64, last64 = wide(x, w, b, d_y, first, d_last)
    b64, lengths = torch.zeros(D, dtype=torch.float64) if b64 is None else b64, lengths or [T] * B
    x64, d64 = torch.nan_to_num(x64), torch.nan_to_num(d64)
    y, state = binding.causal_conv_fwd(x, w, b, silu, n, first, True)
    want, want_state, p, P = ref.conv(x64, w64, b64, silu, lengths, first64)
    p_off = (K + 2) * U * P
    near(y, want, 1.1 * p_off + (2 * p.abs() + 8) * U * want.abs() if silu else p_off, "y")
    assert torch.equal(state.double().cpu(), want_state)
    assert torch.equal(binding.causal_conv_fwd(x, w, b, silu, n, first)[0], y)
    got = binding.causal_conv_bwd(x, w, d_y, b, silu, n, first, d_last, want_d_state=True)
    grads = ref.conv_gradient(x64, w64, b64, silu, lengths, first64, d64, last64)
    s = 1 / (1 + torch.exp(-p))
    e = (d64 * ref.d_silu(p)).abs() if silu else d64.abs()
    e_off = d64.abs() * (0.5 * p_off + (2 * p.abs() + 12) * U * s * (1 + p.abs() * (1 - s))) if silu else 0.0 * d64
    mags = lambda off: ref.conv_gradient(x64.abs(), w64.abs(), b64, silu, lengths, None if first64 is None else first64.abs(), None, None, off)  # noqa: E731
    size, off = mags(e), mags(e_off)
    last = torch.zeros(1, dtype=torch.float64) if last64 is None else last64.abs().max()
    steps = ((K + 2) * U, (128 + 32 + 64) * U, (128 + 32 + 64) * U, (K + 2) * U)
    assert (got[2] is None) == (b is None)
    for name, g, v, m, o, k in zip(("d_x", "d_weight", "d_bias", "d_state"), got, grads, size, off, steps):
        if g is not None:
            near(g, v, m * k + o * 1.001 + U * last * (name in ("d_x", "d_state")), name)
    again = binding.causal_conv_bwd(x, w, d_y, b, silu, n, first, d_last)
    assert again[3] is None and all(torch.equal(a, c) for a, c in zip(again[:2], got[:2]))


@pytest.mark.parametrize("type_", list(seq.TYPES))
@pytest.mark.parametrize("K,D", [(2, 5), (4, 64), (5, 333), (8, 24)])
def test_token_by_token_and_piece_by_piece(K, D, type_):
    """The same bits as the whole sequence: in pieces that hand their state on, and in single tokens with states in a pool."""
    case = (3, 23, D, K, None, True, True, True, False)
    x, w, b, d_y, _, first, d_last = make(case, type_)
    whole, last = binding.causal_conv_fwd(x, w, b, True, None, first, True)
    state, at = first, 0
    for size in (1, 2, 3, 17):
        piece, state = binding.causal_conv_fwd(x[:, at:at + size], w, b, True, None, state, True)
        assert torch.equal(piece, whole[:, at:at + size])
        at += size
    assert torch.equal(state, last)
    pool = torch.full((7, K - 1, D), float("nan"), dtype=x.dtype, device=DEV)
    slots = torch.tensor([5, -1, 0, 7, 2], dtype=torch.int32, device=DEV)
    rows = torch.tensor([0, 0, 1, 0, 2], device=DEV)
    pool[[5, 0, 2]] = first
    for t in range(23):
        y = binding.causal_conv_step(x[rows, t], w, pool, b, True, slots)
        assert torch.equal(y[[0, 2, 4]], whole[:, t]) and (y[[1, 3]] == 0.0).all()
    assert torch.equal(pool[[5, 0, 2]], last) and pool[[1, 3, 4, 6]].isnan().all()
    strided = torch.cat([x[:, 0], x[:, 1]], 1)[:, 1:D + 1]  # slices of a projection; states of their own rows
    own = first.clone()
    assert torch.equal(binding.causal_conv_step(strided, w, own), binding.causal_conv_step(strided.contiguous(), w, first.clone()))
    # errors of a sequence in two pieces: the second's first, its state's error the first's
    d_x, _, _, d_first = binding.causal_conv_bwd(x, w, d_y, b, True, None, first, d_last, True)
    middle = binding.causal_conv_fwd(x[:, :9], w, b, True, None, first, True)[1]
    second = binding.causal_conv_bwd(x[:, 9:], w, d_y[:, 9:], b, True, None, middle, d_last, True)
    assert torch.equal(second[0], d_x[:, 9:])
    if type_ == "fp32":  # (the state's error is rounded to its type between the pieces)
        first_piece = binding.causal_conv_bwd(x[:, :9], w, d_y[:, :9], b, True, None, first, second[3], True)
        assert (first_piece[0] - d_x[:, :9]).abs().max() <= 16 * U * (1 + d_x.abs().max()) and (first_piece[3] - d_first).abs().max() <= 16 * U * (1 + d_first.abs().max())


def test_a_bad_input_reaches_the_tokens_that_see_it():
    x, w = torch.ones(2, 50, 6, device=DEV), torch.ones(6, 4, device=DEV)
    x[1, 20, 3] = float("inf")
    w[3, 1] = 0.0
    y = binding.causal_conv_fwd(x, w)[0]
    assert (~y.isfinite()).nonzero().tolist() == [[1, t, 3] for t in (20, 21, 22, 23)] and y[1, 22, 3].isnan()


def test_captured_calls_replay():
    gen = torch.Generator().manual_seed(9)
    x, w, b = torch.randn(3, 200, 24, generator=gen).to(DEV), torch.randn(24, 4, generator=gen).to(DEV), torch.randn(24, generator=gen).to(DEV)
    pool = torch.zeros(3, 3, 24, device=DEV)

    def call():
        pool.zero_()
        y, state = binding.causal_conv_fwd(x, w, b, True, want_state=True)
        return (y, state, *binding.causal_conv_bwd(x, w, y, b, True)[:3], binding.causal_conv_step(x[:, 0], w, pool, b, True), pool.clone())
    call()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for turn in range(3):
        x.copy_(torch.randn(3, 200, 24, generator=gen))
        want = call()
        for graph, _ in graphs:
            graph.replay()
            call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, c) for a, c in zip(out, want)), turn


def test_refusals():
    x, w, b, n = torch.ones(2, 5, 8, device=DEV), torch.ones(8, 4, device=DEV), torch.ones(8, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    state = torch.ones(2, 3, 8, device=DEV)
    bad = [lambda: binding.causal_conv_fwd(x[0], w), lambda: binding.causal_conv_fwd(x, w[:7]), lambda: binding.causal_conv_fwd(x, w[0]), lambda: binding.causal_conv_fwd(x, w.half()),
           lambda: binding.causal_conv_fwd(x, w, b[:7]), lambda: binding.causal_conv_fwd(x, w, b, lengths=n[:1]), lambda: binding.causal_conv_fwd(x, w, lengths=n.long()),
           lambda: binding.causal_conv_fwd(x, w, initial_state=state[:1]), lambda: binding.causal_conv_fwd(x.half(), w, initial_state=state),
           lambda: binding.causal_conv_fwd(x.transpose(1, 2), w[:5]), lambda: binding.causal_conv_fwd(x.cpu(), w), lambda: binding.causal_conv_fwd(x, w.cpu()),
           lambda: binding.causal_conv_fwd(x.double(), w), lambda: binding.causal_conv_bwd(x, w, x[:1]), lambda: binding.causal_conv_bwd(x, w, x.half()),
           lambda: binding.causal_conv_bwd(x, w, x, d_final_state=state[:, :2]), lambda: binding.causal_conv_step(x[:, 0], w, state[:, :2]),
           lambda: binding.causal_conv_step(x[:, 0], w, state.half()), lambda: binding.causal_conv_step(x[:, 0], w, state, slots=n[:1]), lambda: binding.causal_conv_step(x, w, state)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.causal_conv_fwd(x, torch.ones(8, 9, device=DEV)), lambda: binding.causal_conv_fwd(x, w[:, :1].contiguous()), lambda: binding.causal_conv_fwd(x[:, :0], w),
                 lambda: binding.causal_conv_step(x[:, 0], w, state[:1])):
        with pytest.raises(binding.CnnError):
            call()
