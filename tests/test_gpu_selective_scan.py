"""Selective scan against its definition in 64 bits, within errors that are carried along with it (block_reference.scan)."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U
# B, T, D, N, G, lengths, states, skip and bias, softplus, slices
CASES = [(1, 1, 1, 1, 1, None, False, False, True, False), (2, 1, 6, 4, 2, [1, 0], True, True, True, True), (3, 7, 5, 3, 1, [7, 0, 2], True, True, True, False),
         (2, 9, 70, 16, 2, None, True, True, True, True), (1, 64, 33, 16, 1, None, False, True, False, False), (2, 65, 40, 8, 4, [65, 64], True, True, True, False),
         (1, 300, 20, 16, 2, None, True, True, True, True), (3, 200, 9, 11, 3, [200, 3, 130], False, False, True, False), (2, 130, 24, 32, 1, None, True, True, True, False),
         (1, 90, 34, 64, 2, [77], True, True, True, True), (1, 70, 10, 100, 1, None, True, True, False, False), (2, 20, 260, 128, 1, None, False, True, True, False),
         (40, 30, 130, 16, 1, None, True, True, True, False), (1, 1100, 8, 5, 1, [1099], True, True, True, False), (260, 9, 512, 16, 2, None, False, True, True, False)]


def make(case, type_, seed=0):
    B, T, D, N, G, lengths, states, extras, soft, slices = case
    gen = torch.Generator().manual_seed(seed + T + D + N)
    normal = lambda *shape, dtype=seq.TYPES[type_], by=1.0: (torch.randn(shape, generator=gen) * by).to(dtype).to(DEV)  # noqa: E731
    x = normal(B, T, 2 * D + 1)[:, :, 1:D + 1] if slices else normal(B, T, D)
    dt = normal(B, T, D) if soft else (torch.rand(B, T, D, generator=gen) * 0.3).to(seq.TYPES[type_]).to(DEV)
    bc = normal(B, T, 2 * G * N + 3)
    b, c = (bc[..., 3:3 + G * N].unflatten(2, (G, N)), bc[..., 3 + G * N:].unflatten(2, (G, N))) if slices else (normal(B, T, G, N), normal(B, T, G, N))
    d_y = normal(T, B, D).transpose(0, 1) if slices else normal(B, T, D)
    a = -(torch.rand(D, N, generator=gen) * 3.0 + 0.01).to(DEV)
    skip, bias = (normal(D, dtype=torch.float32), normal(D, dtype=torch.float32) * (1.0 if soft else 0.0) - (2.0 if soft else 0.0)) if extras else (None, None)
    n = None if lengths is None else torch.tensor([v if v < T else v + 7 for v in lengths], dtype=torch.int32, device=DEV)  # above T counts as T
    if n is not None and 0 in lengths:
        n[lengths.index(0)] = -3  # below 0 as 0
    first, d_last = (normal(B, D, N, dtype=torch.float32, by=2.0), normal(B, D, N, dtype=torch.float32)) if states else (None, None)
    for i, v in enumerate(lengths or []):  # what is not read may be anything
        for tensor in (x, dt, b, c, d_y):
            tensor[i, v:] = float("nan")
    return x, dt, a, b, c, skip, bias, d_y, n, first, d_last


def wide(*tensors):
    return [None if t is None else torch.nan_to_num(t.double().cpu()) for t in tensors]


def near(got, want, slack, what):
    seq.near(got, want.numpy(), slack.numpy(), got.dtype, what)


@pytest.mark.parametrize("type_", list(seq.TYPES))
@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c[:6]))
def test_sequences(case, type_):
    (B, T, D, N, G, lengths, states, extras, soft, _), (x, dt, a, b, c, skip, bias, d_y, n, first, d_last) = case, make(case, type_)
    x64, dt64, a64, b64, c64, skip64, bias64, d64, first64, last64 = wide(x, dt, a, b, c, skip, bias, d_y, first, d_last)
    zero = torch.zeros(D, dtype=torch.float64)
    (want, off), (grads, grads_off) = ref.scan(x64, dt64, a64, b64, c64, zero if skip is None else skip64, zero if bias is None else bias64, soft, lengths or [T] * B, first64, d64, last64)
    y, state = binding.selective_scan_fwd(x, dt, a, b, c, skip, bias, soft, n, first, True)
    near(y, want[0], off[0], "y")
    near(state, want[1], off[1], "state")
    y_only = binding.selective_scan_fwd(x, dt, a, b, c, skip, bias, soft, n, first)
    assert y_only[1] is None and torch.equal(y_only[0], y)
    got = binding.selective_scan_bwd(x, dt, a, b, c, d_y, skip, bias, soft, n, first, d_last, want_d_state=True)
    names = ("d_x", "d_dt", "d_a", "d_b", "d_c", "d_skip", "d_dt_bias", "d_state")
    assert [g is None for g in got] == [False] * 5 + [skip is None, bias is None, False]
    for name, g, v, o in zip(names, got, grads, grads_off):
        if g is not None:
            near(g, v, o, name)
    again = binding.selective_scan_bwd(x, dt, a, b, c, d_y, skip, bias, soft, n, first, d_last)
    assert again[7] is None and all(g is None or torch.equal(g, h) for g, h in zip(again[:7], got[:7]))


@pytest.mark.parametrize("type_", list(seq.TYPES))
@pytest.mark.parametrize("D,N,G", [(5, 3, 1), (64, 16, 2), (96, 64, 1), (20, 5, 4), (33, 128, 1), (16, 1, 1)])
def test_token_by_token(D, N, G, type_):
    """Single tokens with states in a pool against the whole sequence, both within their errors; rows without a sequence are zero and change nothing."""
    case = (3, 23, D, N, G, None, True, True, True, False)
    x, dt, a, b, c, skip, bias, _, _, first, _ = make(case, type_)
    want, off = ref.scan(*wide(x, dt, a, b, c, skip, bias), True, [23] * 3, wide(first)[0])
    pool = torch.full((7, D, N), float("nan"), device=DEV)
    slots, rows = torch.tensor([5, -1, 0, 7, 2], dtype=torch.int32, device=DEV), torch.tensor([0, 0, 1, 0, 2], device=DEV)
    pool[[5, 0, 2]] = first
    ys = []
    for t in range(23):
        y = binding.selective_scan_step(x[rows, t], dt[rows, t], a, b[rows, t], c[rows, t], pool, skip, bias, True, slots)
        assert (y[[1, 3]] == 0.0).all()
        ys.append(y[[0, 2, 4]])
    near(torch.stack(ys, 1), want[0], off[0], "y")
    near(pool[[5, 0, 2]], want[1], off[1], "state")
    assert pool[[1, 3, 4, 6]].isnan().all()
    own, again = first.clone(), first.clone()  # states of their own rows; slices of a projection
    bc = torch.cat([b[:, 0].flatten(1), c[:, 0].flatten(1)], 1)
    y = binding.selective_scan_step(x[:, 0], dt[:, 0], a, bc[:, :G * N].unflatten(1, (G, N)), bc[:, G * N:].unflatten(1, (G, N)), own, softplus=False)
    assert torch.equal(y, binding.selective_scan_step(x[:, 0].contiguous(), dt[:, 0].contiguous(), a, b[:, 0].contiguous(), c[:, 0].contiguous(), again, softplus=False))
    assert torch.equal(own, again)


@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_piece_by_piece(type_):
    """Pieces that hand their state on, forwards, and its error, backwards, within the errors of the whole."""
    case = (2, 333, 24, 16, 2, None, True, True, True, False)
    x, dt, a, b, c, skip, bias, d_y, _, first, d_last = make(case, type_)
    (want, off), (grads, grads_off) = ref.scan(*wide(x, dt, a, b, c, skip, bias), True, [333] * 2, *wide(first, d_y, d_last))
    cuts, states, ys = [0, 1, 100, 164, 333], [first], []
    for i, j in zip(cuts, cuts[1:]):
        y, state = binding.selective_scan_fwd(x[:, i:j], dt[:, i:j], a, b[:, i:j], c[:, i:j], skip, bias, initial_state=states[-1], want_state=True)
        ys.append(y), states.append(state)
    near(torch.cat(ys, 1), want[0], off[0], "y")
    near(states[-1], want[1], off[1], "state")
    error, parts = d_last, []
    for i, j, state in list(zip(cuts, cuts[1:], states))[::-1]:
        g = binding.selective_scan_bwd(x[:, i:j], dt[:, i:j], a, b[:, i:j], c[:, i:j], d_y[:, i:j], skip, bias, initial_state=state, d_final_state=error, want_d_state=True)
        parts.insert(0, g)
        error = g[7]
    for k, name in ((0, "d_x"), (1, "d_dt"), (3, "d_b"), (4, "d_c")):
        near(torch.cat([p[k] for p in parts], 1), grads[k], grads_off[k], name)
    near(sum(p[2] for p in parts), grads[2], grads_off[2] + 4 * U * grads[2].abs(), "d_a")
    near(error, grads[7], grads_off[7], "d_state")


def test_state_may_be_updated_in_place():
    x, dt, a, b, c, skip, bias, _, _, first, _ = make((2, 700, 8, 16, 1, None, True, True, True, False), "fp32")
    want = binding.selective_scan_fwd(x, dt, a, b, c, skip, bias, initial_state=first, want_state=True)
    L, stream = binding.lib(), binding._stream()
    for T in (700, 40):  # cut into segments, and whole
        want = binding.selective_scan_fwd(x[:, :T], dt[:, :T], a, b[:, :T], c[:, :T], skip, bias, initial_state=first, want_state=True)
        state, y, shape = first.clone(), torch.empty(2, T, 8, device=DEV), binding.SelectiveScanShape(2, T, 8, 16, 1, 0, 1)
        need = L.cnn_selective_scan_fwd_workspace_bytes(shape)
        assert (need > 0) == (T == 700)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
        row, head = lambda t: binding.Tokens(t.data_ptr(), *t.stride()[:2]), lambda t: binding.Heads(t.data_ptr(), *t.stride()[:3])  # noqa: E731
        p = binding._ptr
        assert L.cnn_selective_scan_fwd(shape, row(x), row(dt), p(a), head(b), head(c), p(skip), p(bias), None, p(state), p(y), p(state), p(ws), need, stream) == 0
        assert torch.equal(y, want[0]) and torch.equal(state, want[1])


def test_a_single_token_of_any_stride():
    """Tokens cut out of something long: their stride is never used, however large."""
    x, a, b = torch.ones(2, 1, 8, device=DEV), -torch.ones(8, 4, device=DEV), torch.ones(2, 1, 2, 4, device=DEV)
    far = lambda t: t.as_strided(t.shape, (t.stride(0), 1 << 40, *t.stride()[2:]))  # noqa: E731
    want, got = binding.selective_scan_fwd(x, x, a, b, b, want_state=True), binding.selective_scan_fwd(far(x), far(x), a, far(b), far(b), want_state=True)
    assert all(torch.equal(v, w) for v, w in zip(want, got))
    w = torch.ones(8, 4, device=DEV)
    assert torch.equal(binding.causal_conv_fwd(far(x), w)[0], binding.causal_conv_fwd(x, w)[0])


def test_extreme_steps():
    """Steps of thousands (the state is forgotten), of next to nothing, a of zero, far negative dt: no NaN, and softplus keeps its small values."""
    D, N = 6, 16
    dt = torch.tensor([[5000.0, 88.0, 21.0, -30.0, -80.0, -200.0]], device=DEV).expand(3, D)[None].contiguous()
    x, b, c = torch.ones(1, 3, D, device=DEV), torch.ones(1, 3, 1, N, device=DEV), torch.ones(1, 3, 1, N, device=DEV)
    a = -torch.rand(D, N, device=DEV) - 0.5
    a[:, 0] = 0.0
    first = torch.ones(1, D, N, device=DEV)
    (want, off), (grads, grads_off) = ref.scan(*wide(x, dt, a, b, c), torch.zeros(D, dtype=torch.float64), torch.zeros(D, dtype=torch.float64), True, [3], *wide(first, x, first))
    y, state = binding.selective_scan_fwd(x, dt, a, b, c, initial_state=first, want_state=True)
    near(y, want[0], off[0], "y")
    near(state, want[1], off[1], "state")
    got = binding.selective_scan_bwd(x, dt, a, b, c, x, initial_state=first, d_final_state=first, want_d_state=True)
    for k, name in ((0, "d_x"), (1, "d_dt"), (2, "d_a"), (3, "d_b"), (4, "d_c"), (7, "d_state")):
        near(got[k], grads[k], grads_off[k], name)
    tiny = binding.selective_scan_fwd(x, dt, a, b, c, want_state=True)[1][0, 3:, 0] / 3  # softplus itself: ln(1 + e) = e there
    assert ((tiny.double().cpu() - torch.exp(dt[0, 0, 3:].double().cpu())).abs() <= 700 * U * torch.exp(dt[0, 0, 3:].double().cpu()) + 1e-37).all()


def test_captured_calls_replay():
    case = (2, 200, 24, 16, 1, None, False, True, True, False)
    x, dt, a, b, c, skip, bias, d_y, _, _, _ = make(case, "fp32")
    pool = torch.zeros(2, 24, 16, device=DEV)

    def call():
        pool.zero_()
        y, state = binding.selective_scan_fwd(x, dt, a, b, c, skip, bias, want_state=True)
        one = binding.selective_scan_step(x[:, 0], dt[:, 0], a, b[:, 0], c[:, 0], pool, skip, bias)
        return (y, state, one, pool.clone(), *binding.selective_scan_bwd(x, dt, a, b, c, d_y, skip, bias)[:7])
    call()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for turn in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(turn)))
        want = call()
        for graph, _ in graphs:
            graph.replay()
            call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(v, w) for v, w in zip(out, want)), turn


def test_refusals():
    x, a, b, n = torch.ones(2, 5, 8, device=DEV), -torch.ones(8, 4, device=DEV), torch.ones(2, 5, 2, 4, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    d, state = torch.ones(8, device=DEV), torch.ones(2, 8, 4, device=DEV)
    fwd, bwd, step = binding.selective_scan_fwd, binding.selective_scan_bwd, binding.selective_scan_step
    bad = [lambda: fwd(x[0], x[0], a, b, b), lambda: fwd(x, x[:1], a, b, b), lambda: fwd(x, x.half(), a, b, b), lambda: fwd(x, x, a[:7], b, b), lambda: fwd(x, x, a[:, :3], b, b),
           lambda: fwd(x, x, a.half(), b, b), lambda: fwd(x, x, a, b[:, :4], b[:, :4]), lambda: fwd(x, x, a, b, b[:, :, :1]), lambda: fwd(x, x, a, b.half(), b.half()),
           lambda: fwd(x, x, a, b, b, d[:7]), lambda: fwd(x, x, a, b, b, d, d.half()), lambda: fwd(x, x, a, b, b, lengths=n.long()), lambda: fwd(x, x, a, b, b, lengths=n[:1]),
           lambda: fwd(x, x, a, b, b, initial_state=state[:1]), lambda: fwd(x.transpose(1, 2), x.transpose(1, 2), a[:5], b, b), lambda: fwd(x.cpu(), x, a, b, b),
           lambda: fwd(x, x, a.cpu(), b, b), lambda: fwd(x.double(), x.double(), a, b.double(), b.double()), lambda: bwd(x, x, a, b, b, x[:1]), lambda: bwd(x, x, a, b, b, x.half()),
           lambda: bwd(x, x, a, b, b, x, d_final_state=state[:, :7]), lambda: step(x[:, 0], x[:, 0], a, b[:, 0], b[:, 0], state[:, :7]),
           lambda: step(x[:, 0], x[:, 0], a, b[:, 0], b[:, 0], state.half()), lambda: step(x[:, 0], x[:, 0], a, b[:, 0], b[:, 0], state, slots=n[:1]), lambda: step(x, x, a, b, b, state)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    b3, wide_b = torch.ones(2, 5, 3, 4, device=DEV), torch.ones(2, 5, 1, 129, device=DEV)
    for call in (lambda: fwd(x, x, a, b3, b3), lambda: fwd(x, x, -torch.ones(8, 129, device=DEV), wide_b, wide_b), lambda: fwd(x[:, :0], x[:, :0], a, b[:, :0], b[:, :0]),
                 lambda: step(x[:, 0], x[:, 0], a, b[:, 0], b[:, 0], state[:1])):
        with pytest.raises(binding.CnnError):
            call()
