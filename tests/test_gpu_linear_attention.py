"""Linear attention, forward, backward and token by token, against the recurrences in 64 bits.

Bounds.  With A the same sums over magnitudes: every sum of n terms in fp32 is off by at most n half steps of A, whatever its order
(Dk terms inside a score, T scores and states inside an output); a power of a decay is off by a few half steps, plus those of its
exponent, which count only while the power itself is not small (T + 64 in all).  What is cut into two pieces of bfloat16 is off by
2^-17 of itself: state and scores of bfloat16 inputs, together 2^-16, and for half, where products of two second pieces are left out
too, 2^-15.  The state itself is fp32 sums of exact products for every type (3 pieces: 2^-24).
"""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DECAYS = [0.96875, 1.0, 0.5, 0.0, 1 - 2.0 ** -12, 0.9]
CUT = {"fp32": 0.0, "bf16": 2.0 ** -16, "fp16": 2.0 ** -15}

# B, T, H, Hk, Dk, Dv, lengths, states, slices of one tensor
CASES = [(1, 1, 1, 1, 1, 1, None, False, False), (2, 5, 3, 1, 7, 9, [5, 0], True, True), (1, 16, 2, 2, 16, 8, None, True, False),
         (1, 64, 2, 2, 32, 32, None, False, True), (2, 65, 4, 2, 33, 40, [64, 65], True, True), (3, 31, 2, 2, 96, 16, [0, 1, 31], True, False),
         (1, 130, 2, 1, 64, 100, None, False, True), (2, 200, 1, 1, 128, 128, [33, 200], True, False), (1, 70, 1, 1, 256, 256, None, True, True),
         (1, 90, 1, 1, 250, 20, None, False, False), (1, 90, 2, 1, 24, 256, [77], True, True),
         # sequences that are cut into segments
         (1, 600, 2, 2, 48, 80, None, True, False), (2, 777, 2, 1, 32, 32, [777, 300], True, True), (1, 1100, 1, 1, 16, 160, [1099], False, False),
         (1, 1025, 3, 3, 64, 64, [512], True, True)]


def make(case, type_, seed=0):
    B, T, H, Hk, Dk, Dv, lengths, states, fused = case
    dtype, gen = ref.TYPES[type_], torch.Generator().manual_seed(seed + T)
    normal = lambda *s: torch.randn(s, generator=gen).to(dtype)  # noqa: E731
    if fused:
        q, k, v, d_o = normal(B, T, H * (Dk + Dv) + Hk * (Dk + Dv)).to(DEV).split([H * Dk, Hk * Dk, Hk * Dv, H * Dv], 2)
        q, k, v, d_o = q.unflatten(2, (H, Dk)), k.unflatten(2, (Hk, Dk)), v.unflatten(2, (Hk, Dv)), d_o.unflatten(2, (H, Dv))
    else:  # heads before tokens in memory
        q, k, v, d_o = (normal(B, h, T, d).to(DEV).transpose(1, 2) for h, d in ((H, Dk), (Hk, Dk), (Hk, Dv), (H, Dv)))
    decay = torch.tensor((DECAYS * 2)[:H], device=DEV)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    state = lambda: torch.randn((B, H, Dk, Dv), generator=gen).to(DEV) if states else None  # noqa: E731
    return q, k, v, decay, d_o, n, state(), state()


def in_64(*tensors):
    return [None if t is None else ref.numpy64(t) for t in tensors]


def magnitudes(*arrays):
    return [None if a is None else np.abs(a) for a in arrays]


def steps(case):
    return 2.0 ** -24 * (case[4] + case[5] + 3 * case[1] + 64)


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("case", CASES, ids=[str(c[:6]) for c in CASES])
def test_forward(case, type_):
    q, k, v, decay, _, n, initial, _ = make(case, type_)
    q64, k64, v64, a64, i64 = in_64(q, k, v, decay, initial)
    want, state = ref.linear_attention(q64, k64, v64, a64, 0.3, case[6], i64)
    size, state_size = ref.linear_attention(*magnitudes(q64, k64, v64, a64), 0.3, case[6], *magnitudes(i64))
    o, last = binding.linear_attention_fwd(q, k, v, decay, 0.3, lengths=n, initial_state=initial, want_state=True)
    assert o.dtype == q.dtype and last.dtype == torch.float32 and o.is_contiguous()
    ref.near(o, want, size * (steps(case) + CUT[type_]), q.dtype, "o %s" % type_)
    ref.near(last, state, state_size * steps(case), torch.float32, "state %s" % type_)
    again, none = binding.linear_attention_fwd(q, k, v, decay, 0.3, lengths=n, initial_state=initial)
    assert none is None and torch.equal(again, o)


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("case", CASES, ids=[str(c[:6]) for c in CASES])
def test_backward(case, type_):
    q, k, v, decay, d_o, n, initial, d_final = make(case, type_)
    arrays = in_64(q, k, v, decay, d_o)
    i64, f64 = in_64(initial, d_final)
    want = ref.linear_attention_gradient(*arrays, 0.3, case[6], i64, f64)
    size = ref.linear_attention_gradient(*magnitudes(*arrays), 0.3, case[6], *magnitudes(i64, f64))
    got = binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, lengths=n, initial_state=initial, d_final_state=d_final, want_d_state=True)
    for name, g, w, m, dtype in zip(("d_q", "d_k", "d_v", "d_state"), got, want, size, [q.dtype] * 3 + [torch.float32]):
        assert g.dtype == dtype and g.is_contiguous()
        cut = 0.0 if name == "d_state" else CUT[type_]
        ref.near(g, w, m * (steps(case) + cut), dtype, "%s %s" % (name, type_))
    again = binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, lengths=n, initial_state=initial, d_final_state=d_final)
    assert again[3] is None and all(torch.equal(x, y) for x, y in zip(again[:3], got[:3]))


# widths of three tiles of 32, and blocks of 96 columns
THREES = [(2, 45, 2, 1, 96, 96, [45, 3], True, True), (1, 333, 2, 2, 80, 96, None, True, True), (1, 100, 3, 1, 77, 90, [99], True, False),
          (1, 700, 1, 1, 96, 160, None, True, False), (2, 640, 2, 1, 64, 88, [600, 33], False, True), (1, 70, 1, 1, 200, 96, None, True, True),
          (1, 65, 1, 1, 24, 72, None, False, False), (1, 390, 1, 1, 128, 192, [388], True, True)]


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("case", THREES, ids=[str(c[:6]) for c in THREES])
def test_widths_of_three_tiles(case, type_):
    test_forward(case, type_)
    test_backward(case, type_)


def test_backward_against_differences_of_the_forward_call():
    """The loss sum(o w) + sum(state u) in fp32, perturbed along random directions: the slope is the gradient's product with them."""
    case = (2, 90, 2, 1, 20, 24, [90, 51], True, False)
    q, k, v, decay, w, n, initial, u = make(case, "fp32")
    decay = torch.tensor([0.96875, 0.9], device=DEV)

    def loss(q, k, v, initial):
        o, state = binding.linear_attention_fwd(q, k, v, decay, 0.3, lengths=n, initial_state=initial, want_state=True)
        return float((o.double() * w.double()).sum() + (state.double() * u.double()).sum())

    grads = binding.linear_attention_bwd(q, k, v, decay, w, 0.3, lengths=n, initial_state=initial, d_final_state=u, want_d_state=True)
    inputs = [q, k, v, initial]
    for i in range(4):
        d = torch.randn(inputs[i].shape, generator=torch.Generator().manual_seed(i)).to(DEV)
        h = 1.0 / 64  # the loss is linear in q, v and the state, and in k: differences are exact to rounding
        up, down = (loss(*[x + s * h * d if j == i else x for j, x in enumerate(inputs)]) for s in (1, -1))
        want = float((grads[i].double() * d.double()).sum())
        size = float((grads[i].double() * d.double()).abs().sum())
        total = float(sum((g.double() * x.double()).abs().sum() for g, x in zip(grads, inputs)))
        # each loss is off by some steps of fp32 of its terms, divided by 2 h
        assert abs((up - down) / (2 * h) - want) <= 2.0 ** -24 * (64 * total / (2 * h) + 256 * size), i


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1), (3, 2, 1, 5, 7), (2, 4, 2, 64, 64), (2, 3, 3, 128, 36), (5, 2, 1, 33, 40), (1, 1, 1, 256, 256),
                                   (4, 2, 2, 100, 30)])
def test_tokens_one_by_one(shape, type_):
    """Steps against the recurrence, with rows that come and go, in slots of a pool that nothing else may touch."""
    B, H, Hk, Dk, Dv = shape
    T, pool = 6, B + 3
    q, k, v, decay, _, _, _, _ = make((B, T, H, Hk, Dk, Dv, None, False, True), type_)
    gen = torch.Generator().manual_seed(9)
    state = torch.randn((pool, H, Dk, Dv), generator=gen).to(DEV)
    before = state.clone()
    slots = torch.randperm(pool, generator=gen)[:B].to(torch.int32)
    lengths = [(3 * b + T) % (T + 1) for b in range(B)]  # a row ends, another goes on
    q64, k64, v64, a64 = in_64(q, k, v, decay)
    initial = ref.numpy64(before)[slots.numpy()]
    want, last = ref.linear_attention(q64, k64, v64, a64, 0.3, lengths, initial)
    size, last_size = ref.linear_attention(*magnitudes(q64, k64, v64, a64), 0.3, lengths, np.abs(initial))
    case = (B, T, H, Hk, Dk, Dv)
    for t in range(T):
        now = torch.tensor([int(s) if t < n else (-1 if b % 2 else pool + 7) for b, (s, n) in enumerate(zip(slots, lengths))], dtype=torch.int32)
        o = binding.linear_attention_step(q[:, t], k[:, t], v[:, t], decay, state, 0.3, slots=now.to(DEV))
        ref.near(o, want[:, t], size[:, t] * steps(case), q.dtype, "o of token %d %s" % (t, type_))
    used = slots.long()
    ref.near(state[used.to(DEV)], last, last_size * steps(case), torch.float32, "state %s" % type_)
    others = [s for s in range(pool) if s not in used.tolist()]
    assert torch.equal(state[others], before[others])


def test_states_larger_than_the_caches():
    """256 MB of states in one call against two calls of half of them, whose tokens are tested above: the same arithmetic."""
    B, H, D = 256, 16, 128
    gen = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn(B, H, D, generator=gen, device=DEV).bfloat16() for _ in range(3))
    state = torch.randn(B + 3, H, D, D, generator=gen, device=DEV)
    decay, other = torch.linspace(0.5, 1.0, H, device=DEV), state.clone()
    slots = torch.randperm(B + 3, generator=gen, device=DEV)[:B].to(torch.int32)
    slots[5], slots[200] = -1, B + 3
    for _ in range(2):
        o = binding.linear_attention_step(q, k, v, decay, state, 0.3, slots=slots)
        halves = [binding.linear_attention_step(q[i:i + 128], k[i:i + 128], v[i:i + 128], decay, other, 0.3, slots=slots[i:i + 128])
                  for i in (0, 128)]
        assert torch.equal(o, torch.cat(halves)) and torch.equal(state, other)
        assert (o[5] == 0).all() and (o[200] == 0).all()


def test_prompt_then_tokens_is_the_whole_sequence():
    case = (2, 700, 2, 2, 64, 96, None, False, True)
    q, k, v, decay, _, _, _, _ = make(case, "fp32")
    whole, last = binding.linear_attention_fwd(q, k, v, decay, 0.3, want_state=True)
    o, state = binding.linear_attention_fwd(q[:, :697], k[:, :697], v[:, :697], decay, 0.3, want_state=True)
    size, state_size = (torch.from_numpy(x).to(DEV) for x in ref.linear_attention(*magnitudes(*in_64(q, k, v, decay)), 0.3))
    assert ((o - whole[:, :697]).abs() <= 2 * steps(case) * size[:, :697]).all()
    for t in range(697, 700):
        o = binding.linear_attention_step(q[:, t], k[:, t], v[:, t], decay, state, 0.3)
        assert ((o - whole[:, t]).abs() <= 2 * steps(case) * size[:, t]).all()
    assert ((state - last).abs() <= 2 * steps(case) * state_size).all()


def test_tokens_past_the_length_are_not_read():
    case = (3, 150, 2, 2, 40, 64, [150, 77, 0], True, False)
    q, k, v, decay, d_o, n, initial, d_final = make(case, "bf16")
    want = binding.linear_attention_fwd(q, k, v, decay, 0.3, n, initial, True)
    d_want = binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, n, initial, d_final, True)
    for x in (q, k, v, d_o):
        x[1, 77:] = float("nan")
        x[2] = float("inf")
    got = binding.linear_attention_fwd(q, k, v, decay, 0.3, n, initial, True)
    d_got = binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, n, initial, d_final, True)
    for x, y in zip(want + d_want, got + d_got):
        assert torch.equal(x, y) and torch.isfinite(x).all()
    assert (got[0][1, 77:] == 0).all() and (got[0][2] == 0).all() and torch.equal(got[1][2], initial[2]) and torch.equal(d_got[3][2], d_final[2])
    # lengths out of range count as none and all
    odd = binding.linear_attention_fwd(q[:1], k[:1], v[:1], decay, 0.3, torch.tensor([1 << 30], dtype=torch.int32, device=DEV), initial[:1])[0]
    assert torch.equal(odd, want[0][:1])
    assert (binding.linear_attention_fwd(q[:1], k[:1], v[:1], decay, 0.3, torch.tensor([-5], dtype=torch.int32, device=DEV))[0] == 0).all()


def test_not_finite_rows_of_queries_stay_alone():
    """A query does not enter the state: the others' rows are as without it."""
    case = (1, 100, 1, 1, 32, 64, None, False, False)
    q, k, v, decay, _, _, _, _ = make(case, "fp32")
    want = binding.linear_attention_fwd(q, k, v, decay)[0]
    q[0, 40] = float("nan")
    got = binding.linear_attention_fwd(q, k, v, decay)[0]
    rest = [t for t in range(100) if t != 40]
    assert got[0, 40].isnan().all() and torch.equal(got[:, rest], want[:, rest])


def test_state_in_place():
    case = (1, 900, 2, 2, 32, 48, None, True, False)  # cut into segments
    q, k, v, decay, _, _, initial, _ = make(case, "bf16")
    L, p = binding.lib(), binding._ptr
    want, last = binding.linear_attention_fwd(q, k, v, decay, 0.3, None, initial, True)
    shape = binding.LinearShape(1, 900, 2, 2, 32, 48, 1)
    heads = lambda t: binding.Heads(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))  # noqa: E731
    need = L.cnn_linear_attention_fwd_workspace_bytes(shape)
    assert need > 0
    o, ws = torch.empty_like(want), torch.empty(need, dtype=torch.uint8, device=DEV)
    assert L.cnn_linear_attention_fwd(shape, heads(q), heads(k), heads(v), p(decay), 0.3, None, p(initial), p(o), p(initial), p(ws), need,
                                      binding._stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(initial, last)


def test_other_stream_and_graph():
    case = (1, 700, 2, 1, 32, 64, None, True, True)
    q, k, v, decay, d_o, _, initial, d_final = make(case, "bf16")
    state = torch.zeros(1, 2, 32, 64, device=DEV)
    everything = lambda s: (binding.linear_attention_fwd(q, k, v, decay, 0.3, None, initial, True) +  # noqa: E731
                            binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, None, initial, d_final, True) +
                            (binding.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, s, 0.3),))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        everything(state)
    side.synchronize()
    state.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(state)
    eager = torch.zeros_like(state)
    for i in range(3):
        q.copy_(torch.randn(q.shape, device=DEV))
        want = everything(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got)) and torch.equal(state, eager), i


@pytest.mark.parametrize("T", [40, 900])
def test_a_scale_of_zero_gives_gradients_of_zero(T):
    """Without states' errors any scale is allowed; 900 tokens are cut into segments."""
    q, k, v, decay, d_o, _, _, _ = make((1, T, 2, 1, 32, 48, None, False, True), "fp32")
    for scale in (0.0, 2.0 ** -140):
        for g in binding.linear_attention_bwd(q, k, v, decay, d_o, scale)[:3]:
            assert torch.isfinite(g).all() and (g.abs() <= 2.0 ** -100).all()


def test_refusals():
    q, k, v = (torch.zeros(2, 3, 4, 8, device=DEV) for _ in range(3))
    decay, fwd = torch.ones(4, device=DEV), binding.linear_attention_fwd
    with pytest.raises(TypeError):
        fwd(None, k, v, decay)
    for bad in ((q[0], k, v, decay), (q.double(), k, v, decay), (q, k.half(), v, decay), (q, k[:, :2], v, decay), (q, k[..., :4], v, decay),
                (q, k, v[:, :, :2], decay), (q, k, v, decay[:2]), (q, k, v, decay.double()), (q.cpu(), k, v, decay),
                (q.transpose(2, 3), k, v, decay), (q.expand(2, 3, 4, 8)[..., :1].expand(2, 3, 4, 8), k, v, decay)):
        with pytest.raises(ValueError):
            fwd(*bad)
    with pytest.raises(binding.CnnError):
        fwd(q, k[:, :, :3], v[:, :, :3], decay)  # 4 query heads on 3
    with pytest.raises(binding.CnnError):
        fwd(q[:, :0], k[:, :0], v[:, :0], decay)
    wide = torch.zeros(1, 1, 1, 257, device=DEV)
    with pytest.raises(binding.CnnError):
        fwd(wide, wide, wide, decay[:1])
    n = torch.zeros(2, dtype=torch.int32, device=DEV)
    for kw in ({"lengths": n.long()}, {"lengths": n[:1]}, {"initial_state": torch.zeros(2, 4, 8, 7, device=DEV)}):
        with pytest.raises(ValueError):
            fwd(q, k, v, decay, **kw)
    with pytest.raises(ValueError):
        binding.linear_attention_bwd(q, k, v, decay, q[:, :2])
    with pytest.raises(binding.CnnError):
        binding.linear_attention_bwd(q, k, v, decay, v, 0.0, want_d_state=True)
    state = torch.zeros(2, 4, 8, 8, device=DEV)
    step = binding.linear_attention_step
    with pytest.raises(ValueError):
        step(q, k, v, decay, state)
    with pytest.raises(ValueError):
        step(q[:, 0], k[:, 0], v[:, 0], decay, state[..., :4])
    with pytest.raises(binding.CnnError):
        step(q[:, 0], k[:, 0], v[:, 0], decay, state[:1])  # a pool of one for two rows
