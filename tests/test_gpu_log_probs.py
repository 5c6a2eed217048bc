"""Log probabilities, entropy, top tokens and their gradient against the definition in 64 bits.

Bounds, in roundings u of fp32, with z = scale (l - max).  z and its exponent are off by 3 |z| u, e = exp(z) by (3 |z| + 2) u of itself; sums take at most 32 additions of
a lane, 6 of a wave, 16 of a workgroup and, joined, 1 + 6 + 4 more with three roundings each: 90 u of a sum of one sign.  So ln sum is off by
(3 E|z| + 92) u and its own 2 u |ln sum|, a log probability by 3 |z| u more.  The entropy's other term is a sum of e z over the sum of e: off by
E|z| (90 + 92 + 3 E|z|) u + E(3 z^2 + 2 |z|) u.  Gradients: p is off by what ln p is, relative to itself, and 2 u + 2 u |ln p| of the exponent."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U
INF = float("inf")
# rows, vocabulary, given, top: one token; a wave's limits; a workgroup's; rows cut into parts, few and many of them
SHAPES = [(1, 1, 1, 1), (3, 7, 1, 7), (37, 60, 1, 33), (11, 128, 2, 40), (21, 129, 1, 50), (70, 256, 1, 5), (9, 511, 3, 64), (5, 513, 1, 20), (4, 2049, 64, 3), (6, 4100, 1, 33), (3, 8193, 2, 64), (2, 32003, 1, 20),
          (3, 32769, 1, 64), (2, 50021, 5, 20), (1, 200003, 256, 40), (300, 40007, 1, 0), (2, 65536, 1, 64), (3, 65537, 2, 7), (2, 131101, 1, 64), (300, 33000, 3, 5)]


def make(shape, type_, seed=0):
    N, V, M, _ = shape
    gen = torch.Generator().manual_seed(seed + N + V)
    logits = torch.randn(N, V, generator=gen) * 3.0
    logits[:, gen.initial_seed() % V] += 9.0
    tokens = torch.randint(0, V, (N, M), generator=gen)
    if M > 1:
        tokens[:, 1] = tokens[:, 0]  # the same token twice
        tokens[0, -1] = -1
        tokens[-1, -1] = V
    return logits.to(seq.TYPES[type_]).to(DEV), (tokens if M > 1 else tokens[:, 0]).contiguous().to(DEV), torch.randn(N, M, generator=gen).to(DEV), torch.randn(N, generator=gen).to(DEV)


def bounds(logits, tokens, scale):
    """Of the log probabilities of all tokens, of the entropy."""
    z = logits * scale
    z = torch.where(torch.isinf(z), torch.zeros_like(z), z - z.amax(1, keepdim=True)).abs()
    lp = ref.log_probs(logits, tokens, scale, 0)[4]
    p = torch.exp(lp)
    mean, square = (p * z).sum(1, keepdim=True), (p * z * z).sum(1, keepdim=True)
    log_sum = torch.log(torch.exp(torch.where(torch.isinf(logits), -INF, -z)).sum(1, keepdim=True)).abs()
    sums = (3 * mean + 94 + 2 * log_sum) * U
    return sums + 3 * z * U, (sums + (mean * (182 + 3 * mean) + 3 * square + 2 * mean) * U + 2 * U * (mean + log_sum))[:, 0]


def check(logits, tokens, d, d_h, scale, top, given_is_finite=True):
    l64, t64 = logits.double().cpu(), tokens.cpu().long().view(len(tokens), -1)
    s64 = float(torch.tensor(scale, dtype=torch.float32))
    lp, entropy, stats, top_lp, top_tokens = binding.log_probs_fwd(logits, tokens, scale, top)
    want = ref.log_probs(l64, t64, s64, top)
    off, h_off = bounds(l64, t64, s64)
    known = (t64 >= 0) & (t64 < logits.shape[1])
    if given_is_finite:
        seq.near(lp.view_as(t64), want[0].numpy(), (off.gather(1, torch.where(known, t64, 0)) * known).numpy(), torch.float32, "log probabilities")
    seq.near(entropy, want[1].numpy(), h_off.numpy(), torch.float32, "entropy")
    if top:
        assert torch.equal(top_tokens.cpu().long(), want[3])
        finite = torch.isfinite(want[2])
        assert torch.equal(torch.isfinite(top_lp.cpu()), finite)
        seq.near(torch.where(finite, top_lp.cpu(), 0.0), torch.where(finite, want[2], 0.0).numpy(), off.gather(1, want[3]).numpy(), torch.float32, "top")
    else:
        assert top_lp is None and top_tokens is None
    for error in (None, d_h):
        got = binding.log_probs_bwd(logits, tokens, stats, d.view_as(lp), error, scale)
        d64, e64 = d.double().cpu().view_as(t64), None if error is None else error.double().cpu()
        want_d = ref.log_probs_gradient(l64, t64, s64, d64, e64)
        p, lps = torch.exp(want[4]), torch.where(torch.isinf(want[4]), 0.0, want[4])
        relative = off + 4 * U + 2 * U * lps.abs()
        total = torch.where(known, d64.abs(), 0.0).sum(1, keepdim=True)
        given = torch.zeros_like(p).scatter_add(1, torch.where(known, t64, 0), torch.where(known, d64.abs(), 0.0))
        slack = p * total * (relative + 16 * U) + given * 8 * U
        if error is not None:
            slack = slack + e64.abs()[:, None] * p * ((lps.abs() + want[1][:, None]) * (relative + 6 * U) + off + h_off[:, None])
        seq.near(got, want_d.numpy(), (abs(s64) * slack).numpy(), got.dtype, "gradient %d" % (error is not None))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_rows(type_, shape):
    logits, tokens, d, d_h = make(shape, type_)
    check(logits, tokens, d, d_h, 0.7, shape[3])


@pytest.mark.parametrize("V", [100, 5000, 70001])
@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_equal_logits_keep_the_order_of_their_tokens(V, type_):
    """Rows of one value (the lists of candidates overflow), of few values, zeros of both signs among them, and of falling ones."""
    gen = torch.Generator().manual_seed(1)
    logits = torch.zeros(5, V)
    logits[1] = torch.randint(-2, 3, (V,), generator=gen) * 0.5
    logits[2] = torch.where(torch.rand(V, generator=gen) < 0.5, -0.0, 0.0)
    logits[3] = -torch.arange(V) * (60.0 / V)
    logits[4] = torch.arange(V) * (60.0 / V)
    tokens = torch.randint(0, V, (5,), generator=gen)
    check(logits.to(seq.TYPES[type_]).to(DEV), tokens.to(torch.int32).to(DEV), torch.randn(5, 1, generator=gen).to(DEV), torch.randn(5, generator=gen).to(DEV), 1.0, 64)


@pytest.mark.parametrize("V", [40, 3000, 66000])
@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_impossible_tokens(V, type_):
    """Masked logits, whole pieces of a row among them; rows of one possible token and of none."""
    gen = torch.Generator().manual_seed(2)
    logits = torch.randn(4, V, generator=gen)
    logits[0, torch.rand(V, generator=gen) < 0.6] = -INF
    logits[0, 0] = 1.0
    logits[1, : V * 9 // 10] = -INF
    logits[2, :] = -INF
    logits[2, V // 3] = -5.0
    logits[3, :] = -INF
    tokens = torch.tensor([0, V - 1, V // 3, 5], dtype=torch.int32)
    check(logits[:3].to(seq.TYPES[type_]).to(DEV), tokens[:3].to(DEV), torch.randn(3, 1, generator=gen).to(DEV), torch.randn(3, generator=gen).to(DEV), 1.3, 9)
    empty = logits[3:].to(seq.TYPES[type_]).to(DEV)
    lp, entropy, stats, top_lp, top = binding.log_probs_fwd(empty, tokens[3:].to(DEV), 1.3, 5)
    assert lp.item() == -INF and entropy.item() == 0.0 and (top_lp == -INF).all() and top.tolist() == [[0, 1, 2, 3, 4]]
    assert (binding.log_probs_bwd(empty, tokens[3:].to(DEV), stats, torch.ones_like(lp), torch.ones_like(entropy), 1.3) == 0.0).all()
    # an impossible token that is asked for
    lp, _, stats, _, _ = binding.log_probs_fwd(logits[1:2].to(seq.TYPES[type_]).to(DEV), tokens[:1].to(DEV), 1.0)
    assert lp.item() == -INF


@pytest.mark.parametrize("V", [1, 300, 5000, 70001])
@pytest.mark.parametrize("bad", [float("nan"), -float("nan"), INF])
def test_bad_logits_show_in_their_row(V, bad):
    """Every result of the row is NaN but padding's; the top tokens are still tokens of the row, each once."""
    logits, tokens, top = torch.randn(3, V, device=DEV), torch.zeros(3, 2, dtype=torch.int64, device=DEV), min(V, 20)
    logits[1, V // 2], tokens[:, 1] = bad, -1
    lp, entropy, stats, top_lp, top_tokens = binding.log_probs_fwd(logits, tokens, 1.0, top)
    d = binding.log_probs_bwd(logits, tokens, stats, torch.ones_like(lp), torch.ones_like(entropy))
    for x in (lp[:, 0], entropy, top_lp.sum(1), d.sum(1)):
        assert x.isnan().tolist() == [False, True, False]
    assert (lp[:, 1] == 0.0).all() and d[1].isnan().all()
    for row in top_tokens.tolist():
        assert len(set(row)) == top and all(0 <= t < V for t in row)
    logits[1] = bad
    lp, entropy, stats, _, top_tokens = binding.log_probs_fwd(logits, tokens, 1.0, top)
    assert lp[1, 0].isnan() and entropy[1].isnan() and len(set(top_tokens[1].tolist())) == top
    assert binding.log_probs_bwd(logits, tokens, stats, torch.ones_like(lp))[1].isnan().all()


@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_strides_leading_dimensions_and_token_types(type_):
    """Rows of a padded vocabulary, at a distance that is no multiple of a pack, and one row for all: as contiguous ones."""
    gen = torch.Generator().manual_seed(4)
    wide = torch.randn(2, 3, 1103, generator=gen).to(seq.TYPES[type_]).to(DEV)
    logits, tokens = wide[..., 3:1000], torch.randint(-2, 1000, (2, 3), generator=gen).to(DEV)
    whole = logits.contiguous()
    a, b = binding.log_probs_fwd(logits, tokens, top=5), binding.log_probs_fwd(whole.view(6, 997), tokens.view(6).to(torch.int32), top=5)
    assert a[0].shape == (2, 3) and a[3].shape == a[4].shape == (2, 3, 5) and a[2].shape == (2, 3, 3)
    for x, y in zip(a, b):
        assert torch.equal(x.view(y.shape), y)
    d = torch.randn(2, 3, generator=gen).to(DEV)
    assert torch.equal(binding.log_probs_bwd(logits, tokens, a[2], d, d).view(6, 997), binding.log_probs_bwd(whole.view(6, 997), tokens.view(6), b[2], d.view(6), d.view(6)))
    row = whole[0, :1].expand(3, 997)
    assert torch.equal(binding.log_probs_fwd(row, tokens[0])[0], binding.log_probs_fwd(row.contiguous(), tokens[0])[0])
    one = binding.log_probs_fwd(whole[0, 0], tokens[0, 0].reshape(()), top=2)  # a row without dimensions in front
    assert one[0].shape == () and torch.equal(one[4], a[4][0, 0, :2])


def test_far_logits_keep_their_differences():
    """A maximum of ten thousand and scales far from 1: what counts are differences."""
    logits = torch.tensor([[10000.0, 10000.5, 9990.0], [-30000.0, -30001.0, -30002.0]], device=DEV)
    lp, entropy, stats, _, _ = binding.log_probs_fwd(logits, torch.tensor([[0, 1, 2]] * 2, device=DEV))
    want = torch.log_softmax(logits.double().cpu(), 1)
    assert (lp.double().cpu() - want).abs().max() <= 200 * U * 12
    d = binding.log_probs_bwd(logits, torch.tensor([0, 0], device=DEV), stats, torch.ones(2, device=DEV))
    assert (d.double().cpu() + want.exp() - torch.tensor([[1.0, 0.0, 0.0]])).abs().max() <= 200 * U * 12
    tiny = binding.log_probs_fwd(logits, torch.tensor([0, 0], device=DEV), scale=1e-30)
    assert (tiny[1] - torch.tensor(3.0).log()).abs().max() < 1e-5
    sharp = binding.log_probs_fwd(logits, torch.tensor([1, 0], device=DEV), scale=1e30)
    assert (sharp[0] == 0.0).all() and (sharp[1] == 0.0).all()


@pytest.mark.parametrize("V", [100, 250, 2584, 40000, 70001])
@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_repeated_calls_give_the_same_bits(V, type_):
    """Whichever lane finds a top token, and whichever writes a given one's result: the same token given and found has one log probability."""
    logits = (torch.randn(700, V, generator=torch.Generator().manual_seed(V)) * 2.5).to(seq.TYPES[type_]).to(DEV)
    tokens = torch.zeros(700, 5, dtype=torch.int32, device=DEV)
    first = binding.log_probs_fwd(logits, tokens, 0.8, 5)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(binding.log_probs_fwd(logits, tokens, 0.8, 5), first))
    assert torch.equal(binding.log_probs_fwd(logits, first[4], 0.8)[0], first[3])


def test_captured_calls_replay():
    gen = torch.Generator().manual_seed(9)
    logits, tokens = torch.randn(5, 70001, generator=gen).to(DEV), torch.randint(0, 70001, (5, 3), generator=gen).to(DEV)
    d, d_h = torch.randn(5, 3, generator=gen).to(DEV), torch.randn(5, generator=gen).to(DEV)

    def call():
        out = binding.log_probs_fwd(logits, tokens, 0.5, 20)
        return (*out, binding.log_probs_bwd(logits, tokens, out[2], d, d_h, 0.5))
    call()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for turn in range(3):
        logits.copy_(torch.randn(5, 70001, generator=gen))
        want = call()
        for graph, _ in graphs:
            graph.replay()
            call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_refusals():
    x, t = torch.ones(4, 24, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    stats, d = torch.zeros(4, 3, device=DEV), torch.ones(4, device=DEV)
    bad = [lambda: binding.log_probs_fwd(x, t[:3]), lambda: binding.log_probs_fwd(x, t.float()), lambda: binding.log_probs_fwd(x.t(), t), lambda: binding.log_probs_fwd(x.cpu(), t),
           lambda: binding.log_probs_fwd(x, t.cpu()), lambda: binding.log_probs_fwd(x.double(), t), lambda: binding.log_probs_fwd(x, t, top=25), lambda: binding.log_probs_fwd(x, t, top=-1),
           lambda: binding.log_probs_bwd(x, t, stats[:3], d), lambda: binding.log_probs_bwd(x, t, stats, d[:3]), lambda: binding.log_probs_bwd(x, t, stats, d, d[:2]),
           lambda: binding.log_probs_bwd(x, t, stats.half(), d), lambda: binding.log_probs_bwd(x, t, stats.cpu(), d)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    big = torch.ones(1, 100, device=DEV)
    for call in (lambda: binding.log_probs_fwd(x, t, scale=0.0), lambda: binding.log_probs_fwd(x, t, scale=float("nan")), lambda: binding.log_probs_fwd(x[:0], t[:0]),
                 lambda: binding.log_probs_fwd(big, t[:1], top=65), lambda: binding.log_probs_fwd(x, t[:, None].expand(4, 257).contiguous()),
                 lambda: binding.log_probs_fwd(big.half().expand(1, 100).new_ones(1, (1 << 24) + 1), t[:1])):
        with pytest.raises(binding.CnnError):
            call()
