"""Norms around a block against their definition in 64 bits.

Bounds, in roundings u of fp32.  A group's sum of squares goes through at most 16 additions of a lane, 6 of a wave and 16 of a workgroup, all
terms of one sign, and the mean's product and eps: 40 u, of which the root keeps half; the root's own steps 4 u; products and weights 4 u.  A
gate's factor: the exponent z log2(e) is rounded twice (|z| 2 u), exponential, sum and reciprocal are within 2 u each, products 2 u.  So a
result is off by (40 + 2 |z|) u of its magnitude, of the sum of magnitudes where it is a difference, and each is rounded once to its type.  The sum r is
off by one rounding of the product and one of the sum before anything else."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U
TYPES = [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")]
# rows, groups, width: one element; narrow teams; a wave, its limits; a workgroup, its limits; the largest; odd ones
SHAPES = [(1, 1, 1), (5, 3, 7), (33, 2, 32), (9, 17, 31), (300, 1, 64), (7, 1, 255), (4, 2, 256), (3, 5, 257), (65, 1, 1000), (3, 1, 1024), (5, 1, 1025),
          (3, 1, 2049), (2, 2, 4096), (3, 1, 4097), (2, 1, 9999), (2, 1, 16384), (2500, 2, 64), (1, 40, 3)]


def normal(gen, *shape, dtype, by=1.0):
    return (torch.randn(shape, generator=gen) * by).to(dtype).to(DEV)


def wide(*tensors):
    return [None if t is None else t.double().cpu() for t in tensors]


def near(got, want, slack, what):
    seq.near(got, want.numpy(), slack.numpy(), got.dtype, what)


def scale_of(s):
    return float(torch.tensor(s, dtype=torch.float32))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_before_a_block(types, shape):
    (N, G, W), (type_, stream) = shape, (seq.TYPES[t] for t in types)
    gen, D, eps, scale = torch.Generator().manual_seed(N + W), G * W, scale_of(1e-5), 0.7
    x, w = normal(gen, N, D, dtype=type_), normal(gen, D, dtype=torch.float32) + 1.0
    res, d_y, d_r = normal(gen, N, D, dtype=stream, by=2.0), normal(gen, N, D, dtype=type_), normal(gen, N, D, dtype=stream)
    if N > 2:
        x[1], res[1] = 0.0, 0.0  # a row of zeros
    x64, w64, res64, d_y64, d_r64 = wide(x, w, res, d_y, d_r)
    s64 = scale_of(scale)
    y, r = binding.add_norm_fwd(x, w, res, scale, 1e-5, G)
    want_y, want_r = ref.add_norm(x64, w64, res64, s64, eps, G)
    sum_off = U * ((s64 * x64).abs() + want_r.abs())
    root = ref.hat(want_r, G, eps)[1]
    sum_part = root * sum_off + want_y.abs() * 0.0 + ref.hat(want_r, G, eps)[0].abs() * ref.group_mean(root * sum_off * ref.hat(want_r, G, eps)[0].abs(), G)
    near(y, want_y, 40 * U * want_y.abs() + sum_part * w64.abs(), "y of a sum")
    near(r, want_r, sum_off, "r")
    y, r = binding.add_norm_fwd(x, w, eps=1e-5, groups=G)
    assert r is x and y.dtype == x.dtype
    want_y = ref.add_norm(x64, w64, None, 1.0, eps, G)[0]
    near(y, want_y, 40 * U * want_y.abs(), "y")
    steps = (60 + N / 16) * U
    for error, by in ((d_r, scale), (d_r, 1.0), (None, scale)):
        got = binding.add_norm_bwd(d_y, res, w, d_r=error, scale=by, eps=1e-5, groups=G)
        want, size = ref.add_norm_gradient(d_y64, res64, w64, None if error is None else d_r64, scale_of(by), eps, G)
        assert (got[0] is got[1]) == (by == 1.0 and type_ == stream) and [g.dtype for g in got] == [type_, stream, torch.float32]
        for name, g, v, m, k in zip(("d_x", "d_residual", "d_weight"), got, want, size, (60 * U, 60 * U, steps + 60 * U)):
            near(g, v, m * k, name)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_behind_a_block(types, shape):
    (N, G, W), (type_, stream) = shape, (seq.TYPES[t] for t in types)
    gen, D, eps, scale = torch.Generator().manual_seed(N + W + 1), G * W, scale_of(1e-5), -0.3
    x, w = normal(gen, N, D, dtype=type_), normal(gen, D, dtype=torch.float32) + 1.0
    gate, res, d_y = normal(gen, N, D, dtype=type_, by=4.0), normal(gen, N, D, dtype=stream), normal(gen, N, D, dtype=stream)
    if N > 2:
        x[1] = 0.0
    x64, w64, gate64, res64, d_y64 = wide(x, w, gate, res, d_y)
    s64, z = scale_of(scale), gate64.abs()
    for gates, adds in ((True, True), (True, False), (False, True), (False, False)):
        y = binding.norm_gate_fwd(x, w, gate if gates else None, res if adds else None, scale, 1e-5, G)
        want = ref.norm_gate(x64, w64, gate64 if gates else None, None, s64, eps, G)
        total = want + res64 if adds else want
        assert y.dtype == (stream if adds else type_)
        near(y, total, (40 + 2 * z * gates) * U * want.abs() + U * total.abs(), "y %d %d" % (gates, adds))
    for gates in (True, False):
        got = binding.norm_gate_bwd(d_y, x, w, gate if gates else None, scale, 1e-5, G)
        want, size = ref.norm_gate_gradient(d_y64, x64, w64, gate64 if gates else None, s64, eps, G)
        most = (60 + 2 * float(z.max())) * U
        assert (got[1] is None) == (not gates)
        for name, g, v, m, k in zip(("d_x", "d_gate", "d_weight"), got, want, size, (most, most, most + (60 + N / 16) * U)):
            if g is not None:
                near(g, v, m * k, name + " %d" % gates)


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_slices_and_leading_dimensions(types):
    """Rows at a distance that is no multiple of a pack, starts in the middle of one, a broadcast row, rows of a transposed batch: as contiguous ones."""
    type_, stream = (seq.TYPES[t] for t in types)
    gen = torch.Generator().manual_seed(5)
    both = normal(gen, 4, 6, 2 * 75 + 1, dtype=type_)
    x, gate = both[..., 1:76], both[..., 76:]
    res, w = normal(gen, 1, 1, 75, dtype=stream).expand(4, 6, 75), normal(gen, 75, dtype=torch.float32)
    plain = [t.contiguous() for t in (x, gate, res)]
    assert torch.equal(binding.norm_gate_fwd(x, w, gate, res, 0.5, groups=3), binding.norm_gate_fwd(plain[0], w, plain[1], plain[2], 0.5, groups=3))
    for a, b in zip(binding.add_norm_fwd(x, w, res, 0.5, groups=3), binding.add_norm_fwd(plain[0], w, plain[2], 0.5, groups=3)):
        assert a.is_contiguous() and torch.equal(a, b)
    for a, b in zip(binding.norm_gate_bwd(res, x, w, gate, 0.5, groups=3), binding.norm_gate_bwd(plain[2], plain[0], w, plain[1], 0.5, groups=3)):
        assert torch.equal(a, b)
    for a, b in zip(binding.add_norm_bwd(x, res, w, res, 0.5, groups=3), binding.add_norm_bwd(plain[0], plain[2], w, plain[2], 0.5, groups=3)):
        assert torch.equal(a, b)
    row = normal(gen, 75, dtype=type_)  # one row without dimensions in front
    assert torch.equal(binding.add_norm_fwd(row, w)[0], binding.add_norm_fwd(row[None], w)[0][0])


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_gradients_of_groups_of_one_element(types):
    """d (1 - n^2) with n next to 1 or -1: what eps leaves is exact to (3 rstd, 12 products and roundings) 60 u of itself, and the type's rounding."""
    type_, stream = (seq.TYPES[t] for t in types)
    gen = torch.Generator().manual_seed(6)
    r, w, d = normal(gen, 9, 20, dtype=stream, by=4.0), normal(gen, 20, dtype=torch.float32), normal(gen, 9, 20, dtype=type_, by=1000.0)
    r64, w64, d64 = wide(r, w, d)
    eps = scale_of(1e-3)
    want = d64 * w64 * eps / (r64 * r64 + eps) ** 1.5
    near(binding.add_norm_bwd(d, r, w, eps=1e-3, groups=20)[1], want, 60 * U * want.abs(), "d_residual")
    x, gate = r.to(type_), normal(gen, 9, 20, dtype=type_)
    x64, z64 = wide(x, gate)
    want = d64 * w64 * ref.silu(z64) * eps / (x64 * x64 + eps) ** 1.5
    near(binding.norm_gate_bwd(d, x, w, gate, eps=1e-3, groups=20)[0], want, (70 + 2 * z64.abs()) * U * want.abs(), "d_x")


def test_a_bad_element_stays_in_its_group():
    x, w = torch.ones(6, 96, device=DEV), torch.ones(96, device=DEV)
    x[2, 40], x[4, 90] = float("nan"), float("inf")
    y = binding.add_norm_fwd(x, w, groups=3)[0].view(6, 3, 32)
    bad = y.isnan().any(2)
    assert bad.nonzero().tolist() == [[2, 1], [4, 2]]
    d_x, _, d_w = binding.add_norm_bwd(torch.ones_like(x), x, w, groups=3)
    assert d_x.view(6, 3, 32).isnan().any(2).nonzero().tolist() == [[2, 1], [4, 2]]
    assert d_w[:32].isfinite().all()


def test_repeated_calls_and_another_stream_give_the_same_bits():
    gen = torch.Generator().manual_seed(8)
    x, d, w = normal(gen, 3000, 160, dtype=torch.bfloat16), normal(gen, 3000, 160, dtype=torch.bfloat16), normal(gen, 160, dtype=torch.float32)
    first = binding.norm_gate_bwd(d, x, w, d, 0.5, groups=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = binding.norm_gate_bwd(d, x, w, d, 0.5, groups=5)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_captured_calls_replay():
    """Two graphs and eager calls between their replays: each has a workspace of its own."""
    gen = torch.Generator().manual_seed(9)
    x, d, w = normal(gen, 700, 64, dtype=torch.float32), normal(gen, 700, 64, dtype=torch.float32), normal(gen, 64, dtype=torch.float32)
    call = lambda: (*binding.add_norm_fwd(x, w, d, 0.5), *binding.add_norm_bwd(d, x, w, x, 0.5), *binding.norm_gate_bwd(d, x, w, d))  # noqa: E731
    call()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for turn in range(3):
        x.copy_(normal(gen, 700, 64, dtype=torch.float32))
        want = call()
        for graph, out in graphs:
            graph.replay()
            call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_refusals():
    x, w = torch.ones(4, 24, device=DEV), torch.ones(24, device=DEV)
    bad = [lambda: binding.add_norm_fwd(x, w, groups=5), lambda: binding.add_norm_fwd(x, w, groups=0), lambda: binding.add_norm_fwd(x, w[:23]),
           lambda: binding.add_norm_fwd(x, w.half()), lambda: binding.add_norm_fwd(x.t(), w[:4]), lambda: binding.add_norm_fwd(x, w, residual=x[:3]),
           lambda: binding.add_norm_fwd(x.half(), w, residual=x.bfloat16()), lambda: binding.add_norm_fwd(x, w, residual=x.half()),
           lambda: binding.add_norm_fwd(x.double(), w), lambda: binding.add_norm_fwd(x.cpu(), w), lambda: binding.add_norm_fwd(x, w.cpu()),
           lambda: binding.norm_gate_fwd(x, w, gate=x.half()), lambda: binding.norm_gate_fwd(x, w, gate=x[:, :23]),
           lambda: binding.norm_gate_bwd(x[:3], x, w), lambda: binding.add_norm_bwd(x, x, w, d_r=x.half()),
           lambda: binding.add_norm_fwd(x.view(2, 2, 24).transpose(0, 1), w)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.add_norm_fwd(x, w, scale=0.5), lambda: binding.add_norm_fwd(x, w, eps=0.0), lambda: binding.add_norm_fwd(x[:0], w),
                 lambda: binding.add_norm_fwd(torch.ones(1, 16385, device=DEV), torch.ones(16385, device=DEV)),
                 lambda: binding.norm_gate_fwd(x, w, scale=float("nan"))):
        with pytest.raises(binding.CnnError):
            call()
    for call in (lambda: binding.add_norm_bwd(None, x, w), lambda: binding.norm_gate_bwd(None, x, w), lambda: binding.add_norm_fwd(None, w)):
        with pytest.raises(TypeError):
            call()
