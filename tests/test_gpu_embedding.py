"""Embedding lookup and its gradient against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# N tokens, V rows, D wide, how the tokens are spread
CASES = [(1, 1, 1, "uniform"), (1, 300, 64, "uniform"), (5, 3, 7, "padding"), (64, 256, 64, "hot"), (63, 10, 6, "one"),
         (1000, 257, 33, "uniform"), (4096, 70, 20, "hot"), (4097, 70, 24, "hot"), (5000, 70000, 8, "uniform"),
         (6000, 300, 520, "one"), (8193, 256, 12, "ascending"), (20000, 17, 16, "hot"), (4500, 5, 9, "padding"),
         (30000, 65537, 4, "zipf"), (9000, 40, 72, "boundary")]


def tokens_of(N, V, spread, seed):
    r = np.random.Generator(np.random.PCG64(seed))
    if spread == "one":
        return np.full(N, V - 1)
    if spread == "padding":
        return np.full(N, -1) if N < 100 else np.where(r.random(N) < 0.5, -7, V)
    if spread == "hot":
        return np.where(r.random(N) < 0.4, V // 2, r.integers(-1, V + 1, N))
    if spread == "ascending":
        return np.arange(N) * V // N
    if spread == "zipf":
        return np.minimum((V ** r.random(N)).astype(np.int64) - 1, V - 1)
    if spread == "boundary":  # runs that end where tiles of 16 and more entries do
        return np.arange(N) // 16 % V
    return r.integers(0, V, N)


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("N,V,D,spread", CASES)
def test_lookup(N, V, D, spread, type_):
    dtype = ref.TYPES[type_]
    table = torch.randn(V, D, generator=torch.Generator().manual_seed(N)).to(dtype)
    t = tokens_of(N, V, spread, N)
    want = ref.embedding(ref.numpy64(table), t, np.float64(np.float32(3.3)))
    for wide in (torch.int32, torch.int64):
        out = binding.embedding_fwd(table.to(DEV), torch.from_numpy(t).to(wide).to(DEV), 3.3)
        assert out.dtype == dtype
        ref.near(out, want, 2.0 ** -24 * np.abs(want), dtype, "lookup %s" % type_)  # the product is rounded to fp32 first


@pytest.mark.parametrize("type_,D", [("bf16", 1024), ("fp32", 224)])
def test_lookup_of_a_long_output(type_, D):
    """Past 96 MB of whole lines of 128 bytes the output goes past the caches; and the row before that."""
    row = D * (4 if type_ == "fp32" else 2)
    for N in ((96 << 20) // row, (96 << 20) // row + 3, 120011):
        table = torch.randn(301, D, generator=torch.Generator().manual_seed(N)).to(DEV, ref.TYPES[type_])
        tokens = (torch.arange(N, device=DEV) * 7919) % 303 - 1
        out = binding.embedding_fwd(table, tokens, 0.5)
        padded = torch.cat([table * 0.5, torch.zeros(1, D, device=DEV, dtype=table.dtype)])
        assert torch.equal(out, padded[torch.where((tokens < 0) | (tokens >= 301), 301, tokens)])


def test_lookup_of_more_rows_than_one_dimension_of_a_grid_holds():
    """Four rows to a workgroup of 256 threads: past 2^26 rows there are 2^32 threads."""
    N, V, D = (1 << 26) + 5, 7, 129
    table = torch.randn(V, D, generator=torch.Generator().manual_seed(0)).to(DEV, torch.bfloat16)
    tokens = (torch.arange(N, dtype=torch.int32, device=DEV) % 11) - 2
    out = binding.embedding_fwd(table, tokens, 2.0)
    padded = torch.cat([table * 2, torch.zeros(1, D, device=DEV, dtype=table.dtype)])
    for first in range(0, N, 1 << 24):  # (a product with a power of two is exact)
        t = tokens[first:first + (1 << 24)].long()
        assert torch.equal(out[first:first + (1 << 24)], padded[torch.where((t < 0) | (t >= V), V, t)]), first


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("N,V,D,spread", CASES)
def test_gradient(N, V, D, spread, type_):
    dtype = ref.TYPES[type_]
    d = torch.randn(N, D, generator=torch.Generator().manual_seed(N + 1)).to(dtype)
    t = tokens_of(N, V, spread, N)
    want, size, terms = ref.embedding_gradient(ref.numpy64(d), t, V, np.float64(np.float32(0.37)))
    d_dev = d.to(DEV)
    got = [binding.embedding_bwd(d_dev, torch.from_numpy(t).to(wide).to(DEV), V, 0.37) for wide in (torch.int32, torch.int64, torch.int64)]
    # m terms are added in fp32 by m - 1 sums, each off by half a step of what is at most the sum of magnitudes; then the scale
    ref.near(got[0], want, 2.0 ** -24 * (terms[:, None] + 1) * size, dtype, "gradient %s" % type_)
    assert torch.equal(got[0], got[1]) and torch.equal(got[1], got[2])  # the order of the sums is fixed
    assert (got[0].cpu()[torch.from_numpy(terms == 0)] == 0).all()


def test_hot_row_is_a_tree_and_not_a_chain():
    """A hundred thousand equal terms of one row: a sum term by term would be off by thousands of half steps."""
    d = torch.full((100000, 4), 0.1, device=DEV)
    got = binding.embedding_bwd(d, torch.zeros(100000, dtype=torch.int32, device=DEV), 2)
    want = 100000 * float(np.float32(0.1))
    assert abs(float(got[0, 0]) - want) <= 64 * 2.0 ** -24 * want and (got[1] == 0).all()


def test_not_finite_stays_in_its_rows():
    d = torch.ones(300, 8, device=DEV)
    d[17], d[200, 3] = float("nan"), float("inf")
    t = torch.arange(300, device=DEV) % 10
    t[17] = -1  # a NaN that belongs to padding
    got = binding.embedding_bwd(d, t, 10).cpu()
    assert not got.isnan().any() and got.isinf().sum() == 1 and got[0, 3] == float("inf")
    table = torch.ones(10, 8, device=DEV)
    table[3] = float("nan")
    out = binding.embedding_fwd(table, torch.tensor([[3, 2], [-1, 10]], device=DEV)).cpu()
    assert out.shape == (2, 2, 8) and out[0, 0].isnan().all() and (out[0, 1] == 1).all() and (out[1] == 0).all()


def test_other_stream_and_graph():
    """On a stream of the caller's, and captured: every replay sees the tokens of its time."""
    d = torch.randn(5000, 40, device=DEV)
    t = torch.randint(0, 50, (5000,), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.embedding_bwd(d, t, 50)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.embedding_bwd(d, t, 50)
        out = binding.embedding_fwd(got, t)
    for k in range(3):
        t.copy_(torch.randint(0, 50, (5000,), device=DEV))
        want = binding.embedding_bwd(d, t, 50)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(out, want[t]), k


def test_refusals():
    table, t = torch.zeros(4, 8, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    for bad in (table.double(), table.t(), table.cpu(), table[0]):
        with pytest.raises(ValueError):
            binding.embedding_fwd(bad, t)
    with pytest.raises(ValueError):
        binding.embedding_fwd(table, t.float())
    with pytest.raises(binding.CnnError):
        binding.embedding_fwd(table, t[:0])
    with pytest.raises(TypeError):
        binding.embedding_fwd(None, t)
    with pytest.raises(ValueError):
        binding.embedding_bwd(torch.zeros(2, 8, device=DEV), t, 4)
    with pytest.raises(binding.CnnError):
        binding.embedding_bwd(torch.zeros(3, 8, device=DEV), t, 0)
