"""Dropout against its definition: the mask bit for bit, the values to one rounding of a product (and a sum)."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [1, 7, 8, 9, 100, 2048, 4095, 4096, 4097, 19200, 100003]


def want_of(x, keep, p, residual=None):
    y = np.where(keep, np.where(keep, ref.numpy64(x), 0.0) / (1.0 - p) if p < 1 else 0.0, 0.0)
    return y if residual is None else y + ref.numpy64(residual)


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.93, 1.0])
def test_against_definition(n, p, type_):
    dtype, seed, offset = ref.TYPES[type_], 0xF123456789ABCDEF, (5 << 32) + n
    gen = torch.Generator().manual_seed(n)
    x, res = (torch.randn(n, generator=gen).to(dtype) for _ in range(2))
    keep = ref.kept(n, p, seed, offset)
    y = binding.dropout_fwd(x.to(DEV), p, seed, offset)
    assert y.dtype == dtype and ((y.cpu() != 0).numpy() == (keep & (x != 0).numpy())).all()
    want = want_of(x, keep, p)
    # 1 / (1 - p) and the product are rounded to fp32; with the residual the sum too
    ref.near(y, want, 2.0 ** -23 * np.abs(want), dtype, "dropout %s" % type_)
    d = binding.dropout_bwd(x.to(DEV), p, seed, offset)
    assert torch.equal(d, y)
    both = binding.dropout_fwd(x.to(DEV), p, seed, offset, residual=res.to(DEV))
    total = want_of(x, keep, p, res)
    ref.near(both, total, 2.0 ** -23 * np.abs(want) + 2.0 ** -24 * np.abs(total), dtype, "with residual %s" % type_)


@pytest.mark.parametrize("type_", ["bf16", "fp16"])
def test_more_than_the_last_cache_holds(type_):
    """Past 256 MB read and written, against the same elements as floats, whose kernel is another: one mask, values exact for p = 1/2."""
    n, dtype = (256 << 20) // 4 + 1003, ref.TYPES[type_]
    x = torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dtype)
    res = x.flip(0)
    want = binding.dropout_fwd(x.float(), 0.5, 11, 12)
    assert torch.equal(binding.dropout_fwd(x, 0.5, 11, 12), want.to(dtype))
    assert torch.equal(binding.dropout_fwd(x, 0.5, 11, 12, residual=res), (want + res.float()).to(dtype))
    small = binding.dropout_fwd(x[:100003].contiguous(), 0.5, 11, 12)
    assert torch.equal(small, want[:100003].to(dtype))


def test_every_bit_of_the_limit_counts():
    """Elements whose high sixteen bits equal the limit's are decided by the low ones: limits around the numbers drawn themselves."""
    n = 4096
    u = ref.numbers(n, 11, 3)
    x = torch.ones(n, device=DEV)
    for e in (0, 5, 1234, 4095):
        for step in (-1, 0, 1):
            p = (int(u[e]) + step) / 2.0 ** 32
            y = binding.dropout_fwd(x, p, 11, 3).cpu().numpy()
            assert ((y != 0) == (u >= np.uint64(int(u[e]) + step))).all(), (e, step)
            assert (y[e] != 0) == (step <= 0)


def test_step_on_the_device_and_graph():
    x, step = torch.randn(5000, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    binding.dropout_fwd(x, 0.3, 9, 100, step=step)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = binding.dropout_fwd(x, 0.3, 9, 100, step=step)
        d = binding.dropout_bwd(x, 0.3, 9, 100, step=step)
    seen = []
    for k in (0, 1, 7):
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, binding.dropout_fwd(x, 0.3, 9, 100 + k)) and torch.equal(d, y)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_dropped_elements_are_zero_whatever_they_hold():
    keep = ref.kept(640, 0.5, 1, 2)
    x = torch.ones(640)
    x[torch.from_numpy(~keep)] = float("nan")
    x[3] = float("inf")
    y = binding.dropout_fwd(x.to(DEV), 0.5, 1, 2).cpu()
    assert not y.isnan().any() and (y[torch.from_numpy(~keep)] == 0).all() and y.isinf().sum() == int(keep[3])


def test_far_elements_have_blocks_of_their_own():
    """Beyond 2^32 elements: the last block of a large tensor against the generator."""
    n = (1 << 32) + 24
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    y = binding.dropout_bwd(x, 0.5, 77, 1)
    far = (y[1 << 32:] != 0).cpu().numpy()
    assert (far == (ref.numbers(24, 77, 1, first=1 << 32) >= np.uint64(1 << 31))).all()
    assert (far != (y[:24] != 0).cpu().numpy()).any()


def test_refusals():
    x = torch.zeros(8, device=DEV)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(binding.CnnError):
            binding.dropout_fwd(x, p, 1)
    with pytest.raises(binding.CnnError):
        binding.dropout_fwd(x[:0], 0.5, 1)
    with pytest.raises(binding.CnnError):
        binding.dropout_bwd(torch.zeros(9, device=DEV)[1:], 0.5, 1)  # not 16-byte aligned
    for bad in (x.double(), x.cpu(), torch.zeros(4, 4, device=DEV)[:, :2]):
        with pytest.raises(ValueError):
            binding.dropout_fwd(bad, 0.5, 1)
    with pytest.raises(ValueError):
        binding.dropout_fwd(x, 0.5, 1, residual=torch.zeros(7, device=DEV))
    with pytest.raises(ValueError):
        binding.dropout_fwd(x, 0.5, 1, step=torch.zeros(2, dtype=torch.int64, device=DEV))
