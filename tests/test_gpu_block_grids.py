"""Kernels of 1024 threads to a workgroup, with more workgroups than one dimension of a grid has: 2^22 of them are 2^32 threads."""
import pytest
import torch

from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_log_probs_of_more_rows_than_one_dimension_has():
    """One row for all, whose tokens all have a log probability: every row's, bit for bit."""
    N, V = (1 << 22) + 3, 8200
    gen = torch.Generator(device=DEV).manual_seed(1)
    row = torch.randn(1, V, generator=gen, device=DEV).to(torch.bfloat16)
    every, entropy, stats, _, _ = binding.log_probs_fwd(row.expand(V, V), torch.arange(V, device=DEV))
    tokens = torch.randint(0, V, (N,), generator=gen, device=DEV)
    got = binding.log_probs_fwd(row.expand(N, V), tokens)
    assert torch.equal(got[0], every[tokens])
    assert (got[1] == entropy[0]).all() and (got[2] == stats[0]).all()


def test_parameters_of_the_scan_in_more_columns_than_one_dimension_has():
    """The sums behind d_a, d_skip and d_dt_bias have D (N + 2) columns, 32 to a workgroup.  The last groups' gradients as by themselves, bit for bit; the first
    and last channels' d_a from its definition, D exp(D a) c d_y h for a single token, some 40 roundings of itself."""
    D, N, per = 1 << 20, 128, 1024
    gen = torch.Generator(device=DEV).manual_seed(2)
    normal = lambda *s: torch.randn(s, generator=gen, device=DEV)  # noqa: E731
    x, dt, d_y = normal(1, 1, D), torch.rand(1, 1, D, generator=gen, device=DEV), normal(1, 1, D)
    a, b, c = -torch.rand(D, N, generator=gen, device=DEV), normal(1, 1, D // per, N), normal(1, 1, D // per, N)
    skip, bias, first = normal(D), torch.zeros(D, device=DEV), normal(1, D, N)
    got = binding.selective_scan_bwd(x, dt, a, b, c, d_y, skip, bias, softplus=False, initial_state=first, want_d_state=True)
    tail, groups = slice(D - 2 * per, D), slice(D // per - 2, D // per)
    cut = lambda t: t[..., tail].contiguous()  # noqa: E731
    alone = binding.selective_scan_bwd(cut(x), cut(dt), a[tail], b[:, :, groups], c[:, :, groups], cut(d_y), skip[tail], bias[tail], softplus=False,
                                       initial_state=first[:, tail], want_d_state=True)
    for name, g, one, part in zip(("d_x", "d_dt", "d_a", "d_b", "d_c", "d_skip", "d_dt_bias", "d_state"), got, alone,
                                  ((..., tail), (..., tail), tail, (..., groups, slice(None)), (..., groups, slice(None)), tail, tail, (slice(None), tail))):
        assert torch.equal(g[part], one), name
    for channels, group in ((slice(0, 64), 0), (slice(D - 64, D), -1)):
        d, h = dt[0, 0, channels, None].double(), first[0, channels].double()
        want = d * torch.exp(d * a[channels].double()) * (c[0, 0, group].double() * d_y[0, 0, channels, None].double()) * h
        assert ((got[2][channels].double() - want).abs() <= 40 * 2.0 ** -24 * want.abs() + 1e-30).all()
