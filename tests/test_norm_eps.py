"""The smallest eps of the norms is the smallest normal number: below it a row of zeros would have no root."""
import math

import pytest
import torch

from paper_1912_05234_amd import binding
from test_block_abi import EINVAL, fake, norm, nul, rows

SMALLEST = 2.0 ** -126
BELOW = [SMALLEST - 2.0 ** -149, 1.1e-38, 1e-40, 2.0 ** -149]


@pytest.mark.parametrize("eps", BELOW)
def test_refused(eps):
    L, s = binding.lib(), norm(eps=eps)
    assert 0.0 < s.eps < SMALLEST and L.cnn_norm_bwd_workspace_bytes(s) == 0
    assert L.cnn_add_norm_fwd(s, rows(), rows(), fake, fake, fake, nul) == L.cnn_norm_gate_fwd(s, rows(), rows(), rows(), fake, fake, nul) == EINVAL
    assert L.cnn_add_norm_bwd(s, rows(), rows(), rows(), fake, fake, fake, fake, fake, 1 << 40, nul) == EINVAL
    assert L.cnn_norm_gate_bwd(s, rows(), rows(), rows(), fake, fake, fake, fake, fake, 1 << 40, nul) == EINVAL
    assert L.cnn_norm_bwd_workspace_bytes(norm(eps=SMALLEST)) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("width", [1, 5, 64, 4097])
@pytest.mark.parametrize("eps", [SMALLEST, 1e-30, 1e-6])
def test_rows_of_zeros(eps, width):
    """n = 0 and d_v = d / sqrt(eps), within two ulps of the root and the product's rounding."""
    x, w, d = torch.zeros(3, width, device="cuda:0"), torch.ones(width, device="cuda:0"), torch.full((3, width), 1e-3, device="cuda:0")
    assert (binding.add_norm_fwd(x, w, eps=eps)[0] == 0.0).all() and (binding.norm_gate_fwd(x, w, gate=d, eps=eps) == 0.0).all()
    d_x, _, d_w = binding.add_norm_bwd(d, x, w, eps=eps)
    want = float(d[0, 0]) / math.sqrt(float(torch.tensor(eps)))
    assert ((d_x.double() - want).abs() <= 4 * 2.0 ** -24 * want).all() and (d_w == 0.0).all()
    d_x, d_gate, d_w = binding.norm_gate_bwd(d, x, w, gate=torch.zeros_like(x), eps=eps)
    assert (d_x == 0.0).all() and (d_gate == 0.0).all() and (d_w == 0.0).all()
