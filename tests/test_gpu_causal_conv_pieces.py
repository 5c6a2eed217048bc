"""The convolution's gradients do not depend on where a call cuts a sequence: pieces give the bits of the whole, in halves too, whose results could be rounded at
once or by way of a float."""
import pytest
import torch

import sequence_reference as seq
from paper_1912_05234_amd import binding
from test_gpu_causal_conv import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", list(seq.TYPES))
@pytest.mark.parametrize("K,D", [(2, 575), (6, 380), (7, 124), (3, 17), (2, 62), (5, 604), (4, 2048), (8, 1500)])
@pytest.mark.parametrize("silu", [True, False])
def test_errors_of_pieces(K, D, silu, type_):
    """Errors of the second piece, and of the first but for the K - 1 inputs that the second one's state takes errors to."""
    x, w, b, d_y, _, first, d_last = make((3, 43, D, K, None, True, True, True, False), type_)
    d_x, _, _, d_first = binding.causal_conv_bwd(x, w, d_y, b, silu, None, first, d_last, True)
    for cut in (9, 16, 31):
        middle = binding.causal_conv_fwd(x[:, :cut], w, b, silu, None, first, True)[1]
        second = binding.causal_conv_bwd(x[:, cut:], w, d_y[:, cut:], b, silu, None, middle, d_last, True)
        assert torch.equal(second[0], d_x[:, cut:]), cut
        one = binding.causal_conv_bwd(x[:, :cut], w, d_y[:, :cut], b, silu, None, first, None, True)
        assert torch.equal(one[0][:, : cut - K + 1], d_x[:, : cut - K + 1]) and torch.equal(one[3], d_first), cut
