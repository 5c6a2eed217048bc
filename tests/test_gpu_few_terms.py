"""The pieces that linear attention cuts its operands into, for every width and number of waves that its kernels are made for: sequences
with few terms, against bounds that one piece fewer goes past (test_few_terms.py)."""
import pytest
import torch

import few_terms
import sequence_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("T", [3, 900])
@pytest.mark.parametrize("Dk,Dv", few_terms.WIDTHS)
def test_pieces(Dk, Dv, T, type_):
    """Rows of whole packs and rows that are none; one pass, and sequences cut into segments."""
    dtype = ref.TYPES[type_]
    for less in (0, 1):
        shape = binding.LinearShape(8, T, 3, 3, Dk - less, Dv - less, list(ref.TYPES).index(type_))
        assert (binding.lib().cnn_linear_attention_bwd_workspace_bytes(shape) > 0) == (T == 900)
        for apart in (False, True):
            data = few_terms.make(T, Dk - less, Dv - less, type_, apart)
            q, k, v, d_o, decay, initial, d_final = (None if x is None else x.to(DEV) for x in data)
            q64, k64, v64, d64, a64, i64, f64 = (None if x is None else ref.numpy64(x) for x in data)
            (want, want_last), (size, last_size) = few_terms.forward(q64, k64, v64, a64, i64)
            o, last = binding.linear_attention_fwd(q, k, v, decay, few_terms.SCALE, initial_state=initial, want_state=True)
            where = " %s, %s" % (type_, "apart" if apart else "together")
            ref.near(o, want, few_terms.slack(T, type_, size), dtype, "o" + where)
            ref.near(last, want_last, few_terms.slack(T, type_, last_size, True), torch.float32, "state" + where)
            wants, sizes = few_terms.backward(q64, k64, v64, d64, a64, i64, f64)
            got = binding.linear_attention_bwd(q, k, v, decay, d_o, few_terms.SCALE, initial_state=initial, d_final_state=d_final, want_d_state=True)
            for name, g, w, m in zip(("d_q", "d_k", "d_v", "d_state"), got, wants, sizes):
                state = name == "d_state"
                ref.near(g, w, few_terms.slack(T, type_, m, state), torch.float32 if state else dtype, name + where)
