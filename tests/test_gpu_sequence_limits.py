"""The sequence operators at the ends of what they take: scales and errors of states far from 1, sizes past 32 bits, parameters that are
no numbers."""
import pytest
import torch

import sequence_reference as ref
from paper_1912_05234_amd import binding
from test_gpu_linear_attention import CUT, in_64, magnitudes, make, steps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("case", [(2, 40, 2, 1, 32, 48, [40, 0], True, False), (1, 21, 1, 1, 20, 7, None, True, True),
                                  (1, 900, 2, 2, 32, 64, None, True, False)], ids=["one pass", "odd widths", "segments"])
@pytest.mark.parametrize("scale,by_d_o,by_final", [(2.0 ** -100, 1.0, 2.0 ** 30), (-2.0 ** -100, 1.0, 2.0 ** 90), (2.0 ** 100, 0.0, 2.0 ** -60),
                                                   (2.0 ** 100, 0.0, 2.0 ** -26)])
def test_errors_of_states_far_from_the_scale(scale, by_d_o, by_final, case, type_):
    """The state's error over the scale is past the range of fp32, the state's error itself and what it leads to are not.  Bounds as in
    test_backward; decays near 1, so that the state's error reaches every token."""
    q, k, v, decay, d_o, n, initial, d_final = make(case, type_)
    decay, d_o, d_final = torch.linspace(0.995, 0.9995, len(decay), device=DEV), d_o * by_d_o, d_final * by_final
    if type_ == "fp16" and by_final > 1.0:  # (whose range ends at 2^16: only the state's own error then)
        k, v = k * 0.0, v * 0.0
    arrays = in_64(q, k, v, decay, d_o)
    i64, f64 = in_64(initial, d_final)
    want = ref.linear_attention_gradient(*arrays, scale, case[6], i64, f64)
    size = ref.linear_attention_gradient(*magnitudes(*arrays), abs(scale), case[6], *magnitudes(i64, f64))
    got = binding.linear_attention_bwd(q, k, v, decay, d_o, scale, lengths=n, initial_state=initial, d_final_state=d_final, want_d_state=True)
    for name, g, w, m, dtype in zip(("d_q", "d_k", "d_v", "d_state"), got, want, size, [q.dtype] * 3 + [torch.float32]):
        cut = 0.0 if name == "d_state" else CUT[type_]
        ref.near(g, w, m * (steps(case) + cut), dtype, "%s far from the scale %s" % (name, type_))


def test_a_table_wider_than_32_bits_count_is_refused():
    """2^32 + 8 columns are not 8."""
    table = torch.empty(1, (1 << 32) + 8, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        binding.embedding_fwd(table, torch.zeros(1, dtype=torch.int32, device=DEV))


def test_more_key_heads_than_32_bits_count_are_refused():
    """2^32 + 2 key heads (one, repeated without memory of its own) are not 2."""
    q, decay = torch.ones(1, 3, 2, 8, device=DEV), torch.ones(2, device=DEV)
    kv = torch.ones(1, 3, 1, 8, device=DEV).expand(1, 3, (1 << 32) + 2, 8)
    with pytest.raises(ValueError):
        binding.linear_attention_fwd(q, kv, kv, decay)
    state = torch.zeros(1, 2, 8, 8, device=DEV)
    with pytest.raises(ValueError):
        binding.linear_attention_step(q[:, 0], kv[:, 0], kv[:, 0], decay, state)


@pytest.mark.parametrize("T", [1, 40, 900])
def test_a_decay_that_is_no_number_shows(T):
    """In every form, also where the sequence is cut into segments (900): NaN in its head's results, nothing in the others'."""
    q, k, v, decay, d_o, _, _, _ = make((1, T, 3, 3, 32, 48, None, False, False), "fp32")
    decay = torch.tensor([0.9, float("nan"), 1.0], device=DEV)
    o, state = binding.linear_attention_fwd(q, k, v, decay, 0.3, want_state=True)
    grads = binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, want_d_state=True)
    pool = torch.zeros(1, 3, 32, 48, device=DEV)
    one = binding.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, pool, 0.3)
    by_head = [o[0].transpose(0, 1), state[0], *(g[0].transpose(0, 1) for g in grads[:3]), grads[3][0], pool[0], one[0]]
    for x in by_head:
        assert x[1].isnan().all() and x[0].isfinite().all() and x[2].isfinite().all()


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("case", [(2, 777, 4, 2, 32, 32, [777, 20], True, True), (1, 1100, 3, 1, 64, 90, [1099], True, False),
                                  (2, 640, 2, 2, 128, 96, [3, 640], True, True)], ids=lambda c: str(c[:6]))
def test_decays_of_zero_in_segments(case, type_):
    """The state is the last token's alone, and the state before the sequence reaches no further than the first: in sequences cut into
    segments, one of them shorter than a segment.  Bounds as in test_forward and test_backward."""
    q, k, v, decay, d_o, n, initial, d_final = make(case, type_)
    decay = torch.tensor([0.0, 1.0, 0.0, 0.5][:case[2]], device=DEV)
    shape = binding.LinearShape(*case[:6], list(ref.TYPES).index(type_))
    assert binding.lib().cnn_linear_attention_fwd_workspace_bytes(shape) > 0
    arrays, (i64, f64) = in_64(q, k, v, decay, d_o), in_64(initial, d_final)
    want = ref.linear_attention(*arrays[:4], 0.3, case[6], i64)
    size = ref.linear_attention(*magnitudes(*arrays[:4]), 0.3, case[6], *magnitudes(i64))
    got = binding.linear_attention_fwd(q, k, v, decay, 0.3, n, initial, True)
    want += ref.linear_attention_gradient(*arrays, 0.3, case[6], i64, f64)
    size += ref.linear_attention_gradient(*magnitudes(*arrays), 0.3, case[6], *magnitudes(i64, f64))
    got += binding.linear_attention_bwd(q, k, v, decay, d_o, 0.3, n, initial, d_final, True)
    for name, g, w, m in zip(("o", "state", "d_q", "d_k", "d_v", "d_state"), got, want, size):
        state = name in ("state", "d_state")
        ref.near(g, w, m * (steps(case) + (0.0 if state else CUT[type_])), torch.float32 if state else q.dtype, "%s %s" % (name, type_))
