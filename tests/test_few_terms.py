"""The bounds of sequences with few terms do tell the number of pieces: what one piece fewer loses goes past them (on the host)."""
import numpy as np
import pytest
import torch

import few_terms
import sequence_reference as ref

WIDTHS = [(32, 32), (31, 30), (96, 64), (64, 128)]


def array(x):
    return None if x is None else ref.numpy64(x)


def past(T, type_, got, exact, size, state=False):
    return few_terms.share(got, exact, few_terms.slack(T, type_, size, state), torch.float32 if state else ref.TYPES[type_])


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("T", [3, 900])
@pytest.mark.parametrize("Dk,Dv", WIDTHS)
def test_states_and_scores_of_fewer_pieces(Dk, Dv, T, type_):
    q, k, v, d_o, decay, initial, d_final = (array(x) for x in few_terms.make(T, Dk, Dv, type_, False))
    (o, _), (o_size, _) = few_terms.forward(q, k, v, decay, initial)
    grads, sizes = few_terms.backward(q, k, v, d_o, decay, initial, d_final)
    fewer = lambda x: few_terms.pieces(x, 2 if type_ == "fp32" else 1)  # noqa: E731
    right = [past(T, type_, o, o, o_size)] + [past(T, type_, g, g, s) for g, s in zip(grads[:3], sizes)]
    assert max(right) <= 1.0  # rounded to the type alone
    cut = few_terms.backward(q, k, v, d_o, decay, fewer(initial), fewer(d_final))[0]
    wrong = [past(T, type_, few_terms.forward(q, k, v, decay, fewer(initial))[0][0], o, o_size)]
    wrong += [past(T, type_, *x) for x in zip(cut[:3], grads, sizes)]
    if T == 3 and type_ != "fp32":  # the second token's scores (tokens of other chunks meet in the state)
        score = lambda s: fewer(np.einsum("bhi,bhi->bh", q[:, 1], k[:, s]) * decay ** (1 - s))[:, :, None] * v[:, s]  # noqa: E731
        rough = o.copy()
        rough[:, 1] = few_terms.SCALE * (np.einsum("bhi,bhij->bhj", q[:, 1], initial) * decay[:, None] ** 2 + score(0) + score(1))
        wrong.append(past(T, type_, rough, o, o_size))
    assert min(wrong) > 1.0, wrong


@pytest.mark.parametrize("type_", list(ref.TYPES))
@pytest.mark.parametrize("T", [3, 900])
@pytest.mark.parametrize("Dk,Dv", WIDTHS)
def test_inputs_and_results_of_fewer_pieces(Dk, Dv, T, type_):
    q, k, v, d_o, decay, _, _ = (array(x) for x in few_terms.make(T, Dk, Dv, type_, True))
    (o, last), (o_size, last_size) = few_terms.forward(q, k, v, decay, None)
    grads, sizes = few_terms.backward(q, k, v, d_o, decay, None, None)
    # states that are results, from decayed rows of v (reversed: of d_o) in two pieces, which no type may do
    passed = (decay[:, None] ** np.arange(T)).T[None, :, :, None]  # of token t from the start, and to the end
    wrong = [past(T, type_, np.einsum("bthi,bthj->bhij", k, few_terms.pieces(v * passed[:, ::-1], 2)), last, last_size, True)]
    rough = few_terms.SCALE * decay[:, None, None] * np.einsum("bthi,bthj->bhij", q, few_terms.pieces(d_o * passed, 2))
    wrong.append(past(T, type_, rough, grads[3], sizes[3], True))
    if type_ == "fp32":
        fewer = lambda x: few_terms.pieces(x, 2)  # noqa: E731
        wrong += [past(T, type_, few_terms.forward(*x, decay, None)[0][0], o, o_size) for x in ((fewer(q), k, v), (q, fewer(k), v), (q, k, fewer(v)))]
        cut = few_terms.backward(q, k, v, fewer(d_o), decay, None, None)[0]
        wrong += [past(T, type_, *x) for x in zip(cut[:3], grads, sizes)]
        if T == 3:  # the score of the second token
            rough = o.copy()
            rough[:, 1] = few_terms.SCALE * fewer(np.einsum("bhi,bhi->bh", q[:, 1], k[:, 0]) * decay)[:, :, None] * v[:, 0]
            wrong.append(past(T, type_, rough, o, o_size))
    assert min(wrong) > 1.0, wrong


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("T", [3, 900])
def test_sums_over_few_tokens_are_the_recurrence(T, apart):
    q, k, v, d_o, decay, initial, d_final = (array(x) for x in few_terms.make(T, 6, 7, "fp32", apart))
    pairs = list(zip(few_terms.forward(q, k, v, decay, initial)[0], ref.linear_attention(q, k, v, decay, few_terms.SCALE, None, initial)))
    pairs += list(zip(few_terms.backward(q, k, v, d_o, decay, initial, d_final)[0],
                      ref.linear_attention_gradient(q, k, v, decay, d_o, few_terms.SCALE, None, initial, d_final)))
    for got, want in pairs:
        assert got.shape == want.shape and np.abs(got - want).max() <= 1e-12 * np.abs(want).max()
