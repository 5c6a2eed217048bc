"""The reference of the sequence operators against what is known of them: published outputs of the generator, differences of a loss,
the quadratic form of linear attention."""
import numpy as np

import sequence_reference as ref


def test_philox_known_answers():
    """Known-answer vectors published with the generator (zeros, ones, digits of pi)."""
    for counter, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]:
        assert tuple(int(w) for w in ref.philox(np.array([counter], np.uint64), key)[0]) == want


def test_numbers_are_uniform_and_share_of_kept():
    n = 1 << 16
    u = ref.numbers(n, 0x1234567890ABCDEF, 7).astype(np.float64) / 2 ** 32
    assert abs(u.mean() - 0.5) < 5 * np.sqrt(1 / 12 / n)
    for p in (0.1, 0.5, 0.9):
        assert abs(ref.kept(n, p, 3, 0).mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
    assert ref.kept(n, 0.0, 3, 0).all() and not ref.kept(n, 1.0, 3, 0).any()
    assert (ref.numbers(64, 5, 9, first=1 << 20) == ref.numbers((1 << 20) + 64, 5, 9)[1 << 20:]).all()


def small(seed, B=2, T=7, H=4, Hk=2, Dk=3, Dv=5):
    r = np.random.Generator(np.random.PCG64(seed))
    return (r.standard_normal((B, T, H, Dk)), r.standard_normal((B, T, Hk, Dk)), r.standard_normal((B, T, Hk, Dv)),
            np.array([1.0, 0.9, 0.5, 0.0]), r.standard_normal((B, H, Dk, Dv)), r.standard_normal((B, T, H, Dv)), r.standard_normal((B, H, Dk, Dv)))


def test_linear_attention_is_the_masked_product():
    q, k, v, decay, initial, _, _ = small(1)
    T = q.shape[1]
    o, state = ref.linear_attention(q, k, v, decay, 0.7, None, initial)
    kk, vv = ref.share(k, 4), ref.share(v, 4)
    e = np.arange(T)[:, None] - np.arange(T)
    for h in range(4):
        w = np.where(e >= 0, decay[h] ** np.maximum(e, 0), 0.0)
        for b in range(2):
            want = (w * (q[b, :, h] @ kk[b, :, h].T)) @ vv[b, :, h] + decay[h] ** (np.arange(T) + 1)[:, None] * (q[b, :, h] @ initial[b, h])
            np.testing.assert_allclose(o[b, :, h], 0.7 * want, rtol=1e-12, atol=1e-12)


def test_gradient_against_differences():
    q, k, v, decay, initial, d_o, d_final = small(2)
    lengths = [7, 4]
    inputs = [q, k, v, initial]

    def loss():
        o, state = ref.linear_attention(inputs[0], inputs[1], inputs[2], decay, 0.7, lengths, inputs[3])
        return (o * d_o).sum() + (state * d_final).sum()

    got = ref.linear_attention_gradient(q, k, v, decay, d_o, 0.7, lengths, initial, d_final)
    r = np.random.Generator(np.random.PCG64(3))
    for x, g in zip(inputs, got):
        for _ in range(30):
            at = tuple(r.integers(0, n) for n in x.shape)
            keep, step = x[at], 1e-4
            x[at] = keep + step
            up = loss()
            x[at] = keep - step
            down = loss()
            x[at] = keep
            assert abs((up - down) / (2 * step) - g[at]) <= 1e-6 * (1 + abs(g[at]))


def test_embedding_gradient_is_the_adjoint():
    r = np.random.Generator(np.random.PCG64(4))
    table, d, tokens = r.standard_normal((9, 5)), r.standard_normal((40, 5)), r.integers(-2, 11, 40)
    g, size, terms = ref.embedding_gradient(d, tokens, 9, 3.0)
    np.testing.assert_allclose((ref.embedding(table, tokens, 3.0) * d).sum(), (g * table).sum(), rtol=1e-12)
    assert terms.sum() == ((tokens >= 0) & (tokens < 9)).sum() and (size >= np.abs(g) - 1e-12).all()
