"""The sequence operators from their definitions, in 64 bits and numpy (the generator in unsigned words), and the bounds of their tests."""
import numpy as np
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    """Largest relative error of one rounding to nearest."""
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Largest absolute error of a rounding among the type's subnormal numbers."""
    return float(torch.finfo(dtype).tiny) * torch.finfo(dtype).eps / 2


def numpy64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def near(got, exact, slack, dtype, what):
    """|got - exact| <= slack + one rounding of a number that is off by at most slack."""
    got = numpy64(got)
    assert got.shape == exact.shape, (what, got.shape, exact.shape)
    assert np.isfinite(got).all(), what
    allowed = slack + half_step(dtype) * (np.abs(exact) + slack) + smallest(dtype)
    worst = np.max(np.abs(got - exact) / allowed) if got.size else 0.0
    print("%s: %.3f of the allowed error" % (what, worst))
    assert worst <= 1.0, (what, worst)


# ---- embedding ------------------------------------------------------------------------------------------------
def embedding(table, tokens, scale):
    out = np.zeros(tokens.shape + (table.shape[1],))
    known = (tokens >= 0) & (tokens < len(table))
    out[known] = table[tokens[known]] * scale
    return out


def embedding_gradient(d_out, tokens, vocab, scale):
    """(gradient, sums of magnitudes, number of terms per row)"""
    d_out, tokens = d_out.reshape(-1, d_out.shape[-1]), tokens.reshape(-1)
    total, size, terms = np.zeros((vocab, d_out.shape[1])), np.zeros((vocab, d_out.shape[1])), np.zeros(vocab)
    for row, token in zip(d_out, tokens):
        if 0 <= token < vocab:
            total[token] += row * scale
            size[token] += np.abs(row * scale)
            terms[token] += 1
    return total, size, terms


# ---- dropout --------------------------------------------------------------------------------------------------
def philox(counter, key):
    """Philox4x32-10 of counter [n, 4] and key (2 words): [n, 4] words."""
    c, k = [np.asarray(counter)[:, i].astype(np.uint64) for i in range(4)], [int(w) for w in key]
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> shift) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, 1)


def numbers(n, seed, offset, first=0):
    """The 32-bit numbers of the elements first .. first + n - 1 (first a multiple of 8)."""
    block = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    halves = []
    for call in (0, 1):
        counter = np.stack([block & np.uint64(0xFFFFFFFF), (block >> np.uint64(32)) | np.uint64(call << 31),
                            np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32 & 0xFFFFFFFF)], 1)
        w = philox(counter, (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
        halves.append(np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n])
    return (halves[0] << np.uint64(16)) | halves[1]


def kept(n, p, seed, offset):
    return numbers(n, seed, offset) >= np.uint64(int(np.floor(p * 2.0 ** 32 + 0.5)))


# ---- linear attention -----------------------------------------------------------------------------------------
def share(x, heads):
    """[B, T, Hk, D] with every head repeated for the query heads that use it."""
    return np.repeat(x, heads // x.shape[2], axis=2)


def linear_attention(q, k, v, decay, scale, lengths=None, initial=None):
    """(o [B, T, H, Dv], state [B, H, Dk, Dv]) token by token."""
    B, T, H, Dk = q.shape
    k, v = share(k, H), share(v, H)
    state = np.zeros((B, H, Dk, v.shape[3])) if initial is None else initial.copy()
    o = np.zeros((B, T, H, v.shape[3]))
    for b in range(B):
        for t in range(T if lengths is None else int(lengths[b])):
            state[b] = state[b] * decay[:, None, None] + k[b, t][:, :, None] * v[b, t][:, None, :]
            o[b, t] = scale * np.einsum("hi,hij->hj", q[b, t], state[b])
    return o, state


def linear_attention_gradient(q, k, v, decay, d_o, scale, lengths=None, initial=None, d_final=None):
    """(d_q, d_k, d_v, d_initial): the error of the state is carried back token by token."""
    B, T, H, Dk = q.shape
    Hk = k.shape[2]
    k, v = share(k, H), share(v, H)
    state = np.zeros((B, H, Dk, v.shape[3])) if initial is None else initial.copy()
    error = np.zeros_like(state) if d_final is None else d_final.copy()
    d_q, d_k, d_v = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        for t in range(n):
            state[b] = state[b] * decay[:, None, None] + k[b, t][:, :, None] * v[b, t][:, None, :]
            d_q[b, t] = scale * np.einsum("hij,hj->hi", state[b], d_o[b, t])
        for t in reversed(range(n)):
            error[b] += scale * q[b, t][:, :, None] * d_o[b, t][:, None, :]
            d_k[b, t] = np.einsum("hij,hj->hi", error[b], v[b, t])
            d_v[b, t] = np.einsum("hij,hi->hj", error[b], k[b, t])
            error[b] *= decay[:, None, None]
    group = lambda x: x.reshape(B, T, Hk, H // Hk, -1).sum(3)  # noqa: E731
    return d_q, group(d_k), group(d_v), error
