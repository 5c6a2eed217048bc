"""Sequences of which almost every element is zero, so that sums have few terms and their bounds few steps: tight enough to tell how many
pieces of bfloat16 the linear attention kernels make of what they multiply.

Three tokens are not zero.  Either (`apart`) each has one element in q, k, v and d_o, and there are no states before or after the
sequence: a result then is one term, or two, of three numbers.  Or q and k are x and -x in two columns, v and d_o in two of theirs, and
the states are one number to 2^-12, so that what a token reads of a state almost cancels, and the second token takes back most of what
the first one wrote: the rounding of a result to its type, which comes last, then hides nothing of what was lost before.
"""
import numpy as np
import torch

import sequence_reference as ref

DECAYS = [1.0, 0.5, 0.984375]
SCALE = 0.3
# Loss of what is cut into two pieces, state and scores of 16-bit types; for half also products of two second pieces.
CUT = {"fp32": 0.0, "bf16": 2.0 ** -16, "fp16": 2.0 ** -15}
# Half steps of fp32.  A product of pieces costs one where it opens a sum and one for each of its six parts where it is added to another
# term, one more for the parts left out; an output is the sum of two terms of the state and two scores for each of three tokens, weighted
# by a power of the decay (four) and scaled.  A state that went through segments has a sum and a power (of up to 900 times 0.023 in the
# exponent: fourteen) more for each token.
STEPS = {3: 36, 900: 48}

# Dk and Dv for every width that the kernels are made for (32, 64, 96, 128, 256 of q and k) and every number of waves
WIDTHS = [(dk, dv) for dk in (32, 64, 96, 128, 256) for dv in (32, 64, 96, 128)]


def tokens(T):
    """Those that are not zero."""
    return [0, 1, 2] if T == 3 else [T // 3, T - 40, T - 2]


def make(T, Dk, Dv, type_, apart):
    """(q, k, v, d_o, decay, initial state, error of the final state): tensors on the host, no states where `apart`"""
    B, H, dtype = 8, 3, ref.TYPES[type_]
    gen = torch.Generator().manual_seed(1000 * T + 300 * Dk + Dv)
    active = tokens(T)

    def rows(D, columns):  # numbers next to 1, of which the pieces leave the most
        x, first = torch.zeros(B, T, H, D), D // 3
        values = ((1.0 + 0.2 * torch.rand((B, 3, H), generator=gen)) * (torch.randint(0, 2, (B, 3, H), generator=gen) * 2 - 1)).to(dtype).float()
        for n, t in enumerate(active):
            x[:, t, :, first + (columns[n] if apart else 0)] = values[:, n]
            if not apart:
                x[:, t, :, D - 1] = -values[:, n]
        return x

    q, k, v, d_o = rows(Dk, (0, 0, 1)), rows(Dk, (0, 1, 2)), rows(Dv, (0, 1, 2)), rows(Dv, (0, 0, 1))
    decay = torch.tensor(DECAYS)
    if apart:
        return *(x.to(dtype) for x in (q, k, v, d_o)), decay, None, None
    by = 1.0 + 0.5 * torch.rand((B, H, 1), generator=gen)
    for a, b in ((k, v), (q, d_o)):  # (b's token is rounded to its type)
        a[:, active[1]], b[:, active[1]] = -by * a[:, active[0]], b[:, active[0]] / by
    state = lambda: (1.0 + 0.2 * torch.rand((B, H, 1, 1), generator=gen)) * (1.0 + 2.0 ** -12 * torch.randn((B, H, Dk, Dv), generator=gen))  # noqa: E731
    return *(x.to(dtype) for x in (q, k, v, d_o)), decay, state(), state()


def magnitudes(*arrays):
    return [None if x is None else np.abs(x) for x in arrays]


def states(k, v, decay, initial):
    """At each token that is not zero, and after the sequence."""
    T, active = k.shape[1], tokens(k.shape[1])
    return [(0.0 if initial is None else decay[:, None, None] ** (t + 1) * initial) + sum(
        decay[:, None, None] ** (t - s) * k[:, s, :, :, None] * v[:, s, :, None, :] for s in active if s <= t) for t in active + [T - 1]]


def scattered(rows, like):
    out = np.zeros(like.shape[:3] + rows[0].shape[2:])
    for t, row in zip(tokens(like.shape[1]), rows):
        out[:, t] = row
    return out


def forward(q, k, v, decay, initial):
    """(o, final state), and the same of magnitudes: arrays of 64 bits"""
    result = []
    for q, k, v, initial in ((q, k, v, initial), magnitudes(q, k, v, initial)):
        *at, last = states(k, v, decay, initial)
        result.append((scattered([SCALE * np.einsum("bhi,bhij->bhj", q[:, t], s) for t, s in zip(tokens(q.shape[1]), at)], q), last))
    return result


def backward(q, k, v, d_o, decay, initial, d_final):
    """Gradients of q, k, v and the initial state, and the same of magnitudes"""
    result = []
    for q, k, v, d_o, initial, d_final in ((q, k, v, d_o, initial, d_final), magnitudes(q, k, v, d_o, initial, d_final)):
        T, active = q.shape[1], tokens(q.shape[1])
        at = states(k, v, decay, initial)
        error = lambda t: (0.0 if d_final is None else decay[:, None, None] ** (T - 1 - t) * d_final) + SCALE * sum(  # noqa: E731
            decay[:, None, None] ** (s - t) * q[:, s, :, :, None] * d_o[:, s, :, None, :] for s in active if s >= t)
        d_q = [SCALE * np.einsum("bhij,bhj->bhi", s, d_o[:, t]) for t, s in zip(active, at)]
        d_k = [np.einsum("bhij,bhj->bhi", error(t), v[:, t]) for t in active]
        d_v = [np.einsum("bhij,bhi->bhj", error(t), k[:, t]) for t in active]
        result.append((*(scattered(rows, q) for rows in (d_q, d_k, d_v)), decay[:, None, None] * error(0)))
    return result


def slack(T, type_, size, state=False):
    return size * (2.0 ** -24 * STEPS[T] + (0.0 if state else CUT[type_]))


def share(got, exact, allowed, dtype):
    """Largest part of what sequence_reference.near allows that `got`, rounded to its type here, takes."""
    got = ref.numpy64(torch.from_numpy(got).to(dtype))
    return float(np.max(np.abs(got - exact) / (allowed + ref.half_step(dtype) * (np.abs(exact) + allowed) + ref.smallest(dtype))))


def pieces(x, n):
    """x as the sum of n bfloat16 numbers, each the nearest to what the ones before left."""
    total, rest = np.zeros_like(x), x
    for _ in range(n):
        piece = ref.numpy64(torch.from_numpy(rest).to(torch.bfloat16))
        total, rest = total + piece, rest - piece
    return total
