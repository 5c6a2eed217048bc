"""The operators around a block from their definitions, in 64 bits: norms, short convolution, selective scan, log probabilities; each
with its gradient written out, and the sums of magnitudes that bound a computation in 32 bits."""
import torch

U = 2.0 ** -24  # one rounding of fp32
LEAST = 2.0 ** -126  # its smallest normal number


def silu(z):
    return z / (1.0 + torch.exp(-z))


def d_silu(z):
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


# ---- norms (rows [N, D], `groups` equal pieces) -----------------------------------------------------------------
def hat(v, groups, eps):
    """(v over its group's root mean square, one over that root, both [N, D])"""
    cut = v.reshape(len(v), groups, -1)
    root = (cut * cut).mean(2, keepdim=True).add(eps).rsqrt().expand_as(cut).reshape(v.shape)
    return v * root, root


def group_mean(x, groups):
    cut = x.reshape(len(x), groups, -1)
    return cut.mean(2, keepdim=True).expand_as(cut).reshape(x.shape)


def norm_gradient(v, error, groups, eps):
    """The error of v for the error of hat(v), and what it is made of in magnitudes."""
    n, root = hat(v, groups, eps)
    return (root * (error - n * group_mean(error * n, groups)),
            root * (error.abs() + n.abs() * group_mean((error * n).abs(), groups)))


def add_norm(x, weight, residual, scale, eps, groups):
    r = x if residual is None else residual + scale * x
    return hat(r, groups, eps)[0] * weight, r


def add_norm_gradient(d_y, r, weight, d_r, scale, eps, groups):
    d, size = norm_gradient(r, d_y * weight, groups, eps)
    if d_r is not None:
        d, size = d + d_r, size + d_r.abs()
    terms = d_y * hat(r, groups, eps)[0]
    return (scale * d, d, terms.sum(0)), (abs(scale) * size, size, terms.abs().sum(0))


def norm_gate(x, weight, gate, residual, scale, eps, groups):
    y = scale * hat(x, groups, eps)[0] * weight
    y = y if gate is None else y * silu(gate)
    return y if residual is None else y + residual


def norm_gate_gradient(d_y, x, weight, gate, scale, eps, groups):
    n = hat(x, groups, eps)[0]
    by = scale if gate is None else scale * silu(gate)
    d, size = norm_gradient(x, d_y * weight * by, groups, eps)
    d_gate = None if gate is None else scale * d_y * n * weight * d_silu(gate)
    terms = d_y * n * by
    return (d, d_gate, terms.sum(0)), (size, None if gate is None else d_gate.abs() + (scale * d_y * n * weight).abs(), terms.abs().sum(0))


# ---- short convolution (x [B, T, D], weight [D, K], states [B, K - 1, D], lengths a list) --------------------------------
def _inputs(x, initial, b, n, K):
    head = torch.zeros(K - 1, x.shape[2], dtype=x.dtype) if initial is None else initial[b]
    return torch.cat([head, x[b, :n]])


def conv(x, weight, bias, active, lengths, initial):
    """(y, final state, p, sums of magnitudes of p)"""
    (B, T, D), K = x.shape, weight.shape[1]
    y, p, size, state = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x), torch.zeros(B, K - 1, D, dtype=x.dtype)
    for b, n in enumerate(lengths):
        seen = _inputs(x, initial, b, n, K)
        for t in range(n):
            terms = torch.cat([seen[t:t + K] * weight.t(), bias[None]])
            p[b, t], size[b, t] = terms.sum(0), terms.abs().sum(0)
        state[b] = seen[n:]
        y[b, :n] = silu(p[b, :n]) if active else p[b, :n]
    return y, state, p, size


def conv_gradient(x, weight, bias, active, lengths, initial, d_y, d_final, off=None):
    """(d_x, d_weight, d_bias, d_initial) for errors of p in magnitudes where `off` gives them (in place of d_y times silu'), else the gradient."""
    (B, T, D), K = x.shape, weight.shape[1]
    p = conv(x, weight, bias, active, lengths, initial)[2]
    e = (d_y * d_silu(p) if active else d_y) if off is None else off
    d_x, d_w, d_b, d_first = torch.zeros_like(x), torch.zeros_like(weight), torch.zeros_like(bias), torch.zeros(B, K - 1, D, dtype=x.dtype)
    for b, n in enumerate(lengths):
        seen, d_seen = _inputs(x, initial, b, n, K), torch.zeros(K - 1 + n, D, dtype=x.dtype)
        for k in range(K):
            d_seen[k:k + n] += e[b, :n] * weight[:, k]
            d_w[:, k] += (e[b, :n] * seen[k:k + n]).sum(0)
        if d_final is not None:
            d_seen[n:] += d_final[b]
        d_b += e[b, :n].sum(0)
        d_first[b], d_x[b, :n] = d_seen[:K - 1], d_seen[K - 1:]
    return d_x, d_w, d_b, d_first


# ---- selective scan (x, dt [B, T, D], a [D, N], b, c [B, T, G, N], states [B, D, N], lengths a list) ---------------------------
def softplus(z):
    return torch.logaddexp(z, torch.zeros_like(z))


def scan(x, dt, a, b, c, skip, dt_bias, soft, lengths, initial, d_y=None, d_final=None):
    """((y, final state), their errors in 32 bits), and with d_y the gradients (d_x, d_dt, d_a, d_b, d_c, d_skip, d_dt_bias, d_initial) and theirs.

    Errors are carried along, in roundings U of what is added.  z is rounded once and the exponent of softplus twice, so D is off by (3 |z| + 8) U of
    itself (by U |z| without softplus), a decay by |D a| (3 |z| + 10) + 2 roundings, D x b by 3 |z| + 11; where sequences are cut, a segment's decay
    from the sum of its D is off by no more, and a decay below 2^-126, the smallest normal number, may be 0.  So a state's error, and an adjoint's, is the last one's decayed and (|D a| + 1) (3 |z| + 12) + 4 roundings of its magnitude.  Sums over n take up to N
    + 4 roundings, over channels 6 of a wave and D / 4 of waves, over tokens and sequences 64 of a segment, 32 + 64 of the rest."""
    (B, T, D), (G, N) = x.shape, b.shape[2:]
    zeros = lambda *s: torch.zeros(s, dtype=x.dtype)  # noqa: E731
    b, c = b.repeat_interleave(D // G, 2), c.repeat_interleave(D // G, 2)
    inside = torch.arange(T)[None, :] < torch.tensor(lengths)[:, None]
    z = dt + dt_bias
    delta = torch.where(inside[..., None], softplus(z) if soft else z, 0.0)
    rough = (3 * z.abs() + 12)[..., None] * U  # of D, of products with it
    x = torch.where(inside[..., None], x, 0.0)
    b, c = torch.where(inside[..., None, None], b, 0.0), torch.where(inside[..., None, None], c, 0.0)
    h, size, off = (zeros(B, D, N) if initial is None else initial), zeros(B, D, N) if initial is None else initial.abs(), zeros(B, D, N)
    hs, sizes, offs, decays, steps = [h], [size], [off], [], []
    for t in range(T):
        decay, u = torch.exp(delta[:, t, :, None] * a), (delta[:, t] * x[:, t])[..., None] * b[:, t]
        step = ((delta[:, t, :, None] * a).abs() + 1) * rough[:, t] + 4 * U
        h, size = decay * h + u, decay * size + u.abs()
        off = decay * off + size * step + LEAST * sizes[-1]
        hs.append(h), sizes.append(size), offs.append(off), decays.append(decay), steps.append(step)
    stack = lambda v: torch.stack(v, 1)  # noqa: E731
    H, M, E, A, S = stack(hs), stack(sizes), stack(offs), stack(decays), stack(steps)
    y = (H[:, 1:] * c).sum(3) + skip * x
    y_off = (c.abs() * (E[:, 1:] + (N + 4) * U * M[:, 1:])).sum(3) + 2 * U * (skip * x).abs()
    forward = (torch.where(inside[..., None], y, 0.0), H[:, -1]), (torch.where(inside[..., None], y_off, 0.0), E[:, -1])
    if d_y is None:
        return forward
    d_y = torch.where(inside[..., None], d_y, 0.0)
    q, q_size, q_off = (zeros(B, D, N) if d_final is None else d_final), zeros(B, D, N) if d_final is None else d_final.abs(), zeros(B, D, N)
    gs, g_sizes, g_offs = [], [], []
    for t in reversed(range(T)):
        g, g_size = q + c[:, t] * d_y[:, t, :, None], q_size + (c[:, t] * d_y[:, t, :, None]).abs()
        g_off = q_off + 2 * U * g_size
        q, q_size, q_off = A[:, t] * g, A[:, t] * g_size, A[:, t] * (g_off + g_size * S[:, t]) + LEAST * g_size
        gs.append(g), g_sizes.append(g_size), g_offs.append(g_off)
    back = lambda v: torch.stack(v[::-1], 1)  # noqa: E731
    g, gm, ge = back(gs), back(g_sizes), back(g_offs)
    sums = (N + 8) * U
    gb, gb_size = (g * b).sum(3), (gm * b.abs()).sum(3)
    gb_off = (ge * b.abs()).sum(3) + sums * gb_size
    along, along_size = A * g * H[:, :-1], A * gm * M[:, :-1]
    along_off = A * (ge * M[:, :-1] + gm * E[:, :-1]) + along_size * S + LEAST * gm * M[:, :-1]
    r, d_size = rough[..., 0], delta.abs()
    d_x, d_x_off = delta * gb + skip * d_y, d_size * (gb_off + r * gb_size) + 2 * U * (skip * d_y).abs()
    dd = x * gb + (along * a).sum(3)
    dd_size = x.abs() * gb_size + (along_size * a.abs()).sum(3)
    dd_off = x.abs() * gb_off + (a.abs() * (along_off + sums * along_size)).sum(3) + 3 * U * dd_size
    slope = 1 / (1 + torch.exp(-z)) if soft else torch.ones_like(z)
    d_dt, d_dt_size, d_dt_off = dd * slope, dd_size * slope, slope * (dd_off + r * dd_size)
    share = lambda v: v.unflatten(2, (G, D // G)).sum(3)  # noqa: E731
    u, u_size = (delta * x)[..., None], (delta * x)[..., None].abs()
    channels, tokens = (6 + D / 4) * U, (64 + 32 + 64) * U
    total = lambda v: v.sum((0, 1))  # noqa: E731
    masked = lambda v: torch.where(inside[..., None], v, 0.0)  # noqa: E731
    grads = (masked(d_x), masked(d_dt), total(along * delta[..., None]), share(g * u), share(H[:, 1:] * d_y[..., None]), total(d_y * x), total(masked(d_dt)), q)
    off = (masked(d_x_off), masked(d_dt_off), total(d_size[..., None] * (along_off + along_size * (rough + tokens))),
           share(u_size * (ge + gm * (rough + channels))), share(d_y[..., None].abs() * (E[:, 1:] + channels * M[:, 1:])), tokens * total((d_y * x).abs()),
           total(masked(d_dt_off + tokens * d_dt_size)), q_off)
    return forward, (grads, off)


# ---- log probabilities (rows [N, V], tokens [N, M]) ----------------------------------------------------------------
def log_probs(logits, tokens, scale, top):
    """(log probabilities of the tokens, entropy, log probabilities of the top ones, their tokens, all log probabilities)"""
    z = logits * scale
    m = z.amax(1, keepdim=True)
    none = torch.isinf(m) & (m < 0)
    z = torch.where(none, z, z - m)
    lp = torch.where(none, z, z - torch.log(torch.exp(z).sum(1, keepdim=True)))
    p = torch.exp(lp)
    known = (tokens >= 0) & (tokens < logits.shape[1])
    given = torch.where(known, lp.gather(1, torch.where(known, tokens, 0)), torch.zeros((), dtype=lp.dtype))
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    order = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :top]
    return given, entropy, lp.gather(1, order), order, lp


def log_probs_gradient(logits, tokens, scale, d_given, d_entropy):
    lp = log_probs(logits, tokens, scale, 0)[4]
    p = torch.exp(lp)
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    known = (tokens >= 0) & (tokens < logits.shape[1])
    g = torch.where(known, d_given, torch.zeros_like(d_given))
    d = -p * g.sum(1, keepdim=True)
    d = d.scatter_add(1, torch.where(known, tokens, 0), g)
    if d_entropy is not None:
        d = d - d_entropy[:, None] * (plp - p * plp.sum(1, keepdim=True))
    none = torch.isinf(logits).all(1, keepdim=True) & (logits < 0).all(1, keepdim=True)
    return torch.where(none, torch.zeros_like(d), scale * d)
