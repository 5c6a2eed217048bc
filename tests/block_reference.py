"""The operators around a block from their definitions, in 64 bits: norms, short convolution, selective scan, log probabilities; each
with its gradient written out, and the sums of magnitudes that bound a computation in 32 bits."""
import torch

U = 2.0 ** -24  # one rounding of fp32


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
