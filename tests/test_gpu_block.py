"""The operators around a block together, as a model that predicts the next pixel uses them: embedding, norm, projection, short convolution, selective scan,
gated norm, the scaled residual and its norm, logits, log probabilities; its gradients, its form token by token, and its step captured into a graph."""
import pytest
import torch

import block_reference as ref
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEVELS, WIDTH, INNER, STATES, TAPS, SCALE = 40, 24, 48, 16, 4, 0.5


def parameters(seed=0):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s, by=1.0: torch.randn(s, generator=gen) * by  # noqa: E731
    p = {"table": normal(LEVELS, WIDTH), "w1": normal(WIDTH, by=0.1) + 1, "w_in": normal(2 * INNER, WIDTH, by=WIDTH ** -0.5), "taps": normal(INNER, TAPS, by=0.5),
         "bias": normal(INNER, by=0.1), "w_p": normal(INNER + 2 * STATES, INNER, by=INNER ** -0.5), "a": -torch.arange(1.0, STATES + 1).repeat(INNER, 1) * 0.3,
         "skip": normal(INNER), "dt_bias": normal(INNER, by=0.5) - 2, "w_g": normal(INNER, by=0.1) + 1, "w_out": normal(WIDTH, INNER, by=INNER ** -0.5),
         "w2": normal(WIDTH, by=0.1) + 1, "v": normal(LEVELS, WIDTH, by=WIDTH ** -0.5)}
    return {k: v.to(DEV) for k, v in p.items()}


def rows(x):
    return x.reshape(-1, x.shape[-1])


def forward(p, tokens, answers):
    """(loss, what the backward pass needs): the mean of -log p of the answers, less a tenth of the mean entropy."""
    x = binding.embedding_fwd(p["table"], tokens)
    n1, _ = binding.add_norm_fwd(x, p["w1"])
    u, z = binding.fc_fwd(rows(n1), p["w_in"]).view(*tokens.shape, 2 * INNER).split(INNER, 2)
    c, _ = binding.causal_conv_fwd(u, p["taps"], p["bias"], True)
    dt, b, cc = binding.fc_fwd(rows(c), p["w_p"]).view(*tokens.shape, -1).split([INNER, STATES, STATES], 2)
    b, cc = b.unflatten(2, (1, STATES)), cc.unflatten(2, (1, STATES))
    y, _ = binding.selective_scan_fwd(c, dt, p["a"], b, cc, p["skip"], p["dt_bias"])
    g = binding.norm_gate_fwd(y, p["w_g"], gate=z, groups=2)
    o = binding.fc_fwd(rows(g), p["w_out"]).view_as(x)
    n2, r = binding.add_norm_fwd(o, p["w2"], residual=x, scale=SCALE)
    logits = binding.fc_fwd(rows(n2), p["v"]).view(*tokens.shape, LEVELS)
    lp, h, stats, _, _ = binding.log_probs_fwd(logits, answers)
    return -lp.mean() - 0.1 * h.mean(), (tokens, answers, x, n1, u, z, c, dt, b, cc, y, g, r, n2, logits, stats, lp)


def gradient(p, saved):
    tokens, answers, x, n1, u, z, c, dt, b, cc, y, g, r, n2, logits, stats, lp = saved
    d = {}
    each = torch.full_like(lp, 1.0 / lp.numel())
    d_logits = binding.log_probs_bwd(logits, answers, stats, -each, d_entropy=-0.1 * each)
    d["v"], _ = binding.fc_bwd_weight(rows(n2), rows(d_logits), want_bias=False)
    d_n2 = binding.fc_bwd_input(rows(d_logits), p["v"]).view_as(n2)
    d_o, d_x, d["w2"] = binding.add_norm_bwd(d_n2, r, p["w2"], scale=SCALE)
    d["w_out"], _ = binding.fc_bwd_weight(rows(g), rows(d_o), want_bias=False)
    d_y, d_z, d["w_g"] = binding.norm_gate_bwd(binding.fc_bwd_input(rows(d_o), p["w_out"]).view_as(g), y, p["w_g"], gate=z, groups=2)
    d_c, d_dt, d["a"], d_b, d_cc, d["skip"], d["dt_bias"], _ = binding.selective_scan_bwd(c, dt, p["a"], b, cc, d_y, p["skip"], p["dt_bias"])
    d_p = torch.cat([rows(d_dt), d_b.view(-1, STATES), d_cc.view(-1, STATES)], 1)
    d["w_p"], _ = binding.fc_bwd_weight(rows(c), d_p, want_bias=False)
    d_c = d_c + binding.fc_bwd_input(d_p, p["w_p"]).view_as(d_c)
    d_u, d["taps"], d["bias"], _ = binding.causal_conv_bwd(u, p["taps"], d_c, p["bias"], True)
    d_uz = torch.cat([rows(d_u), rows(d_z)], 1)
    d["w_in"], _ = binding.fc_bwd_weight(rows(n1), d_uz, want_bias=False)
    d_x1, _, d["w1"] = binding.add_norm_bwd(binding.fc_bwd_input(d_uz, p["w_in"]).view_as(x), x, p["w1"], d_r=d_x)
    d["table"] = binding.embedding_bwd(d_x1, tokens, LEVELS)
    return d


def in_64(p, tokens, answers):
    """The same loss in 64 bits from the definitions, one sequence at a time."""
    loss = 0.0
    for b in range(len(tokens)):
        x = p["table"][tokens[b]]
        n1 = ref.hat(x, 1, 1e-6)[0] * p["w1"]
        u, z = (n1 @ p["w_in"].t()).split(INNER, 1)
        seen = torch.cat([torch.zeros(TAPS - 1, INNER, dtype=u.dtype), u])
        c = ref.silu(p["bias"] + sum(seen[k:k + len(u)] * p["taps"][:, k] for k in range(TAPS)))
        dt, bb, cc = (c @ p["w_p"].t()).split([INNER, STATES, STATES], 1)
        delta, h, ys = torch.logaddexp(dt + p["dt_bias"], torch.zeros_like(dt)), torch.zeros(INNER, STATES, dtype=u.dtype), []
        for t in range(len(u)):
            h = torch.exp(delta[t][:, None] * p["a"]) * h + (delta[t] * c[t])[:, None] * bb[t]
            ys.append(h @ cc[t] + p["skip"] * c[t])
        g = ref.norm_gate(torch.stack(ys), p["w_g"], z, None, 1.0, 1e-6, 2)
        r = x + SCALE * (g @ p["w_out"].t())
        lp = torch.log_softmax((ref.hat(r, 1, 1e-6)[0] * p["w2"]) @ p["v"].t(), 1)
        loss = loss - lp.gather(1, answers[b][:, None]).sum() + 0.1 * (lp.exp() * lp).sum()
    return loss / tokens.numel()


def batch(B, T, seed=1):
    tokens = torch.randint(0, LEVELS, (B, T + 1), generator=torch.Generator().manual_seed(seed)).to(torch.int32).to(DEV)
    return tokens[:, :-1].contiguous(), tokens[:, 1:].contiguous()


@pytest.mark.parametrize("T", [1, 3, 70, 200])
def test_gradients(T):
    """Each operator's results are off by at most some 300 roundings of what they are made of (its own tests), and ten of them follow one another: a gradient
    is off by less than 2^-12 of its norm."""
    p, (tokens, answers) = parameters(), batch(3, T)
    loss, saved = forward(p, tokens, answers)
    got = gradient(p, saved)
    p64 = {k: v.double().cpu().requires_grad_(True) for k, v in p.items()}
    want = in_64(p64, tokens.cpu().long(), answers.cpu().long())
    assert abs(loss.item() - want.item()) <= 2.0 ** -12 * abs(want.item())
    grads = dict(zip(p64, torch.autograd.grad(want, list(p64.values()))))
    for name, g in grads.items():
        off = (got[name].double().cpu() - g).norm()
        print(name, "%.2e" % (off / g.norm().clamp(min=1e-30)).item())
        assert off <= 2.0 ** -12 * g.norm() + 1e-12, name


def test_token_by_token():
    """A token at a time, in place, with the sequences in any slots: the logits of the whole sequences, the top token among them."""
    p, (tokens, answers) = parameters(), batch(3, 60)
    _, saved = forward(p, tokens, answers)
    logits = saved[14]
    slots = torch.tensor([4, 0, 3], dtype=torch.int32, device=DEV)
    last, state = torch.zeros(5, TAPS - 1, INNER, device=DEV), torch.zeros(5, INNER, STATES, device=DEV)
    for t in range(60):
        x = binding.embedding_fwd(p["table"], tokens[:, t].contiguous())
        u, z = binding.fc_fwd(binding.add_norm_fwd(x, p["w1"])[0], p["w_in"]).split(INNER, 1)
        c = binding.causal_conv_step(u, p["taps"], last, p["bias"], True, slots)
        dt, b, cc = binding.fc_fwd(c, p["w_p"]).split([INNER, STATES, STATES], 1)
        y = binding.selective_scan_step(c, dt, p["a"], b.unflatten(1, (1, STATES)), cc.unflatten(1, (1, STATES)), state, p["skip"], p["dt_bias"], slots=slots)
        o = binding.fc_fwd(binding.norm_gate_fwd(y, p["w_g"], gate=z, groups=2), p["w_out"])
        one = binding.fc_fwd(binding.add_norm_fwd(o, p["w2"], residual=x, scale=SCALE)[0], p["v"])
        assert (one - logits[:, t]).abs().max() <= 2.0 ** -12 * logits[:, t].abs().max(), t
        given = binding.log_probs_fwd(one, answers[:, t].contiguous(), top=1)
        assert torch.equal(given[4][:, 0].long(), one.argmax(1))
    assert (last[[1, 2]] == 0.0).all() and (state[[1, 2]] == 0.0).all()


def test_step_in_a_graph():
    """Loss and gradients captured once and replayed with other tokens, with eager steps between the replays: the eager results, bit for bit."""
    p, (tokens, answers) = parameters(), batch(4, 90)

    def step():
        loss, saved = forward(p, tokens, answers)
        return [loss, *gradient(p, saved).values()]
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (5, 6, 7):
        for to, new in zip((tokens, answers), batch(4, 90, seed)):
            to.copy_(new)
        want = step()
        graph.replay()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), seed
