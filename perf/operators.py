"""Performance cases of the sequence operators: embedding, dropout and linear attention (paper_1912_05234_amd.binding).

The images of this framework can be read as sequences: 784 pixels, one token of 256 grey levels each, 100 sequences to a
batch.  The operators that such a classifier needs beside the fully connected and logistic calls, each in both directions:

  embed_fwd     rows of a table looked up by token and scaled; a token outside the table (padding) gives a row of zeros
  embed_bwd     gradient of the table: every row the scaled sum of the output errors of its tokens
  drop_fwd      dropout with the mask of a counter-based generator, added to a residual stream
  drop_bwd      its gradient, from the same counters
  linear_fwd    linear attention with a decay for each head over whole sequences (prompts, training)
  linear_bwd    its gradients
  linear_step   one token of each sequence against a pool of states, updated in place (serving)

`run` computes them with elementary torch operations where `own` is false, and calls the framework where it is true.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}

PIXELS = 28 * 28     # tokens of one image
LEVELS = 256         # grey levels, the vocabulary of pixel tokens
BATCH = 100          # images of a training batch
WIDTH = 64           # of the classifier over pixel sequences: two heads of 32


def listed():
    return [
        # The next pixel of 64 streams: the smallest lookup, where latency is everything.
        {"name": "embed_fwd_64_pixels", "kind": "embed_fwd", "N": 64, "V": LEVELS, "D": WIDTH, "type": "fp32", "dist": "pixels"},
        # A long batch of text over a large vocabulary, in bfloat16.
        {"name": "embed_fwd_text", "kind": "embed_fwd", "N": 131071, "V": 50021, "D": 1024, "type": "bf16", "dist": "zipf"},
        # The gradient of the pixel classifier's table: few rows, one of them (the background) with a third of all tokens.
        {"name": "embed_bwd_pixels", "kind": "embed_bwd", "N": BATCH * PIXELS, "V": LEVELS, "D": WIDTH, "type": "fp32", "dist": "pixels"},
        # The gradient of a text model's table: many rows, most with few tokens, some with none; a width that is no power of two.
        {"name": "embed_bwd_text", "kind": "embed_bwd", "N": 65521, "V": 32003, "D": 1000, "type": "bf16", "dist": "zipf"},
        # Dropout in front of the image classifier's output layer, backward, at the paper's batch.
        {"name": "drop_bwd_192x100", "kind": "drop_bwd", "n": BATCH * 192, "p": 0.5, "type": "fp32"},
        # Dropout of a layer's output on its way into the residual stream; an odd number of elements.
        {"name": "drop_fwd_residual", "kind": "drop_fwd", "n": 8191 * 8193, "p": 0.1, "type": "bf16", "residual": True},
        # A prompt: two long sequences, slices of one projection, and the state that generation goes on from.
        {"name": "linear_fwd_prompt", "kind": "linear_fwd", "B": 2, "T": 8192, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "type": "bf16",
         "fused": True, "ragged": False, "states": "out"},
        # The classifier over pixel sequences of different lengths, empty ones among them.
        {"name": "linear_fwd_pixels", "kind": "linear_fwd", "B": BATCH, "T": PIXELS, "H": 2, "Hk": 2, "Dk": 32, "Dv": 32, "type": "fp32",
         "fused": False, "ragged": True, "states": "none"},
        # Its training step.
        {"name": "linear_bwd_pixels", "kind": "linear_bwd", "B": BATCH, "T": PIXELS, "H": 2, "Hk": 2, "Dk": 32, "Dv": 32, "type": "fp32",
         "fused": False, "ragged": False, "states": "none"},
        # Training on pieces of long sequences in fp16: shared key heads, an odd length, states handed from piece to piece.
        {"name": "linear_bwd_pieces", "kind": "linear_bwd", "B": 3, "T": 2047, "H": 12, "Hk": 4, "Dk": 64, "Dv": 96, "type": "fp16",
         "fused": True, "ragged": False, "states": "both"},
        # One stream, one token.
        {"name": "linear_step_1", "kind": "linear_step", "B": 1, "pool": 1, "H": 8, "Hk": 8, "Dk": 64, "Dv": 64, "type": "fp32"},
        # A server's batch: 256 rows, some without a sequence, states scattered over a pool of 300.
        {"name": "linear_step_256", "kind": "linear_step", "B": 256, "pool": 300, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "type": "bf16"},
    ]


# The most that a drawn case may ask for: the largest listed one of its family.
EMBED_CAP, DROP_CAP, LINEAR_CAP, STEP_CAP = 5.0e8, 4.0e8, 2.6e8, 5.3e8


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_bwd", "drop_fwd", "drop_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "linear_bwd", "linear_step"])
    type_ = rng.choice(["fp32", "bf16", "fp16"])
    if kind.startswith("embed"):
        while True:
            case = {"kind": kind, "N": _log_int(rng, 1, 131072), "V": _log_int(rng, 10, 60000), "D": _log_int(rng, 8, 2048), "type": type_,
                    "dist": rng.choice(["zipf", "pixels", "uniform"])}
            if rng.random() < 0.7:
                case["D"] = max(8, case["D"] // 8 * 8)
            if work(case)["bytes"] <= EMBED_CAP:
                return case
    if kind.startswith("drop"):
        residual = kind == "drop_fwd" and rng.random() < 0.6
        most = int(DROP_CAP / (BYTES[type_] * (3 if residual else 2)))
        case = {"kind": kind, "n": _log_int(rng, 100, most), "p": rng.choice([0.05, 0.1, 0.25, 0.5, round(rng.uniform(0.01, 0.95), 4)]), "type": type_}
        return {**case, "residual": residual} if kind == "drop_fwd" else case
    while True:
        Hk, group = rng.choice([1, 2, 3, 4, 8, 12, 16]), rng.choice([1, 1, 1, 2, 3])
        Dk, Dv = (rng.choice([16, 32, 64, 64, 80, 96, 128, 128, rng.randint(8, 160), 256]) for _ in range(2))
        if kind == "linear_step":
            B = _log_int(rng, 1, 512)
            case = {"kind": kind, "B": B, "pool": B + rng.randint(0, 40), "H": Hk * group, "Hk": Hk, "Dk": Dk, "Dv": Dv, "type": type_}
            if work(case)["bytes"] <= STEP_CAP:
                return case
            continue
        case = {"kind": kind, "B": _log_int(rng, 1, 100), "T": _log_int(rng, 1, 8192), "H": Hk * group, "Hk": Hk, "Dk": Dk, "Dv": Dv, "type": type_,
                "fused": rng.random() < 0.5, "ragged": rng.random() < 0.5, "states": rng.choice(["none", "out", "both"])}
        w = work(case)
        if w["bytes"] <= LINEAR_CAP and w["flops"] <= 2.0e10:
            return case


def _tokens(case, gen):
    """Tokens as they come: pixel levels with a large background, words by Zipf's law, or uniform; three in a hundred are padding (-1)."""
    N, V, dist = case["N"], case["V"], case["dist"]
    u = torch.rand(N, generator=gen, device=DEV, dtype=torch.float64)
    if dist == "pixels":
        t = ((u * 1.5 - 0.5).clamp_(min=0.0) * V).long().clamp_(max=V - 1)
        return t.to(torch.int32)
    if dist == "zipf":
        cdf = (1.0 / (torch.arange(V, device=DEV, dtype=torch.float64) + 2.7)).cumsum(0)
        t = torch.searchsorted(cdf, u * cdf[-1]).clamp_(max=V - 1)
        t = torch.randperm(V, generator=gen, device=DEV)[t]  # frequent words are anywhere in the table
    else:
        t = (u * V).long().clamp_(max=V - 1)
    return torch.where(torch.rand(N, generator=gen, device=DEV) < 0.03, torch.full_like(t, -1), t)


def _decays(H):
    """1 - 2^-5 for the first head, 1 - 2^-12 for the last."""
    steps = torch.arange(H, device=DEV, dtype=torch.float64) * (7.0 / max(1, H - 1))
    return (1.0 - torch.exp2(-5.0 - steps)).float()


def prepare(case, seed):
    kind, type_ = case["kind"], TYPES[case["type"]]
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, dtype=type_, by=1.0):
        return torch.randn(shape, generator=gen, device=DEV).mul_(by).to(dtype)

    s = {"case": case}
    if kind.startswith("embed"):
        s["tokens"], s["scale"] = _tokens(case, gen), math.sqrt(case["D"])
        if kind == "embed_fwd":
            s["table"] = normal(case["V"], case["D"], by=case["D"] ** -0.5)
        else:
            s["d_out"] = normal(case["N"], case["D"])
        return s
    if kind.startswith("drop"):
        s["x"] = normal(case["n"])
        s["residual"] = normal(case["n"]) if case.get("residual") else None
        s["seed"], s["offset"] = 0x1912052340000000 + seed, seed % 1000  # of the run, and of the step and layer
        return s
    B, H, Hk, Dk, Dv = (case[k] for k in ("B", "H", "Hk", "Dk", "Dv"))
    s["decay"], s["scale"] = _decays(H), Dk ** -0.5
    if kind == "linear_step":
        s["q"], s["k"], s["v"] = normal(B, H, Dk), normal(B, Hk, Dk), normal(B, Hk, Dv)
        s["state"] = normal(case["pool"], H, Dk, Dv, dtype=torch.float32, by=4.0)
        s["slots"] = torch.randperm(case["pool"], generator=gen, device=DEV)[:B].to(torch.int32)
        if B > 1:
            s["slots"][torch.rand(B, generator=gen, device=DEV) < 0.05] = -1
        return s
    T = case["T"]
    if case["fused"]:  # slices of one projection's output
        both = normal(B, T, H * Dk + Hk * (Dk + Dv))
        q, k, v = both.split([H * Dk, Hk * Dk, Hk * Dv], dim=2)
        s["q"], s["k"], s["v"] = q.unflatten(2, (H, Dk)), k.unflatten(2, (Hk, Dk)), v.unflatten(2, (Hk, Dv))
    else:
        s["q"], s["k"], s["v"] = normal(B, T, H, Dk), normal(B, T, Hk, Dk), normal(B, T, Hk, Dv)
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device=DEV).to(torch.int32)
    both = case["states"] == "both"
    s["initial"] = normal(B, H, Dk, Dv, dtype=torch.float32, by=4.0) if both else None
    if kind == "linear_bwd":
        s["d_o"] = normal(B, T, H, Dv)
        s["d_final"] = normal(B, H, Dk, Dv, dtype=torch.float32) if both else None
    return s


def run(s):
    return _framework(s) if own else _plain(s)


def _framework(s):
    from paper_1912_05234_amd import binding
    case = s["case"]
    kind = case["kind"]
    if kind == "embed_fwd":
        return binding.embedding_fwd(s["table"], s["tokens"], s["scale"])
    if kind == "embed_bwd":
        return binding.embedding_bwd(s["d_out"], s["tokens"], case["V"], s["scale"])
    if kind == "drop_fwd":
        return binding.dropout_fwd(s["x"], case["p"], s["seed"], s["offset"], residual=s["residual"])
    if kind == "drop_bwd":
        return binding.dropout_bwd(s["x"], case["p"], s["seed"], s["offset"])
    if kind == "linear_step":
        o = binding.linear_attention_step(s["q"], s["k"], s["v"], s["decay"], s["state"], s["scale"], slots=s["slots"])
        return {"o": o, "state": s["state"]}
    if kind == "linear_fwd":
        o, state = binding.linear_attention_fwd(s["q"], s["k"], s["v"], s["decay"], s["scale"], lengths=s["lengths"],
                                                initial_state=s["initial"], want_state=case["states"] != "none")
        return {"o": o, "state": state}
    d_q, d_k, d_v, d_state = binding.linear_attention_bwd(s["q"], s["k"], s["v"], s["decay"], s["d_o"], s["scale"], lengths=s["lengths"],
                                                          initial_state=s["initial"], d_final_state=s["d_final"],
                                                          want_d_state=case["states"] == "both")
    return {"d_q": d_q, "d_k": d_k, "d_v": d_v, "d_state": d_state}


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _plain(s):
    case = s["case"]
    kind, type_ = case["kind"], TYPES[case["type"]]
    if kind.startswith("embed"):
        tokens = s["tokens"].long()
        known = (tokens >= 0) & (tokens < case["V"])
        if kind == "embed_fwd":
            rows = s["table"][torch.where(known, tokens, 0)].float() * s["scale"]
            return torch.where(known[:, None], rows, 0.0).to(type_)
        # differences of running sums at the ends of each token's run, in 64 bits: up to a hundred thousand errors to a sum
        tokens, order = torch.where(known, tokens, case["V"]).sort(stable=True)
        sums = torch.nn.functional.pad(s["d_out"][order].t().double().contiguous().cumsum(1), (1, 0))
        ends = torch.searchsorted(tokens, torch.arange(case["V"] + 1, device=DEV))
        return (sums[:, ends].diff(dim=1) * s["scale"]).t().to(type_).contiguous()
    if kind.startswith("drop"):
        y = torch.where(_kept(case["n"], case["p"], s["seed"], s["offset"]), s["x"].float() * (1.0 / (1.0 - case["p"])), 0.0)
        return (y if s["residual"] is None else y + s["residual"].float()).to(type_)
    group, scale = case["H"] // case["Hk"], s["scale"]
    if kind == "linear_step":
        q, k, v = s["q"].float(), s["k"].float().repeat_interleave(group, 1), s["v"].float().repeat_interleave(group, 1)
        active, at = (s["slots"] >= 0)[:, None, None], s["slots"].clamp(min=0).long()
        new = s["state"][at] * s["decay"][:, None, None] + k[..., None] * v[..., None, :]
        o = torch.where(active, (new * q[..., None]).sum(2) * scale, 0.0)
        row = torch.full((case["pool"] + 1,), -1, device=DEV)  # of each slot; the last one collects the inactive rows
        row[torch.where(s["slots"] >= 0, at, case["pool"])] = torch.arange(case["B"], device=DEV)
        row = row[:-1, None, None, None]
        s["state"].copy_(torch.where(row >= 0, new[row.flatten().clamp(min=0)], s["state"]))
        return {"o": o.to(type_), "state": s["state"]}
    B, T = case["B"], case["T"]
    lengths = torch.full((B,), T, device=DEV) if s["lengths"] is None else s["lengths"].long()
    inside = (torch.arange(T, device=DEV) < lengths[:, None])[:, None, :, None]
    there = lambda x: torch.where(inside, x.float().transpose(1, 2), 0.0)  # noqa: E731  [B, heads, T, width], zeros past the length
    q, k, v = there(s["q"]), there(s["k"]).repeat_interleave(group, 1), there(s["v"]).repeat_interleave(group, 1)
    back = lambda x: x.transpose(1, 2).to(type_).contiguous()  # noqa: E731
    lam = s["decay"].double()
    if kind == "linear_fwd":
        o = _chunked(q, k, v, lam, s["initial"]) * scale
        state = _last_state(k, v, lam, s["initial"], lengths) if case["states"] != "none" else None
        return {"o": back(torch.where(inside, o, 0.0)), "state": state}
    d_o = there(s["d_o"])
    order = (lengths[:, None] - 1 - torch.arange(T, device=DEV)).clamp_(min=0)
    turn = lambda x: torch.where(inside, x.gather(2, order[:, None, :, None].expand_as(x)), 0.0)  # noqa: E731  time reversed
    # an error of the last state stands one decay ahead of where the reversed sequence would have a state before its first token
    ahead = None if s["d_final"] is None else s["d_final"] / (scale * s["decay"][:, None, None])
    flip = lambda x: None if x is None else x.transpose(2, 3).contiguous()  # noqa: E731
    rq, rk, rv, rd = turn(q), turn(k), turn(v), turn(d_o)
    d_q = torch.where(inside, _chunked(d_o, v, k, lam, flip(s["initial"])), 0.0) * scale
    d_k = turn(_chunked(rv, rd, rq, lam, flip(ahead))) * scale
    d_v = turn(_chunked(rk, rq, rd, lam, ahead)) * scale
    shared = lambda x: x.unflatten(1, (case["Hk"], group)).sum(2)  # noqa: E731
    d_state = None
    if case["states"] == "both":
        d_state = _last_state(rq, rd, lam, ahead, lengths) * (scale * s["decay"][:, None, None])
        d_state = torch.where((lengths > 0)[:, None, None, None], d_state, s["d_final"])
    return {"d_q": back(d_q), "d_k": back(shared(d_k)), "d_v": back(shared(d_v)), "d_state": d_state}


def _chunked(q, k, v, lam, s0, C=128):
    """o_t = sum_{s <= t} lam^(t - s) (q_t . k_s) v_s + lam^(t + 1) q_t s0: inside chunks of C tokens as a masked product, between
    them through the states at the chunks' starts, all at once.  Powers of the decays in 64 bits."""
    T, n = q.shape[2], -(-q.shape[2] // C)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, n * C - T)).unflatten(2, (n, C))  # noqa: E731
    q, k, v = cut(q), cut(k), cut(v)
    i, c = torch.arange(C, device=DEV), torch.arange(n, device=DEV)
    power = lambda e: torch.where(e >= 0, lam.view(-1, *([1] * e.dim())) ** e.clamp(min=0), 0.0).float()  # noqa: E731
    scores = q.matmul(k.transpose(-1, -2).contiguous()) * power(i[:, None] - i)[:, None]
    added = (k * power(C - 1 - i)[:, None, :, None]).transpose(-1, -2).contiguous().matmul(v)
    states = power((c[:, None] - 1 - c) * C).matmul(added.flatten(3)).view_as(added)
    if s0 is not None:
        states = states + power(c * C)[..., None, None] * s0[:, :, None]
    o = scores.matmul(v) + (q * power(i + 1)[:, None, :, None]).matmul(states)
    return o.flatten(2, 3)[:, :, :T]


def _last_state(k, v, lam, s0, lengths):
    e = lengths[:, None] - 1 - torch.arange(k.shape[2], device=DEV)  # tokens still to come, [B, T]
    w = torch.where(e[:, None] >= 0, lam[None, :, None] ** e[:, None].clamp(min=0), 0.0).float()
    state = (k * w[..., None]).transpose(-1, -2).contiguous().matmul(v)
    return state if s0 is None else state + (lam[None, :, None, None] ** lengths[:, None, None, None]).float() * s0


def _kept(n, p, seed, offset):
    """The generator's decision on n elements, in 64-bit integers: eight elements to a block, sixteen high bits of each element's
    number from one call of the generator, sixteen low bits from another."""
    block = torch.arange(-(-n // 8), device=DEV)
    number = (_halves(block, 0, seed, offset) << 16) | _halves(block, 1, seed, offset)
    return number.flatten()[:n] >= int(math.floor(p * 2.0 ** 32 + 0.5))


def _halves(block, call, seed, offset):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) of the counters (block, call * 2^31 in the second word, offset): the four words
    as eight halves, low half first."""
    low = 0xFFFFFFFF
    c0, c1 = block & low, (block >> 32) | (call << 31)
    c2, c3 = torch.full_like(block, offset & low), torch.full_like(block, (offset >> 32) & low)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        h0, l0 = _product(c0, 0xD2511F53)
        h1, l1 = _product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).flatten(1)


def _product(a, m):
    """High and low 32 bits of a * m, both below 2^32."""
    upper = a * (m >> 16) + ((a * (m & 0xFFFF)) >> 16)
    return upper >> 16, (a * m) & 0xFFFFFFFF


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    wide = {name: x.double() for name, x in s.items() if torch.is_tensor(x) and x.is_floating_point()}
    if kind == "embed_fwd":
        table = torch.cat([wide["table"] * s["scale"], torch.zeros(1, case["D"], device=DEV, dtype=torch.float64)])
        tokens = s["tokens"].long()
        return table[torch.where((tokens < 0) | (tokens >= case["V"]), case["V"], tokens)]
    if kind == "embed_bwd":
        total = torch.zeros(case["V"], case["D"], device=DEV, dtype=torch.float64)
        known = (s["tokens"] >= 0) & (s["tokens"] < case["V"])
        return total.index_add_(0, s["tokens"][known].long(), wide["d_out"][known]) * s["scale"]
    if kind.startswith("drop"):
        keep = torch.from_numpy(_kept_by_words(case["n"], case["p"], s["seed"], s["offset"])).to(DEV)
        y = wide["x"] / (1.0 - case["p"]) * keep
        return y + wide["residual"] if "residual" in wide else y
    H, group, scale = case["H"], case["H"] // case["Hk"], s["scale"]
    lam = wide["decay"][:, None, None]
    if kind == "linear_step":
        o, state = torch.zeros(case["B"], H, case["Dv"], device=DEV, dtype=torch.float64), wide["state"]
        for b, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                k, v = wide["k"][b].repeat_interleave(group, 0), wide["v"][b].repeat_interleave(group, 0)
                state[slot] = state[slot] * lam + torch.einsum("hi,hj->hij", k, v)
                o[b] = torch.einsum("hi,hij->hj", wide["q"][b], state[slot]) * scale
        return {"o": o, "state": state}
    B, T, Hk = case["B"], case["T"], case["Hk"]
    lengths = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    active = torch.arange(T, device=DEV)[:, None] < torch.tensor(lengths, device=DEV)
    zeros = lambda *shape: torch.zeros(shape, device=DEV, dtype=torch.float64)  # noqa: E731
    k, v = wide["k"].repeat_interleave(group, 2), wide["v"].repeat_interleave(group, 2)
    state = wide["initial"] if s["initial"] is not None else zeros(B, H, case["Dk"], case["Dv"])
    if kind == "linear_fwd":
        o = zeros(B, T, H, case["Dv"])
        for t in range(max(lengths)):
            on = active[t][:, None, None, None]
            state = torch.where(on, state * lam + k[:, t, :, :, None] * v[:, t, :, None, :], state)
            o[:, t] = (wide["q"][:, t, :, None] @ state)[:, :, 0] * (active[t][:, None, None] * scale)
        return {"o": o, "state": state if case["states"] != "none" else None}
    d_o = wide["d_o"]
    d_q, d_k, d_v = zeros(B, T, H, case["Dk"]), zeros(B, T, H, case["Dk"]), zeros(B, T, H, case["Dv"])
    for t in range(max(lengths)):
        on = active[t][:, None, None, None]
        state = torch.where(on, state * lam + k[:, t, :, :, None] * v[:, t, :, None, :], state)
        d_q[:, t] = (state @ d_o[:, t, :, :, None])[..., 0] * (active[t][:, None, None] * scale)
    d_state = wide["d_final"] if s["d_final"] is not None else torch.zeros_like(state)
    for t in reversed(range(max(lengths))):
        on = active[t][:, None, None, None]
        d_state = torch.where(on, d_state + scale * wide["q"][:, t, :, :, None] * d_o[:, t, :, None, :], d_state)
        d_k[:, t] = (d_state @ v[:, t, :, :, None])[..., 0] * active[t][:, None, None]
        d_v[:, t] = (k[:, t, :, None] @ d_state)[:, :, 0] * active[t][:, None, None]
        d_state = torch.where(on, d_state * lam, d_state)
    d_k, d_v = (x.view(B, T, Hk, group, -1).sum(3) for x in (d_k, d_v))
    return {"d_q": d_q, "d_k": d_k, "d_v": d_v, "d_state": d_state if case["states"] == "both" else None}


def _kept_by_words(n, p, seed, offset):
    """The same decision in unsigned words on the host; the second call only for the blocks where the first leaves one open."""
    limit = int(math.floor(p * 2.0 ** 32 + 0.5))

    def words(block, call):
        u = np.uint64
        low, c = u(0xFFFFFFFF), [block & u(0xFFFFFFFF), (block >> u(32)) | u(call << 31), np.full_like(block, offset & 0xFFFFFFFF),
                                 np.full_like(block, offset >> 32)]
        key = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
        for _ in range(10):
            first, second = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)  # exact: below 2^64
            c = [second >> u(32) ^ c[1] ^ u(key[0]), second & low, first >> u(32) ^ c[3] ^ u(key[1]), first & low]
            key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
        return np.stack(c, 1).astype("<u4").view("<u2").astype(np.int64)

    high = np.concatenate([words(np.arange(a, min(a + (1 << 20), -(-n // 8)), dtype=np.uint64), 0) for a in range(0, -(-n // 8), 1 << 20)])
    keep, open_ = high > limit >> 16, high == limit >> 16
    blocks = np.flatnonzero(open_.any(1))
    if len(blocks):
        low = words(blocks.astype(np.uint64), 1)
        keep[blocks] |= open_[blocks] & (low >= (limit & 0xFFFF))
    return keep.reshape(-1)[:n]


def work(case):
    """Every input read once, every output written once; of a table only the rows that can be asked for."""
    kind, e = case["kind"], BYTES[case["type"]]
    if kind.startswith("embed"):
        N, V, D, t = case["N"], case["V"], case["D"], 4 if case["dist"] == "pixels" else 8
        rows = N + min(N, V) if kind == "embed_fwd" else N + V
        return {"bytes": float(N * t + rows * D * e), "flops": float(N * D)}
    if kind.startswith("drop"):
        return {"bytes": float(case["n"] * e * (3 if case.get("residual") else 2)), "flops": float(case["n"])}
    B, H, Hk, Dk, Dv = (case[k] for k in ("B", "H", "Hk", "Dk", "Dv"))
    if kind == "linear_step":
        return {"bytes": float(B * (H * Dk * Dv * 8 + (H + Hk) * Dk * e + (H + Hk) * Dv * e)), "flops": 4.0 * B * H * Dk * Dv}
    T, states = case["T"], {"none": 0, "out": 1, "both": 2}[case["states"]] * B * H * Dk * Dv * 4
    tokens = B * T
    read = tokens / 2 if case["ragged"] else tokens  # lengths are uniform between 0 and T
    if kind == "linear_fwd":
        return {"bytes": float(read * (H * Dk + Hk * Dk + Hk * Dv) * e + tokens * H * Dv * e + states), "flops": 4.0 * read * H * Dk * Dv}
    states = states if case["states"] != "both" else states // 2 * 3
    return {"bytes": float(read * (H * Dk + Hk * Dk + Hk * Dv + H * Dv) * e + tokens * (H * Dk + Hk * Dk + Hk * Dv) * e + states),
            "flops": 10.0 * read * H * Dk * Dv}
