"""Log probabilities of logits and scales far from 1, all of them finite: masks that are numbers, temperatures next to 0, differences past the largest number.

What counts are differences: the bounds are those of test_gpu_log_probs.py, in roundings of the scaled difference z to the row's largest logit, however large
logits and scale are.  Where a single exponential and a factor behind the sum stand for exp(z), their exponents are off by at most 2^-9, which costs the
entropy's difference t - rest s no more than 2^-9 of the 180 u of its two sums.  No probability of these rows lies between 0 and 2^-126."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding
from test_gpu_log_probs import bounds, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# of a few lanes, a wave, several waves, a workgroup's last form, several parts
VOCABULARIES = [3, 200, 5000, 32003, 70001]
LOWEST = {"fp32": -torch.finfo(torch.float32).max, "bf16": -torch.finfo(torch.bfloat16).max, "fp16": -torch.finfo(torch.float16).max}


def run(logits, tokens, type_, scale, top):
    gen, by = torch.Generator().manual_seed(0), max(scale, 1.0) if type_ == "fp16" else 1.0  # (a gradient is the scale times errors: halves end at 65504)
    d, d_h = (torch.randn(tokens.shape, generator=gen) / by).to(DEV), (torch.randn(len(logits), generator=gen) / by).to(DEV)
    check(logits.to(seq.TYPES[type_]).to(DEV), tokens.to(DEV), d, d_h, scale, top)


def masked(V, value, gen):
    """Rows of which a few tokens are left, spread over the row; its first tenth; its last token; none."""
    logits = torch.randn(4, V, generator=gen).clamp(-3, 3)
    logits[0, torch.rand(V, generator=gen) > 200 / V] = value
    logits[0, V // 2] = 1.0
    logits[1, max(V // 10, 1):] = value
    logits[2, :-1] = value
    logits[3] = value
    return logits, torch.stack([torch.tensor([V // 2, 0, V - 1, V // 3]), torch.randint(0, V, (4,), generator=gen)], 1)


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("value,scale", [(-1e4, 1.0), (-1e9, 10.0), (-1e10, 1.0), (-1e10, 0.8), (-1e30, 0.8), (-1e30, 0.5), (-3e38, 1.0), (-1e9, 1e6)])
@pytest.mark.parametrize("type_", ["fp32", "bf16"])
def test_masks_that_are_numbers(type_, value, scale, V):
    run(*masked(V, value, torch.Generator().manual_seed(V)), type_, scale, min(V, 20))


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("scale", [1.0, 0.3, 1e5, 3e6])
def test_masks_of_halves(scale, V):
    """Their lowest value is -65504: past 2^32 with such scales."""
    run(*masked(V, LOWEST["fp16"], torch.Generator().manual_seed(V)), "fp16", scale, min(V, 20))


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("scale", [10.0 ** k for k in range(3, 31, 3)] + [3e8, 1e28])
@pytest.mark.parametrize("type_", list(seq.TYPES))
def test_temperatures_next_to_0(type_, scale, V):
    """Maxima that are no powers of two, of both signs, alone and three times; the rest below them."""
    logits = torch.randn(5, V, generator=torch.Generator().manual_seed(V)).clamp(-3, 3)
    for n, m in enumerate((20.3, 33.1, -17.7, 20.3, -17.7)):
        if m < 0:
            logits[n] -= 30.0
        for at in ((V // 2,) if n < 3 else (0, V // 3, V - 1)):
            logits[n, at] = m
    tokens = torch.stack([torch.full((5,), V // 2), torch.zeros(5, dtype=torch.int64)], 1)
    run(logits, tokens, type_, scale, min(V, 5))


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("size", [1e8, 1e10, 1e16, 1e25, 1e30, 3e38])
@pytest.mark.parametrize("type_", ["fp32", "bf16"])
def test_large_logits(type_, size, V):
    """A large maximum among ordinary logits; all of them large, alike to a few roundings or of either sign, at scales that leave differences of some units too."""
    gen = torch.Generator().manual_seed(V)
    logits = torch.randn(4, V, generator=gen)
    logits[0, V // 2] = size
    logits[1] = size * (1 - torch.randint(0, 4, (V,), generator=gen) * 2.0 ** -8)
    logits[2] = -logits[1]
    logits[3] = (logits[3].clamp(-3, 3) / 3) * size
    tokens = torch.randint(0, V, (4, 2), generator=gen)
    for scale in (1.0, 30.0 / size):
        if size * scale * 2 < 3e38:  # (else log probabilities are no numbers)
            run(logits, tokens, type_, scale, min(V, 5))


@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("type_", ["fp32", "bf16"])
def test_differences_past_the_largest_number(type_, V):
    """The type's lowest value and its largest in one row: their difference is no number, its product with a scale below 1/2 is one."""
    gen = torch.Generator().manual_seed(V)
    logits = torch.where(torch.rand(3, V, generator=gen) < 0.5, LOWEST[type_], -LOWEST[type_])
    logits[0] = LOWEST[type_]
    logits[0, V // 2] = -LOWEST[type_]
    logits[:, 0] = LOWEST[type_]
    tokens = torch.stack([torch.zeros(3, dtype=torch.int64), torch.full((3,), V // 2)], 1)
    for scale in (0.4, 1e-30, 1e-38):
        run(logits, tokens, type_, scale, min(V, 5))


@pytest.mark.parametrize("V", VOCABULARIES)
def test_nothing_is_lost_below_the_direct_form(V):
    """Scaled maxima of up to 2^24, where exponents are taken by one operation or by two: entropies of k equal logits, ln k, within the bounds."""
    logits = torch.full((25, V), -50.0)
    logits[:, ::max(V // 7, 1)] = 1.0
    logits = logits * torch.tensor([1.37 * 2.0 ** k for k in range(25)])[:, None]
    tokens = torch.zeros(25, 1, dtype=torch.int64)
    lp, entropy, _, _, _ = binding.log_probs_fwd(logits.to(DEV), tokens.to(DEV))
    l64 = logits.double()
    want = ref.log_probs(l64, tokens, 1.0, 0)
    off, h_off = bounds(l64, tokens, 1.0)
    seq.near(lp, want[0].numpy(), off.gather(1, tokens).numpy(), torch.float32, "log probabilities")
    seq.near(entropy, want[1].numpy(), h_off.numpy(), torch.float32, "entropy")
