"""What the compiler made of the kernels around a block (host-only, no GPU needed)."""
import re

from test_compiled_kernels import KERNELS

BLOCK = {n: k for n, k in KERNELS.items() if re.search("norm_forward|norm_backward|conv_tokens|conv_one_token|selective_|logp_|fold_kernel", n)}


def test_every_kernel_is_there():
    count = lambda what: sum(what in n for n in BLOCK)  # noqa: E731
    assert count("norm_forward") >= 60 and count("norm_backward") >= 60 and count("conv_tokens_kernel") == count("conv_tokens_backward") == 21
    assert count("logp_part") >= 50 and count("logp_backward") >= 15 and count("selective_gradient") == 18 and count("selective_tokens") >= 50


def test_scratch_memory_is_for_the_widest_groups_and_a_few_scans():
    """Groups of more than 4096 elements, whose sixteen waves share a compute unit's registers, and gradients of the scan: a few registers."""
    spilling = {n: k[".private_segment_fixed_size"] for n, k in BLOCK.items() if k[".private_segment_fixed_size"]}
    wide = {n: b for n, b in spilling.items() if "norm_" in n}
    assert set(spilling) - set(wide) <= {n for n in BLOCK if "selective_gradient" in n}, spilling
    assert all(KERNELS[n][".max_flat_workgroup_size"] == 1024 and b <= 512 for n, b in wide.items()), wide
    assert all(b <= 96 for n, b in spilling.items() if n not in wide), spilling
