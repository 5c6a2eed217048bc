"""What the compiler made of the kernels of the operators on sequences (host-only, no GPU needed)."""
import re

from test_compiled_kernels import KERNELS, REGISTERS

SEQUENCE = sorted(n for n in KERNELS if re.search("scan_kernel|carry_kernel|share_kernel|step_kernel|embed_|sort_|dropout_kernel", n) and "train" not in n)

# Forms of floats of 96 and 128 columns that two waves to a SIMD leave too few registers: bytes of scratch per lane.
SPILLING = {"cnn::linear::scan_kernel<float, 128, 2, false, false, true>": 200, "cnn::linear::scan_kernel<float, 128, 2, true, false, true>": 100,
            "cnn::linear::scan_kernel<float, 128, 3, false, false, true>": 50, "cnn::linear::scan_kernel<float, 128, 3, true, false, true>": 50,
            "cnn::linear::scan_kernel<float, 96, 2, false, false, true>": 50, "cnn::linear::scan_kernel<float, 96, 2, true, false, true>": 50}


def test_every_kernel_is_there():
    assert sum("scan_kernel" in n for n in SEQUENCE) >= 15 * 2 * (2 + 3 + 3) and len(SEQUENCE) > 260


def test_scratch_memory_is_for_the_widest_floats_alone():
    more = {n: KERNELS[n][".private_segment_fixed_size"] for n in SEQUENCE if KERNELS[n][".private_segment_fixed_size"] > SPILLING.get(n, 0)}
    assert not more, more


def test_two_waves_of_a_scan_fit_a_simd():
    """What the plan of the segments counts on: widths of 256 have a SIMD to themselves."""
    for name in SEQUENCE:
        if "scan_kernel" in name:
            waves = 1 if re.search(r"<float, 256|Li256E", name) else 2
            assert KERNELS[name][".vgpr_count"] <= REGISTERS // waves, name
