"""Norms of more bytes than the last cache holds, in rows of whole packs: these go past the caches.  Single rows are the same bits as in small calls, which do not.

The weights' gradients against 64 bits: the products' 60 u as in test_gpu_norm.py, N / 256 rows at most added up one by one by each lane, 8 of a workgroup side by
side, and 32 + 32 of the workgroups' rows."""
import pytest
import torch

import block_reference as ref
import sequence_reference as seq
from paper_1912_05234_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = ref.U
LAST_CACHE = 1 << 28
# rows, groups, width: teams of a wave or less, of 256 and of 1024 lanes, of one pack and of several
SHAPES = [(24001, 32, 64), (24001, 8, 256), (24001, 1, 2048), (9001, 1, 5120), (6007, 1, 8192), (3001, 1, 16384)]
TYPES = [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")]


def filled(*shape, dtype, seed):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


def gradient_of_weights(d_y, v, by, groups):
    """(sums over rows of d_y by n, sums of magnitudes), a thousand rows at a time."""
    total, size = 0.0, 0.0
    for i in range(0, len(v), 1000):
        rows = slice(i, i + 1000)
        terms = d_y[rows].double() * by(rows) * ref.hat(v[rows].double(), groups, float(torch.tensor(1e-5)))[0]
        total, size = total + terms.sum(0), size + terms.abs().sum(0)
    return total.cpu().numpy(), size.cpu().numpy()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_rows_past_the_caches(types, shape):
    (N, G, W), (type_, stream) = shape, (seq.TYPES[t] for t in types)
    D = G * W
    assert 3 * N * D * torch.finfo(type_).bits // 8 >= LAST_CACHE  # two inputs and a result at least, of `type`
    x = filled(N, D + 8, dtype=type_, seed=1)[:, 3:D + 3]  # (whole packs from row to row, whatever the first one's address)
    d, gate, w = filled(N, D, dtype=type_, seed=2), filled(N, D, dtype=type_, seed=3), filled(D, dtype=torch.float32, seed=4)
    r, d_r = filled(N, D, dtype=stream, seed=5), filled(N, D, dtype=stream, seed=6)
    calls = {"add_norm_fwd": (lambda s: binding.add_norm_fwd(x[s], w, r[s], 0.5, 1e-5, G), 2),
             "add_norm_bwd": (lambda s: binding.add_norm_bwd(d[s], r[s], w, d_r[s], 0.5, 1e-5, G), 2),
             "norm_gate_fwd": (lambda s: (binding.norm_gate_fwd(x[s], w, gate[s], r[s], 0.5, 1e-5, G),), 1),
             "norm_gate_bwd": (lambda s: binding.norm_gate_bwd(d_r[s], x[s], w, gate[s], 0.5, 1e-5, G), 2)}
    for name, (call, count) in calls.items():
        got = call(slice(0, N))
        for rows in (slice(0, 40), slice(N // 2, N // 2 + 40), slice(N - 40, N)):
            for i, (g, one) in enumerate(zip(got[:count], call(rows))):
                assert torch.equal(g[rows], one), (name, i, rows)
        if name.endswith("bwd"):
            v, error, by = (r, d, lambda s: 1.0) if name == "add_norm_bwd" else (x, d_r, lambda s: 0.5 * ref.silu(gate[s].double()))
            want, size = gradient_of_weights(error, v, by, G)
            most = 0.0 if name == "add_norm_bwd" else 2 * float(gate.abs().max())
            seq.near(got[2], want, size * (60 + most + N / 256 + 8 + 64) * U, torch.float32, name + " d_weight")
