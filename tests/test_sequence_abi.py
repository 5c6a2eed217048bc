"""Host-side checks of the sequence operators' entry points: what is refused before anything touches the device."""
import ctypes

from paper_1912_05234_amd import binding

EINVAL, EWS = -1, -2
nul, fake, odd = ctypes.c_void_p(None), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)  # never dereferenced


def test_embedding_refusals():
    L = binding.lib()
    fwd = lambda table=fake, tokens=fake, out=fake, N=4, V=5, D=8, type_=0: L.cnn_embedding_fwd(table, tokens, out, N, V, D, type_, 0, 1.0, nul)  # noqa: E731
    for bad in ({"table": nul}, {"tokens": nul}, {"out": nul}, {"table": odd}, {"out": odd}, {"tokens": odd}, {"N": 0}, {"N": 1 << 31},
                {"V": 0}, {"V": 1 << 31}, {"D": 0}, {"D": 65537}, {"type_": 3}, {"type_": -1}):
        assert fwd(**bad) == EINVAL, bad
    q = L.cnn_embedding_bwd_workspace_bytes
    assert q(0, 5, 8, 0) == q(4, 0, 8, 0) == q(4, 5, 0, 0) == q(4, 5, 8, 7) == q(1 << 31, 5, 8, 0) == 0
    need = q(10000, 500, 64, 0)
    assert 0 < need <= 64 << 20
    bwd = lambda d=fake, ws=fake, n=need, N=10000, type_=0: L.cnn_embedding_bwd(d, fake, fake, N, 500, 64, type_, 1, 1.0, ws, n, nul)  # noqa: E731
    assert bwd(n=need - 1) == EWS
    for bad in ({"d": nul}, {"ws": nul}, {"ws": odd}, {"N": -1}, {"type_": 9}):
        assert bwd(**bad) == EINVAL, bad


def test_dropout_refusals():
    L = binding.lib()
    fwd = lambda x=fake, r=nul, y=fake, n=8, t=0, p=0.5, step=nul: L.cnn_dropout_fwd(x, r, y, n, t, p, 1, 2, step, nul)  # noqa: E731
    for bad in ({"x": nul}, {"y": nul}, {"x": odd}, {"y": odd}, {"r": odd}, {"n": 0}, {"n": (1 << 40) + 1}, {"t": 3}, {"p": -0.01}, {"p": 1.01},
                {"p": float("nan")}, {"step": odd}):
        assert fwd(**bad) == EINVAL, bad
    assert L.cnn_dropout_bwd(nul, fake, 8, 0, 0.5, 1, 2, nul, nul) == EINVAL
    assert L.cnn_dropout_bwd(fake, fake, 8, 0, 2.0, 1, 2, nul, nul) == EINVAL
