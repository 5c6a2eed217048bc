"""Host-side checks of the entry points around a block: what is refused before anything touches the device, and the workspaces."""
import ctypes

from paper_1912_05234_amd import binding

EINVAL, EWS = -1, -2
nul, fake, odd = ctypes.c_void_p(None), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)  # never dereferenced


def rows(data=0x1002, row=77):
    return binding.Rows(data, row)


def norm(rows=100, groups=3, width=32, type_=1, stream=1, scale=0.5, eps=1e-6):
    return binding.NormShape(rows, groups, width, type_, stream, scale, eps)


BAD_NORMS = [{"rows": 0}, {"rows": 1 << 31}, {"groups": 0}, {"width": 0}, {"width": 16385}, {"groups": 1 << 16, "width": 17}, {"type_": 3}, {"type_": -1},
             {"type_": 1, "stream": 2}, {"type_": 0, "stream": 1}, {"stream": 5}, {"eps": 0.0}, {"eps": -1.0}, {"eps": float("nan")},
             {"eps": float("inf")}, {"scale": float("nan")}, {"scale": float("inf")}]
BAD_ROWS = [rows(data=0), rows(data=0x1001), rows(row=-1)]


def test_norm_refusals():
    L = binding.lib()
    add = lambda s=norm(), x=rows(), res=rows(), w=fake, y=fake, r=fake: L.cnn_add_norm_fwd(s, x, res, w, y, r, nul)  # noqa: E731
    addb = lambda s=norm(), d=rows(), r=rows(), dr=rows(), w=fake, dx=fake, res=fake, dw=fake, ws=fake, n=1 << 40: L.cnn_add_norm_bwd(  # noqa: E731
        s, d, r, dr, w, dx, res, dw, ws, n, nul)
    gate = lambda s=norm(), x=rows(), g=rows(), res=rows(), w=fake, y=fake: L.cnn_norm_gate_fwd(s, x, g, res, w, y, nul)  # noqa: E731
    gateb = lambda s=norm(), d=rows(), x=rows(), g=rows(), w=fake, dx=fake, dg=fake, dw=fake, ws=fake, n=1 << 40: L.cnn_norm_gate_bwd(  # noqa: E731
        s, d, x, g, w, dx, dg, dw, ws, n, nul)
    assert add(s=None) == addb(s=None) == gate(s=None) == gateb(s=None) == EINVAL
    assert add(x=None) == addb(d=None) == addb(r=None) == gate(x=None) == gateb(d=None) == gateb(x=None) == EINVAL
    for bad in BAD_NORMS:
        s = norm(**bad)
        assert add(s=s) == addb(s=s) == gate(s=s) == gateb(s=s) == EINVAL and L.cnn_norm_bwd_workspace_bytes(s) == 0, bad
    for r in BAD_ROWS:
        assert add(x=r) == add(res=r) == addb(d=r) == addb(r=r) == addb(dr=r) == gate(x=r) == gate(g=r) == gate(res=r) == gateb(d=r) == gateb(x=r) == gateb(g=r) == EINVAL
    for p in (nul, odd):
        assert add(w=p) == add(y=p) == addb(w=p) == addb(res=p) == addb(dw=p) == gate(w=p) == gate(y=p) == gateb(w=p) == gateb(dx=p) == gateb(dw=p) == gateb(dg=p) == EINVAL
    assert add(r=odd) == addb(dx=odd) == addb(ws=odd) == EINVAL
    # without a residual there is nothing to scale, to return or of another type
    assert add(res=None) == add(res=None, r=nul) == add(s=norm(scale=1.0), res=None) == add(s=norm(scale=1.0, stream=0), res=None, r=nul) == EINVAL
    assert gateb(g=None) == EINVAL  # a gate's gradient without a gate
    need = L.cnn_norm_bwd_workspace_bytes(norm())
    assert need and addb(n=need - 1) == gateb(n=need - 1) == addb(ws=nul) == gateb(ws=nul) == EWS


def test_norm_workspaces():
    """A row of partial sums for every workgroup along the rows; none where there is one."""
    q = binding.lib().cnn_norm_bwd_workspace_bytes
    assert q(norm(rows=1)) == 0 and q(norm(rows=2, groups=1)) == 0 and q(None) == 0
    assert q(norm(rows=1 << 20, groups=1, width=64)) == 1024 * 64 * 4
    assert q(norm(rows=1 << 20, groups=1, width=4096)) == 1024 * 4096 * 4
    assert q(norm(rows=1 << 20, groups=64, width=16384)) == 4 * 64 * 16384 * 4


def conv(B=3, T=50, D=20, K=4, type_=1, silu=1):
    return binding.CausalConvShape(B, T, D, K, type_, silu)


def tokens(data=0x1002, batch=1000, token=20):
    return binding.Tokens(data, batch, token)


BAD_CONVS = [{"B": 0}, {"T": 0}, {"D": 0}, {"D": (1 << 20) + 1}, {"K": 1}, {"K": 9}, {"type_": 3}, {"type_": -1}, {"B": 1 << 16, "T": 1 << 15}]
BAD_TOKENS = [tokens(data=0), tokens(data=0x1001), tokens(batch=-1), tokens(token=-1)]


def test_conv_refusals():
    L = binding.lib()
    fwd = lambda s=conv(), x=tokens(), w=fake, b=fake, n=fake, i=fake, y=fake, f=fake: L.cnn_causal_conv_fwd(s, x, w, b, n, i, y, f, nul)  # noqa: E731
    bwd = lambda s=conv(), x=tokens(), d=tokens(), w=fake, b=fake, n=fake, i=fake, f=fake, dx=fake, dw=fake, db=fake, di=fake, ws=fake, size=1 << 40: (  # noqa: E731
        L.cnn_causal_conv_bwd(s, x, d, w, b, n, i, f, dx, dw, db, di, ws, size, nul))
    step = lambda s=conv(T=1), x=tokens(), w=fake, b=fake, st=fake, pool=3, slots=nul, y=fake: L.cnn_causal_conv_step(s, x, w, b, st, pool, slots, y, nul)  # noqa: E731
    assert fwd(s=None) == fwd(x=None) == bwd(s=None) == bwd(x=None) == bwd(d=None) == step(s=None) == step(x=None) == EINVAL
    for bad in BAD_CONVS:
        assert fwd(s=conv(**bad)) == bwd(s=conv(**bad)) == EINVAL and L.cnn_causal_conv_bwd_workspace_bytes(conv(**bad)) == 0, bad
        if "T" not in bad:
            assert step(s=conv(**{"T": 1, **bad})) == EINVAL, bad
    for x in BAD_TOKENS:
        assert fwd(x=x) == bwd(x=x) == bwd(d=x) == step(x=x) == EINVAL
    for p in (nul, odd):
        assert fwd(w=p) == fwd(y=p) == bwd(w=p) == bwd(dx=p) == bwd(dw=p) == bwd(ws=p) == step(w=p) == step(st=p) == step(y=p) == EINVAL
    assert fwd(b=odd) == fwd(n=odd) == fwd(i=odd) == fwd(f=odd) == bwd(b=odd) == bwd(n=odd) == bwd(i=odd) == bwd(f=odd) == bwd(db=odd) == bwd(di=odd) == EINVAL
    assert step(b=odd) == step(slots=odd) == step(pool=0) == step(pool=2) == step(s=conv(T=2)) == step(pool=(1 << 30) + 1) == EINVAL
    need = L.cnn_causal_conv_bwd_workspace_bytes(conv())
    assert need % (20 * 5 * 4) == 0 and 0 < need and bwd(size=need - 1) == EWS and L.cnn_causal_conv_bwd_workspace_bytes(None) == 0


def scan(B=3, T=50, D=20, N=16, G=2, type_=1, soft=1):
    return binding.SelectiveScanShape(B, T, D, N, G, type_, soft)


def heads(data=0x1002, batch=1600, token=32, head=16):
    return binding.Heads(data, batch, token, head)


BAD_SCANS = [{"B": 0}, {"T": 0}, {"D": 0}, {"N": 0}, {"N": 129}, {"G": 0}, {"G": 3}, {"type_": 3}, {"type_": -1}, {"B": 1 << 20, "T": 1, "D": 32}, {"B": 1 << 16, "T": 1 << 15}]
BAD_HEADS = [heads(data=0), heads(data=0x1001), heads(batch=-1), heads(token=-1), heads(head=-1)]


def test_scan_refusals():
    L = binding.lib()
    fwd = lambda s=scan(), x=tokens(), dt=tokens(), a=fake, b=heads(), c=heads(), k=fake, z=fake, n=fake, i=fake, y=fake, f=fake, ws=fake, size=1 << 40: (  # noqa: E731
        L.cnn_selective_scan_fwd(s, x, dt, a, b, c, k, z, n, i, y, f, ws, size, nul))
    bwd = lambda s=scan(), x=tokens(), dt=tokens(), a=fake, b=heads(), c=heads(), d=tokens(), k=fake, z=fake, n=fake, i=fake, f=fake, o=(fake,) * 8, ws=fake, size=1 << 40: (  # noqa: E731
        L.cnn_selective_scan_bwd(s, x, dt, a, b, c, d, k, z, n, i, f, *o, ws, size, nul))
    step = lambda s=scan(T=1), x=tokens(), dt=tokens(), a=fake, b=heads(), c=heads(), k=fake, z=fake, st=fake, pool=3, slots=nul, y=fake: (  # noqa: E731
        L.cnn_selective_scan_step(s, x, dt, a, b, c, k, z, st, pool, slots, y, nul))
    assert fwd(s=None) == bwd(s=None) == step(s=None) == EINVAL
    for bad in BAD_SCANS:
        s = scan(**bad)
        assert fwd(s=s) == bwd(s=s) == EINVAL and L.cnn_selective_scan_fwd_workspace_bytes(s) == L.cnn_selective_scan_bwd_workspace_bytes(s) == 0, bad
        if bad.get("T", 1) == 1:
            assert step(s=scan(**{"T": 1, **bad})) == EINVAL, bad
    for x in [None, tokens(token=(1 << 26) + 1)] + BAD_TOKENS:
        assert fwd(x=x) == fwd(dt=x) == bwd(x=x) == bwd(dt=x) == bwd(d=x) == step(x=x) == step(dt=x) == EINVAL
    for h in [None, heads(token=(1 << 26) + 1)] + BAD_HEADS:
        assert fwd(b=h) == fwd(c=h) == bwd(b=h) == bwd(c=h) == step(b=h) == step(c=h) == EINVAL
    for p in (nul, odd):
        assert fwd(a=p) == fwd(y=p) == bwd(a=p) == bwd(ws=p) == step(a=p) == step(st=p) == step(y=p) == EINVAL
        for i in range(5):
            assert bwd(o=(fake,) * i + (p,) + (fake,) * (7 - i)) == EINVAL, i
    for name in ("k", "z", "n", "i"):
        assert fwd(**{name: odd}) == bwd(**{name: odd}) == EINVAL
    assert fwd(f=odd) == fwd(ws=odd) == bwd(f=odd) == bwd(o=(fake,) * 5 + (odd, fake, fake)) == bwd(o=(fake,) * 7 + (odd,)) == step(k=odd) == step(z=odd) == EINVAL
    assert step(slots=odd) == step(pool=0) == step(pool=2) == step(s=scan(T=2)) == step(pool=(1 << 30) + 1) == EINVAL
    need = L.cnn_selective_scan_bwd_workspace_bytes(scan())
    assert need and bwd(size=need - 1) == EWS
    long = scan(B=1, T=8192)
    need = L.cnn_selective_scan_fwd_workspace_bytes(long)
    assert need and fwd(s=long, size=need - 1) == fwd(s=long, ws=nul) == EWS


def test_scan_workspaces():
    """Forward none where the channels fill the chip, or a sequence is short; backward always, for the partial sums."""
    L = binding.lib()
    fwd, bwd = L.cnn_selective_scan_fwd_workspace_bytes, L.cnn_selective_scan_bwd_workspace_bytes
    assert fwd(scan(T=64)) == 0 and fwd(scan(B=128, T=10000, D=2048)) == 0 and fwd(None) == bwd(None) == 0
    assert bwd(scan(T=1)) > 0 and bwd(scan(T=8192)) > 128 * 3 * 20 * 16 * 4 * 2


def logp(rows=100, vocab=1000, given=2, top=5, type_=1, wide=1, scale=1.0):
    return binding.LogProbsShape(rows, vocab, given, top, type_, wide, scale)


BAD_LOGP = [{"rows": 0}, {"rows": 1 << 31}, {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"given": 0}, {"given": 257}, {"top": -1}, {"top": 65}, {"vocab": 4}, {"type_": 3},
            {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}]


def test_log_probs_refusals():
    L = binding.lib()
    fwd = lambda s=logp(), x=rows(), t=fake, lp=fake, h=fake, st=fake, tl=fake, tt=fake, ws=fake, n=1 << 40: L.cnn_log_probs_fwd(  # noqa: E731
        s, x, t, lp, h, st, tl, tt, ws, n, nul)
    bwd = lambda s=logp(), x=rows(), t=fake, st=fake, d=fake, dh=fake, o=fake: L.cnn_log_probs_bwd(s, x, t, st, d, dh, o, nul)  # noqa: E731
    assert fwd(s=None) == fwd(x=None) == bwd(s=None) == bwd(x=None) == EINVAL
    for bad in BAD_LOGP:
        assert fwd(s=logp(**bad)) == bwd(s=logp(**bad)) == EINVAL and L.cnn_log_probs_fwd_workspace_bytes(logp(**bad)) == 0, bad
    for r in BAD_ROWS:
        assert fwd(x=r) == bwd(x=r) == EINVAL
    for p in (nul, odd):
        assert fwd(t=p) == fwd(lp=p) == fwd(tl=p) == fwd(tt=p) == bwd(t=p) == bwd(o=p) == EINVAL  # (tokens of eight bytes)
    half = ctypes.c_void_p(0x1002)
    assert bwd(st=nul) == bwd(d=nul) == bwd(st=half) == bwd(d=half) == bwd(dh=half) == fwd(s=logp(wide=0), t=half) == EINVAL
    assert fwd(h=odd) == fwd(st=odd) == fwd(ws=odd) == EINVAL
    long = logp(vocab=100000)
    need = L.cnn_log_probs_fwd_workspace_bytes(long)
    assert need and fwd(s=long, n=need - 1) == fwd(s=long, ws=nul) == EWS


def test_log_probs_workspaces():
    """None for rows that a workgroup holds; sums and keys of the parts of longer ones."""
    q = binding.lib().cnn_log_probs_fwd_workspace_bytes
    assert q(logp(vocab=65536)) == q(logp(vocab=32768, type_=0)) == q(logp(rows=1000, vocab=16384, type_=0)) == 0 and q(None) == 0
    assert q(logp(rows=1, vocab=65537, top=0)) >= 2 * 12 and q(logp(rows=1, vocab=32769, top=0, type_=0)) >= 2 * 12
    assert q(logp(rows=1, vocab=1 << 24, top=64)) >= 512 * (12 + 64 * 8)
