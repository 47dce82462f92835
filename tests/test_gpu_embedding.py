"""The embedding lookup and its gradient by sorted tokens against a plain implementation in 64 bits, element by element.

Bounds.  Lookup: one fp32 product, then the rounding of the output: 2^-23 and, for bf16, 2^-8 of the value (half a step
each, and one more for the product).  Gradient: the n rows of a token are added in fp32 in a fixed order, every addition off by
at most 2^-24 of a running magnitude that stays below S = sum |dy|; chunks of positions are joined by more of the same additions, so
at most n of them in a chain; then the product with the scale and the rounding: (n + 4) 2^-24 scale S + the
output's half step.  Accumulating adds one addition more."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
F32, BF = torch.float32, torch.bfloat16


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def guarded(shape, dtype):
    """A buffer with a filled margin behind it."""
    n = int(np.prod(shape))
    base = torch.full((n + 512,), 3.0, dtype=dtype, device="cuda")
    return base[:n].view(shape), base[n:]


def workspace(n):
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    return ws[:n], ws[n:]


def some_ids(rng, T, V, kind):
    if kind == "uniform":
        ids = rng.integers(0, V, T)
    elif kind == "text":                                # frequencies as in text
        ids = np.minimum((2.7 * ((V + 2.7) / 2.7) ** rng.random(T) - 2.7).astype(np.int64), V - 1)
    elif kind == "one":                                 # the same token everywhere
        ids = np.full(T, V // 2)
    elif kind == "ends":                                # first and last row only
        ids = np.where(rng.random(T) < 0.5, 0, V - 1)
    else:                                               # half of the positions are padding
        ids = np.where(rng.random(T) < 0.5, -1 - rng.integers(0, 200, T), rng.integers(0, V, T))
    return ids.astype(np.int64)


def grad64(ids, dy, V, scale):
    """(gradient, sum of magnitudes, rows a token has) in 64 bits."""
    out, mag, cnt = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1])), np.zeros(V)
    keep = (ids >= 0) & (ids < V)
    np.add.at(out, ids[keep], dy[keep])
    np.add.at(mag, ids[keep], np.abs(dy[keep]))
    np.add.at(cnt, ids[keep], 1)
    return scale * out, abs(scale) * mag, cnt


def check_grad(T, d, V, dtype, gdtype, idt, kind, scale, accumulate, seed=0):
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(seed)
    ids = some_ids(rng, T, V, kind)
    dy = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(dtype)
    out, margin = guarded((V, d), gdtype)
    base = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)).cuda().to(gdtype)
    out.copy_(base if accumulate else torch.full_like(base, float("nan")))
    ws, ws_margin = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    dev_ids = torch.from_numpy(ids).to(idt).cuda()
    B.embedding_backward(dev_ids, dy, out, ws, scale=scale, accumulate=accumulate)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    assert bool((margin == 3).all()) and bool((ws_margin == 0xA5).all())
    ref, mag, cnt = grad64(ids, f64(dy), V, scale)
    tol = (cnt[:, None] + 4) * U * mag
    got = f64(out)
    if accumulate:
        b = f64(base)
        assert np.array_equal(got[cnt == 0], b[cnt == 0])
        ref = ref + b
        tol = tol + 2 * U * (np.abs(b) + mag)
    else:
        assert not got[cnt == 0].any()
    tol = tol + HALF[gdtype] * (np.abs(ref) + tol)
    assert (np.abs(got - ref) <= tol).all()
    first = out.clone()                                 # the same bits again, on a workspace the first call has used
    out.copy_(base if accumulate else torch.full_like(base, float("nan")))
    B.embedding_backward(dev_ids, dy, out, ws, scale=scale, accumulate=accumulate)
    assert torch.equal(out, first)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [(1, 8, 1), (1, 2048, 32000), (3, 72, 5), (33, 1536, 1001), (300, 64, 100003), (4097, 520, 700)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_lookup(T, d, V, dtype, idt):
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(T)
    ids = some_ids(rng, T, V, "padding")
    ids[0], ids[-1] = V - 1, 0
    table = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)).cuda().to(dtype)
    for scale in (1.0, d ** 0.5, -0.3):
        y, margin = guarded((T, d), dtype)
        y.fill_(float("nan"))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.embedding(torch.from_numpy(ids).to(idt).cuda(), table, y, scale=scale, status=status)
        assert int(status) == 0 and bool((margin == 3).all())
        ref = np.where((ids >= 0)[:, None], f64(table)[np.maximum(ids, 0)] * np.float64(np.float32(scale)), 0.0)
        assert (np.abs(f64(y) - ref) <= (2.0 ** -23 + HALF[dtype]) * np.abs(ref)).all()


# (T, d, V): one position, fewer than a warp, ragged chunks, one chunk over, more than one pass of the sort, wide rows,
# chunks of 16 to 128 positions, vocabularies of one to three digits of the sort
GRADS = [(1, 8, 1), (1, 2048, 32000), (7, 64, 3), (31, 136, 1001), (257, 1536, 1023), (1000, 520, 1024), (4096, 72, 50), (4097, 72, 5000),
         (9001, 264, 100003), (20000, 64, 40), (40000, 40, 70000), (70001, 24, 1500000), (513, 4104, 300)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", GRADS)
@pytest.mark.parametrize("kind", ["uniform", "text", "one", "padding"])
def test_gradient(T, d, V, kind):
    check_grad(T, d, V, BF, F32, torch.int64, kind, 1.0, False, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("gdtype", [BF, F32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_gradient_types(dtype, gdtype, accumulate, idt):
    for T, d, V, kind in [(5, 64, 9, "ends"), (777, 328, 2000, "text"), (3000, 64, 300, "padding")]:
        check_grad(T, d, V, dtype, gdtype, idt, kind, -1.75, accumulate, seed=T)


@pytest.mark.gpu
def test_gradient_is_the_derivative():
    """Of sum(dy * y) with respect to the table, by differences: y is linear in it."""
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(3)
    T, d, V = 40, 16, 12
    ids = torch.from_numpy(some_ids(rng, T, V, "padding")).cuda()
    table, dy = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((V, d), (T, d)))
    out, y = torch.empty(V, d, device="cuda"), torch.empty(T, d, device="cuda")
    ws, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    B.embedding_backward(ids, dy, out, ws, scale=2.0)

    def objective(t):
        B.embedding(ids, t, y, scale=2.0)
        return float((y.double() * dy.double()).sum())
    for v, c in [(0, 0), (5, 3), (11, 15)]:
        up, down = table.clone(), table.clone()
        up[v, c] += 0.5
        down[v, c] -= 0.5
        # differences of sums of T d fp32 products, each rounded to 2^-24 of at most 2 * 4.5 * 5
        assert abs(objective(up) - objective(down) - float(out[v, c])) <= T * d * 2.0 ** -24 * 45 * 2


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 100, 5000])
def test_ids_past_the_table_are_reported_and_left_out(T):
    from paper_2409_12210_b200 import binding as B
    d, V = 64, 50
    rng = np.random.default_rng(T)
    for idt, far in [(torch.int32, 2 ** 31 - 1), (torch.int64, 2 ** 40 + 3), (torch.int64, V)]:
        ids = rng.integers(0, V, T)
        ids[T // 2] = far
        table, dy = torch.randn(V, d, device="cuda"), torch.randn(T, d, device="cuda")
        y, status = torch.full((T, d), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        dev = torch.from_numpy(ids).to(idt).cuda()
        B.embedding(dev, table, y, status=status)
        assert B.check_workspace_status(status) == B.MODSE_ERR_DEVICE_BOUNDS
        assert not bool(y[T // 2].any())
        out = torch.empty(V, d, device="cuda")
        ws, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
        B.embedding_backward(dev, dy, out, ws)
        assert B.check_workspace_status(ws) == B.MODSE_ERR_DEVICE_BOUNDS
        ref, mag, cnt = grad64(ids, f64(dy), V, 1.0)
        assert (np.abs(f64(out) - ref) <= (cnt[:, None] + 4) * U * mag).all()
        B.embedding_backward(dev.clamp(max=V - 1), dy, out, ws)      # the next call starts with a clean word
        assert B.check_workspace_status(ws) == B.MODSE_OK


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_rows():
    from paper_2409_12210_b200 import binding as B
    T, d, V = 300, 64, 20
    rng = np.random.default_rng(8)
    ids = rng.integers(0, V, T)
    dy = rng.standard_normal((T, d)).astype(np.float32)
    ids[10], dy[10, 5], ids[20], dy[20, 6], ids[30], dy[30, :] = 3, np.nan, 4, np.inf, -1, np.nan
    out = torch.empty(V, d, device="cuda")
    ws, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    B.embedding_backward(torch.from_numpy(ids).cuda(), torch.from_numpy(dy).cuda(), out, ws)
    bad = ~np.isfinite(f64(out))
    assert bad[3, 5] and bad[4, 6] and bad.sum() == 2


@pytest.mark.gpu
def test_no_tokens():
    from paper_2409_12210_b200 import binding as B
    out = torch.ones(40, 64, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    empty = torch.empty(0, 64, device="cuda")
    ws, _ = workspace(1024)
    B.embedding_backward(none, empty, out, ws, accumulate=True)
    assert bool((out == 1).all()) and B.check_workspace_status(ws) == B.MODSE_OK
    B.embedding_backward(none, empty, out, ws)
    assert not bool(out.any())
    B.embedding(none, out, empty)


@pytest.mark.gpu
def test_rows_past_32_bits():
    """A table and a gradient of more than 2^31 elements."""
    from paper_2409_12210_b200 import binding as B
    d, V = 2048, 1_100_000
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.zeros(V, d, dtype=BF, device="cuda")
    table[-3:].normal_(generator=g)
    ids = torch.tensor([V - 1, 0, V - 3, V - 1, -1], device="cuda")
    y = torch.empty(5, d, dtype=BF, device="cuda")
    B.embedding(ids, table, y)
    assert torch.equal(y[0], table[-1]) and torch.equal(y[2], table[-3]) and not bool(y[1].any()) and not bool(y[4].any())
    ws, _ = workspace(B.embedding_backward_workspace_bytes(5, d, V))
    table.fill_(1)
    B.embedding_backward(ids, y, table, ws)
    assert torch.equal(table[-3], y[2]) and torch.equal(table[-1].float(), (2 * y[0].float()))
    assert int(torch.count_nonzero(table[:-3])) == 0 and not bool(table[-2].any())


@pytest.mark.gpu
def test_replayed_graph_and_side_stream():
    """A captured call follows what the buffers hold, beside calls on another stream with a workspace of their own."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 1000, 256, 400
    rng = np.random.default_rng(5)
    mk = lambda: torch.from_numpy(some_ids(rng, T, V, "text")).cuda()
    ids, dy, table = mk(), torch.randn(T, d, device="cuda"), torch.randn(V, d, device="cuda")
    y, out = torch.empty(T, d, device="cuda"), torch.empty(V, d, device="cuda")
    ws, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    ws2, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    other, out2 = mk(), torch.empty(V, d, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.embedding(ids, table, y)
        B.embedding_backward(ids, dy, out, ws)
    side = torch.cuda.Stream()
    for _ in range(3):
        ids.copy_(mk())
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            B.embedding_backward(other, dy, out2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(y, table[ids])
        for i, o in ((ids, out), (other, out2)):
            ref, mag, cnt = grad64(i.cpu().numpy(), f64(dy), V, 1.0)
            assert (np.abs(f64(o) - ref) <= (cnt[:, None] + 4) * U * mag).all()


@pytest.mark.gpu
def test_rows_written_by_the_kernel_ahead():
    """Table, ids and dy come from kernels right ahead, again and again, with nothing in between."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 2048, 512, 600
    y, out = torch.empty(T, d, device="cuda"), torch.empty(V, d, device="cuda")
    ws, _ = workspace(B.embedding_backward_workspace_bytes(T, d, V))
    ids, table = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(V, d, device="cuda")
    ramp = torch.arange(T, device="cuda")
    seen = []
    for step in range(30):
        ids.copy_((ramp * (step + 1)) % V)
        table.fill_(step + 1)
        B.embedding(ids, table, y)
        B.embedding_backward(ids, y, out, ws)
        seen.append((torch.bincount(ids, minlength=V), out.clone()))
    for step, (count, o) in enumerate(seen):
        assert torch.equal(o, (count.float() * (step + 1))[:, None].expand(V, d))      # whole numbers below 2^24: exact


def test_refusals_need_no_gpu():
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    lib = B.load()
    p = 0x1000

    def fwd(dtype=B.MODSE_BF16, T=4, d=64, V=10, ids=p, width=8, table=p, y=p, status=None):
        return lib.modse_embedding(dtype, T, d, V, ids, width, table, 1.0, y, status, None)

    def bwd(dtype=B.MODSE_BF16, T=4, d=64, V=10, ids=p, width=8, dy=p, gd=B.MODSE_F32, out=p, ws=p, n=1 << 30):
        return lib.modse_embedding_backward(dtype, T, d, V, ids, width, dy, 1.0, gd, 0, out, ws, n, None)

    bad = [dict(dtype=B.MODSE_E4M3), dict(T=-1), dict(T=2 ** 30 + 1), dict(d=60), dict(d=0), dict(V=0), dict(V=2 ** 30 + 1), dict(width=2),
           dict(ids=None), dict(ids=p + 4)]
    for kw in bad + [dict(table=None), dict(table=p + 8), dict(y=None), dict(y=p + 8), dict(status=p + 2)]:
        assert fwd(**kw) == B.MODSE_ERR_INVALID_ARG, kw
    for kw in bad + [dict(gd=B.MODSE_E4M3), dict(dy=None), dict(dy=p + 8), dict(out=None), dict(out=p + 8), dict(ws=None),
                     dict(ws=p + 16)]:
        assert bwd(**kw) == B.MODSE_ERR_INVALID_ARG, kw
    assert fwd(d=32776) == bwd(d=32776) == B.MODSE_ERR_UNSUPPORTED
    need = B.embedding_backward_workspace_bytes(4, 64, 10)
    assert need > 0 and bwd(n=need - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    assert fwd(T=0) == B.MODSE_OK
    for args in [(-1, 64, 10), (4, 60, 10), (4, 64, 0), (4, 32776, 10)]:
        assert B.embedding_backward_workspace_bytes(*args) == 0
    sizes = [B.embedding_backward_workspace_bytes(T, 64, 10) for T in range(1, 9000, 7)] + \
            [B.embedding_backward_workspace_bytes(T, 64, 10) for T in range(9000, 300000, 511)]
    assert sizes == sorted(sizes)


def test_wrong_tensors_are_refused():
    from paper_2409_12210_b200 import binding as B
    table = torch.zeros(10, 64)
    with pytest.raises(ValueError):
        B.embedding(torch.zeros(3, dtype=torch.int64), table, torch.zeros(3, 64))        # not on a CUDA device
    with pytest.raises(ValueError):
        B.embedding_backward(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 64), table, None)


@pytest.mark.gpu
def test_wrong_tensors_are_refused_on_the_device():
    from paper_2409_12210_b200 import binding as B
    mk = lambda *s, dt=F32: torch.zeros(*s, dtype=dt, device="cuda")
    ids, table, y, ws = mk(3, dt=torch.int64), mk(10, 64), mk(3, 64), mk(1 << 16, dt=torch.uint8)
    for call in (lambda: B.embedding(mk(4, dt=torch.int64), table, y), lambda: B.embedding(ids.cpu(), table, y),
                 lambda: B.embedding(ids, table, mk(3, 64, dt=BF)), lambda: B.embedding(ids, table.T, y),
                 lambda: B.embedding(ids, table[:, ::2], mk(3, 32)), lambda: B.embedding_backward(ids, y, mk(10, 72), ws),
                 lambda: B.embedding_backward(ids, y, table, ws.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.embedding(ids.short(), table, y), lambda: B.embedding(ids, table.half(), y.half()),
                 lambda: B.embedding_backward(ids, y, table.double(), ws)):
        with pytest.raises(TypeError):
            call()
