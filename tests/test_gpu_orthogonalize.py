"""Orthogonalised updates (modse_orthogonalize) against the iteration in 64 bits.

Bound.  The documented roundings are: factors of the products in fp16 (2^-11 of a value; X's as its leading half), X carried in 22 bits, fp32
accumulation, one rounding of the result to bf16 (2^-8).  What the first two do to the result depends on the spectrum, so
the test runs the iteration in 64 bits with exactly these roundings put in by hand; its distance E from the iteration
without them is the size of the error they cause.  A kernel that accumulates in another order meets other instances of
the same roundings, so its own error before the last rounding is held to 2 E in norm, and an element to 10 times the
root mean square of that, each plus the last rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

A, B_, C = MUON = (3.4445, -4.7750, 2.0315)
U32 = 2.0 ** -23


def iterate(G, steps=5, k=MUON, eps=1e-7, rounded=False):
    def fp16(t, s):
        return (t * s).half().double() / s if rounded else t

    X = G.double()
    X = X / (X.norm() + eps)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    if rounded:
        hi = fp16(X, 4096.0)
        X = hi + fp16(X - hi, 4096.0)
    for i in range(steps):
        Xh = fp16(X, 4096.0)
        M = fp16(Xh @ Xh.T, 1024.0)
        # the step as it is computed: (a I + b A + c A^2) in fp16 times the leading half of X, plus a times the rest
        P = fp16(k[0] * torch.eye(len(M), dtype=M.dtype, device=M.device) + k[1] * M + k[2] * (M @ M), 1024.0)
        X = P @ Xh + k[0] * (X - Xh)
        if rounded and i + 1 < steps:
            hi = fp16(X, 4096.0)
            X = hi + fp16(X - hi, 4096.0)
    return X.T if tall else X


def check(out, G, scale=1.0, **kw):
    ref, emu = iterate(G, **kw) * scale, iterate(G, rounded=True, **kw) * scale
    long = max(G.shape)
    # the fp32 sums: at most `long` additions a product, three products a step, amplified like the other errors (8 covers
    # the worst slope of the last steps): far below E except where E happens to vanish (a 1 x 1 matrix, powers of two)
    err = 2 * (emu - ref).norm() + 8 * 3 * 5 * min(long, 64) * U32 * ref.norm()
    got = out.double()
    assert float((got - ref).norm()) <= float(err + 2.0 ** -8 * ref.norm())
    rms = err / max(1, ref.numel()) ** 0.5
    bad = (got - ref).abs() > 10 * rms + 2.0 ** -8 * ref.abs() * 1.01
    assert not bool(bad.any()), (int(bad.sum()), float((got - ref).abs().max()), float(rms))


def gaussian(r, c, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(r, c, generator=g) * 0.02).to(dtype).cuda()


def low_rank(r, c, rank, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(r, rank, generator=g) @ torch.randn(rank, c, generator=g) * 0.01).to(dtype).cuda()


def run(grads, **kw):
    from paper_2409_12210_b200 import binding as B
    outs = [torch.full(g.shape, 7.0, dtype=torch.bfloat16, device="cuda") for g in grads]
    n = B.orthogonalize_workspace_bytes([g.shape for g in grads])
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    B.orthogonalize(grads, outs, ws[:n], **kw)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    assert bool((ws[n:] == 0xA5).all())
    return outs


SHAPES = [(1, 1), (1, 77), (77, 1), (8, 8), (9, 200), (200, 9), (64, 96), (160, 64), (130, 130), (257, 300), (300, 257),
          (512, 520), (1000, 264), (256, 4099), (640, 2048), (2816, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_one_matrix(shape, dtype):
    G = gaussian(*shape, seed=3, dtype=dtype)
    out, = run([G])
    check(out, G)
    again, = run([G])
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,rank", [((256, 700), 4), ((700, 256), 32), ((512, 512), 200), ((96, 64), 1)])
def test_rank_deficient(shape, rank):
    """What the rank leaves empty stays empty: noise there would be amplified by a^5."""
    G = low_rank(*shape, rank, seed=4)
    out, = run([G])
    check(out, G)


@pytest.mark.gpu
def test_decaying_spectrum_and_singular_values():
    g = torch.Generator().manual_seed(5)
    u, _, v = torch.linalg.svd(torch.randn(300, 500, generator=g, dtype=torch.float64), full_matrices=False)
    G = ((u * torch.logspace(0, -4, 300, dtype=torch.float64)) @ v).float().cuda()
    out, = run([G])
    check(out, G)
    full = gaussian(200, 600, 6)
    out, = run([full])
    s = torch.linalg.svdvals(out.double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25          # where Muon's polynomial leaves them


@pytest.mark.gpu
def test_a_set_of_diverse_matrices_with_scales():
    """More matrices than one launch holds, wide and tall ones mixed; every one as if it were alone in its group."""
    shapes = [(96, 64), (64, 160), (257, 40), (1, 5), (128, 128), (300, 520), (33, 700)] * 3
    grads = [gaussian(r, c, 10 + i, torch.float32) for i, (r, c) in enumerate(shapes)]
    scales = [0.25 + 0.1 * i for i in range(len(shapes))]
    for out, G, s in zip(run(grads, scales=scales), grads, scales):
        check(out, G, scale=float(np.float32(s)))


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 4, 5])
@pytest.mark.parametrize("shape", [(2400, 64), (100, 2900), (127, 3840), (5376, 112), (128, 3841), (9, 20001)])
def test_long_thin_matrices(shape, steps):
    """Clusters of sixteen blocks, with two copies of X and in place, at the ends of what they hold and past it."""
    G = gaussian(*shape, seed=12, dtype=torch.float32)
    out, = run([G], steps=steps)
    check(out, G, steps=steps)
    again, = run([G], steps=steps)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("sets", [1, 6])
def test_a_set_of_long_and_short_thin_matrices(sets):
    grads = [gaussian(r, c, 20 + i) for i, (r, c) in enumerate([(100, 4000), (3, 3), (1800, 75), (16, 500), (90, 90), (3500, 120)] * sets)]
    for out, G in zip(run(grads), grads):
        check(out, G)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 8, 13])
def test_column_blocks(dtype, offset):
    """Gradients and updates as column blocks of wider matrices, aligned or not; the columns beside them stay."""
    from paper_2409_12210_b200 import binding as B
    wide = torch.randn(70, 401, device="cuda").to(dtype)
    target = torch.full((70, 333), 7.0, dtype=torch.bfloat16, device="cuda")
    g, u = wide[:, offset:offset + 200], target[:, offset:offset + 200]
    ws = torch.empty(B.orthogonalize_workspace_bytes([(70, 200)]), dtype=torch.uint8, device="cuda")
    B.orthogonalize([g], [u], ws)
    check(u, g)
    assert bool((target[:, :offset] == 7).all()) and bool((target[:, offset + 200:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1100, 1104])
def test_column_blocks_of_every_alignment_in_one_launch(cols, dtype):
    """Grouped products with updates as column blocks of wider matrices: 1100 columns end inside a 16-byte piece, and the
    columns beside a block stay whatever the alignment of its rows; of 1104 columns the aligned blocks leave by TMA and the
    others by plain stores, so that a warp's two staging buffers pass from one kind to the other.  Gradients as blocks of
    wider matrices too, aligned and not; 240 tiles, so that every CTA pair has several."""
    from paper_2409_12210_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(17)
    places = [0, 1, 8, 13, 0, 3, 16, 8, 2, 0, 24, 5, 0, 7, 8, 11]
    wide = [torch.randn(600, 1136, generator=g, device="cuda").to(dtype) * 0.02 for _ in places]
    targets = [torch.full((600, 1128 + (i % 3)), 7.0, dtype=torch.bfloat16, device="cuda") for i in range(len(places))]
    grads = [w[:, (5 * o) % 32:(5 * o) % 32 + cols] for w, o in zip(wide, places)]
    ups = [t[:, o:o + cols] for t, o in zip(targets, places)]
    assert {t.data_ptr() % 16 == 0 and t.stride(0) % 8 == 0 for t in ups} == {True, False}
    ws = torch.empty(B.orthogonalize_workspace_bytes([(600, cols)] * 16), dtype=torch.uint8, device="cuda")
    B.orthogonalize(grads, ups, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    for u, m, t, o in zip(ups, grads, targets, places):
        check(u, m)
        assert bool((t[:, :o] == 7).all()) and bool((t[:, o + cols:] == 7).all())
    first = [u.clone() for u in ups]
    B.orthogonalize(grads, ups, ws)
    assert all(torch.equal(a, b) for a, b in zip(first, ups))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1300, 2100), (2203, 2100), (2100, 2203), (2900, 2904)])
def test_tiles_cut_along_the_contraction(shape):
    """On 74 CTA pairs: 36 narrow tiles of X X^T in two pieces each; the last 7 tiles of the step, wide and tall, written by
    plain stores into a column block; the last 4 of 78 symmetric tiles of X X^T and of the polynomial."""
    from paper_2409_12210_b200 import binding as B
    G = gaussian(*shape, seed=18)
    target = torch.full((shape[0], shape[1] + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    out = target[:, 3:3 + shape[1]]
    n = B.orthogonalize_workspace_bytes([shape])
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    B.orthogonalize([G], [out], ws[:n])
    assert B.check_workspace_status(ws) == B.MODSE_OK and bool((ws[n:] == 0xA5).all())
    check(out, G)
    assert bool((target[:, :3] == 7).all()) and bool((target[:, 3 + shape[1]:] == 7).all())
    first = out.clone()
    B.orthogonalize([G], [out], ws[:n])
    assert torch.equal(first, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,sizes", [(256, (128, 384, 192, 320)), (64, (96, 160, 112, 144)), (520, (272, 304, 144, 432))])
def test_updates_of_a_layer(d, sizes, dtype):
    """The expert matrices of a layer against the iteration in 64 bits: rows of the gate and up gradients, column blocks of
    the down gradients, a scale a matrix; grouped products, the one-kernel form, and widths above and below the d_model."""
    from paper_2409_12210_b200 import binding as B
    layer = B.ModseLayer(d, list(sizes), 2)
    S = sum(sizes)
    grads = [gaussian(S, d, 21, dtype), gaussian(S, d, 22, dtype), gaussian(d, S, 23, dtype)]
    ups = [torch.full(g.shape, 7.0, dtype=torch.bfloat16, device="cuda") for g in grads]
    n = layer.orthogonalize_workspace_bytes()
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = [[0.5 + 0.25 * e, 1.0, 2.0 - 0.25 * e] for e in range(len(sizes))]
    layer.orthogonalize_wgrads(*grads, *ups, ws[:n], scales=scales)
    assert B.check_workspace_status(ws) == B.MODSE_OK and bool((ws[n:] == 0xA5).all())
    off = 0
    for e, h in enumerate(sizes):
        rows, cols = slice(off, off + h), (slice(None), slice(off, off + h))
        for j, at in enumerate((rows, rows, cols)):
            check(ups[j][at], grads[j][at], scale=scales[e][j])
        off += h
    layer.destroy()


@pytest.mark.gpu
@pytest.mark.parametrize("steps,k", [(1, MUON), (8, MUON), (12, (1.5, -0.5, 0.0)), (3, (1.875, -1.25, 0.375))])
def test_other_coefficients(steps, k):
    G = gaussian(120, 200, 7, torch.float32)
    out, = run([G], steps=steps, coefficients=k)
    check(out, G, steps=steps, k=k)


@pytest.mark.gpu
def test_zero_tiny_huge_and_nan():
    z = torch.zeros(40, 64, device="cuda")
    tiny, huge = gaussian(40, 64, 8, torch.float32) * 1e-30, gaussian(40, 64, 8, torch.float32) * 1e25
    bad = gaussian(40, 64, 9, torch.float32)
    bad[3, 5] = float("nan")
    outs = run([z, tiny, huge, bad])
    assert bool((outs[0] == 0).all())
    assert bool(torch.isnan(outs[3]).all())
    check(outs[2], huge)
    assert float(outs[1].abs().max()) < 1e-18                       # eps swamps a norm of 1e-30
    out, = run([tiny], eps=0.0)
    check(out, tiny, eps=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(40, 64), (200, 300)])
def test_norms_and_eps_at_the_ends_of_fp32(shape):
    """One kernel and grouped products: zeros with an eps below the normal range, matrices of subnormal numbers, and sums of
    squares far past fp32."""
    zeros = torch.zeros(*shape, device="cuda")
    for eps in (1e-36, 1e-38, 1e-44):
        out, = run([zeros], eps=eps)
        assert bool((out == 0).all())
    tiny = gaussian(*shape, 8, torch.float32) * 1e-37
    assert 0 < float(tiny.abs().max()) < 2.0 ** -126 * 1.5
    huge = gaussian(*shape, 9, torch.float32).sign() * 3e38
    for G in (tiny, huge):
        out, = run([G], eps=0.0)
        check(out, G, eps=0.0)


@pytest.mark.gpu
def test_one_row_with_the_longest_row_distance():
    """A single row's distance to the next is never used; grouped products (65536 columns do not fit the one-kernel form)."""
    import ctypes

    from paper_2409_12210_b200 import binding as B
    G, out = gaussian(1, 65536, 14), torch.full((1, 65536), 7.0, dtype=torch.bfloat16, device="cuda")
    far = (1 << 40) - 8
    arr = (B._Matrix * 1)(B._Matrix(G.data_ptr(), out.data_ptr(), far, far, 1, 65536, 1.0))
    n = B.load().modse_orthogonalize_workspace_bytes(1, arr)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    st = B.load().modse_orthogonalize(B.MODSE_BF16, 1, arr, 5, (ctypes.c_float * 3)(*MUON), 1e-7, ws.data_ptr(), n,
                                      torch.cuda.current_stream().cuda_stream)
    assert st == B.MODSE_OK and B.check_workspace_status(ws) == B.MODSE_OK
    check(out, G)


@pytest.mark.gpu
def test_replay_in_a_graph():
    from paper_2409_12210_b200 import binding as B
    G = gaussian(300, 500, 11)
    ref, = run([G])
    buf, out = torch.zeros_like(G), torch.empty_like(ref)
    ws = torch.empty(B.orthogonalize_workspace_bytes([(300, 500)]), dtype=torch.uint8, device="cuda")
    B.orthogonalize([G], [out], ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.orthogonalize([buf], [out], ws)
    out.zero_()
    buf.copy_(G)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


@pytest.mark.gpu
def test_binding_refusals():
    from paper_2409_12210_b200 import binding as B
    G, out = gaussian(16, 24, 0), torch.empty(16, 24, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.orthogonalize_workspace_bytes([(16, 24)]), dtype=torch.uint8, device="cuda")
    for bad in [([G.t()], [out.t()]), ([G], [out.float()]), ([G], [out[:, :8]]), ([G, G.float()], [out, out]), ([G], []),
                ([G.cpu()], [out.cpu()])]:
        with pytest.raises(ValueError):
            B.orthogonalize(*bad, ws)
    with pytest.raises(B.ModseError):
        B.orthogonalize([G], [out], ws[:256])
    with pytest.raises(B.ModseError):
        B.orthogonalize([G], [out], ws, coefficients=(9.0, 0.0, 0.0))
    B.orthogonalize([], [], ws)


def test_refusals_need_no_gpu():
    import ctypes

    from paper_2409_12210_b200 import binding as B
    from paper_2409_12210_b200 import build
    build.build()
    lib = B.load()
    p = 0x10000
    inv = B.MODSE_ERR_INVALID_ARG
    need = B.orthogonalize_workspace_bytes([(16, 24)])
    assert need > 0 and need % 256 == 0
    assert B.orthogonalize_workspace_bytes([]) > 0
    for shape in [(0, 4), (4, 0), (-1, 4), (1 << 21, 4), (1 << 18, 1 << 18)]:
        assert B.orthogonalize_workspace_bytes([shape]) == 0
    # a set in groups: the workspace is the largest group's, not the sum
    assert B.orthogonalize_workspace_bytes([(16, 24)] * 64) == B.orthogonalize_workspace_bytes([(16, 24)] * 16)

    def call(dtype=B.MODSE_F32, n=1, steps=5, k=MUON, eps=1e-7, ws=p, size=None, grad=p, update=p, ldg=24, ldu=24, rows=16,
             cols=24, scale=1.0, null=False):
        arr = (B._Matrix * 1)(B._Matrix(grad, update, ldg, ldu, rows, cols, scale))
        kk = None if k is None else (ctypes.c_float * 3)(*k)
        return lib.modse_orthogonalize(dtype, n, None if null else arr, steps, kk, eps, ws, need if size is None else size, None)

    assert call(n=0) == B.MODSE_OK
    assert call(size=need - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    nan = float("nan")
    for bad in [dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(null=True), dict(steps=0), dict(steps=65), dict(k=None),
                dict(k=(nan, 0, 0)), dict(eps=-1.0), dict(eps=nan), dict(ws=None), dict(ws=p + 128), dict(grad=None),
                dict(update=None), dict(grad=p + 2), dict(update=p + 1), dict(ldg=23), dict(ldu=23), dict(rows=0),
                dict(cols=0), dict(scale=nan)]:
        assert call(**bad) == inv, bad
    for k in [(8.0, 0.0, 0.0), (3.0, 3.0, 3.0), (1.0, 100.0, -100.0)]:
        assert call(k=k) == B.MODSE_ERR_UNSUPPORTED, k
    layer = B.ModseLayer(64, [96, 160, 112, 144], 2)
    full = layer.orthogonalize_workspace_bytes()
    assert full > 0 and lib.modse_orthogonalize_wgrads_workspace_bytes(None) == 0
    k3 = (ctypes.c_float * 3)(*MUON)
    g = B._WGrads(None, p, p, p)
    f = lambda *a: lib.modse_orthogonalize_wgrads(*a, None)
    assert f(None, B.MODSE_F32, g, g, None, 5, k3, 1e-7, p, full) == inv
    assert f(layer._h, B.MODSE_F32, None, g, None, 5, k3, 1e-7, p, full) == inv
    assert f(layer._h, B.MODSE_F32, B._WGrads(None, p, None, p), g, None, 5, k3, 1e-7, p, full) == inv
    assert f(layer._h, B.MODSE_F32, g, g, None, 5, k3, 1e-7, p, full - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    layer.destroy()


def test_what_the_one_kernel_form_holds():
    """Sets in the one-kernel form need the head of the workspace alone: sixteen blocks a matrix for up to seven matrices,
    eight for more; columns in steps of sixteen a block."""
    from paper_2409_12210_b200 import binding as B
    from paper_2409_12210_b200 import build
    build.build()
    head = B.orthogonalize_workspace_bytes([(1, 1)])
    for count, ends in [(8, {64: 3968, 96: 2048, 112: 1408, 128: 896}), (7, {64: 12544, 96: 6912, 112: 5376, 128: 3840})]:
        for short, long in ends.items():
            for shape in ((short, long), (long, short)):
                assert B.orthogonalize_workspace_bytes([shape] * count) == head, shape
            assert B.orthogonalize_workspace_bytes([(short, long + 1)] * count) > head
        assert B.orthogonalize_workspace_bytes([(129, 130)] * count) > head
