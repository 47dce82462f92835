"""Residual addition with root-mean-square norm (modse_add_rms_norm and its gradient) against a plain implementation in
64 bits, element by element.

Bounds.  An output is rounded once, by at most eps/2 of its value (bf16 2^-8, fp32 2^-24, e4m3 2^-4); before that it
carries the fp32 arithmetic of a row: a sum of d squares added in at most d/32 + 20 steps, a square root, a division
and three products, each off by at most 2^-23 of its value - FP = (d/32 + 40) 2^-23 covers all of it relative to the
magnitudes that are added (for dx those are the two terms of the difference and dsum, not the result)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

E4M3_MAX = 448.0
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SHAPES = [(1, 8), (1, 2048), (2, 64), (3, 264), (7, 520), (300, 1024), (5, 1032), (513, 2048), (4, 4104), (3, 8200),
          (2, 16392), (700, 256)]


def torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def fp_bound(d):
    return (d / 32 + 40) * 2.0 ** -23


def reference(x, r, w, eps):
    s = x if r is None else x + r
    rstd = 1 / np.sqrt((s * s).mean(1) + eps)
    y = s * rstd[:, None] * (1 if w is None else w)
    return s, rstd, y


def reference_bwd(s, w, dy, dsum, eps):
    d = s.shape[1]
    m = (s * s).mean(1, keepdims=True) + eps
    u = dy * (1 if w is None else w)
    first, second = u / np.sqrt(m), s * (u * s).sum(1, keepdims=True) / (d * m ** 1.5)
    # the mean's own terms may cancel: what it can be off by goes with the sum of their magnitudes
    mag = np.abs(first) + np.abs(s) * np.abs(u * s).sum(1, keepdims=True) / (d * m ** 1.5)
    dx = first - second + (0 if dsum is None else dsum)
    n = s / np.sqrt(m)
    return dx, mag + (0 if dsum is None else np.abs(dsum)), (dy * n).sum(0), np.abs(dy * n).sum(0)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def e4m3_grid(v):
    mag = np.maximum(np.abs(v), 2.0 ** -30)
    step = np.exp2(np.maximum(np.floor(np.log2(mag)), -6.0) - 3.0)
    return np.clip(np.round(v / step) * step, -E4M3_MAX, E4M3_MAX), step


def inputs(T, d, dtype, seed, scale=1.0):
    rng = np.random.default_rng(seed)
    dt = torch_dtype(dtype)
    mk = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda", dt)
    x = mk(T, d) * scale
    x[:, ::37] *= 20
    return x, mk(T, d), mk(d), mk(T, d), mk(T, d)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("residual,weight", [(True, True), (False, True), (True, False)])
def test_forward(T, d, dtype, residual, weight):
    from paper_2409_12210_b200 import binding as B
    x, r, w, _, _ = inputs(T, d, dtype, 1)
    r, w = (r if residual else None), (w if weight else None)
    s, y = torch.full_like(x, 7), torch.full_like(x, 7)
    q = torch.zeros(T, d, dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.zeros(T, device="cuda")
    B.add_rms_norm(x, r, w, 1e-5, sum_out=s, y=y, y8=q, y_scale=sc)
    rs, _, ry = reference(f64(x), None if r is None else f64(r), None if w is None else f64(w), 1e-5)
    # fp32 sum of two numbers, one rounding more in bf16
    assert np.all(np.abs(f64(s) - rs) <= np.abs(rs) * (HALF[dtype] + 2.0 ** -24))
    # an element of s is off by half an ulp of itself; that passes through to y like the rest of the row's arithmetic
    fp = fp_bound(d)
    assert np.all(np.abs(f64(y) - ry) <= np.abs(ry) * (HALF[dtype] * (1 + fp) + fp))
    rscale = np.abs(ry).max(1) / E4M3_MAX
    np.testing.assert_allclose(sc.cpu().numpy(), rscale, rtol=fp + 2.0 ** -23)
    grid, step = e4m3_grid(ry / rscale[:, None])
    diff = np.abs(f64(q) - grid)
    # within one step of the grid everywhere, and off the reference's grid point only where it lies next to a border
    border = np.abs(np.abs(ry / rscale[:, None]) / step % 1 - 0.5) <= 4 * fp * (np.abs(ry / rscale[:, None]) / step + 1)
    assert np.all(diff <= step * 1.01)
    assert np.all((diff == 0) | border)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES + [(5000, 512), (6000, 2048)])
@pytest.mark.parametrize("dsum,weight", [(True, True), (False, True), (True, False)])
def test_backward(T, d, dtype, dsum, weight):
    from paper_2409_12210_b200 import binding as B
    s, add, w, dy, _ = inputs(T, d, dtype, 2)
    add, w = (add if dsum else None), (w if weight else None)
    dx = torch.full_like(s, 7)
    dw = torch.full((d,), 7.0, device="cuda")
    n = B.add_rms_norm_backward_workspace_bytes(T, d)
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    B.add_rms_norm_backward(s, w, 1e-5, dy, add, dx, dw, ws[:n])
    opt = lambda t: None if t is None else f64(t)
    rdx, mag, rdw, dwmag = reference_bwd(f64(s), opt(w), f64(dy), opt(add), 1e-5)
    fp = fp_bound(d)
    assert np.all(np.abs(f64(dx) - rdx) <= np.abs(rdx) * HALF[dtype] + mag * fp * (1 + HALF[dtype]))
    # T terms, each off by FP, added in at most T/16 + 100 steps per partial sum and run
    assert np.all(np.abs(f64(dw) - rdw) <= dwmag * (fp + (T / 16 + 100) * 2.0 ** -23))
    assert bool((ws[n:] == 0xA5).all())
    again = torch.empty_like(dw)
    B.add_rms_norm_backward(s, w, 1e-5, dy, add, dx, again, ws[:n])
    assert torch.equal(again, dw)


@pytest.mark.gpu
def test_backward_against_differences():
    """The gradient of sum(dy * y) along random directions by central differences of the 64-bit forward."""
    from paper_2409_12210_b200 import binding as B
    s, _, w, dy, _ = inputs(6, 72, "f32", 3)
    dx, dw = torch.empty_like(s), torch.empty(72, device="cuda")
    ws = torch.empty(B.add_rms_norm_backward_workspace_bytes(6, 72), dtype=torch.uint8, device="cuda")
    B.add_rms_norm_backward(s, w, 1e-3, dy, None, dx, dw, ws)
    S, W, G = f64(s), f64(w), f64(dy)
    loss = lambda a, b: (reference(a, None, b, 1e-3)[2] * G).sum()
    rng = np.random.default_rng(0)
    for _ in range(4):
        u, v, h = rng.standard_normal(S.shape), rng.standard_normal(W.shape), 1e-5
        num = (loss(S + h * u, W) - loss(S - h * u, W)) / (2 * h)
        assert abs(num - (f64(dx) * u).sum()) <= 1e-4 * np.abs(f64(dx) * u).sum()
        num = (loss(S, W + h * v) - loss(S, W - h * v)) / (2 * h)
        assert abs(num - (f64(dw) * v).sum()) <= 1e-4 * np.abs(f64(dw) * v).sum()


@pytest.mark.gpu
def test_rows_of_zeros_infinities_and_nan():
    from paper_2409_12210_b200 import binding as B
    x = torch.randn(6, 256, device="cuda").bfloat16()
    x[0] = 0
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    x[3] = 1e-38
    w = torch.ones(256, device="cuda").bfloat16()
    y = torch.empty_like(x)
    q, sc = torch.empty(6, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, device="cuda")
    B.add_rms_norm(x, None, w, 0.0, y=y, y8=q, y_scale=sc)
    assert bool(torch.isnan(sc[1:3]).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[1, 3]))
    assert bool(torch.isnan(sc[0]))                       # 0/0: the mean square of a row of zeros is 0 and eps is 0
    B.add_rms_norm(x, None, w, 1e-5, y=y, y8=q, y_scale=sc)
    assert float(sc[0]) == 0 and bool((q[0].float() == 0).all()) and bool((y[0] == 0).all())
    # a row whose norm is far below the normal range's scale still has finite bytes that stand for it
    assert bool(torch.isfinite(q[3].float()).all())
    back = q[3].float() * sc[3]
    assert bool(((back - y[3].float()).abs() <= y[3].float().abs() * (2.0 ** -4 + 2.0 ** -8) + 1e-44).all())
    assert bool(torch.isfinite(y[4:].float()).all()) and bool(torch.isfinite(sc[4:]).all())


@pytest.mark.gpu
def test_in_place_streams_and_replay():
    from paper_2409_12210_b200 import binding as B
    x, r, w, dy, ds = inputs(37, 2048, "bf16", 4)
    y0, s0 = torch.empty_like(x), torch.empty_like(x)
    B.add_rms_norm(x, r, w, 1e-5, sum_out=s0, y=y0)
    stream, r2, y = r.clone(), r.clone(), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.add_rms_norm(x, r2, w, 1e-5, sum_out=r2, y=y)          # the residual stream is updated in place
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(r2, s0) and torch.equal(y, y0)
    # the same in a captured graph, replayed on a refreshed residual stream; backward with dx written over dsum
    ws = torch.empty(B.add_rms_norm_backward_workspace_bytes(37, 2048), dtype=torch.uint8, device="cuda")
    dx0, dw0 = torch.empty_like(x), torch.empty(2048, device="cuda")
    B.add_rms_norm_backward(s0, w, 1e-5, dy, ds, dx0, dw0, ws)
    buf, g, dw = stream.clone(), ds.clone(), torch.empty(2048, device="cuda")
    y.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.add_rms_norm(x, buf, w, 1e-5, sum_out=buf, y=y)
        B.add_rms_norm_backward(buf, w, 1e-5, dy, g, g, dw, ws)
    for _ in range(2):
        buf.copy_(stream)
        g.copy_(ds)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(buf, s0) and torch.equal(y, y0) and torch.equal(g, dx0) and torch.equal(dw, dw0)


@pytest.mark.gpu
def test_empty_batch_and_binding_refusals():
    from paper_2409_12210_b200 import binding as B
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    B.add_rms_norm(x, None, None, 1e-5, y=torch.empty_like(x))
    dw = torch.ones(64, device="cuda")
    B.add_rms_norm_backward(x, None, 1e-5, x, None, x, dw, torch.empty(4096, dtype=torch.uint8, device="cuda"))
    assert bool((dw == 0).all())
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(y=torch.empty(4, 128, dtype=torch.bfloat16, device="cuda")[:, ::2]),
                dict(y=torch.empty(4, 64, device="cuda")), dict(y=torch.empty(3, 64, dtype=torch.bfloat16, device="cuda")),
                dict(y=torch.empty(4, 64, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            B.add_rms_norm(x, None, None, 1e-5, **bad)
    with pytest.raises(B.ModseError):
        B.add_rms_norm(x, None, None, 1e-5)


def test_refusals_need_no_gpu():
    from paper_2409_12210_b200 import binding as B
    from paper_2409_12210_b200 import build
    build.build()
    lib = B.load()
    p = 0x10000
    f = lambda *a: lib.modse_add_rms_norm(*a, None)
    ok = (B.MODSE_BF16, 4, 64, p, p, p, 1e-5, p, p, p, p)
    for i, v in [(0, 2), (0, 7), (1, -1), (1, (1 << 30) + 1), (2, 0), (2, 60), (2, -8), (3, None), (3, p + 8), (4, p + 2),
                 (5, p + 4), (6, -1.0), (6, float("nan")), (6, float("inf")), (7, p + 8), (8, p + 8), (9, p + 8),
                 (9, None), (10, None), (10, p + 2)]:
        a = list(ok)
        a[i] = v
        assert f(*a) == B.MODSE_ERR_INVALID_ARG, (i, v)
    assert f(B.MODSE_BF16, 4, 32776, p, p, p, 1e-5, p, p, p, p) == B.MODSE_ERR_UNSUPPORTED
    assert f(B.MODSE_BF16, 4, 64, p, p, p, 1e-5, None, None, None, None) == B.MODSE_ERR_INVALID_ARG
    assert f(B.MODSE_BF16, 0, 64, None, None, None, 1e-5, None, None, None, None) == B.MODSE_OK
    g = lambda *a: lib.modse_add_rms_norm_backward(*a, None)
    need = B.add_rms_norm_backward_workspace_bytes(4, 64)
    assert need >= 256 and B.add_rms_norm_backward_workspace_bytes(-1, 64) == 0
    assert B.add_rms_norm_backward_workspace_bytes(4, 63) == 0
    ok = (B.MODSE_F32, 4, 64, p, p, 1e-5, p, p, p, p, p, need)
    for i, v in [(0, 2), (1, -1), (2, 12), (3, None), (3, p + 8), (4, p + 8), (5, -1.0), (6, None), (6, p + 4), (7, p + 4),
                 (8, None), (8, p + 4), (9, p + 4), (10, None), (10, p + 16)]:
        a = list(ok)
        a[i] = v
        assert g(*a) == B.MODSE_ERR_INVALID_ARG, (i, v)
    a = list(ok)
    a[11] = need - 1
    assert g(*a) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(ValueError):
        B.add_rms_norm(torch.zeros(4, 64), None, None, 1e-5, y=torch.zeros(4, 64))       # no CPU path
    with pytest.raises(ValueError):
        B.add_rms_norm(torch.zeros(64), None, None, 1e-5, y=torch.zeros(64))
    with pytest.raises(TypeError):
        B.add_rms_norm(torch.zeros(4, 64, dtype=torch.float16), None, None, 1e-5, y=torch.zeros(4, 64))
