"""The dense product with bias, activation and residual (modse_linear and its gradient) against a plain implementation
in 64 bits, element by element.

Bounds.  Products of 16- or 8-bit numbers are exact in fp32; K of them are added in fp32, each addition off by at most
2^-23 of the running magnitude (tensor cores may truncate), which stays below S = sum_k |x w|: K 2^-23 S, and a few more
roundings for scales, bias and residual: ACC = (K + 64) 2^-23 times the sum of all magnitudes.  An activation changes an
error by at most 1.13 (the largest slope of gelu and silu is below that) and adds its own arithmetic, 2^-20 of |z|.  An
output is rounded once, to bf16: 2^-8 of its value.  In backward dz is rounded to bf16 before it enters a product: 2^-8
of every term."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

ACTS = ["none", "relu", "gelu", "silu"]
BF, U = 2.0 ** -8, 2.0 ** -23
# (T, d_in, d_out): one token, few, ragged tiles, one tile over, several tiles with a tail, many tiles
SHAPES = [(1, 8, 8), (1, 2048, 2048), (3, 136, 264), (17, 4096, 24), (32, 512, 1000), (33, 64, 136), (64, 1024, 4096),
          (127, 200, 72), (129, 80, 520), (257, 648, 1032), (300, 2816, 2048), (1000, 256, 384), (2500, 512, 2048),
          (200, 2048, 264), (1100, 72, 1032), (1100, 136, 1032)]      # tiles shared by two and by four pairs of CTAs


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def phi(z):
    return 0.5 * (1 + np.vectorize(math.erf)(z / math.sqrt(2)))


def act64(z, name):
    return {"none": lambda: z, "relu": lambda: np.maximum(z, 0), "gelu": lambda: z * phi(z),
            "silu": lambda: z / (1 + np.exp(-z))}[name]()


def slope64(z, name):
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return phi(z) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def rand(rng, *shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).cuda()


def guarded(shape, dtype=torch.bfloat16):
    """A buffer with a filled margin behind it."""
    n = int(np.prod(shape))
    base = torch.full((n + 512,), 3.0, dtype=dtype, device="cuda")
    return base[:n].view(shape), base[n:]


def workspace(n):
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    return ws[:n], ws[n:]


def check_forward(T, k, n, f8, act, bias, residual, save, seed=0):
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(seed)
    x, w = rand(rng, T, k), rand(rng, n, k, std=k ** -0.5)
    sx = sw = None
    if f8:
        sx, sw = rand(rng, T).abs() + 0.1, rand(rng, n).abs() + 0.1
        x, w = x.to(torch.float8_e4m3fn), (w * math.sqrt(k)).to(torch.float8_e4m3fn)
        sw *= k ** -0.5
    else:
        x, w = x.bfloat16(), w.bfloat16()
    b = rand(rng, n).bfloat16() if bias else None
    r = rand(rng, T, n).bfloat16() if residual else None
    y, y_margin = guarded((T, n))
    z, z_margin = guarded((T, n))
    ws, ws_margin = workspace(B.linear_workspace_bytes(x.dtype, T, k, n))
    B.linear(x, w, y, ws, bias=b, residual=r, activation=act, z=z if save else None, x_scale=sx, w_scale=sw)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    X, W = f64(x), f64(w)
    if f8:
        X, W = X * f64(sx)[:, None], W * f64(sw)[:, None]
    zz, mag = X @ W.T, np.abs(X) @ np.abs(W).T
    if bias:
        zz, mag = zz + f64(b), mag + np.abs(f64(b))
    rr = f64(r) if residual else 0.0
    yy = act64(zz, act) + rr
    acc = (k + 64) * U * mag
    if save:
        assert np.all(np.abs(f64(z) - zz) <= BF * np.abs(zz) + acc * (1 + BF))
    tol = BF * np.abs(yy) + (1.13 * acc + 2.0 ** -20 * np.abs(zz) + U * np.abs(rr)) * (1 + BF)
    bad = np.abs(f64(y) - yy) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())
    for m in (y_margin, z_margin):
        assert bool((m == 3).all())
    assert bool((ws_margin == 0xA5).all())
    again = torch.empty_like(y)
    B.linear(x, w, again, ws, bias=b, residual=r, activation=act, x_scale=sx, w_scale=sw)
    assert torch.equal(again, y)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act,bias,residual,save", [("none", False, False, False), ("gelu", True, False, True),
                                                    ("silu", True, True, True), ("relu", False, True, False)])
def test_forward_bf16(shape, act, bias, residual, save):
    check_forward(*shape, False, act, bias, residual, save)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(T, (k + 15) // 16 * 16, n) for T, k, n in SHAPES])
@pytest.mark.parametrize("act,bias,residual,save", [("none", False, True, False), ("silu", True, False, True)])
def test_forward_e4m3(shape, act, bias, residual, save):
    check_forward(*shape, True, act, bias, residual, save)


def run_backward(T, k, n, act, want=("dx", "dw", "db"), seed=1):
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(seed)
    x, w, dy = rand(rng, T, k).bfloat16(), rand(rng, n, k, std=k ** -0.5).bfloat16(), rand(rng, T, n).bfloat16()
    z = rand(rng, T, n).bfloat16()
    z.view(-1)[::7] = 0
    dx, m1 = guarded((T, k))
    dw, m2 = guarded((n, k))
    db, m3 = guarded((n,), torch.float32)
    ws, m4 = workspace(B.linear_backward_workspace_bytes(T, k, n))
    B.linear_backward(x, w, dy, z if act != "none" else None, act, dx if "dx" in want else None,
                      dw if "dw" in want else None, db if "db" in want else None, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    for m in (m1, m2, m3):
        assert bool((m == 3).all())
    assert bool((m4 == 0xA5).all())
    return x, w, dy, z, dx, dw, db


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act", ACTS)
def test_backward(shape, act):
    T, k, n = shape
    x, w, dy, z, dx, dw, db = run_backward(T, k, n, act)
    X, W, G, Z = f64(x), f64(w), f64(dy), f64(z)
    dz = G * slope64(Z, act)
    # dz carries its own arithmetic (2^-19 of dy; slopes are at most 1.13) and, inside the products, one rounding to bf16
    own = 2.0 ** -19 * np.abs(G)
    term = np.abs(dz) * BF + own * (1 + BF) if act != "none" else 0 * np.abs(dz)
    for got, ref, err, mag, terms in ((dx, dz @ W, term @ np.abs(W), np.abs(dz) @ np.abs(W), n),
                                      (dw, dz.T @ X, term.T @ np.abs(X), np.abs(dz).T @ np.abs(X), T)):
        tol = BF * np.abs(ref) + (err + (terms + 64) * U * (mag + err)) * (1 + BF)
        bad = np.abs(f64(got) - ref) > tol
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())
    tol = own.sum(0) + (T / 8 + 200) * U * (np.abs(dz) + own).sum(0)
    assert np.all(np.abs(f64(db) - dz.sum(0)) <= tol)


# Shapes some of whose tiles are cut along the contraction on 74 CTA pairs (at least 32 k-blocks, and a last round that leaves
# room): the last 6, 7 or 16 of more tiles than pairs in two pieces, ragged edges among them; few tiles in two to eight pieces.
CUT = [(2500, 2304, 2048), (2100, 2056, 2056), (1000, 2048, 1032), (64, 5632, 2048), (40, 8448, 1032), (33, 8448, 136)]
CUT8 = [(2500, 4112, 2056), (1000, 4096, 1032), (40, 16400, 136)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", CUT)
@pytest.mark.parametrize("act,bias,residual,save", [("silu", True, True, True), ("relu", True, False, False)])
def test_cut_tiles_bf16(shape, act, bias, residual, save):
    check_forward(*shape, False, act, bias, residual, save)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", CUT8)
@pytest.mark.parametrize("act,bias,residual,save", [("none", False, True, False), ("silu", True, False, True)])
def test_cut_tiles_e4m3(shape, act, bias, residual, save):
    check_forward(*shape, True, act, bias, residual, save)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2100, 2056, 2056), (300, 2304, 2304)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_cut_tiles_backward(shape, act):
    """dx and dw in one launch whose last tiles are cut; dx alone of the second shape, in 128-column tiles."""
    test_backward(shape, act)
    full, part = run_backward(*shape, act), run_backward(*shape, act, ("dx",))
    assert torch.allclose(full[4].float(), part[4].float(), rtol=2.0 ** -7, atol=1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2500, 2304, 2048), (40, 8448, 1032)])
def test_cut_tiles_in_graphs(shape):
    """The counters that find a strip's last piece are zero again after every launch: replays, two graphs with a workspace
    each running at once, and eager calls between them."""
    from paper_2409_12210_b200 import binding as B
    T, k, n = shape
    rng = np.random.default_rng(15)
    xs = [rand(rng, T, k).bfloat16() for _ in range(3)]
    w, r = rand(rng, n, k, std=k ** -0.5).bfloat16(), rand(rng, T, n).bfloat16()
    size = B.linear_workspace_bytes(w.dtype, T, k, n)
    wss = [workspace(size) for _ in range(3)]
    refs = []
    for x in xs:
        y = torch.empty_like(r)
        B.linear(x, w, y, wss[2][0], residual=r, activation="silu")
        refs.append(y)
    sides = [torch.cuda.Stream() for _ in range(2)]
    ins, outs, graphs = [torch.zeros_like(xs[0]) for _ in sides], [torch.empty_like(r) for _ in sides], []
    torch.cuda.synchronize()
    for side, x, y, ws in zip(sides, ins, outs, wss):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.linear(x, w, y, ws[0], residual=r, activation="silu")
        graphs.append(graph)
    for i in range(3):
        for j, (side, graph) in enumerate(zip(sides, graphs)):
            with torch.cuda.stream(side):
                ins[j].copy_(xs[(i + j) % 3])
                for _ in range(4):
                    graph.replay()
        torch.cuda.synchronize()
        for j in range(2):
            assert torch.equal(outs[j], refs[(i + j) % 3])
        B.linear(xs[i], w, outs[0], wss[0][0], residual=r, activation="silu")
        assert B.check_workspace_status(wss[0][0]) == B.MODSE_OK and torch.equal(outs[0], refs[i])
        torch.cuda.synchronize()
    assert all(bool((margin == 0xA5).all()) for _, margin in wss)


@pytest.mark.gpu
def test_512_row_tiles():
    """Shapes whose products run on 512-row tiles: a ragged last tile with one 256-row half, column edges, a tail dealt out
    as halves (forward) and two products in one launch with more than one round (backward)."""
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(11)
    T, k, n = 19300, 1544, 1000
    x, w, b = rand(rng, T, k).bfloat16(), rand(rng, n, k, std=k ** -0.5).bfloat16(), rand(rng, n).bfloat16()
    y, margin = guarded((T, n))
    ws, ws_margin = workspace(B.linear_workspace_bytes(x.dtype, T, k, n))
    B.linear(x, w, y, ws, bias=b, activation="relu")
    assert B.check_workspace_status(ws) == B.MODSE_OK
    ref = (x.double() @ w.double().T + b.double()).clamp_min(0)
    mag = x.double().abs() @ w.double().abs().T + b.double().abs()
    assert bool(((y.double() - ref).abs() <= BF * ref + (k + 64) * U * mag * (1 + BF)).all())
    assert bool((margin == 3).all()) and bool((ws_margin == 0xA5).all())
    T, k, n = 9300, 2056, 1544
    x, w, dy, _, dx, dw, db = run_backward(T, k, n, "none")
    X, W, G = x.double(), w.double(), dy.double()
    for got, ref, mag, terms in ((dx, G @ W, G.abs() @ W.abs(), n), (dw, G.T @ X, G.abs().T @ X.abs(), T)):
        assert bool(((got.double() - ref).abs() <= BF * ref.abs() + (terms + 64) * U * mag * (1 + BF)).all())
    assert bool(((db.double() - G.sum(0)).abs() <= (T / 8 + 200) * U * G.abs().sum(0)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("db",), ("dx", "db")])
def test_backward_outputs_that_are_not_wanted_are_left_alone(want):
    full = run_backward(257, 648, 1032, "silu")
    part = run_backward(257, 648, 1032, "silu", want)
    for name, a, b in (("dx", full[4], part[4]), ("dw", full[5], part[5]), ("db", full[6], part[6])):
        if name in want:
            # which pieces a cut tile is summed from depends on the products of the launch: one bf16 step at most
            assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-5)
        else:
            assert bool((b == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes_against_differences(act):
    """dbias of a batch of one token is the slope itself (dy = 1): central differences of the 64-bit activation."""
    from paper_2409_12210_b200 import binding as B
    z = torch.linspace(-6, 6, 1024).bfloat16().cuda().view(1, 1024)
    z[0, 512] = 0.25                                       # away from relu's corner
    dy, db = torch.ones_like(z), torch.empty(1024, device="cuda")
    ws = torch.empty(B.linear_backward_workspace_bytes(1, 8, 1024), dtype=torch.uint8, device="cuda")
    x, w = torch.zeros(1, 8, device="cuda").bfloat16(), torch.zeros(1024, 8, device="cuda").bfloat16()
    B.linear_backward(x, w, dy, z, act, None, None, db, ws)
    Z, h = f64(z)[0], 1e-6
    keep = np.abs(Z) > 1e-4
    num = (act64(Z + h, act) - act64(Z - h, act)) / (2 * h)
    assert np.all(np.abs(f64(db) - num)[keep] <= 1e-6)


@pytest.mark.gpu
def test_far_activations_and_special_values():
    """The activations' ends: no NaN from exp overflowing, NaN and infinities pass through a row and stay in it."""
    from paper_2409_12210_b200 import binding as B
    x = torch.zeros(5, 64, device="cuda").bfloat16()
    x[0, 0], x[1, 0], x[2, 0], x[3, 1] = 3e4, -3e4, float("nan"), 1.0
    w = torch.zeros(16, 64, device="cuda").bfloat16()
    w[:, 0] = 1
    ws = torch.empty(B.linear_workspace_bytes(x.dtype, 5, 64, 16), dtype=torch.uint8, device="cuda")
    y = torch.empty(5, 16, device="cuda").bfloat16()
    for act in ACTS:
        B.linear(x, w, y, ws, activation=act)
        assert bool((y[0] == x[0, 0]).all()) and bool(torch.isnan(y[2]).all())
        assert bool((y[1] == (x[1, 0] if act == "none" else 0)).all())
        assert bool((y[3:] == 0).all())


def tail64(z, name):
    """gelu, silu and their slopes without cancellation, for z < 0."""
    if name == "silu":
        s = np.exp(z) / (1 + np.exp(z))
        return z * s, s * (1 + z * (1 - s))
    q = 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2))
    return z * q, q + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [8, 40])
@pytest.mark.parametrize("act,low", [("gelu", -12.75), ("silu", -86.0)])
def test_left_tails_of_the_activations(act, low, T):
    """Far left the functions go to zero and keep their leading digits.  Bound relative to the value: one rounding to bf16
    (none for dbias), 6.1e-5 for the approximation of the tail, and the exponential's argument, off by two roundings of at
    most 2^-24 |q|, |q| <= 128 log2(e) 2^-1 .. 125: 2 * 125 * 2^-24 ln 2 = 1.1e-5, with a few units of the approximate
    functions 2^-22 each: 1e-4 in all.  The slope adds terms of opposite sign: q and z phi, both relative to |z| phi."""
    from paper_2409_12210_b200 import binding as B
    z = torch.linspace(low, -0.5, 8 * T).bfloat16().cuda().view(T, 8)
    x, w = torch.zeros(T, 8, device="cuda").bfloat16(), torch.eye(8, device="cuda").bfloat16()
    x.copy_(z)                                     # z = x I, exactly
    y, saved = torch.empty_like(z), torch.empty_like(z)
    ws = torch.empty(B.linear_workspace_bytes(x.dtype, T, 8, 8), dtype=torch.uint8, device="cuda")
    B.linear(x, w, y, ws, activation=act, z=saved)
    assert torch.equal(saved, z)
    Z = f64(z)
    ref, slope = tail64(Z, act)
    assert np.all(np.abs(f64(y) - ref) <= (BF + 1e-4) * np.abs(ref))
    n = 8 * T
    flat, dy, db = z.view(1, n), torch.ones(1, n, device="cuda").bfloat16(), torch.empty(n, device="cuda")
    ws = torch.empty(B.linear_backward_workspace_bytes(1, 8, n), dtype=torch.uint8, device="cuda")
    x, w = torch.zeros(1, 8, device="cuda").bfloat16(), torch.zeros(n, 8, device="cuda").bfloat16()
    B.linear_backward(x, w, dy, flat, act, None, None, db, ws)
    size = np.abs(Z) * np.exp(-Z * Z / 2) if act == "gelu" else (1 - Z) * np.exp(Z)
    assert np.all(np.abs(f64(db) - slope.ravel()) <= 1e-4 * size.ravel())


@pytest.mark.gpu
def test_relu_masks_infinities_and_nan_in_the_incoming_gradient():
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(7)
    T, k, n = 70, 72, 136
    x, w, z, dy = (rand(rng, *s).bfloat16() for s in ((T, k), (n, k), (T, n), (T, n)))
    z[:, ::5] = 0
    z[0, 1], z[1, 2] = -float("inf"), -1.0
    clean, dirty = torch.where(z > 0, dy, 0), dy.clone()
    for i, v in enumerate((float("inf"), -float("inf"), float("nan"))):
        dirty.view(-1)[i::3] = torch.where(z.view(-1)[i::3] > 0, dirty.view(-1)[i::3], v)
    outs = []
    for g in (clean, dirty):
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda")
        ws = torch.empty(B.linear_backward_workspace_bytes(T, k, n), dtype=torch.uint8, device="cuda")
        B.linear_backward(x, w, g, z, "relu", dx, dw, db, ws)
        outs.append((dx, dw, db))
    assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(*outs))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 40])
def test_infinities_go_where_the_limits_are(T):
    from paper_2409_12210_b200 import binding as B
    inf = float("inf")
    x = torch.zeros(T, 8, device="cuda").bfloat16()
    x[0, 0], x[1, 0], x[2, 0] = inf, -inf, float("nan")
    w = torch.zeros(16, 8, device="cuda").bfloat16()
    w[:, 0] = 1
    y, z = torch.empty(T, 16, device="cuda").bfloat16(), torch.empty(T, 16, device="cuda").bfloat16()
    ws = torch.empty(B.linear_workspace_bytes(x.dtype, T, 8, 16), dtype=torch.uint8, device="cuda")
    back = torch.empty(B.linear_backward_workspace_bytes(1, 8, 16), dtype=torch.uint8, device="cuda")
    db, one = torch.empty(16, device="cuda"), torch.ones(1, 16, device="cuda").bfloat16()
    for act in ACTS:
        B.linear(x, w, y, ws, activation=act, z=z)
        assert bool((z[0] == inf).all()) and bool((z[1] == -inf).all()) and bool(torch.isnan(z[2]).all())
        assert bool((y[0] == inf).all()) and bool((y[1] == (-inf if act == "none" else 0)).all())
        assert bool(torch.isnan(y[2]).all()) and bool((y[3:] == 0).all())
        if act != "none":
            for row, slope in ((0, 1.0), (1, 0.0)):
                B.linear_backward(x[:1], w, one, z[row:row + 1], act, None, None, db, back)
                assert bool((db == slope).all())


@pytest.mark.gpu
def test_in_place_residual_replay_and_two_streams():
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(5)
    x, w, r = rand(rng, 300, 512).bfloat16(), rand(rng, 512, 512, std=0.05).bfloat16(), rand(rng, 300, 512).bfloat16()
    n = B.linear_workspace_bytes(x.dtype, 300, 512, 512)
    wss = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ref = torch.empty_like(r)
    B.linear(x, w, ref, wss[0], residual=r, activation="silu")
    stream = r.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.linear(x, w, stream, wss[0], residual=stream, activation="silu")
    for _ in range(3):
        stream.copy_(r)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(stream, ref)
    # two calls at once, a workspace each
    outs = [torch.empty_like(r) for _ in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for side, out, ws in zip(sides, outs, wss):
            with torch.cuda.stream(side):
                B.linear(x, w, out, ws, residual=r, activation="silu")
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 24, 300, 2500])
def test_a_chain_of_overlapped_calls_reads_what_the_call_before_it_wrote(T):
    """Norm and 8-bit product in turn on the same buffers, inputs changing from call to call and nothing waited for: rows
    and scales are those of the norm just ahead, whose kernel is still running when the product's starts."""
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(T)
    k, n, calls = 512, 1032, 24
    xs = [rand(rng, T, k).bfloat16() * (1 + i) for i in range(calls)]
    w, sw = rand(rng, n, k).to(torch.float8_e4m3fn), rand(rng, n).abs() + 0.1
    q, sc = torch.empty(T, k, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, device="cuda")
    ws = torch.empty(B.linear_workspace_bytes(q.dtype, T, k, n), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(T, n, device="cuda").bfloat16() for _ in range(2 * calls)]

    def step(x, y):
        B.add_rms_norm(x, None, None, 1.0, y8=q, y_scale=sc)       # eps 1: the rows' size stays in the result
        B.linear(q, w, y, ws, x_scale=sc, w_scale=sw)

    for x, y in zip(xs, outs):
        step(x, y)
        torch.cuda.synchronize()
    for x, y in zip(xs, outs[calls:]):
        step(x, y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, outs[calls:]))
    assert not torch.equal(outs[0], outs[1])


@pytest.mark.gpu
def test_empty_batch_and_binding_refusals():
    from paper_2409_12210_b200 import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w, y = torch.empty(0, 64, **bf), torch.zeros(32, 64, **bf), torch.empty(0, 32, **bf)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    B.linear(x, w, y, ws)
    dw, db = torch.ones(32, 64, **bf), torch.ones(32, device="cuda")
    B.linear_backward(x, w, y, y, "gelu", x, dw, db, ws)
    assert bool((dw == 0).all()) and bool((db == 0).all())
    x, y = torch.zeros(4, 64, **bf), torch.empty(4, 32, **bf)
    with pytest.raises(ValueError):
        B.linear(x, w.t().contiguous().t(), y, ws)
    with pytest.raises(ValueError):
        B.linear(x, w, y, ws, bias=torch.zeros(32, device="cuda"))
    with pytest.raises(ValueError):
        B.linear(x, w, y, ws, z=torch.empty(4, 31, **bf))
    with pytest.raises(B.ModseError):
        B.linear(x, w, y, ws[:64])
    with pytest.raises(KeyError):
        B.linear(x, w, y, ws, activation="tanh")
    with pytest.raises(TypeError):
        B.linear(x.float(), w.float(), y, ws)


@pytest.mark.gpu
def test_a_workspace_for_the_largest_batch_serves_the_smaller_ones():
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(13)
    k, n, most = 2048, 1408, 8192
    w = rand(rng, n, k, std=k ** -0.5).bfloat16()
    ws, margin = workspace(B.linear_workspace_bytes(w.dtype, most, k, n))
    back, back_margin = workspace(B.linear_backward_workspace_bytes(most, k, n))
    for T in (1, 33, 500, 2048, 3300, 8192):
        x, dy = rand(rng, T, k).bfloat16(), rand(rng, T, n).bfloat16()
        outs = []
        for a, b in ((ws, back), (None, None)):
            a = workspace(B.linear_workspace_bytes(w.dtype, T, k, n))[0] if a is None else a
            b = workspace(B.linear_backward_workspace_bytes(T, k, n))[0] if b is None else b
            y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w)
            B.linear(x, w, y, a)
            B.linear_backward(x, w, dy, None, "none", dx, dw, None, b)
            assert B.check_workspace_status(a) == B.MODSE_OK and B.check_workspace_status(b) == B.MODSE_OK
            outs.append((y, dx, dw))
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert bool((margin == 0xA5).all()) and bool((back_margin == 0xA5).all())


def test_workspace_sizes_never_fall_with_the_batch():
    from paper_2409_12210_b200 import binding as B
    from paper_2409_12210_b200 import build
    build.build()
    batches = list(range(1, 2000, 37)) + [2048, 2304, 4096, 6144, 8192, 8193, 12000, 16384, 20000, 65536, 1 << 20]
    for k, n in [(2048, 5632), (5632, 2048), (2048, 2048), (8448, 1024), (64, 64), (512, 8448), (1536, 2816), (8192, 136)]:
        for size in (lambda T: B.linear_workspace_bytes(torch.bfloat16, T, k, n),
                     lambda T: B.linear_workspace_bytes(torch.float8_e4m3fn, T, k, n),
                     lambda T: B.linear_backward_workspace_bytes(T, k, n)):
            sizes = [size(T) for T in batches]
            assert sizes == sorted(sizes) and sizes[0] > 0


def test_refusals_need_no_gpu():
    from paper_2409_12210_b200 import binding as B
    from paper_2409_12210_b200 import build
    build.build()
    lib = B.load()
    p = 0x10000
    need = lib.modse_linear_workspace_bytes(B.MODSE_BF16, 4, 64, 32)
    assert need > 0 and need % 256 == 0
    for bad in [(B.MODSE_F32, 4, 64, 32), (9, 4, 64, 32), (B.MODSE_BF16, -1, 64, 32), (B.MODSE_BF16, 4, 60, 32),
                (B.MODSE_BF16, 4, 64, 36), (B.MODSE_BF16, 4, 0, 32), (B.MODSE_BF16, 4, 64, 0), (B.MODSE_E4M3, 4, 72, 32),
                (B.MODSE_BF16, 1 << 30, 64, 1 << 26)]:
        assert lib.modse_linear_workspace_bytes(*bad) == 0, bad

    def call(dtype=B.MODSE_BF16, T=4, k=64, n=32, act=0, ws=p, size=None, x=p, w=p, x_scale=None, w_scale=None, bias=p,
             residual=p, z=p, y=p, none=False):
        args = B._Linear(x, w, x_scale, w_scale, bias, residual, z, y)
        return lib.modse_linear(dtype, T, k, n, act, None if none else args, ws, need if size is None else size, None)

    inv = B.MODSE_ERR_INVALID_ARG
    assert call(T=0) == B.MODSE_OK
    assert call(dtype=B.MODSE_F32) == B.MODSE_ERR_UNSUPPORTED
    assert call(size=need - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    for bad in [dict(none=True), dict(act=-1), dict(act=4), dict(dtype=5), dict(T=-1), dict(k=60), dict(n=12), dict(x=None),
                dict(w=None), dict(y=None), dict(x=p + 8), dict(w=p + 8), dict(bias=p + 2), dict(residual=p + 8),
                dict(z=p + 4), dict(y=p + 8), dict(ws=None), dict(ws=p + 64), dict(x_scale=p), dict(w_scale=p),
                dict(dtype=B.MODSE_E4M3), dict(dtype=B.MODSE_E4M3, x_scale=p), dict(dtype=B.MODSE_E4M3, w_scale=p),
                dict(dtype=B.MODSE_E4M3, x_scale=p + 2, w_scale=p), dict(dtype=B.MODSE_E4M3, x_scale=p, w_scale=p + 4)]:
        assert call(**bad) == inv, bad

    need_b = lib.modse_linear_backward_workspace_bytes(4, 64, 32)
    assert need_b > 0
    for bad in [(-1, 64, 32), (4, 60, 32), (4, 64, 33), (4194241, 64, 32)]:
        assert lib.modse_linear_backward_workspace_bytes(*bad) == 0, bad

    def back(T=4, k=64, n=32, act=2, ws=p, size=None, x=p, w=p, dy=p, z=p, dx=p, dw=p, dbias=p, none=False):
        args = B._LinearGrads(x, w, dy, z, dx, dw, dbias)
        return lib.modse_linear_backward(T, k, n, act, None if none else args, ws, need_b if size is None else size, None)

    assert back(size=need_b - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    for bad in [dict(none=True), dict(act=4), dict(T=-1), dict(k=4), dict(n=4), dict(x=None), dict(w=None), dict(dy=None),
                dict(z=None), dict(x=p + 8), dict(w=p + 8), dict(dy=p + 8), dict(z=p + 8), dict(dx=p + 8), dict(dw=p + 8),
                dict(dbias=p + 2), dict(ws=None), dict(ws=p + 16), dict(dx=None, dw=None, dbias=None)]:
        assert back(**bad) == inv, bad
    assert lib.modse_check_workspace_status(None, None) == inv


@pytest.mark.gpu
@pytest.mark.parametrize("T,k", [(300, 256), (300, 2048), (20000, 256), (18944, 1544)])
def test_a_wait_that_runs_out_is_reported_and_the_gpu_stays_usable(T, k):
    """The producers of one CTA pair are told to load nothing for one item: nothing of theirs is in flight, their consumers
    give up after the (shortened) limit, the kernel returns and the host reads the time-out; the next call is correct."""
    from paper_2409_12210_b200 import binding as B
    rng = np.random.default_rng(9)
    n = 1024 if k > 1000 else 512
    x, w = rand(rng, T, k).bfloat16(), rand(rng, n, k, std=0.06).bfloat16()
    y, ref = torch.empty(T, n, device="cuda").bfloat16(), torch.empty(T, n, device="cuda").bfloat16()
    ws = torch.empty(B.linear_workspace_bytes(x.dtype, T, k, n), dtype=torch.uint8, device="cuda")
    B.linear(x, w, ref, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    B.debug_set_wait_limit_ms(50)
    B.debug_skip_tile_loads(6, 0)
    try:
        B.linear(x, w, y, ws)
        assert B.check_workspace_status(ws) == B.MODSE_ERR_DEVICE_TIMEOUT
    finally:
        B.debug_set_wait_limit_ms(2000)
        B.debug_skip_tile_loads(-1, -1)
    B.linear(x, w, y, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    assert torch.equal(y, ref)
