"""The softmax cross entropy over a vocabulary and its gradient against a plain implementation in 64 bits, element by
element.

Bounds.  A logit is a sum of d exact products in fp32, each addition off by at most 2^-23 of a magnitude below S = sum |x w|
(tensor cores may truncate): ez = (d + 8) 2^-23 S.  Forward: lse moves by at most the largest ez of the row; a term 2^(z log2 e - M) carries the
rounding of its exponent, at most 2^-24 (|z| + 130) log2 e, and 2^-22 of the exponential (all but nothing below 2^-126); sums of V / 128 runs of 128 in a
fixed order add (160 + V / 128) 2^-24, the logarithm and the product with ln 2 2^-22 of |lse| + 1.  loss is their difference, rounded.
Gradient: dz = f (p - [v = label]) with p off by p (ez + the same exponent and exponential terms), then rounded to bf16 once, 2^-8 of it (and
at most 2^-126 f below the normal range of fp32); the products add (K + 64) 2^-23 of the sum of their magnitudes and the output's 2^-8."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

BF, U = 2.0 ** -8, 2.0 ** -24
L2E = 1.4426950408889634


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def guarded(shape, dtype):
    n = int(np.prod(shape))
    base = torch.full((n + 512,), 3.0, dtype=dtype, device="cuda")
    return base[:n].view(shape), base[n:]


def workspace(n):
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    return ws[:n], ws[n:]


def problem(T, d, V, seed=0, std=2.0):
    rng = np.random.default_rng(seed)
    w = torch.from_numpy((rng.standard_normal((V, d)) * std * d ** -0.5).astype(np.float32)).bfloat16()
    labels = rng.integers(0, V, T)
    x = rng.standard_normal((T, d)) + 1.5 * rng.random((T, 1)) * w.float().numpy()[labels]
    labels = np.where(rng.random(T) < 0.2, -1 - rng.integers(0, 200, T), labels)
    return torch.from_numpy(x.astype(np.float32)).bfloat16().cuda(), w.cuda(), labels


def logits64(x, w):
    """Logits and the sums of the magnitudes of their terms in 64 bits, on the device."""
    a, b = x.double(), w.double()
    return a @ b.T, a.abs() @ b.abs().T


def exponent_error(z):
    return 2 * U * (z.abs() + 130) * L2E + 2.0 ** -21


def forward64(x, w, labels):
    """(loss, lse, bound of lse, bound of loss) in 64 bits."""
    z, S = logits64(x, w)
    d, V = x.shape[1], w.shape[0]
    ez = (d + 8) * 2.0 ** -23 * S
    lse = torch.logsumexp(z, 1)
    e_lse = ez.max(1).values + exponent_error(z).max(1).values + (160 + V / 128) * U + 2.0 ** -22 * (lse.abs() + 1)
    lab = torch.from_numpy(np.clip(labels, 0, V - 1)).cuda()[:, None]
    counted = torch.from_numpy((labels >= 0) & (labels < V)).cuda()
    loss = torch.where(counted, lse - z.gather(1, lab)[:, 0], 0.0)
    e_loss = e_lse + ez.gather(1, lab)[:, 0] + U * loss.abs()
    return loss, lse, e_lse, torch.where(counted, e_loss, 0.0)


def check_forward(T, d, V, idt=torch.int64, seed=0):
    from paper_2409_12210_b200 import binding as B
    x, w, labels = problem(T, d, V, seed)
    (loss, m0), (lse, m1) = guarded((T,), torch.float32), guarded((T,), torch.float32)
    total, m2 = guarded((2,), torch.float32)
    ws, m3 = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    lab = torch.from_numpy(labels).to(idt).cuda()
    B.cross_entropy(x, w, lab, loss, lse, ws, total=total)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    for m in (m0, m1, m2):
        assert bool((m == 3).all())
    assert bool((m3 == 0xA5).all())
    rloss, rlse, e_lse, e_loss = forward64(x, w, labels)
    assert bool(((lse.double() - rlse).abs() <= e_lse).all())
    assert bool(((loss.double() - rloss).abs() <= e_loss).all())
    assert float(total[1]) == (labels >= 0).sum()
    assert abs(float(total[0]) - float(loss.double().sum())) <= 2.0 ** -23 * float(loss.double().abs().sum())
    first = [t.clone() for t in (loss, lse, total)]
    B.cross_entropy(x, w, lab, loss, lse, ws, total=total)          # the same bits on a used workspace
    assert all(torch.equal(a, b) for a, b in zip(first, (loss, lse, total)))
    loss.fill_(5)
    B.cross_entropy(x, w, lab, loss, lse, ws)
    assert torch.equal(loss, first[0]) and torch.equal(lse, first[1])


# (T, d, V): one token, one word, fewer than a run, runs and tiles with ragged ends, tiles cut along the contraction
# (74 CTA pairs, left-over tiles), several rounds
SHAPES = [(1, 8, 1), (1, 2048, 5000), (3, 64, 7), (24, 2048, 9001), (31, 72, 129), (127, 200, 300), (257, 648, 1003),
          (300, 4096, 2048), (1000, 256, 3001), (2049, 64, 50), (513, 1536, 20000), (5000, 128, 1000)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_forward(T, d, V):
    check_forward(T, d, V, seed=T + V)


@pytest.mark.gpu
def test_forward_takes_32_bit_labels():
    check_forward(200, 136, 777, torch.int32)


def check_backward(T, d, V, idt=torch.int64, weighted=False, mean=True, scale=1.0, want=("dx", "dw"), seed=0):
    from paper_2409_12210_b200 import binding as B
    x, w, labels = problem(T, d, V, seed)
    rng = np.random.default_rng(seed + 1)
    lab = torch.from_numpy(labels).to(idt).cuda()
    _, rlse, _, _ = forward64(x, w, labels)
    lse = rlse.float()
    count = max(int((labels >= 0).sum()), 1)
    total = torch.tensor([1.0, count], device="cuda") if mean else None
    dloss = torch.from_numpy((rng.random(T) - 0.3).astype(np.float32)).cuda() if weighted else None
    (dx, m0), (dw, m1) = guarded((T, d), torch.bfloat16), guarded((V, d), torch.bfloat16)
    dx.fill_(float("nan"))
    dw.fill_(float("nan"))
    ws, m2 = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    call = lambda: B.cross_entropy_backward(x, w, lab, lse, dx if "dx" in want else None, dw if "dw" in want else None, ws,
                                            dloss=dloss, total=total, scale=scale)
    call()
    assert B.check_workspace_status(ws) == B.MODSE_OK
    assert bool((m0 == 3).all()) and bool((m1 == 3).all()) and bool((m2 == 0xA5).all())
    z, S = logits64(x, w)
    f = torch.from_numpy((labels >= 0).astype(np.float64) * scale / (count if mean else 1)).cuda()
    if weighted:
        f = f * dloss.double()
    p = torch.exp(z - rlse[:, None])
    onehot = torch.zeros_like(p)
    at = torch.from_numpy(np.nonzero(labels >= 0)[0]).cuda()
    onehot[at, torch.from_numpy(labels[labels >= 0]).cuda()] = 1.0
    dz = f[:, None] * (p - onehot)
    # lse is handed over rounded, 2^-24 of itself, and once more times log2 e
    edz = f.abs()[:, None] * (p * ((d + 8) * 2.0 ** -23 * S + exponent_error(z) + 3 * U * L2E * rlse.abs()[:, None]) + 2 * U * (p + onehot) + 2.0 ** -126)
    edz = edz + 2 * U * dz.abs()
    unrounded = edz                 # of dz before its rounding to bf16
    edz = edz + BF * (dz.abs() + edz)
    xd, wd = x.double(), w.double()
    if "dx" in want:
        ref = dz @ wd
        tol = edz @ wd.abs() + (V + 64) * 2.0 ** -23 * (dz.abs() @ wd.abs())
        assert bool(((dx.double() - ref).abs() <= tol + BF * (ref.abs() + tol)).all())
        assert not bool(dx[torch.from_numpy(labels < 0).cuda()].any())
        # far inside those bounds on the whole: one rounding of dz and one of the output, each at most 2^-8 / sqrt(3) in norm,
        # on top of what the fp32 arithmetic ahead of them is off by.  That part does not shrink with the result: with
        # p = 1 - q the difference p - 1 = -q keeps p's error of (ez + exponent terms) p, however small q is (a vocabulary of
        # one word has q = 0 and p = 1 + 3e-7).
        fp32 = unrounded @ wd.abs() + (V + 64) * 2.0 ** -23 * (dz.abs() @ wd.abs())
        assert float((dx.double() - ref).norm()) <= 1.5 * 2.0 ** -8 / 3 ** 0.5 * 2 ** 0.5 * float(ref.norm()) + float(fp32.norm())
    else:
        assert bool(dx.isnan().all())
    if "dw" in want:
        ref = dz.T @ xd
        tol = edz.T @ xd.abs() + (T + 64) * 2.0 ** -23 * (dz.abs().T @ xd.abs())
        assert bool(((dw.double() - ref).abs() <= tol + BF * (ref.abs() + tol)).all())
        fp32 = unrounded.T @ xd.abs() + (T + 64) * 2.0 ** -23 * (dz.abs().T @ xd.abs())
        assert float((dw.double() - ref).norm()) <= 1.5 * 2.0 ** -8 / 3 ** 0.5 * 2 ** 0.5 * float(ref.norm()) + float(fp32.norm())
    else:
        assert bool(dw.isnan().all())
    first = dx.clone(), dw.clone()
    call()
    if "dx" in want:
        assert torch.equal(dx, first[0])
    if "dw" in want:
        assert torch.equal(dw, first[1])


# one piece and several, the last of them narrower; odd vocabularies; dx cut along the vocabulary; short contractions
GRADS = [(1, 8, 1), (1, 256, 3001), (3, 64, 7), (24, 512, 9001), (31, 72, 129), (127, 200, 300), (257, 648, 1003),
         (300, 1024, 2048), (1000, 256, 3001), (2049, 64, 50), (9000, 64, 15001), (16500, 72, 9001), (35000, 64, 4500)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", GRADS)
def test_gradient(T, d, V):
    check_backward(T, d, V, seed=T + V)


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(weighted=True), dict(mean=False, scale=-0.25), dict(idt=torch.int32, weighted=True, mean=False),
                                dict(want=("dx",)), dict(want=("dw",))])
@pytest.mark.parametrize("T,d,V", [(50, 128, 333), (9000, 64, 15001)])
def test_gradient_forms(T, d, V, kw):
    check_backward(T, d, V, **kw)


@pytest.mark.gpu
def test_gradient_is_the_derivative():
    """Of the mean loss, by differences along random directions."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 60, 64, 200
    x, w, labels = problem(T, d, V, 4)
    lab = torch.from_numpy(labels).cuda()
    loss, lse, total = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.cross_entropy(x, w, lab, loss, lse, ws, total=total)
    B.cross_entropy_backward(x, w, lab, lse, dx, dw, wsb, total=total)

    def mean(a, b):
        return float(forward64(a, b, labels)[0].sum()) / float(total[1])
    g = torch.Generator(device="cuda").manual_seed(0)
    for which in (0, 1):
        t = (x, w)[which].double()
        v = torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64)
        args = lambda s: (t + s * v, w) if which == 0 else (x, t + s * v)
        h = 1e-5
        slope = (mean(*args(h)) - mean(*args(-h))) / (2 * h)
        got = (dx, dw)[which].double()
        # each element of the gradient carries two bf16 roundings; the difference's own error is about h^2
        assert abs(slope - float((got * v).sum())) <= 3 * 2.0 ** -8 * float((got.abs() * v.abs()).sum()) ** 1.0 * 0.2 + 1e-7


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 9000])
def test_labels_past_the_vocabulary_are_reported_and_left_out(T):
    from paper_2409_12210_b200 import binding as B
    d, V = 64, 300
    x, w, labels = problem(T, d, V, 7)
    labels[T // 2] = V - 1
    for idt, far in [(torch.int32, V), (torch.int64, 2 ** 40 + 1)]:
        bad, none = labels.copy(), labels.copy()
        bad[T // 2], none[T // 2] = far, -1
        outs = []
        for lab, want in ((bad, B.MODSE_ERR_DEVICE_BOUNDS), (none, B.MODSE_OK)):
            lab = torch.from_numpy(lab).to(idt).cuda()
            loss, lse, total = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, device="cuda")
            ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
            wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
            dx, dw = torch.empty_like(x), torch.empty_like(w)
            B.cross_entropy(x, w, lab, loss, lse, ws, total=total)
            B.cross_entropy_backward(x, w, lab, lse, dx, dw, wsb, scale=0.5)
            assert B.check_workspace_status(ws) == want and B.check_workspace_status(wsb) == want
            outs.append((loss, lse, total, dx, dw))
        assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.gpu
def test_infinities_nan_and_rows_that_do_not_count():
    from paper_2409_12210_b200 import binding as B
    T, d, V = 10, 64, 500
    x, w, _ = problem(T, d, V, 9)
    w[:, 0] = 1.0
    w[7, 0] = -1.0
    labels = torch.arange(T, device="cuda")
    inf = float("inf")
    x[0, 3] = float("nan")          # a NaN: all of the row
    x[1, 0] = inf                   # logits of +inf, and one of -inf
    x[2, 0] = -inf                  # logits of -inf but one
    x[3, 3], labels[3] = float("nan"), -100
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    total = torch.empty(2, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    B.cross_entropy(x, w, labels, loss, lse, ws, total=total)
    assert bool(lse[[0, 3]].isnan().all()) and bool(loss[0].isnan()) and float(loss[3]) == 0.0
    assert float(lse[1]) == inf and float(lse[2]) == inf
    rest = torch.tensor([4, 5, 6, 7, 8, 9], device="cuda")
    ref = forward64(x[rest], w, labels[rest].cpu().numpy())
    assert bool(((loss[rest].double() - ref[0]).abs() <= ref[3]).all()) and float(total[1]) == T - 1
    # the rows of the gradient stay apart: what does not count or has no weight gives nothing
    dloss = torch.ones(T, device="cuda")
    dloss[:3] = 0
    wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.cross_entropy_backward(x, w, labels, lse, dx, None, wsb, dloss=dloss)
    assert not bool(dx[:4].any()) and bool(torch.isfinite(dx.float()).all()) and bool(dx[4:].any(1).all())


@pytest.mark.gpu
def test_large_logits_neither_overflow_nor_vanish():
    """Logits of hundreds: the exponentials of the raw numbers would overflow."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 70, 64, 1000
    x, w, labels = problem(T, d, V, 11, std=60.0)
    lab = torch.from_numpy(labels).cuda()
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    for sign in (1.0, -1.0):
        B.cross_entropy(x * sign, w, lab, loss, lse, ws)
        rloss, rlse, e_lse, e_loss = forward64(x * sign, w, labels)
        assert bool(((lse.double() - rlse).abs() <= e_lse).all()) and bool(((loss.double() - rloss).abs() <= e_loss).all())


@pytest.mark.gpu
def test_no_tokens_and_nothing_counted():
    from paper_2409_12210_b200 import binding as B
    d, V = 64, 100
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w, none, f = torch.empty(0, d, **bf), torch.randn(V, d, **bf), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    ws, _ = workspace(1 << 16)
    total, dw = torch.ones(2, device="cuda"), torch.ones(V, d, **bf)
    B.cross_entropy(x, w, none, f, f, ws, total=total)
    assert B.check_workspace_status(ws) == B.MODSE_OK and not bool(total.any())
    B.cross_entropy_backward(x, w, none, f, x, dw, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK and not bool(dw.any())
    T = 40
    x, lab = torch.randn(T, d, **bf), torch.full((T,), -1, device="cuda")
    loss, lse = torch.ones(T, device="cuda"), torch.empty(T, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    B.cross_entropy(x, w, lab, loss, lse, ws, total=total)
    assert not bool(loss.any()) and not bool(total.any())
    wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    dx, dw = torch.ones_like(x), torch.ones_like(w)
    B.cross_entropy_backward(x, w, lab, lse, dx, dw, wsb, total=total)      # a mean of nothing: no gradient
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.gpu
def test_replayed_graph_and_side_stream():
    from paper_2409_12210_b200 import binding as B
    T, d, V = 700, 256, 3000
    mk = lambda seed: problem(T, d, V, seed)
    x, w, labels = mk(0)
    lab = torch.from_numpy(labels).cuda()
    new = lambda *s: torch.empty(*s, device="cuda")
    loss, lse, total, dx, dw = new(T), new(T), new(2), torch.empty_like(x), torch.empty_like(w)
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    torch.cuda.synchronize()

    def step():
        B.cross_entropy(x, w, lab, loss, lse, ws, total=total)
        B.cross_entropy_backward(x, w, lab, lse, dx, dw, wsb, total=total)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    ws2, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    loss2, lse2 = new(T), new(T)
    for seed in (1, 2, 3):
        a, b, c = mk(seed)
        x.copy_(a); w.copy_(b); lab.copy_(torch.from_numpy(c))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            B.cross_entropy(x, w, lab, loss2, lse2, ws2)
        torch.cuda.synchronize()
        first = [t.clone() for t in (loss, lse, total, dx, dw)]
        step()
        assert all(torch.equal(p, q) for p, q in zip(first, (loss, lse, total, dx, dw)))
        assert torch.equal(loss2, loss) and torch.equal(lse2, lse)
        rloss, _, _, e_loss = forward64(x, w, c)
        assert bool(((loss.double() - rloss).abs() <= e_loss).all())


def test_refusals_need_no_gpu():
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    lib, p = B.load(), 0x1000

    def fwd(T=4, d=64, V=10, ws=p, n=1 << 30, **kw):
        a = dict(x=p, w=p, labels=p, loss=p, lse=p, total=p, label_bytes=8)
        a.update(kw)
        return lib.modse_cross_entropy(T, d, V, B._CrossEntropy(**a), ws, n, None)

    def bwd(T=4, d=64, V=10, ws=p, n=1 << 30, **kw):
        a = dict(x=p, w=p, labels=p, lse=p, dloss=p, total=p, dx=p, dw=p, scale=1.0, label_bytes=8)
        a.update(kw)
        return lib.modse_cross_entropy_backward(T, d, V, B._CrossEntropyGrads(**a), ws, n, None)

    bad = [dict(T=-1), dict(d=60), dict(d=0), dict(V=0), dict(V=2 ** 28 + 1), dict(T=2 ** 28 + 1), dict(T=2 ** 28, V=2 ** 28),
           dict(label_bytes=2), dict(x=None), dict(x=p + 8), dict(w=None), dict(w=p + 8), dict(labels=None), dict(labels=p + 4),
           dict(lse=None), dict(lse=p + 2), dict(total=p + 2), dict(ws=None), dict(ws=p + 16)]
    for kw in bad + [dict(loss=None), dict(loss=p + 2)]:
        assert fwd(**kw) == B.MODSE_ERR_INVALID_ARG, kw
    for kw in bad + [dict(dx=p + 8), dict(dw=p + 8), dict(dx=None, dw=None), dict(dloss=p + 2)]:
        assert bwd(**kw) == B.MODSE_ERR_INVALID_ARG, kw
    assert lib.modse_cross_entropy(4, 64, 10, None, p, 1 << 30, None) == B.MODSE_ERR_INVALID_ARG
    assert lib.modse_cross_entropy_backward(4, 64, 10, None, p, 1 << 30, None) == B.MODSE_ERR_INVALID_ARG
    for size, call in ((B.cross_entropy_workspace_bytes, fwd), (B.cross_entropy_backward_workspace_bytes, bwd)):
        need = size(4, 64, 10)
        assert need > 0 and call(n=need - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
        for args in [(-1, 64, 10), (4, 60, 10), (4, 64, 0)]:
            assert size(*args) == 0


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    from paper_2409_12210_b200 import binding as B
    mk = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    bf = torch.bfloat16
    x, w, lab, v, ws = mk(4, 64, dt=bf), mk(10, 64, dt=bf), mk(4, dt=torch.int64), mk(4), mk(1 << 20, dt=torch.uint8)
    for call in (lambda: B.cross_entropy(x, w.float(), lab, v, v, ws), lambda: B.cross_entropy(x, w[:, :56], lab, v, v, ws),
                 lambda: B.cross_entropy(x, w, lab[:3], v, v, ws), lambda: B.cross_entropy(x, w, lab.cpu(), v, v, ws),
                 lambda: B.cross_entropy(x, w, lab, v.double(), v, ws), lambda: B.cross_entropy(x.float(), w, lab, v, v, ws),
                 lambda: B.cross_entropy(x, w, lab, v, v, ws, total=mk(3)),
                 lambda: B.cross_entropy_backward(x, w, lab, v, x.T, w, ws),
                 lambda: B.cross_entropy_backward(x, w, lab, v, x, w, ws, dloss=mk(5))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        B.cross_entropy(x, w, lab.float(), v, v, ws)


@pytest.mark.gpu
def test_a_vocabulary_past_32_bits():
    """More than 2^31 elements in w and dw: logits of zero but for the last rows."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 6, 2048, 1_100_003
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[-3:] = torch.randn(3, d, generator=g, device="cuda").bfloat16() * 0.1
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    labels = torch.tensor([V - 1, V - 2, V - 3, 0, -1, V - 1], device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    B.cross_entropy(x, w, labels, loss, lse, ws)
    z = x.double() @ w[-3:].double().T
    ref = torch.logsumexp(torch.cat([z, torch.full((T, 1), float(np.log(V - 3)), dtype=torch.float64, device="cuda")], 1), 1)
    own = torch.stack([z[0, 2], z[1, 1], z[2, 0], z[3, 0] * 0, z[4, 0] * 0, z[5, 2]])
    want = torch.where(labels >= 0, ref - own, 0.0)
    # logits of at most 30, each off by (d + 8) 2^-23 of a sum of magnitudes below 200
    assert float((lse.double() - ref).abs().max()) <= 0.06 and float((loss.double() - want).abs().max()) <= 0.1
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    B.cross_entropy_backward(x, w, labels, lse, dx, dw, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    dz = torch.exp(z - ref[:, None]) * (labels >= 0)[:, None]
    for t, c in ((0, 2), (1, 1), (2, 0), (5, 2)):
        dz[t, c] -= 1
    got, exact = dw[-3:].double(), dz.T @ x.double()
    assert float((got - exact).norm()) <= 0.02 * float(exact.norm())
    exact = dz @ w[-3:].double()
    assert float((dx.double() - exact).norm()) <= 0.02 * float(exact.norm())
    # the row of token 3's label, and one that nobody names: p x summed over the counted rows
    p0 = torch.exp(-ref) * (labels >= 0)
    far = dw[V // 2].double()
    assert float((far - p0 @ x.double()).norm()) <= 0.02 * float(far.norm())


@pytest.mark.gpu
def test_an_expired_wait_is_reported():
    from paper_2409_12210_b200 import binding as B
    T, d, V = 40, 64, 300
    x, w, labels = problem(T, d, V, 7)
    lab = torch.from_numpy(labels).cuda()
    loss, lse, dx, dw = torch.empty(T, device="cuda"), torch.zeros(T, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    wsb, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    B.debug_set_wait_limit_ms(50)
    B.debug_skip_tile_loads(6, 0)
    try:
        B.cross_entropy(x, w, lab, loss, lse, ws)
        assert B.check_workspace_status(ws) == B.MODSE_ERR_DEVICE_TIMEOUT
        B.cross_entropy_backward(x, w, lab, lse, dx, dw, wsb)
        assert B.check_workspace_status(wsb) == B.MODSE_ERR_DEVICE_TIMEOUT
    finally:
        B.debug_skip_tile_loads(-1, -1)
        B.debug_set_wait_limit_ms(2000)
    B.cross_entropy(x, w, lab, loss, lse, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    rloss, _, _, e_loss = forward64(x, w, labels)
    assert bool(((loss.double() - rloss).abs() <= e_loss).all())


@pytest.mark.gpu
def test_a_factor_that_all_rows_share_costs_no_precision():
    """A mean over 7372 tokens, or weights that are all 1 / 3: the gradient is as exact as that of the sum."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 500, 128, 900
    x, w, labels = problem(T, d, V, 13)
    lab = torch.from_numpy(labels).cuda()
    _, rlse, _, _ = forward64(x, w, labels)
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    z, _ = logits64(x, w)
    p = torch.exp(z - rlse[:, None])
    at = np.nonzero(labels >= 0)[0]
    p[torch.from_numpy(at).cuda(), torch.from_numpy(labels[at]).cuda()] -= 1
    p *= torch.from_numpy((labels >= 0).astype(np.float64)).cuda()[:, None]
    third = torch.full((T,), 1 / 3, device="cuda")
    for kw, f in ((dict(total=torch.tensor([1.0, 7372.0], device="cuda")), 1 / 7372), (dict(dloss=third), float(third[0])), (dict(scale=0.1), float(np.float32(0.1)))):
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        B.cross_entropy_backward(x, w, lab, rlse.float(), dx, dw, ws, **kw)
        for got, ref in ((dx, f * p @ w.double()), (dw, f * p.T @ x.double())):
            # dz and the output are rounded to bf16 once each, 2^-8 / sqrt(3) of a typical element at most: together 0.0032, on
            # average over the positions inside a binade 0.0024; a shared factor's own rounding would come on top, up to 0.0039
            assert float((got.double() - ref).norm()) <= 0.0028 * float(ref.norm())


# Few rows go through a kernel of their own: tiles of 8 rows of w to 128, one or several a block, the last one cut; one to many
# column blocks, odd numbers of them and a last one that is cut
@pytest.mark.gpu
@pytest.mark.parametrize("d,V", [(8, 1), (64, 9), (72, 1184), (1000, 1185), (192, 18944), (64, 18945), (136, 40003), (4096, 700)])
def test_forward_of_few_rows(d, V):
    for T in (1, 2, 15, 16, 17, 32, 33):
        check_forward(T, d, V, torch.int32 if T % 2 else torch.int64, seed=T)


@pytest.mark.gpu
def test_few_rows_in_the_workspace_of_many():
    from paper_2409_12210_b200 import binding as B
    for d, V in ((64, 1184), (256, 3001)):
        sizes = [B.cross_entropy_workspace_bytes(T, d, V) for T in range(1, 80)]
        assert sizes == sorted(sizes)
        x, w, labels = problem(79, d, V, V)
        lab, (ws, guard) = torch.from_numpy(labels).cuda(), workspace(sizes[-1])
        rloss, rlse, e_lse, e_loss = forward64(x, w, labels)
        for T in (79, 20, 64, 1, 33, 32):
            loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
            B.cross_entropy(x[:T], w, lab[:T], loss, lse, ws)
            assert bool(((loss.double() - rloss[:T]).abs() <= e_loss[:T]).all()) and bool(((lse.double() - rlse[:T]).abs() <= e_lse[:T]).all())
        assert bool((guard == 0xA5).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 30])
def test_an_expired_wait_of_few_rows_is_reported(T):
    """One tile is not asked for: nothing is in flight when its block gives up."""
    from paper_2409_12210_b200 import binding as B
    x, w, labels = problem(T, 640, 40000, 7)
    lab, (ws, _) = torch.from_numpy(labels).cuda(), workspace(B.cross_entropy_workspace_bytes(T, 640, 40000))
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    B.debug_set_wait_limit_ms(50)
    B.debug_skip_tile_loads(6, 200)
    try:
        B.cross_entropy(x, w, lab, loss, lse, ws)
        assert B.check_workspace_status(ws) == B.MODSE_ERR_DEVICE_TIMEOUT
    finally:
        B.debug_skip_tile_loads(-1, -1)
        B.debug_set_wait_limit_ms(2000)
    B.cross_entropy(x, w, lab, loss, lse, ws)
    rloss, _, _, e_loss = forward64(x, w, labels)
    assert B.check_workspace_status(ws) == B.MODSE_OK and bool(((loss.double() - rloss).abs() <= e_loss).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d,V", [(8192, 300), (5000, 7200), (8192, 7000)])       # long rows: either way, by the tiles' height
def test_forward_of_few_long_rows(d, V):
    for T in (1, 32):
        check_forward(T, d, V, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("weight", [float("inf"), float("nan")])
def test_a_weight_without_measure_is_seen_where_it_belongs(weight):
    """One row weighs infinitely much or NaN and the others nothing, or as ever: its own gradient shows it, theirs do not."""
    from paper_2409_12210_b200 import binding as B
    T, d, V = 40, 64, 300
    x, w, labels = problem(T, d, V, 3)
    labels[:] = np.arange(T) % V
    lab = torch.from_numpy(labels).cuda()
    _, rlse, _, _ = forward64(x, w, labels)
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    for others in (0.0, 0.5):
        dloss = torch.full((T,), others, device="cuda")
        dloss[7] = weight
        dx, dw, ref = torch.empty_like(x), torch.empty_like(w), torch.empty_like(x)
        B.cross_entropy_backward(x, w, lab, rlse.float(), dx, dw, ws, dloss=dloss)
        assert not bool(torch.isfinite(dx[7]).any()) and not bool(torch.isfinite(dw.float()).any())
        dloss[7] = 0
        B.cross_entropy_backward(x, w, lab, rlse.float(), ref, None, ws, dloss=dloss)
        keep = torch.arange(T, device="cuda") != 7
        assert torch.equal(dx[keep], ref[keep]) and bool(torch.isfinite(ref.float()).all())


@pytest.mark.gpu
def test_forward_of_many_rows_past_32_bits():
    from paper_2409_12210_b200 import binding as B
    T, d, V = 300, 2048, 1_050_001
    g = torch.Generator(device="cuda").manual_seed(4)
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[-5:] = (torch.randn(5, d, generator=g, device="cuda") * 0.1).bfloat16()
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    labels = V - 1 - torch.arange(T, device="cuda") % 5
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    B.cross_entropy(x, w, labels, loss, lse, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    z = x.double() @ w[-5:].double().T
    ref = torch.logsumexp(torch.cat([z, torch.full((T, 1), float(np.log(V - 5)), dtype=torch.float64, device="cuda")], 1), 1)
    want = ref - z.gather(1, (labels - (V - 5))[:, None])[:, 0]
    # a logit is off by (d + 8) 2^-23 of its magnitudes' sum, which is below 200 here, twice; the sum of V / 128 runs by (160 + V / 128) 2^-24
    assert float((lse.double() - ref).abs().max()) <= 0.06 and float((loss.double() - want).abs().max()) <= 0.1
