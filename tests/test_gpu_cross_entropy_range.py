"""The cross entropy and its gradient over the range of logits that the header promises, against 64 bits.

Rows of x and w with one number that is not zero make logits that are one exact product, whatever order sums take: nothing is
left but the softmax's own arithmetic.  Bounds.  z - top is rounded once, 2^-24 of it; where the exponential is not all but zero
(2^-130) it is below 130 / log2 e, and so is its product with log2 e, rounded once more: 2 2^-24 130 of the exponential, whose
own arithmetic takes 2^-21; the runs add (160 + V / 128) 2^-24, the logarithm 2^-22 of at most 13.  lse and loss are one rounded sum each on
top, 2^-24 of themselves.  A probability of the gradient is exp(z - lse) of the lse handed over: off by the same of itself."""
import numpy as np
import pytest

from test_gpu_cross_entropy import check_backward, workspace

torch = pytest.importorskip("torch")

U, BF = 2.0 ** -24, 2.0 ** -8
EXPONENT = 2 * U * 130 + 2.0 ** -21


def exact_problem(T, V, size, seed=0, d=8):
    """Logits x[t, 0] w[v, 0] of magnitudes up to `size`, of either sign."""
    rng = np.random.default_rng(seed)
    x, w = torch.zeros(T, d, dtype=torch.bfloat16), torch.zeros(V, d, dtype=torch.bfloat16)
    x[:, 0] = torch.from_numpy((size ** 0.5 * rng.choice([-1, 1], T)).astype(np.float32)).bfloat16()
    w[:, 0] = torch.from_numpy((size ** 0.5 * rng.uniform(0.5, 1, V)).astype(np.float32)).bfloat16()
    return x.cuda(), w.cuda(), torch.from_numpy(rng.integers(0, V, T)).cuda()


def forward(x, w, labels):
    from paper_2409_12210_b200 import binding as B
    T, d, V = *x.shape, w.shape[0]
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ws, _ = workspace(B.cross_entropy_workspace_bytes(T, d, V))
    B.cross_entropy(x, w, labels, loss, lse, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    return loss, lse


# A few rows and many go through kernels of their own.
@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 30, 70, 300])
@pytest.mark.parametrize("V", [3, 1000])
@pytest.mark.parametrize("size", [1.0, 200.0, 1e5, 1e7, 1.5e9, 3.1e9, 8657043456.0, 1e20, 1.9e38])
def test_forward_of_exact_logits(T, V, size):
    x, w, labels = exact_problem(T, V, size, T + V)
    z = x.double() @ w.double().T
    top, at = z.max(1)
    labels[::2] = at[::2]                            # the right answer, or any other
    loss, lse = forward(x, w, labels)
    rlse = torch.logsumexp(z, 1)
    rloss = rlse - z.gather(1, labels[:, None])[:, 0]
    e = EXPONENT + (160 + V / 128) * U + 2.0 ** -22 * 13
    assert bool(((lse.double() - rlse).abs() <= e + U * rlse.abs()).all())
    assert bool(((loss.double() - rloss).abs() <= e + U * rlse.abs() + U * rloss.abs()).all())
    # where one word has all the weight, lse is its logit, and so is the loss of another word their distance
    alone = ((top[:, None] - z) > 110).sum(1) == V - 1
    assert torch.equal(lse[alone].double(), top.float()[alone].double())
    assert not bool(loss[alone & (labels == at)].any())
    assert bool(alone.any()) or size < 1e5 or V > 3      # (among many words the largest number comes more than once)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(1, 8), (24, 200), (70, 200), (500, 1032)])
def test_a_vocabulary_of_one_word_has_no_loss(T, d):
    from paper_2409_12210_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T)
    for std in (1.0, 15.0):
        x = (torch.randn(T, d, generator=g, device="cuda") * std).bfloat16()
        w = torch.randn(1, d, generator=g, device="cuda").bfloat16()
        labels = torch.zeros(T, dtype=torch.int64, device="cuda")
        loss, lse = forward(x, w, labels)
        assert not bool(loss.any())


@pytest.mark.gpu
@pytest.mark.parametrize("T,V", [(5, 3), (40, 1000), (300, 1000), (9000, 9001)])
@pytest.mark.parametrize("size", [1.0, 200.0, 1e5, 1e7, 1e8, 3.1e9, 1e20])
def test_gradient_of_exact_logits(T, V, size):
    """dx alone, against probabilities of the lse handed over; the columns behind the first one are there to be zeros."""
    from paper_2409_12210_b200 import binding as B
    x, w, labels = exact_problem(T, V, size, T + V)
    w[:, 1] = 1.0                                    # x[:, 1] is 0, so that dx[:, 1] is the sum of dz, of moderate terms
    d = x.shape[1]
    z = x.double() @ w.double().T
    _, lse = forward(x, w, labels)
    top, at = z.max(1)
    labels[::2] = at[::2]
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    B.cross_entropy_backward(x, w, labels, lse, dx, dw, ws)
    p = torch.exp(z - lse.double()[:, None])
    assert float(p.max()) <= 1.0
    dz = p.scatter_add(1, labels[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device="cuda"))
    edz = p * EXPONENT + U * dz.abs()
    edz = edz + BF * (dz.abs() + edz) + 2.0 ** -126
    for got, ref, tol in ((dx, dz @ w.double(), edz @ w.double().abs() + (V + 64) * 2.0 ** -23 * (dz.abs() @ w.double().abs())),
                          (dw, dz.T @ x.double(), edz.T @ x.double().abs() + (T + 64) * 2.0 ** -23 * (dz.abs().T @ x.double().abs()))):
        assert bool(((got.double() - ref).abs() <= tol + BF * (ref.abs() + tol)).all())
    # one word has all the weight and is the right one: nothing to learn
    alone = (((top[:, None] - z) > 130).sum(1) == V - 1) & (labels == at)
    assert not bool(dx[alone].any())


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [(8, 2048, 1000), (24, 4096, 1000), (70, 2048, 1), (2051, 4096, 1000), (300, 648, 1)])
@pytest.mark.parametrize("size", [30.0, 3e5, 3e12])
def test_no_probability_is_above_one(T, d, V, size):
    """Logits of 1e5 to 1e26 out of sums that round: forward and backward cut them at different places in some of these shapes.
    For the word that has all the weight, and is the right one, dz is p - 1, between -1 and 0; dx is that times its row of w."""
    from paper_2409_12210_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T + d)
    x, w = ((torch.randn(n, d, generator=g, device="cuda") * size).bfloat16() for n in (T, V))
    z = x.double() @ w.double().T
    top, at = z.max(1)
    # alone by more than the rounding of any sum
    S = x.double().abs() @ w.double().abs().T
    alone = (((top[:, None] - z) > 110 + 2 * (d + 8) * 2.0 ** -23 * S).sum(1) == V - 1)
    assert bool(alone.any())
    _, lse = forward(x, w, at)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    B.cross_entropy_backward(x, w, at, lse, dx, dw, ws)
    row = w[at].double()
    dz = (dx.double() * row).sum(1) / row.square().sum(1)
    assert bool(torch.isfinite(dx.float()).all()) and bool(torch.isfinite(dw.float()).all())
    # dz and the elements of dx are rounded to bf16 once each
    assert bool((dz[alone] <= 0).all()) and bool((dz[alone] >= -1 - 2 * BF).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 9000])
def test_a_scale_of_zero_gives_nothing(T):
    """f is 0 in every row, so that NaN and infinite logits give nothing either."""
    from paper_2409_12210_b200 import binding as B
    d, V = 64, 9001
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.randn(T, d, generator=g, device="cuda").bfloat16(), torch.randn(V, d, generator=g, device="cuda").bfloat16()
    labels = torch.arange(T, device="cuda") % V
    _, lse = forward(x, w, labels)
    lse[3], lse[4], lse[5] = float("nan"), float("inf"), float("-inf")
    ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
    total = torch.tensor([1.0, T], device="cuda")
    for kw in (dict(), dict(total=total), dict(dloss=torch.rand(T, device="cuda"))):
        dx, dw = torch.ones_like(x), torch.ones_like(w)
        B.cross_entropy_backward(x, w, labels, lse, dx, dw, ws, scale=0.0, **kw)
        assert not bool(dx.any()) and not bool(dw.any())


# More rows are worked off in narrower pieces, which need less; the sizes do not fall all the same.
@pytest.mark.parametrize("d,V", [(2048, 32000), (1536, 100003), (64, 9001), (520, 3100), (4096, 1000), (8, 1)])
def test_workspace_sizes_never_fall_with_the_rows(d, V):
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    rows = list(range(0, 400)) + list(range(400, 9000, 7)) + list(range(9000, 70000, 331)) + [670, 671, 672, 2096, 2097, 2098, 4096]
    for size in (B.cross_entropy_workspace_bytes, B.cross_entropy_backward_workspace_bytes):
        sizes = [size(T, d, V) for T in sorted(rows)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    # what the header says of the gradient's: a piece's dz and up to eight sums of dx, beside cut tiles and a number a row
    for T in (1, 300, 2097, 8192, 30000):
        sums = 8 * ((T + 31) // 32 * 32) * ((d + 31) // 32 * 32) * 4
        most = 2 * max(2 ** 26 + 255 * T, 2048 * T) + sums + 128 * 2 ** 18 + 4 * T + 2 ** 16
        assert B.cross_entropy_backward_workspace_bytes(T, d, V) <= most


@pytest.mark.gpu
def test_few_rows_of_the_gradient_in_the_workspace_of_many():
    from paper_2409_12210_b200 import binding as B
    d, V, most = 72, 32000, 4096
    x, w, labels = (t.contiguous() for t in exact_problem(most, V, 200.0, 1, d))
    _, lse = forward(x, w, labels)
    ws, guard = workspace(B.cross_entropy_backward_workspace_bytes(most, d, V))
    for T in (4096, 2097, 2098, 1, 33, 700):
        own, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
        outs = []
        for buf in (ws, own):
            dx, dw = torch.empty_like(x[:T]), torch.empty_like(w)
            B.cross_entropy_backward(x[:T], w, labels[:T], lse[:T], dx, dw, buf)
            assert B.check_workspace_status(buf) == B.MODSE_OK
            outs.append((dx, dw))
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert bool((guard == 0xA5).all())


# Gradients of training size: dx and dw come out of tiles of 512 rows, dx on top of the piece ahead (two pieces, a sum each), out of
# four sums that are joined (one piece), both (two pieces, two sums each), and both in tiles of 256 rows (100003 words); rows, words
# and columns all end inside a tile, and the last round of tiles is halved in the second and third of them.
@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [(5000, 2056, 20011), (2051, 1544, 30011), (4649, 936, 26151), (2051, 1536, 100003)])
def test_gradient_of_training_size(T, d, V):
    check_backward(T, d, V, weighted=T == 2051, seed=V)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 3000])
def test_rows_of_x_that_do_not_count(T):
    """Their dz is 0 whatever their logits are: nothing reaches dx, and dw = dz^T x is as if they were zeros but for the columns
    where they hold an infinity or a NaN, which 0 times is a NaN."""
    from paper_2409_12210_b200 import binding as B
    d, V = 136, 9001
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.randn(T, d, generator=g, device="cuda").bfloat16(), torch.randn(V, d, generator=g, device="cuda").bfloat16()
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels[[3, 4, T - 1]] = torch.tensor([-1, -100, -1], device="cuda")
    x[[3, 4, T - 1]] = 0
    outs = []
    for bad in (False, True):
        if bad:
            x[3, 3], x[4, 0], x[4, 100], x[T - 1, 70] = float("nan"), float("inf"), 1e30, float("-inf")
        loss, lse = forward(x, w, labels)
        ws, _ = workspace(B.cross_entropy_backward_workspace_bytes(T, d, V))
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        B.cross_entropy_backward(x, w, labels, lse, dx, dw, ws)
        outs.append((loss, dx, dw))
    (loss, dx, dw), (loss2, dx2, dw2) = outs
    assert torch.equal(loss, loss2) and torch.equal(dx, dx2) and not bool(dx2[[3, 4, T - 1]].any())
    apart = torch.ones(d, dtype=torch.bool, device="cuda")
    apart[[0, 3, 70]] = False
    assert torch.equal(dw[:, apart], dw2[:, apart]) and bool(dw2[:, ~apart].isnan().all())
