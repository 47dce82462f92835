"""modse_decode where a router logit is NaN, against the definition: softmax over the kept logits, the NaN first among them."""
import pytest

from test_gpu_decode import BF, F32, Problem, run, check

torch = pytest.importorskip("torch")


# routing by a thread a token and by a warp a token, in a kernel of its own; extents that are multiples of 64 and others
NAN_LAYERS = [(64, (96, 160, 112, 144), BF), (64, (96, 160, 112, 144), F32), (192, (64, 128, 192), BF), (64, (32,) * 40, BF),
              (128, (64,) * 40, BF), (64, (16,) * 200, F32)]


@pytest.mark.gpu
@pytest.mark.parametrize("d,widths,dtype", NAN_LAYERS)
@pytest.mark.parametrize("k", [1, 2])
def test_a_nan_logit_is_taken_and_seen(d, widths, dtype, k):
    """One expert's row of the router holds a NaN: every token meets it, and its output says so."""
    N = len(widths)
    p = Problem(d, widths, k, dtype, seed=N)
    layer = p.layer()
    for e in {0, 1, N // 2, N - 1}:
        p.w[0].copy_(Problem(d, widths, k, dtype, seed=N).w[0])
        z = p.logits(p.x)
        z[:, e] = -float("inf")
        second = z.argmax(1)
        p.w[0][e, 3] = float("nan")
        for T in (1, 5, 12, 32):
            y, idx, gate = run(p, T, layer, dtype)
            assert bool((idx[:, 0] == e).all()) and bool(gate.isnan().all()) and bool(y.isnan().all())
            if k == 2:
                assert torch.equal(idx[:, 1].long(), second[:T])
    # two of them: the lower index first
    p.w[0][0, 5] = float("nan")
    p.w[0][N - 1, 5] = float("nan")
    y, idx, _ = run(p, 12, layer, dtype)
    assert bool((idx[:, 0] == 0).all()) and bool(y.isnan().all())
    layer.destroy()
