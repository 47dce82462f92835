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


# The second product has a group of rows of W_down for a block: of 128 rows by TMA, of 16 otherwise.  More groups than blocks
# (148 and 444 at most): a block takes several, one after the other.
@pytest.mark.gpu
@pytest.mark.parametrize("d,widths,dtype", [(19072, (64, 128), BF), (40000, (128, 64), BF), (7208, (48, 16), BF), (7208, (48, 16), F32)])
def test_more_groups_of_rows_than_blocks(d, widths, dtype):
    p = Problem(d, widths, 2, dtype, seed=d)
    for T in (1, 3, 12, 32):
        check(p, T)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 12, 25])
@pytest.mark.parametrize("d,widths", [(64, (64, 128, 192, 64)), (576, (128, 384, 192, 320))])
def test_a_row_of_nan_or_infinity_stays_alone_in_whole_column_blocks(T, d, widths):
    p = Problem(d, widths, 2, BF, seed=T)
    layer = p.layer()
    clean, idx, _ = run(p, T, layer, BF)
    rest = [t for t in range(T) if t != 3]
    for bad in (float("nan"), float("inf")):
        x = p.x.clone()
        p.x[3, 5] = bad
        y, idx2, _ = run(p, T, layer, BF)
        assert torch.equal(y[rest], clean[rest]) and torch.equal(idx2[rest], idx[rest])
        assert not bool(torch.isfinite(y[3].float()).any()) and bool((idx2[3] >= 0).all()) and bool((idx2[3] < 4).all())
        p.x.copy_(x)
    layer.destroy()


@pytest.mark.gpu
def test_host_threads_that_share_a_layer():
    """Four threads, a stream and a workspace each, all at once."""
    import threading
    p = Problem(256, (128, 384, 192, 320), 2, BF)
    layer = p.layer()
    want = [torch.empty_like(p.x[:T]) for T in (1, 7, 16, 32)]
    ws = [layer.alloc_decode_workspace(BF) for _ in want]
    for y, w in zip(want, ws):
        layer.decode(*p.w, p.x[:len(y)], y, w)
    got = [torch.zeros_like(y) for y in want]
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    layer.decode(*p.w, p.x[:len(got[i])], got[i], ws[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:                       # shown by the assertion below
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and all(torch.equal(a, b) for a, b in zip(got, want))
    layer.destroy()
