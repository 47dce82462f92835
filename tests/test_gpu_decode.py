"""modse_decode - the layer for the few tokens of a generation step - against the layer's formulas in 64 bits, element by
element, and against modse_forward.

Bounds.  A product sums d exact (bf16) or once rounded (fp32) terms in fp32: (d + 8) 2^-23 of the sum S of their magnitudes.  A
gate's slope in a logit is at most g (1 - g), and two logits move it; its own arithmetic costs 2^-21 of it.  silu's slope is below 1.1, its
arithmetic 2^-21 of |a|.  The hidden value is rounded once (bf16: 2^-8 of it, fp32: 2^-24); the second product adds (sum of widths + 64)
2^-23 of its magnitudes, and the output its rounding.  Inputs keep the k-th and k+1-st logits of a token 1e-3 apart, so
that the routing is the same."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

F32, BF = torch.float32, torch.bfloat16
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
U23, U21 = 2.0 ** -23, 2.0 ** -21
BENCH = (2816, 8448, 3520, 7744, 4224, 7040, 4928, 6336)


class Problem:
    def __init__(self, d, widths, k, dtype, seed=0, noise=None, T=32):
        rng = np.random.default_rng(seed)
        mk = lambda *s, std=1.0: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32)).cuda().to(dtype)
        N, S = len(widths), sum(widths)
        self.d, self.widths, self.k, self.dtype, self.noise = d, widths, k, dtype, noise
        self.w = (mk(N, d, std=d ** -0.5), mk(S, d, std=d ** -0.5), mk(S, d, std=d ** -0.5), mk(d, S, std=(S / N) ** -0.5))
        self.wn = mk(N, d, std=d ** -0.5) if noise else None
        x = mk(T, d)
        for _ in range(20 if k < N else 0):
            z = self.logits(x).sort(dim=1, descending=True).values
            close = ((z[:, :k] - z[:, 1:k + 1]).min(1).values < 1e-3).nonzero()[:, 0]
            if len(close) == 0:
                break
            x[close] = mk(len(close), d)
        self.x = x

    def logits(self, x):
        z = x.double() @ self.w[0].double().T
        if self.noise:
            s = torch.nn.functional.softplus(x.double() @ self.wn.double().T)
            z = z + self.noise[0] * s / (s.square().mean(1, keepdim=True) + self.noise[1]).sqrt()
        return z

    def layer(self, out_f32=False):
        from paper_2409_12210_b200 import binding as B
        layer = B.ModseLayer(self.d, self.widths, self.k)
        if self.noise:
            layer.set_noise_gate(self.wn, *self.noise)
        layer.set_output_f32(out_f32)
        return layer

    def reference(self, x, out_dtype):
        """(y, bound of y, idx, gate, bound of gate) in 64 bits."""
        d, k = self.d, self.k
        z = self.logits(x)
        order = z.sort(dim=1, descending=True, stable=True)
        idx, gate = order.indices[:, :k], torch.softmax(order.values[:, :k], 1)
        ez = (d + 8) * U23 * (x.double().abs() @ self.w[0].double().abs().T)
        if self.noise:
            # the second term is gamma times a number of at most sqrt(N) whose slope in u is at most 2 sqrt(N) / |s|: softplus of
            # a unit normal keeps |s| / sqrt(N) above 0.5 here
            eu = (d + 8) * U23 * (x.double().abs() @ self.wn.double().abs().T)
            ez = ez + abs(self.noise[0]) * (4 * eu.max(1, keepdim=True).values * len(self.widths) ** 0.5 + U21 * len(self.widths) ** 0.5)
        e_top = ez.gather(1, idx).sum(1, keepdim=True)
        eg = gate * (1 - gate) * 1.1 * e_top + U21 * gate
        y, mag, err = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for _ in range(3))
        off = 0
        for e, h in enumerate(self.widths):
            t, j = (idx == e).nonzero(as_tuple=True)
            if len(t):
                r, wg, wu, wd = x[t].double(), *(m[off:off + h].double() for m in self.w[1:3]), self.w[3][:, off:off + h].double()
                a, b = r @ wg.T, r @ wu.T
                ea, eb = (d + 8) * U23 * (r.abs() @ wg.abs().T), (d + 8) * U23 * (r.abs() @ wu.abs().T)
                g, dg = gate[t, j][:, None], eg[t, j][:, None]
                silu = a * torch.sigmoid(a)
                v = g * silu * b
                ev = g * ((1.1 * ea + U21 * a.abs()) * b.abs() + silu.abs() * eb) + dg * (silu * b).abs() + 4 * U23 * v.abs()
                ev = ev + HALF[self.dtype] * (v.abs() + ev)
                y.index_add_(0, t, v @ wd.T)
                mag.index_add_(0, t, v.abs() @ wd.abs().T)
                err.index_add_(0, t, ev @ wd.abs().T)
            off += h
        tol = err + (sum(self.widths) + 64) * U23 * mag
        return y, tol + HALF[out_dtype] * (y.abs() + tol), idx, gate, eg


def same_bits(a, b):                                      # NaN equal to themselves
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def run(p, T, layer, out_dtype):
    from paper_2409_12210_b200 import binding as B
    base = torch.full((T * p.d + 512,), 3.0, dtype=out_dtype, device="cuda")
    y = base[:T * p.d].view(T, p.d)
    idx, gate = torch.full((T, p.k), -7, dtype=torch.int32, device="cuda"), torch.full((T, p.k), -7.0, device="cuda")
    code = B.MODSE_F32 if p.dtype == F32 else B.MODSE_BF16
    n = layer.decode_workspace_bytes(code, T)
    ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    call = lambda: layer.decode(*p.w, p.x[:T], y, ws[:n], topk_idx=idx, topk_gate=gate)
    call()
    first = y.clone()
    assert bool((base[T * p.d:] == 3).all()) and bool((ws[n:] == 0xA5).all())
    call()                                                # the same bits on a used workspace
    assert same_bits(first, y)
    y.fill_(1)
    layer.decode(*p.w, p.x[:T], y, ws[:n])                # without the routing
    assert same_bits(first, y)
    return y, idx, gate


def check(p, T, out_f32=False):
    layer = p.layer(out_f32)
    out_dtype = F32 if out_f32 else p.dtype
    y, idx, gate = run(p, T, layer, out_dtype)
    ry, tol, ridx, rgate, eg = p.reference(p.x[:T], out_dtype)
    assert torch.equal(idx.long(), ridx)
    assert bool(((gate.double() - rgate).abs() <= eg).all())
    assert bool(((y.double() - ry).abs() <= tol).all())
    # far inside the worst case on the whole: the hidden value's rounding and the output's, each at most half step / sqrt(3) in norm
    scale = float(ry.norm())
    fp32 = 1e-5
    assert float((y.double() - ry).norm()) <= (1.3 * (HALF[p.dtype] ** 2 + HALF[out_dtype] ** 2) ** 0.5 / 3 ** 0.5 + fp32) * scale
    layer.destroy()


# (d, widths, top_k): tiny, widths of 16 and odd multiples of it, one expert, many experts, widths that end inside a load
LAYERS = [(64, (96, 160, 112, 144), 2), (8, (16,), 1), (8, (16, 32), 2), (72, (48, 16, 208), 1), (200, (64, 128), 2), (1000, (176,), 1),
          (136, (16,) * 33, 2), (256, (64, 32) * 8, 2), (64, (16,) * 256, 2), (512, (1040, 16, 2000), 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("d,widths,k", LAYERS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_small_layers(d, widths, k, dtype):
    p = Problem(d, widths, k, dtype, seed=d + len(widths))
    for T in (1, 2, 7, 8, 9, 16, 17, 31, 32):
        check(p, T)


@pytest.mark.gpu
@pytest.mark.parametrize("d,widths,k,T", [(2048, BENCH, 2, 1), (2048, BENCH, 2, 5), (2048, BENCH, 2, 32), (1536, (2112, 6336, 2624, 5824), 1, 19),
                                          (2048, (5632,), 1, 32), (4096, (1024, 4096), 2, 12)])
@pytest.mark.parametrize("out_f32", [False, True])
def test_large_layers(d, widths, k, T, out_f32):
    check(Problem(d, widths, k, BF, seed=T), T, out_f32)


@pytest.mark.gpu
@pytest.mark.parametrize("widths", [(64, 96, 32, 48), (32,) * 20, (16,) * 40])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_second_router_term(widths, dtype):
    p = Problem(256, widths, 2, dtype, seed=len(widths), noise=(0.7, 1e-6))
    for T in (1, 9, 32):
        check(p, T)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [1, 2])
def test_agrees_with_forward(k):
    from paper_2409_12210_b200 import binding as B
    p = Problem(256, (128, 384, 192, 320), k, BF, seed=k)
    layer = p.layer()
    y, idx, gate = run(p, 32, layer, BF)
    ws = layer.alloc_workspace(BF, 32, False)
    ref = torch.empty_like(y)
    layer.forward(*p.w, p.x, ref, ws, False)
    rt = layer.get_routing(ws, 32)
    assert torch.equal(idx, rt["topk_idx"]) and float((gate - rt["topk_gate"]).abs().max()) <= 1e-5
    _, tol, _, _, _ = p.reference(p.x, BF)
    assert bool(((y.double() - ref.double()).abs() <= 2 * tol).all())
    assert layer.check_device_status(ws) == B.MODSE_OK
    layer.destroy()


@pytest.mark.gpu
@pytest.mark.parametrize("N", [2, 8, 40])
def test_equal_logits_go_to_the_lower_index(N):
    p = Problem(64, (32,) * N, 2, BF)
    p.w[0][:] = p.w[0][0]
    layer = p.layer()
    for T in (1, 20):
        y, idx, gate = run(p, T, layer, BF)
        assert bool((idx == torch.tensor([0, 1], device="cuda")).all()) and bool((gate == 0.5).all())
    layer.destroy()


@pytest.mark.gpu
def test_all_tokens_to_one_expert():
    p = Problem(128, (64, 2048, 32), 1, BF)
    p.w[0].zero_()
    p.w[0][1] = p.x[0].sign()
    p.x[:] = p.x.abs() * p.x[0].sign()
    check(p, 32)


@pytest.mark.gpu
def test_a_row_of_nan_or_infinity_stays_alone():
    p = Problem(64, (96, 160, 112, 144), 2, BF)
    layer = p.layer()
    clean, idx, _ = run(p, 12, layer, BF)
    for bad in (float("nan"), float("inf")):
        x = p.x.clone()
        p.x[3, 5] = bad
        y, idx2, _ = run(p, 12, layer, BF)
        rest = [t for t in range(12) if t != 3]
        assert torch.equal(y[rest], clean[rest]) and torch.equal(idx2[rest], idx[rest])
        assert not bool(torch.isfinite(y[3].float()).any()) and bool((idx2[3] >= 0).all()) and bool((idx2[3] < 4).all())
        p.x.copy_(x)
    layer.destroy()


@pytest.mark.gpu
def test_replayed_graph_and_streams_that_share_a_layer():
    p = Problem(256, (128, 384, 192, 320), 2, BF, T=32)
    layer = p.layer()
    x, y = p.x[:4].clone(), torch.empty(4, 256, dtype=BF, device="cuda")
    ws, ws2 = layer.alloc_decode_workspace(BF), layer.alloc_decode_workspace(BF)
    y2 = torch.empty(20, 256, dtype=BF, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.decode(*p.w, x, y, ws)
    whole, _, _ = run(p, 32, layer, BF)
    side = torch.cuda.Stream()
    for i in (0, 8, 20):
        x.copy_(p.x[i:i + 4])
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            layer.decode(*p.w, p.x[12:32], y2, ws2)
        torch.cuda.synchronize()
        ref, tol, _, _, _ = p.reference(p.x[i:i + 4], BF)
        assert bool(((y.double() - ref).abs() <= tol).all())
        ref, tol, _, _, _ = p.reference(p.x[12:32], BF)
        assert bool(((y2.double() - ref).abs() <= tol).all())
    layer.destroy()


@pytest.mark.gpu
def test_a_saved_forward_survives_a_decode():
    """The layer object is only read: backward still finds the forward it belongs to."""
    from paper_2409_12210_b200 import binding as B
    p = Problem(256, (128, 384, 192, 320), 2, BF)
    layer = p.layer()
    y, dx, dx2 = (torch.empty_like(p.x) for _ in range(3))
    grads = [torch.empty(p.w[0].shape, device="cuda")] + [torch.empty_like(w) for w in p.w[1:]]
    ws = layer.alloc_workspace(BF, 32, True)
    dy = torch.randn_like(p.x)
    layer.forward(*p.w, p.x, y, ws, True)
    layer.backward(*p.w, p.x, dy, dx, *grads, ws)
    launches = layer.last_launch_count()
    layer.decode(*p.w, p.x[:3], torch.empty_like(p.x[:3]), layer.alloc_decode_workspace(BF, 3))
    layer.backward(*p.w, p.x, dy, dx2, *grads, ws)
    assert torch.equal(dx, dx2) and layer.last_launch_count() == launches
    layer.destroy()


@pytest.mark.gpu
def test_rows_written_by_the_kernel_ahead():
    p = Problem(256, (128, 384), 2, BF)
    layer = p.layer()
    x, ws = torch.empty(8, 256, dtype=BF, device="cuda"), layer.alloc_decode_workspace(BF, 8)
    chain = []
    for i in range(20):
        x.copy_(p.x[i:i + 8])
        y = torch.empty_like(x)
        layer.decode(*p.w, x, y, ws)
        layer.decode(*p.w, y, x, ws)          # rows that the call ahead has written, over the rows it read
        chain.append((y, x.clone()))
    for i, (y, x2) in enumerate(chain):
        one, two = torch.empty_like(y), torch.empty_like(y)
        layer.decode(*p.w, p.x[i:i + 8].contiguous(), one, ws)
        torch.cuda.synchronize()
        layer.decode(*p.w, one, two, ws)
        assert torch.equal(one, y) and torch.equal(two, x2)
    layer.destroy()


def test_refusals_need_no_gpu():
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    lib, p = B.load(), 0x1000
    layer = B.ModseLayer(64, (96, 160, 112, 144), 2)
    w = B._Weights(p, p, p, p)

    def call(h=layer._h, dtype=B.MODSE_BF16, w=w, x=p, T=4, y=p, idx=p, gate=p, ws=p, n=1 << 30):
        return lib.modse_decode(h, dtype, ctypes.byref(w) if w is not None else None, x, T, y, idx, gate, ws, n, None)

    for kw in [dict(h=None), dict(dtype=B.MODSE_E4M3), dict(w=None), dict(T=-1), dict(x=None), dict(x=p + 8), dict(y=None), dict(y=p + 8),
               dict(idx=p + 2), dict(gate=p + 2), dict(ws=None), dict(ws=p + 16), dict(w=B._Weights(None, p, p, p)),
               dict(w=B._Weights(p, p + 8, p, p))]:
        assert call(**kw) == B.MODSE_ERR_INVALID_ARG, kw
    assert call(T=33) == B.MODSE_ERR_UNSUPPORTED and call(T=0) == B.MODSE_OK
    need = layer.decode_workspace_bytes(B.MODSE_BF16, 4)
    assert need > 0 and call(n=need - 1) == B.MODSE_ERR_WORKSPACE_TOO_SMALL
    sizes = [layer.decode_workspace_bytes(B.MODSE_BF16, T) for T in range(33)]
    assert sizes == sorted(sizes) and sizes[1] > 0
    assert layer.decode_workspace_bytes(B.MODSE_BF16, 33) == 0 == layer.decode_workspace_bytes(B.MODSE_E4M3, 3)
    layer.destroy()


@pytest.mark.gpu
def test_wrong_tensors_are_refused():
    from paper_2409_12210_b200 import binding as B
    p = Problem(64, (96, 160, 112, 144), 2, BF)
    layer = p.layer()
    x, y, ws = p.x[:4], torch.empty_like(p.x[:4]), layer.alloc_decode_workspace(BF)
    wr, wg, wu, wd = p.w
    for call in (lambda: layer.decode(wr, wg, wu, wd.T, x, y, ws), lambda: layer.decode(wr, wg.float(), wu, wd, x, y, ws),
                 lambda: layer.decode(wr, wg, wu, wd, x[:, :56], y, ws), lambda: layer.decode(wr, wg, wu, wd, x, y.float(), ws),
                 lambda: layer.decode(wr, wg, wu, wd, x.cpu(), y, ws), lambda: layer.decode(wr, wg, wu, wd, x, y, ws, topk_idx=y),
                 lambda: layer.decode(wr, wg, wu, wd, x, y, ws.cpu())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.ModseError):
        big = torch.zeros(33, 64, dtype=BF, device="cuda")
        layer.decode(wr, wg, wu, wd, big, torch.empty_like(big), ws)
    layer.destroy()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 12, 25])
def test_an_expired_wait_is_reported_and_the_next_call_is_right(T):
    """One block of the first kernel asks for no weights: nothing is in flight when its warps give up."""
    from paper_2409_12210_b200 import binding as B
    p = Problem(256, (128, 384, 192, 320), 2, BF)
    layer = p.layer()
    y, ws = torch.empty_like(p.x[:T]), layer.alloc_decode_workspace(BF)
    good = torch.empty_like(y)
    layer.decode(*p.w, p.x[:T], good, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    B.debug_set_wait_limit_ms(50)
    B.debug_skip_tile_loads(7, 0)
    try:
        layer.decode(*p.w, p.x[:T], y, ws)
        assert B.check_workspace_status(ws) == B.MODSE_ERR_DEVICE_TIMEOUT
    finally:
        B.debug_skip_tile_loads(-1, -1)
        B.debug_set_wait_limit_ms(2000)
    layer.decode(*p.w, p.x[:T], y, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK and torch.equal(y, good)
    layer.destroy()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 20])
def test_weights_past_32_bits(T):
    """An expert whose weights begin behind 2^31 elements of the three matrices."""
    d, widths = 2048, (1_060_864, 64)
    p = Problem(d, (64, 64), 1, BF, seed=T)
    small = p.w
    S = sum(widths)
    wg, wu, wd = torch.zeros(S, d, dtype=BF, device="cuda"), torch.zeros(S, d, dtype=BF, device="cuda"), torch.zeros(d, S, dtype=BF, device="cuda")
    wg[-64:], wu[-64:], wd[:, -64:] = small[1][-64:], small[2][-64:], small[3][:, -64:]
    wr = torch.zeros(2, d, dtype=BF, device="cuda")
    wr[1] = p.x[0].sign()
    x = (p.x.abs() * p.x[0].sign())[:T].contiguous()
    from paper_2409_12210_b200 import binding as B
    big, little = B.ModseLayer(d, widths, 1), B.ModseLayer(d, (64, 64), 1)
    y, ref = torch.empty_like(x), torch.empty_like(x)
    idx = torch.empty(T, 1, dtype=torch.int32, device="cuda")
    big.decode(wr, wg, wu, wd, x, y, big.alloc_decode_workspace(BF, T), topk_idx=idx)
    little.decode(wr, *small[1:], x, ref, little.alloc_decode_workspace(BF, T))
    assert bool((idx == 1).all())
    # the same products in runs of other lengths: fp32 sums of 64 terms, then one rounding to bf16
    assert bool(((y.float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 1e-5).all()) and bool(ref.any())
    big.destroy()
    little.destroy()


# Extents that are multiples of 64: d of one, three and an odd number of column blocks, more experts than a block's own routing
# takes, experts narrower and wider than others by far, rows of x too long to be held
BLOCKED = [(64, (64,), 1), (64, (64, 128), 2), (192, (320, 64, 128), 2), (320, (64,) * 9, 2), (128, (64,) * 40, 2), (576, (64, 1984), 1),
           (8192, (64, 128), 2), (16384, (64, 192), 2), (1088, (704, 64, 128, 960), 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("d,widths,k", BLOCKED)
def test_layers_of_whole_column_blocks(d, widths, k):
    p = Problem(d, widths, k, BF, seed=d + len(widths))
    for T in (1, 3, 8, 9, 16, 17, 32):
        check(p, T, out_f32=T % 2 == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("widths", [(64, 128, 192), (64,) * 40])
def test_second_router_term_of_whole_column_blocks(widths):
    p = Problem(192, widths, 2, BF, seed=len(widths), noise=(0.7, 1e-6))
    for T in (1, 8, 10, 32):
        check(p, T)


@pytest.mark.gpu
def test_tokens_past_the_last_row_are_left_alone():
    """Fewer tokens than the workspace was sized for, with the hidden rows of an earlier, larger call still in it."""
    from paper_2409_12210_b200 import binding as B
    p = Problem(256, (128, 384, 192, 320), 2, BF, seed=3)
    layer, ws = p.layer(), None
    ws = layer.alloc_decode_workspace(BF)
    for T in (32, 5, 20, 1, 32):
        y, fresh = torch.full((32, p.d), 9.0, dtype=BF, device="cuda"), torch.empty(T, p.d, dtype=BF, device="cuda")
        layer.decode(*p.w, p.x[:T], y[:T], ws)
        layer.decode(*p.w, p.x[:T], fresh, layer.alloc_decode_workspace(BF, T))
        assert torch.equal(y[:T], fresh) and bool((y[T:] == 9).all())
    assert B.check_workspace_status(ws) == B.MODSE_OK
    layer.destroy()
