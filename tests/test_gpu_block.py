"""The operators around the layer used together, as one block of a model uses them: a projection back onto the residual
stream, the norm, the MoDSE layer, the whole way back, and the orthogonalised updates of the expert matrices - against
the same chain in 64 bits, step by step on the values the step before it wrote."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2409_12210_b200 import inputs as I

import helpers as H

pytestmark = pytest.mark.gpu

CFG = I.LayerConfig("block", "bf16", 256, (128, 384, 192, 320), 2, 333, seed=21, weight_std=0.05)
BF = 2.0 ** -8


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def near(got, ref, rel=2e-2):
    """The layer's own bar: largest error beyond one bf16 rounding, in units of the tensor's root mean square."""
    err = np.abs(f64(got) - ref) - BF * np.abs(ref)
    assert err.max() <= rel * np.sqrt((ref * ref).mean())


def test_block_forward_backward_and_updates():
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    inp, _ = H.screened(CFG)
    T, d = CFG.n_tokens, CFG.d_model
    bf = dict(dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(0)
    mk = lambda *s, std=1.0: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32)).to(**bf)
    stream, attn, wo, gamma = mk(T, d), mk(T, d), mk(d, d, std=d ** -0.5), mk(d, std=0.1) + 1
    w = B.pack_weights(inp, "cuda")
    layer = B.ModseLayer(d, CFG.ffn_sizes, CFG.top_k)
    new = lambda *s: torch.empty(*s, **bf)
    u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    # forward: s = stream + attn wo^T; n = norm(s); y = layer(n); out = s + y with the next block's norm
    s, n, y, out, nxt = new(T, d), new(T, d), new(T, d), new(T, d), new(T, d)
    lws = u8(B.linear_workspace_bytes(torch.bfloat16, T, d, d))
    B.linear(attn, wo, s, lws, residual=stream)
    B.add_rms_norm(s, None, gamma, 1e-5, y=n)
    ws = layer.alloc_workspace(torch.bfloat16, T, True)
    layer.forward(*w, n, y, ws, True)
    B.add_rms_norm(y, s, gamma, 1e-5, sum_out=out, y=nxt)
    # backward from a gradient of nxt and one that arrives along the residual stream
    dnxt, dres = mk(T, d), mk(T, d)
    dsum, dn, ds, dgamma, dgamma2 = new(T, d), new(T, d), new(T, d), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    nws = u8(B.add_rms_norm_backward_workspace_bytes(T, d))
    B.add_rms_norm_backward(out, gamma, 1e-5, dnxt, dres, dsum, dgamma2, nws)     # gradient of y and of s alike
    dwr = torch.empty(w[0].shape, dtype=torch.float32, device="cuda")
    dwg, dwu, dwd = (torch.empty_like(t) for t in w[1:])
    layer.backward(*w, n, dsum, dn, dwr, dwg, dwu, dwd, ws)
    B.add_rms_norm_backward(s, gamma, 1e-5, dn, dsum, ds, dgamma, nws)
    dattn, dwo = new(T, d), new(d, d)
    bws = u8(B.linear_backward_workspace_bytes(T, d, d))
    B.linear_backward(attn, wo, ds, None, "none", dattn, dwo, None, bws)
    ups = [torch.empty_like(t) for t in (dwg, dwu, dwd)]
    ows = u8(layer.orthogonalize_workspace_bytes())
    layer.orthogonalize_wgrads(dwg, dwu, dwd, *ups, ows)
    for st in (layer.check_device_status(ws), B.check_workspace_status(lws), B.check_workspace_status(bws),
               B.check_workspace_status(ows)):
        assert st == B.MODSE_OK

    # each step from what the step before it wrote
    def norm(a):
        return a / np.sqrt((a * a).mean(1, keepdims=True) + 1e-5) * f64(gamma)

    def norm_back(a, g):
        m = (a * a).mean(1, keepdims=True) + 1e-5
        u = g * f64(gamma)
        return u / np.sqrt(m) - a * (u * a).mean(1, keepdims=True) / m ** 1.5

    near(s, f64(stream) + f64(attn) @ f64(wo).T, 1e-4)
    near(n, norm(f64(s)), 1e-4)
    near(out, f64(s) + f64(y), 1e-4)
    near(nxt, norm(f64(s) + f64(y)), 1e-4)
    near(dsum, norm_back(f64(out), f64(dnxt)) + f64(dres), 1e-4)
    near(ds, norm_back(f64(s), f64(dn)) + f64(dsum), 1e-4)
    near(dattn, f64(ds) @ f64(wo), 1e-4)
    near(dwo, f64(ds).T @ f64(attn), 1e-4)
    # the layer inside the block gives what it gives on its own
    y2, dx2 = new(T, d), new(T, d)
    ws2 = layer.alloc_workspace(torch.bfloat16, T, True)
    layer.forward(*w, n, y2, ws2, True)
    again = [torch.empty_like(t) for t in (dwg, dwu, dwd)]
    layer.backward(*w, n, dsum, dx2, dwr, *again, ws2)
    assert torch.equal(y2, y) and torch.equal(dx2, dn) and torch.equal(again[0], dwg) and torch.equal(again[2], dwd)
    # the updates are those of the experts' matrices one by one
    off = 0
    for h in CFG.ffn_sizes:
        views = [(dwg[off:off + h], ups[0][off:off + h]), (dwu[off:off + h], ups[1][off:off + h]),
                 (dwd[:, off:off + h], ups[2][:, off:off + h])]
        for g, u in views:
            one = torch.empty(g.shape, **bf)
            B.orthogonalize([g], [one], u8(B.orthogonalize_workspace_bytes([g.shape])))
            scale = float(one.float().pow(2).mean().sqrt())
            assert float((one.float() - u.float()).abs().max()) <= 0.05 * scale
            sv = torch.linalg.svdvals(u.double())
            assert float(sv.max()) < 1.3
        off += h
    scales = [[0.5, 2.0, 1.0]] * len(CFG.ffn_sizes)
    twice = [torch.empty_like(t) for t in ups]
    layer.orthogonalize_wgrads(dwg, dwu, dwd, *twice, ows, scales=scales)
    assert torch.equal(twice[0], ups[0] * 0.5) and torch.equal(twice[1], ups[1] * 2) and torch.equal(twice[2], ups[2])
    layer.destroy()


def test_eight_bit_rows_from_the_norm_into_the_product():
    """Serving: the norm's 8-bit rows and scales go straight into the 8-bit product."""
    from paper_2409_12210_b200 import binding as B, build
    build.build()
    for T in (1, 5, 40, 300):
        rng = np.random.default_rng(T)
        mk = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()
        x, r, gamma, w = mk(T, 512).bfloat16(), mk(T, 512).bfloat16(), mk(512).bfloat16(), mk(264, 512)
        sw = w.abs().amax(1) / 448
        w8 = (w / sw[:, None]).to(torch.float8_e4m3fn)
        s, q = torch.empty_like(x), torch.empty(T, 512, dtype=torch.float8_e4m3fn, device="cuda")
        sc, y = torch.empty(T, device="cuda"), torch.empty(T, 264, dtype=torch.bfloat16, device="cuda")
        B.add_rms_norm(x, r, gamma, 1e-5, sum_out=s, y8=q, y_scale=sc)
        ws = torch.empty(B.linear_workspace_bytes(q.dtype, T, 512, 264), dtype=torch.uint8, device="cuda")
        B.linear(q, w8, y, ws, x_scale=sc, w_scale=sw)
        ref = (f64(q) * f64(sc)[:, None]) @ (f64(w8) * f64(sw)[:, None]).T
        near(y, ref, 1e-4)
        # against the unquantised chain: each factor is off by at most 2^-4 of itself (2^-10 of the row's top below the
        # e4m3 normals, which are at 2^-15 of it), so a sum of 512 products of independent errors stays within
        # 5 sqrt(512) (2^-4 + 2^-4) / sqrt(3) of a typical product
        a = f64(x) + f64(r)
        plain = (a / np.sqrt((a * a).mean(1, keepdims=True) + 1e-5) * f64(gamma)) @ f64(w).T
        typical = np.sqrt((plain * plain).mean() / 512)
        assert np.abs(f64(y) - plain).max() <= 5 * np.sqrt(512) * 2 ** -3 / np.sqrt(3) * typical


def test_offsets_past_32_bits():
    """More than 2^31 elements in a tensor: the last rows come out as they do on their own."""
    from paper_2409_12210_b200 import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    T, d = 1_050_003, 2056                                          # 2.16e9 elements
    x = torch.empty(T, d, **bf)
    x[-5:].normal_(generator=g)
    x[:-5] = 1
    w = torch.ones(d, **bf)
    y, tail = torch.zeros(T, d, **bf), torch.empty(5, d, **bf)
    B.add_rms_norm(x, None, w, 1e-5, y=y)
    B.add_rms_norm(x[-5:].contiguous(), None, w, 1e-5, y=tail)
    # another number of rows may take another shape of block, so sums may differ in their last bits: one bf16 step at most
    assert torch.allclose(y[-5:].float(), tail.float(), rtol=2.0 ** -7, atol=0)
    dw = torch.empty(d, device="cuda")
    ws = torch.empty(B.add_rms_norm_backward_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")
    dx = y                                                          # the gradient over the norm's output
    dy_tail, x_tail = y[-5:].clone(), x[-5:].clone()
    B.add_rms_norm_backward(x, w, 1e-5, y, None, dx, dw, ws)
    ref = torch.empty(5, d, **bf)
    B.add_rms_norm_backward(x_tail, w, 1e-5, dy_tail, None, ref, None)      # no weight gradient: no workspace
    scale = float(ref.float().abs().max())
    assert float((dx[-5:].float() - ref.float()).abs().max()) <= 2.0 ** -7 * scale
    del x, y, dx
    T, k, n = 262_147, 64, 8200                                     # 2.15e9 outputs
    x, w, b = torch.randn(T, k, generator=g, device="cuda").bfloat16(), torch.randn(n, k, generator=g, device="cuda").bfloat16(), torch.zeros(n, **bf)
    y = torch.zeros(T, n, **bf)
    ws = torch.empty(B.linear_workspace_bytes(x.dtype, T, k, n), dtype=torch.uint8, device="cuda")
    r = torch.zeros(T, n, **bf)
    r[-3:] = 1
    B.linear(x, w, y, ws, bias=b, residual=r)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    ref = x[-3:].double() @ w.double().T + 1
    assert bool(((y[-3:].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-3).all())
    del r
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda")
    ws = torch.empty(B.linear_backward_workspace_bytes(T, k, n), dtype=torch.uint8, device="cuda")
    B.linear_backward(x, w, y, y, "relu", dx, dw, db, ws)
    assert B.check_workspace_status(ws) == B.MODSE_OK
    dz = (y[-3:] * (y[-3:] > 0)).double()
    ref, mag = dz @ w.double(), dz.abs() @ w.double().abs()
    assert bool(((dx[-3:].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (n + 64) * 2.0 ** -23 * mag).all())


def test_calls_with_nothing_to_do_leave_a_clean_status_word():
    from paper_2409_12210_b200 import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x, w, y = torch.empty(0, 64, **bf), torch.zeros(32, 64, **bf), torch.empty(0, 32, **bf)
    dw, db = torch.ones(32, 64, **bf), torch.ones(32, device="cuda")
    calls = [lambda ws: B.linear(x, w, y, ws), lambda ws: B.linear_backward(x, w, y, y, "gelu", x, dw, db, ws),
             lambda ws: B.orthogonalize([], [], ws)]
    for call in calls:
        ws = torch.full((1 << 20,), 0xA5, dtype=torch.uint8, device="cuda")
        call(ws)
        assert B.check_workspace_status(ws) == B.MODSE_OK
        assert bool((ws[4:] == 0xA5).all())


FIRST_CALLS = """
import torch
from paper_2409_12210_b200 import binding as B
bf = dict(dtype=torch.bfloat16, device="cuda")
x, w, g = torch.randn(300, 256, **bf), torch.randn(512, 256, **bf), torch.randn(256, **bf)
s, y, dx, dg = torch.empty_like(x), torch.empty(300, 512, **bf), torch.empty_like(x), torch.empty(256, device="cuda")
dw, db, u, t = torch.empty_like(w), torch.empty(512, device="cuda"), torch.empty_like(w), torch.empty(64, 96, **bf)
u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
w1, w2, w3 = u8(B.add_rms_norm_backward_workspace_bytes(300, 256)), u8(B.linear_workspace_bytes(x.dtype, 300, 256, 512)), u8(B.linear_backward_workspace_bytes(300, 256, 512))
w4, w5 = u8(B.orthogonalize_workspace_bytes([(512, 256)])), u8(B.orthogonalize_workspace_bytes([(64, 96)]))
m = torch.randn(64, 96, **bf)
def block():
    B.add_rms_norm(x, x, g, 1e-5, y=s)
    B.linear(s, w, y, w2)
    B.linear(s[:3], w, y[:3], w2)
    B.linear_backward(s, w, y, y, "silu", dx, dw, db, w3)
    B.add_rms_norm_backward(x, g, 1e-5, dx, None, dx, dg, w1)
    B.orthogonalize([dw], [u], w4)
    B.orthogonalize([m], [t], w5)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    block()
graph.replay()
torch.cuda.synchronize()
first = [v.clone() for v in (s, y, dx, dw, db, dg, u, t)]
for v in (s, y, dx, dw, db, dg, u, t):
    v.zero_()
block()
torch.cuda.synchronize()
for a, b in zip(first, (s, y, dx, dw, db, dg, u, t)):
    assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) and bool((a != 0).any())
print("same")
"""


def test_first_calls_of_a_process_inside_a_capture():
    """Nothing has to be called once before it is captured, and a replay gives what the calls give."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "same" in out.stdout, out.stderr[-2000:]
