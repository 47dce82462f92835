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
