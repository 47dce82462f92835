"""A small language model made of the library's calls: token ids through the embedding, the norm, the MoDSE layer and the norm into the
cross entropy over the vocabulary, all the way back into the one table that embedding and head share, and the same model
one token at a time - each step against 64 bits on the values the step before it wrote."""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF = 2.0 ** -8


def near(got, ref, rel=1e-4):
    """Largest error beyond one bf16 rounding, in units of the tensor's root mean square."""
    err = (got.double() - ref).abs() - BF * ref.abs()
    assert float(err.max()) <= rel * float(ref.square().mean().sqrt())


def norm64(a, gamma):
    a = a.double()
    return a / (a.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma.double()


def norm_back64(a, gamma, g):
    a, u = a.double(), g.double() * gamma.double()
    m = a.square().mean(1, keepdim=True) + 1e-5
    return u / m.sqrt() - a * (u * a).mean(1, keepdim=True) / m ** 1.5


class Model:
    d, V, widths, k, scale = 256, 3001, (128, 384, 192, 320), 2, 16.0

    def __init__(self):
        from paper_2409_12210_b200 import binding as B, build
        build.build()
        g = torch.Generator(device="cuda").manual_seed(5)
        mk = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
        S, d = sum(self.widths), self.d
        self.table = mk(self.V, d, std=d ** -0.5)
        self.g1, self.g2 = (1 + mk(d, std=0.1)).bfloat16(), (1 + mk(d, std=0.1)).bfloat16()
        self.w = (mk(len(self.widths), d, std=d ** -0.5), mk(S, d, std=d ** -0.5), mk(S, d, std=d ** -0.5), mk(d, S, std=(S / 4) ** -0.5))
        self.layer = B.ModseLayer(d, self.widths, self.k)


def u8(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def test_training_step():
    from paper_2409_12210_b200 import binding as B
    m = Model()
    T, d, V = 700, m.d, m.V
    rng = np.random.default_rng(1)
    ids = torch.from_numpy(np.where(rng.random(T) < 0.05, -1, rng.integers(0, 200, T))).cuda()
    labels = torch.from_numpy(np.where(rng.random(T) < 0.1, -100, rng.integers(0, V, T))).cuda()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    new = lambda *s: torch.empty(*s, **bf)
    h0, n1, y, h1, n2 = (new(T, d) for _ in range(5))
    loss, lse, total = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, device="cuda")
    ws, wsl, wsb = m.layer.alloc_workspace(torch.bfloat16, T, True), u8(B.cross_entropy_workspace_bytes(T, d, V)), u8(B.cross_entropy_backward_workspace_bytes(T, d, V))
    B.embedding(ids, m.table, h0, scale=m.scale)
    B.add_rms_norm(h0, None, m.g1, 1e-5, y=n1)
    m.layer.forward(*m.w, n1, y, ws, True)
    B.add_rms_norm(y, h0, m.g2, 1e-5, sum_out=h1, y=n2)
    B.cross_entropy(n2, m.table, labels, loss, lse, wsl, total=total)
    # back: the head's gradient, down to the rows of the embedding, added to it
    dn2, dh1, dn1, dh0, dtable = new(T, d), new(T, d), new(T, d), new(T, d), new(V, d)
    dg1, dg2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    nws, wse = u8(B.add_rms_norm_backward_workspace_bytes(T, d)), u8(B.embedding_backward_workspace_bytes(T, d, V))
    grads = [torch.empty(m.w[0].shape, device="cuda")] + [torch.empty_like(t) for t in m.w[1:]]
    B.cross_entropy_backward(n2, m.table, labels, lse, dn2, dtable, wsb, total=total)
    head = dtable.clone()
    B.add_rms_norm_backward(h1, m.g2, 1e-5, dn2, None, dh1, dg2, nws)
    m.layer.backward(*m.w, n1, dh1, dn1, *grads, ws)
    B.add_rms_norm_backward(h0, m.g1, 1e-5, dn1, dh1, dh0, dg1, nws)
    B.embedding_backward(ids, dh0, dtable, wse, scale=m.scale, accumulate=True)
    for st in (m.layer.check_device_status(ws), *(B.check_workspace_status(t) for t in (wsl, wsb, wse))):
        assert st == B.MODSE_OK

    keep = (ids >= 0)[:, None]
    near(h0, torch.where(keep, m.table[ids.clamp(min=0)].double() * m.scale, 0.0))
    near(n1, norm64(h0, m.g1))
    near(n2, norm64(h0.double() + y.double(), m.g2))
    z = n2.double() @ m.table.double().T
    rlse = torch.logsumexp(z, 1)
    counted = labels >= 0
    want = torch.where(counted, rlse - z.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    assert float((loss.double() - want).abs().max()) <= 1e-4 and float(total[1]) == int(counted.sum())
    assert abs(float(total[0]) - float(want.sum())) <= 1e-5 * float(want.sum())
    dz = torch.exp(z - rlse[:, None])
    dz[torch.arange(T, device="cuda")[counted], labels[counted]] -= 1
    dz *= (counted.double() / counted.sum())[:, None]
    near(dn2, dz @ m.table.double(), 5e-2)          # dz is rounded to bf16 on the way: 2^-8 of every term
    near(head, dz.T @ n2.double(), 5e-2)
    near(dh1, norm_back64(h1, m.g2, dn2))
    near(dh0, norm_back64(h0, m.g1, dn1) + dh1.double())
    rows = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, ids.clamp(min=0), dh0.double() * m.scale * keep)
    near(dtable, head.double() + rows)
    untouched = torch.ones(V, dtype=torch.bool, device="cuda")
    untouched[ids[ids >= 0]] = False
    assert torch.equal(dtable[untouched], head[untouched])

    # the whole step changes the loss as its gradient says: along the table's gradient, by differences in 64 bits of the head alone
    step = 1e-3
    slope = float((head.double().square()).sum())

    def mean_loss(table):
        zz = n2.double() @ table.T
        return float((torch.logsumexp(zz, 1) - zz.gather(1, labels.clamp(min=0)[:, None])[:, 0])[counted].mean())
    t64 = m.table.double()
    diff = (mean_loss(t64 + step * head.double()) - mean_loss(t64 - step * head.double())) / (2 * step)
    assert abs(diff - slope) <= 0.02 * abs(slope)
    m.layer.destroy()


def test_generation_agrees_with_the_batch():
    """Rows of a prompt one step at a time, through the layer's form for few tokens, and scored by the head."""
    from paper_2409_12210_b200 import binding as B
    m = Model()
    T, d, V = 64, m.d, m.V
    ids = torch.from_numpy(np.random.default_rng(2).integers(0, V, T)).cuda()
    labels = ids.roll(-1)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    new = lambda t: torch.empty(t, d, **bf)

    def run(rows, decode):
        t = len(rows)
        h0, n1, y, h1, n2 = (new(t) for _ in range(5))
        loss, lse = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        B.embedding(ids[rows].contiguous(), m.table, h0, scale=m.scale)
        B.add_rms_norm(h0, None, m.g1, 1e-5, y=n1)
        if decode:
            m.layer.decode(*m.w, n1, y, m.layer.alloc_decode_workspace(torch.bfloat16, t))
        else:
            m.layer.forward(*m.w, n1, y, m.layer.alloc_workspace(torch.bfloat16, t, False), False)
        B.add_rms_norm(y, h0, m.g2, 1e-5, sum_out=h1, y=n2)
        B.cross_entropy(n2, m.table, labels[rows].contiguous(), loss, lse, u8(B.cross_entropy_workspace_bytes(t, d, V)))
        return n2, loss
    whole, loss = run(list(range(T)), False)
    for rows in ([0], [5], list(range(8)), list(range(20, 33)), list(range(32, 64))):
        part, l2 = run(rows, True)
        # both round the gated hidden values and the layer's output to bf16, in sums of another order
        near(part, whole[rows].double(), 3e-2)
        assert float((l2 - loss[rows]).abs().max()) <= 0.05
    m.layer.destroy()


FIRST_CALLS = """
import torch
from paper_2409_12210_b200 import binding as B
bf = dict(dtype=torch.bfloat16, device="cuda")
g = torch.Generator(device="cuda").manual_seed(0)
mk = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).bfloat16()
T, d, V, widths = 300, 256, 2000, (128, 384)
table, w = mk(V, d), (mk(2, d), mk(512, d), mk(512, d), mk(d, 512))
ids, labels = torch.randint(0, V, (T,), generator=g, device="cuda"), torch.randint(0, V, (T,), generator=g, device="cuda")
layer = B.ModseLayer(d, widths, 2)
u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
w1, w2, w3 = u8(B.cross_entropy_workspace_bytes(T, d, V)), u8(B.cross_entropy_backward_workspace_bytes(T, d, V)), u8(B.embedding_backward_workspace_bytes(T, d, V))
w4, w5 = layer.alloc_decode_workspace(torch.bfloat16), layer.alloc_decode_workspace(torch.bfloat16)
x, dx, dw, y = torch.empty(T, d, **bf), torch.empty(T, d, **bf), torch.empty(V, d, **bf), torch.empty(T, d, **bf)
loss, lse, total = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, device="cuda")
outs = (x, y, loss, lse, total, dx, dw)
def step():
    B.embedding(ids, table, x, scale=16.0)
    layer.decode(*w, x[:4], y[:4], w4)
    layer.decode(*w, x[4:30], y[4:30], w5)
    layer.decode(*w, x[30:42], y[30:42], w4)
    B.cross_entropy(x, table, labels, loss, lse, w1, total=total)
    B.cross_entropy_backward(x, table, labels, lse, dx, dw, w2, total=total)
    B.embedding_backward(ids, dx, dw, w3, accumulate=True)
y.zero_()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
first = [v.clone() for v in outs]
graph.replay()
torch.cuda.synchronize()
for a, b in zip(first, outs):
    assert torch.equal(a, b)
for v in outs:
    v.zero_()
step()
torch.cuda.synchronize()
for a, b in zip(first, outs):
    assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) and bool((a != 0).any())
print("same")
"""


def test_first_calls_of_a_process_inside_a_capture():
    """Nothing has to be called once before it is captured, and a replay gives what the calls give."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "same" in out.stdout, out.stderr[-2000:]
