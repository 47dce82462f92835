"""The operators at the two ends of a model built from MoDSE layers, and the layer for a few tokens, as they are measured:
the embedding lookup and its gradient, the softmax cross entropy over the vocabulary straight from the hidden rows and its
gradient, and one call of a whole MoDSE layer on the tokens of a generation step.

``run`` computes a case in plain torch operations in 32 bits or, where ``own`` is true, through the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ID_DTYPES = {"i32": torch.int32, "i64": torch.int64}
# the benchmark's expert widths (width sum of adjacent pairs 11264) and those of the tiny configuration
WIDTHS = (2816, 8448, 3520, 7744, 4224, 7040, 4928, 6336)
TINY_WIDTHS = (96, 160, 112, 144)
VOCABULARY = 32000


def _embed(name, tokens, d, vocabulary, dtype, ids):
    return {"name": name, "op": "embed", "tokens": tokens, "d": d, "vocabulary": vocabulary, "dtype": dtype, "ids": ids}


def _embed_bwd(name, tokens, d, vocabulary, dtype, grad, ids):
    return {"name": name, "op": "embed_bwd", "tokens": tokens, "d": d, "vocabulary": vocabulary, "dtype": dtype,
            "grad": grad, "ids": ids}


def _loss(name, tokens, d, vocabulary, ids):
    return {"name": name, "op": "loss", "tokens": tokens, "d": d, "vocabulary": vocabulary, "ids": ids}


def _loss_bwd(name, tokens, d, vocabulary, ids, weighted):
    return {"name": name, "op": "loss_bwd", "tokens": tokens, "d": d, "vocabulary": vocabulary, "ids": ids,
            "weighted": weighted}


def _decode(name, tokens, d, widths, top_k, dtype):
    return {"name": name, "op": "decode", "tokens": tokens, "d": d, "widths": ",".join(str(h) for h in widths),
            "top_k": top_k, "dtype": dtype}


def listed():
    d = 2048
    return [
        # the last tokens of a batch of requests: nothing but latency
        _embed("embed_step_32", 32, d, VOCABULARY, "bf16", "i64"),
        # a large batch of prompts: every row read and written once
        _embed("embed_prompt_64k", 65536, d, VOCABULARY, "bf16", "i32"),
        # the benchmark's training batch, the gradient kept in 32 bits for accumulation over micro-batches
        _embed_bwd("embed_bwd_16k", 16384, d, VOCABULARY, "bf16", "f32", "i64"),
        # a ragged batch at the 300M width over a large vocabulary of odd size: most rows of the gradient are zeros
        _embed_bwd("embed_bwd_ragged", 5003, 1536, 100003, "bf16", "bf16", "i32"),
        # scoring the drafted tokens of a few requests: the head's bytes
        _loss("loss_score_24", 24, d, VOCABULARY, "i64"),
        # the benchmark's training batch
        _loss("loss_train_16k", 16384, d, VOCABULARY, "i64"),
        # both gradients of a training batch, mean over the counted tokens
        _loss_bwd("loss_bwd_8k", 8192, d, VOCABULARY, "i64", False),
        # a ragged batch at the 300M width over a large vocabulary of odd size, tokens with weights of their own
        _loss_bwd("loss_bwd_ragged", 2051, 1536, 100003, "i32", True),
        # the tiny configuration: launch-bound
        _decode("decode_tiny", 4, 64, TINY_WIDTHS, 2, "f32"),
        # one generated token through the benchmark layer: the bytes of two experts
        _decode("decode_token", 1, d, WIDTHS, 2, "bf16"),
        # a batch of generated tokens: the bytes of all experts
        _decode("decode_batch_32", 32, d, WIDTHS, 2, "bf16"),
        # a small batch at the 300M width, one expert a token
        _decode("decode_top1_7", 7, 1536, (2112, 6336, 2624, 5824), 1, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_bwd", "embed_bwd", "loss", "loss", "loss_bwd", "loss_bwd", "decode", "decode", "decode"))
    ids = rng.choice(("i32", "i64"))
    if op == "embed":
        d = 8 * _log(rng, 8, 512)
        c = _embed("", min(_log(rng, 1, 65536), 65536 * 2048 // d), d, _log(rng, 256, 131072),
                   rng.choice(("bf16", "bf16", "f32")), ids)
    elif op == "embed_bwd":
        d = 8 * _log(rng, 8, 512)
        vocabulary = min(_log(rng, 256, 131072), 100003 * 2048 // d)
        c = _embed_bwd("", min(_log(rng, 1, 32768), 16384 * 2048 // d), d, vocabulary, rng.choice(("bf16", "bf16", "f32")),
                       rng.choice(("bf16", "f32")), ids)
    elif op == "loss":
        d, vocabulary = 8 * _log(rng, 8, 512), _log(rng, 1000, 131072)
        c = _loss("", max(1, min(_log(rng, 1, 16384), 16384 * 2048 * VOCABULARY // (d * vocabulary))), d, vocabulary, ids)
    elif op == "loss_bwd":
        d, vocabulary = 8 * _log(rng, 8, 512), _log(rng, 1000, 131072)
        c = _loss_bwd("", max(1, min(_log(rng, 1, 16384), 8192 * 2048 * VOCABULARY // (d * vocabulary))), d, vocabulary, ids,
                      rng.random() < 0.5)
    else:
        experts = rng.choice((1, 2, 4, 8, 8, 16))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        d = 128 * _log(rng, 1, 20 if dtype == "bf16" else 4)
        top = max(64, min(8448, 45056 * 2048 // (d * experts)))
        widths = [min(top, 64 * _log(rng, 1, 132)) for _ in range(experts)]
        c = _decode("", rng.choice((1, 1, 2, rng.randint(3, 16), rng.randint(17, 32))), d, widths,
                    min(experts, rng.choice((1, 2, 2))), dtype)
    del c["name"]
    return c


def _ids(g, n, vocabulary, dtype):
    """Token ids with the frequencies of text: the r-th most frequent in proportion to 1 / (r + 2.7)."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (2.7 * ((vocabulary + 2.7) / 2.7) ** u - 2.7).long().clamp_(0, vocabulary - 1)
    # a vocabulary is not sorted by frequency: spread the ranks by a multiplication modulo a prime
    return ((rank * 7919) % vocabulary).to(ID_DTYPES[dtype])


def _lse(x, w):
    """log sum exp of the rows of x w^T, a piece of rows at a time."""
    return torch.cat([torch.logsumexp((p.float() @ w.float().T).double(), 1) for p in x.split(2048)])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    st = dict(case)
    op = case["op"]
    if op in ("embed", "embed_bwd"):
        t, d, v, dt = case["tokens"], case["d"], case["vocabulary"], DTYPES[case["dtype"]]
        ids = _ids(g, t, v, case["ids"])
        # a few positions of a batch are padding
        st["tok"] = torch.where(torch.rand(t, generator=g, device="cuda") < 0.02, -1, ids).to(ids.dtype)
        st["scale"] = math.sqrt(d) if op == "embed" else 1.0
        if op == "embed":
            st["table"] = normal(v, d, std=d ** -0.5).to(dt)
        else:
            st["dy"] = normal(t, d).to(dt)
    elif op in ("loss", "loss_bwd"):
        t, d, v = case["tokens"], case["d"], case["vocabulary"]
        w = normal(v, d, std=2 * d ** -0.5)
        labels = _ids(g, t, v, case["ids"])
        # hidden rows lean towards the right answer, some hardly and some a lot
        x = normal(t, d) + 2 * torch.rand(t, 1, generator=g, device="cuda") * w[labels.long()]
        st["x"], st["w"] = x.bfloat16(), w.bfloat16()
        # the tokens of the prompts are not scored
        st["tok"] = torch.where(torch.rand(t, generator=g, device="cuda") < 0.1, -100, labels).to(labels.dtype)
        if op == "loss_bwd":
            counted = st["tok"] >= 0
            st["lse"] = _lse(st["x"], st["w"]).float()
            st["total"] = torch.stack((st["lse"][counted].sum(), counted.sum().float()))
            st["dloss"] = torch.rand(t, generator=g, device="cuda") + 0.5 if case["weighted"] else None
    else:
        t, d, k, dt = case["tokens"], case["d"], case["top_k"], DTYPES[case["dtype"]]
        widths = _widths(case)
        wide = sum(widths)
        st["wr"] = normal(len(widths), d, std=d ** -0.5).to(dt)
        st["wg"], st["wu"] = normal(wide, d, std=d ** -0.5).to(dt), normal(wide, d, std=d ** -0.5).to(dt)
        st["wd"] = normal(d, wide, std=(wide / len(widths)) ** -0.5).to(dt)
        x = normal(t, d).to(dt)
        # tokens whose choice of experts hangs on the last bits of a logit are drawn again
        for _ in range(6 if k < len(widths) else 0):
            z = (x.double() @ st["wr"].double().T).sort(1, descending=True).values
            close = (z[:, :k] - z[:, 1:k + 1]).min(1, keepdim=True).values < 1e-4
            x = torch.where(close, normal(t, d).to(dt), x)
        st["x"] = x
        if own:
            from paper_2409_12210_b200 import binding as B
            st["layer"] = B.ModseLayer(d, widths, k)
    return st


def _widths(case):
    return [int(h) for h in case["widths"].split(",")]


# ---- plain forms ------------------------------------------------------------
def _plain_embed(st):
    ids, table = st["tok"].long(), st["table"]
    y = table[ids.clamp_min(0)].float() * st["scale"]
    return {"y": torch.where((ids >= 0)[:, None], y, 0.0).to(table.dtype)}


def _plain_embed_bwd(st):
    ids, dy = st["tok"].long(), st["dy"].float() * st["scale"]
    dy = torch.where((ids >= 0)[:, None], dy, 0.0)
    out = torch.zeros(st["vocabulary"], st["d"], dtype=torch.float32, device=dy.device)
    return {"dtable": out.index_add_(0, ids.clamp_min(0), dy).to(DTYPES[st["grad"]])}


def _plain_loss(st):
    labels = st["tok"].long()
    z = st["x"].float() @ st["w"].float().T
    top = z.max(1, keepdim=True).values
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    counted = labels >= 0
    loss = torch.where(counted, lse - z.gather(1, labels.clamp_min(0)[:, None])[:, 0], 0.0)
    total = torch.stack((loss.double().sum(), counted.double().sum())).float()
    return {"loss": loss, "lse": lse, "total": total}


def _plain_loss_bwd(st):
    labels = st["tok"].long()
    x, w = st["x"].float(), st["w"].float()
    factor = (labels >= 0).float() / st["total"][1]
    if st["dloss"] is not None:
        factor = factor * st["dloss"]
    dz = torch.exp(x @ w.T - st["lse"][:, None])
    rows = torch.arange(len(labels), device=x.device)
    dz[rows, labels.clamp_min(0)] -= 1.0          # rows that are not counted are multiplied by zero below
    dz *= factor[:, None]
    return {"dx": (dz @ w).bfloat16(), "dw": (dz.T @ x).bfloat16()}


def _plain_decode(st):
    # without a question to the host which experts were chosen, all of them see all tokens; a gate of zero drops what was not
    x, k = st["x"].float(), st["top_k"]
    widths = _widths(st)
    z = x @ st["wr"].float().T
    left, idx, kept = z.clone(), [], []
    for _ in range(k):                            # ties go to the lowest index
        i = torch.argmax(left, 1, keepdim=True)
        idx.append(i)
        kept.append(z.gather(1, i))
        left.scatter_(1, i, -math.inf)
    idx, kept = torch.cat(idx, 1), torch.cat(kept, 1)
    e = torch.exp(kept - kept[:, :1])
    gate = e / e.sum(1, keepdim=True)
    per_expert = torch.zeros_like(z).scatter_(1, idx, gate)
    a, b = x @ st["wg"].float().T, x @ st["wu"].float().T
    h = a / (1 + torch.exp(-a)) * b
    off = 0
    for e, width in enumerate(widths):
        h[:, off:off + width] *= per_expert[:, e:e + 1]
        off += width
    y = h @ st["wd"].float().T
    return {"y": y.to(st["x"].dtype), "idx": idx.int(), "gate": gate}


# ---- the framework's calls --------------------------------------------------
def _own_embed(st):
    from paper_2409_12210_b200 import binding as B
    ids, table = st["tok"], st["table"]
    if "o" not in st:
        st["o"] = {"y": torch.empty(ids.shape[0], table.shape[1], dtype=table.dtype, device=table.device)}
    B.embedding(ids, table, st["o"]["y"], scale=st["scale"])
    return st["o"]


def _own_embed_bwd(st):
    from paper_2409_12210_b200 import binding as B
    ids, dy = st["tok"], st["dy"]
    if "o" not in st:
        shape = (st["vocabulary"], dy.shape[1])
        st["o"] = {"dtable": torch.empty(shape, dtype=DTYPES[st["grad"]], device=dy.device)}
        st["ws"] = torch.empty(B.embedding_backward_workspace_bytes(dy.shape[0], shape[1], shape[0]), dtype=torch.uint8,
                               device=dy.device)
    B.embedding_backward(ids, dy, st["o"]["dtable"], st["ws"], scale=st["scale"])
    return st["o"]


def _own_loss(st):
    from paper_2409_12210_b200 import binding as B
    x, w = st["x"], st["w"]
    if "o" not in st:
        new = lambda n: torch.empty(n, dtype=torch.float32, device=x.device)
        st["o"] = {"loss": new(x.shape[0]), "lse": new(x.shape[0]), "total": new(2)}
        st["ws"] = torch.empty(B.cross_entropy_workspace_bytes(x.shape[0], x.shape[1], w.shape[0]), dtype=torch.uint8,
                               device=x.device)
    o = st["o"]
    B.cross_entropy(x, w, st["tok"], o["loss"], o["lse"], st["ws"], total=o["total"])
    return o


def _own_loss_bwd(st):
    from paper_2409_12210_b200 import binding as B
    x, w = st["x"], st["w"]
    if "o" not in st:
        st["o"] = {"dx": torch.empty_like(x), "dw": torch.empty_like(w)}
        st["ws"] = torch.empty(B.cross_entropy_backward_workspace_bytes(x.shape[0], x.shape[1], w.shape[0]),
                               dtype=torch.uint8, device=x.device)
    o = st["o"]
    B.cross_entropy_backward(x, w, st["tok"], st["lse"], o["dx"], o["dw"], st["ws"], dloss=st["dloss"], total=st["total"])
    return o


def _own_decode(st):
    layer, x = st["layer"], st["x"]
    if "o" not in st:
        t, k = x.shape[0], st["top_k"]
        st["o"] = {"y": torch.empty_like(x), "idx": torch.empty(t, k, dtype=torch.int32, device=x.device),
                   "gate": torch.empty(t, k, dtype=torch.float32, device=x.device)}
        st["ws"] = layer.alloc_decode_workspace(x.dtype, t, x.device)
    o = st["o"]
    layer.decode(st["wr"], st["wg"], st["wu"], st["wd"], x, o["y"], st["ws"], topk_idx=o["idx"], topk_gate=o["gate"])
    return o


_PLAIN = {"embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "loss": _plain_loss, "loss_bwd": _plain_loss_bwd,
          "decode": _plain_decode}
_OWN = {"embed": _own_embed, "embed_bwd": _own_embed_bwd, "loss": _own_loss, "loss_bwd": _own_loss_bwd,
        "decode": _own_decode}


def run(state):
    if own:
        return _OWN[state["op"]](state)
    return _PLAIN[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------
def work(case):
    op = case["op"]
    if op == "decode":
        t, d, k, e = case["tokens"], case["d"], case["top_k"], 2 if case["dtype"] == "bf16" else 4
        widths = _widths(case)
        n, wide = len(widths), sum(widths)
        # experts that t tokens meet, on average over choices that favour none
        met = 1 - (1 - k / n) ** t
        return {"bytes": int(e * (3 * d * wide * met + n * d + 2 * t * d) + 8 * t * k), "flops": 6 * d * t * k * wide // n}
    t, d, v, i = case["tokens"], case["d"], case["vocabulary"], 4 if case["ids"] == "i32" else 8
    if op == "embed":
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": t * (d * e + i) + min(t, v) * d * e, "flops": t * d}
    if op == "embed_bwd":
        return {"bytes": t * (d * (2 if case["dtype"] == "bf16" else 4) + i) + v * d * (2 if case["grad"] == "bf16" else 4),
                "flops": t * d}
    if op == "loss":
        return {"bytes": 2 * d * (t + v) + t * (i + 8) + 8, "flops": 2 * t * d * v}
    # the logits are not kept, so they are computed again before the two products of the gradient
    return {"bytes": 4 * d * (t + v) + t * (i + 4 + 4 * case["weighted"]), "flops": 6 * t * d * v}


# ---- the definitions in 64 bits ---------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    dbl = lambda name: st[name].double()
    if op == "embed":
        rows = torch.zeros(case["tokens"], case["d"], dtype=torch.float64, device="cuda")
        at = torch.nonzero(st["tok"] >= 0)[:, 0]
        rows[at] = st["table"].index_select(0, st["tok"][at].long()).double() * st["scale"]
        return {"y": rows}
    if op == "embed_bwd":
        # the rows sorted by token; a token's gradient is the difference of two running sums
        order = torch.argsort(st["tok"].long(), stable=True)
        order = order[st["tok"][order] >= 0]
        run_sum = torch.zeros(len(order) + 1, case["d"], dtype=torch.float64, device="cuda")
        torch.cumsum(dbl("dy")[order], 0, out=run_sum[1:])
        count = torch.bincount(st["tok"][order].long(), minlength=case["vocabulary"])
        ends = torch.cumsum(count, 0)
        out = (run_sum[ends] - run_sum[ends - count]) * st["scale"]
        return {"dtable": torch.where(count[:, None] > 0, out, 0.0)}
    if op in ("loss", "loss_bwd"):
        x, w, tok = dbl("x"), dbl("w"), st["tok"].long()
        keep = (tok >= 0).double()
        if op == "loss":
            loss, lse = [], []
            for rows, lab in zip(x.split(2048), tok.split(2048)):
                z = torch.einsum("td,vd->tv", rows, w)
                lse.append(torch.logsumexp(z, 1))
                loss.append(torch.where(lab >= 0, lse[-1] - (rows * w[lab.clamp_min(0)]).sum(1), 0.0))
            loss = torch.cat(loss)
            return {"loss": loss, "lse": torch.cat(lse), "total": torch.stack((loss.sum(), keep.sum()))}
        dx, dw = [], torch.zeros_like(w)
        g = keep / keep.sum()
        if st["dloss"] is not None:
            g = g * dbl("dloss")
        for rows, lab, f in zip(x.split(1024), tok.split(1024), g.split(1024)):
            p = torch.softmax(torch.einsum("td,vd->tv", rows, w), 1)
            p.scatter_add_(1, lab.clamp_min(0)[:, None], torch.full_like(f, -1.0)[:, None])
            p = f[:, None] * p
            dx.append(torch.einsum("tv,vd->td", p, w))
            dw += torch.einsum("tv,td->vd", p, rows)
        return {"dx": torch.cat(dx), "dw": dw}
    x, k, widths = dbl("x"), case["top_k"], _widths(case)
    z = torch.einsum("td,nd->tn", x, dbl("wr"))
    order = torch.sort(z, dim=1, descending=True, stable=True)
    idx, gate = order.indices[:, :k], torch.softmax(order.values[:, :k], 1)
    y = torch.zeros_like(x)
    off = 0
    for e, width in enumerate(widths):
        token, slot = torch.nonzero(idx == e, as_tuple=True)
        if len(token):
            rows = x[token]
            a = rows @ st["wg"][off:off + width].double().T
            b = rows @ st["wu"][off:off + width].double().T
            out = (a * torch.sigmoid(a) * b) @ st["wd"][:, off:off + width].double().T
            y.index_add_(0, token, out * gate[token, slot][:, None])
        off += width
    return {"y": y, "idx": idx.int(), "gate": gate}
