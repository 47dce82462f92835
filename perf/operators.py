"""The operators around the MoDSE layer, as they are measured: the residual addition with the root-mean-square norm
(forward with 16/32-bit and 8-bit outputs, backward), the dense product with bias, activation and residual in its
epilogue (forward in bf16 and from 8-bit rows, backward), and the orthogonalised update of the expert matrices.

``run`` computes a case in plain torch operations in 32 bits or, where ``own`` is true, through the framework's calls.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
NORM_EPS = 1e-5
NS_COEFFS = (3.4445, -4.7750, 2.0315)
NS_STEPS = 5
NS_EPS = 1e-7
ACTIVATIONS = ("none", "relu", "gelu", "silu")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# the benchmark's expert widths (width sum of adjacent pairs 11264) and those of the tiny configuration
WIDTHS = (2816, 8448, 3520, 7744, 4224, 7040, 4928, 6336)
TINY_WIDTHS = (96, 160, 112, 144)


def _norm(name, tokens, d, dtype, out, residual=True):
    return {"name": name, "op": "norm", "tokens": tokens, "d": d, "dtype": dtype, "out": out, "residual": residual}


def _norm_bwd(name, tokens, d, dtype, dsum):
    return {"name": name, "op": "norm_bwd", "tokens": tokens, "d": d, "dtype": dtype, "dsum": dsum}


def _linear(name, tokens, k, n, dtype, act, bias, residual, save):
    return {"name": name, "op": "linear", "tokens": tokens, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias,
            "residual": residual, "save": save}


def _linear_bwd(name, tokens, k, n, act, bias):
    return {"name": name, "op": "linear_bwd", "tokens": tokens, "k": k, "n": n, "act": act, "bias": bias}


def _orth(name, shapes, dtype, strided):
    """shapes: "RxC" a matrix, comma-separated; strided: a matrix with fewer rows than columns is a column block of a wider one."""
    return {"name": name, "op": "orth", "shapes": ",".join("%dx%d" % s for s in shapes), "dtype": dtype, "strided": strided}


def listed():
    d = 2048
    return [
        # one generated token, ready for an 8-bit product: nothing but latency
        _norm("norm_token_8bit", 1, d, "bf16", "q"),
        # the benchmark's training batch: the sum is kept for backward, the norm is the layer's input
        _norm("norm_train_16k", 16384, d, "bf16", "y"),
        # the largest batch, serving a prompt: the sum and the 8-bit rows of the next product
        _norm("norm_prompt_64k_8bit", 65536, d, "bf16", "q"),
        # backward of the training batch; the residual path brings a gradient of its own
        _norm_bwd("norm_bwd_16k", 16384, d, "bf16", True),
        # one token through a square projection with the residual stream added: the weights' bytes
        _linear("linear_token", 1, d, d, "bf16", "none", True, True, False),
        # a batch of generated tokens on 8-bit weights
        _linear("linear_decode_8bit", 24, d, 5632, "e4m3", "silu", True, False, False),
        # the training batch through an activated product, pre-activations kept for backward
        _linear("linear_train_16k", 16384, d, 5632, "bf16", "gelu", True, False, True),
        # a ragged prompt on 8-bit rows and weights, back onto the residual stream
        _linear("linear_prompt_8bit", 4099, 5632, d, "e4m3", "none", False, True, False),
        # both gradients of the training product
        _linear_bwd("linear_bwd_8k", 8192, d, 5632, "gelu", True),
        # a small ragged batch at the 300M width
        _linear_bwd("linear_bwd_ragged", 1001, 1536, 2816, "silu", True),
        # the tiny configuration's gate matrices: launch-bound
        _orth("orth_tiny", [(h, 64) for h in TINY_WIDTHS], "f32", False),
        # two expert pairs of the benchmark layer: gate gradients (tall) and down gradients (column blocks)
        _orth("orth_experts", [(h, d) for h in WIDTHS[:4]] + [(d, h) for h in WIDTHS[:4]], "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_bwd", "linear", "linear", "linear_bwd", "orth", "orth"))
    if op in ("norm", "norm_bwd"):
        d = 8 * _log(rng, 8, 1024)
        tokens = _log(rng, 1, min(65536, (32768 if op == "norm_bwd" else 65536) * 2048 // max(d, 2048)))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if dtype == "f32":
            tokens = max(1, tokens // 2)
        if op == "norm":
            c = _norm("", tokens, d, dtype, rng.choice(("y", "q", "yq")), rng.random() < 0.8)
        else:
            c = _norm_bwd("", tokens, d, dtype, rng.random() < 0.7)
    elif op == "linear":
        dtype = rng.choice(("bf16", "e4m3"))
        k, n = 16 * _log(rng, 4, 528), 8 * _log(rng, 8, 1056)
        tokens = max(1, min(_log(rng, 1, 16384), 16384 * 2048 * 5632 // (k * n)))
        c = _linear("", tokens, k, n, dtype, rng.choice(ACTIVATIONS), rng.random() < 0.6, rng.random() < 0.5,
                    dtype == "bf16" and rng.random() < 0.4)
    elif op == "linear_bwd":
        k, n = 8 * _log(rng, 8, 1056), 8 * _log(rng, 8, 1056)
        tokens = max(1, min(_log(rng, 1, 16384), 8192 * 2048 * 5632 // (k * n)))
        c = _linear_bwd("", tokens, k, n, rng.choice(ACTIVATIONS), rng.random() < 0.6)
    else:
        short = _log(rng, 64, 2048)
        count = rng.randint(1, 4 if short > 1024 else 8)
        shapes = []
        for _ in range(count):
            long = _log(rng, 64, 8448)
            shapes.append((short, long) if rng.random() < 0.5 else (long, short))
        c = _orth("", shapes, rng.choice(("bf16", "f32")), rng.random() < 0.5)
    del c["name"]
    return c


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _quantise_rows(t):
    """8-bit rows and the scale of each, as a checkpoint or an earlier kernel leaves them."""
    scale = t.abs().amax(1).clamp_min(1e-12) / E4M3_MAX
    return (t / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    st = dict(case)
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        t, d, dt = case["tokens"], case["d"], DTYPES[case["dtype"]]
        # a residual stream: a few channels are much larger than the rest
        channels = torch.where(torch.rand(d, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        st["x"] = (normal(t, d) * channels).to(dt)
        st["weight"] = (1 + normal(d, std=0.2)).to(dt)
        if op == "norm":
            st["r"] = normal(t, d, std=0.5).to(dt) if case["residual"] else None
        else:
            st["dy"] = normal(t, d).to(dt)
            st["ds"] = normal(t, d).to(dt) if case["dsum"] else None
    elif op == "linear":
        t, k, n = case["tokens"], case["k"], case["n"]
        x, w = normal(t, k), normal(n, k, std=k ** -0.5)
        if case["dtype"] == "e4m3":
            st["x"], st["sx"] = _quantise_rows(x)
            st["w"], st["sw"] = _quantise_rows(w)
        else:
            st["x"], st["w"], st["sx"], st["sw"] = x.bfloat16(), w.bfloat16(), None, None
        st["b"] = normal(n, std=0.5).bfloat16() if case["bias"] else None
        st["r"] = normal(t, n).bfloat16() if case["residual"] else None
    elif op == "linear_bwd":
        t, k, n = case["tokens"], case["k"], case["n"]
        st["x"], st["w"] = normal(t, k).bfloat16(), normal(n, k, std=k ** -0.5).bfloat16()
        st["z"] = normal(t, n).bfloat16() if case["act"] != "none" else None
        st["dy"] = normal(t, n).bfloat16()
    else:
        dt = DTYPES[case["dtype"]]
        grads = []
        for r, c in _shapes(case):
            # a gradient: a few strong directions over a noise floor
            low = normal(r, 16) @ normal(16, c)
            m = (low * 0.02 + normal(r, c, std=0.01)).to(dt)
            if case["strided"] and r < c:
                wide = torch.zeros(r, c + 64, dtype=dt, device="cuda")
                wide[:, 32:32 + c] = m
                m = wide[:, 32:32 + c]
            grads.append(m)
        st["grads"] = grads
    return st


# ---- plain forms ------------------------------------------------------------
def _act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_norm(st):
    dt = st["x"].dtype
    s = st["x"].float()
    if st["r"] is not None:
        s = s + st["r"].float()
    y = s * torch.rsqrt((s * s).mean(1, keepdim=True) + NORM_EPS) * st["weight"].float()
    out = {"sum": s.to(dt)} if st["r"] is not None else {}
    if "y" in st["out"]:
        out["y"] = y.to(dt)
    if "q" in st["out"]:
        scale = y.abs().amax(1) / E4M3_MAX
        out["scale"] = scale
        out["q"] = (y / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return out


def _plain_norm_bwd(st):
    s, dy, w = st["x"].float(), st["dy"].float(), st["weight"].float()
    rstd = torch.rsqrt((s * s).mean(1, keepdim=True) + NORM_EPS)
    n = s * rstd
    u = dy * w
    dx = rstd * (u - n * (u * n).mean(1, keepdim=True))
    if st["ds"] is not None:
        dx = dx + st["ds"].float()
    return {"dx": dx.to(st["x"].dtype), "dweight": (dy * n).sum(0)}


def _plain_linear(st):
    z = st["x"].float() @ st["w"].float().T
    if st["sx"] is not None:
        z = z * st["sx"][:, None] * st["sw"]
    if st["b"] is not None:
        z = z + st["b"].float()
    y = _act(z, st["act"])
    if st["r"] is not None:
        y = y + st["r"].float()
    return {"y": y.bfloat16(), "z": z.bfloat16()} if st["save"] else {"y": y.bfloat16()}


def _plain_linear_bwd(st):
    dz = st["dy"].float()
    if st["z"] is not None:
        dz = dz * _act_grad(st["z"].float(), st["act"])
    out = {"dx": (dz @ st["w"].float()).bfloat16(), "dw": (dz.T @ st["x"].float()).bfloat16()}
    if st["bias"]:
        out["db"] = dz.sum(0)
    return out


def _plain_orth(st):
    a, b, c = NS_COEFFS
    outs = []
    for g in st["grads"]:
        tall = g.shape[0] > g.shape[1]
        x = g.float().T if tall else g.float()
        x = x / (torch.sqrt((x * x).sum()) + NS_EPS)
        for _ in range(NS_STEPS):
            m = x @ x.T
            m = b * m + c * (m @ m)
            x = a * x + m @ x
        outs.append((x.T if tall else x).bfloat16())
    return outs


# ---- the framework's calls --------------------------------------------------
def _own_norm(st):
    from paper_2409_12210_b200 import binding as B
    o = st.get("o")
    if o is None:
        x = st["x"]
        o = st["o"] = {"sum": torch.empty_like(x)} if st["r"] is not None else {}
        if "y" in st["out"]:
            o["y"] = torch.empty_like(x)
        if "q" in st["out"]:
            o["q"] = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
            o["scale"] = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    B.add_rms_norm(st["x"], st["r"], st["weight"], NORM_EPS, sum_out=o.get("sum"), y=o.get("y"), y8=o.get("q"),
                   y_scale=o.get("scale"))
    return o


def _own_norm_bwd(st):
    from paper_2409_12210_b200 import binding as B
    x = st["x"]
    if "o" not in st:
        st["o"] = {"dx": torch.empty_like(x), "dweight": torch.empty(x.shape[1], dtype=torch.float32, device=x.device)}
        st["ws"] = torch.empty(B.add_rms_norm_backward_workspace_bytes(*x.shape), dtype=torch.uint8, device=x.device)
    o = st["o"]
    B.add_rms_norm_backward(x, st["weight"], NORM_EPS, st["dy"], st["ds"], o["dx"], o["dweight"], st["ws"])
    return o


def _own_linear(st):
    from paper_2409_12210_b200 import binding as B
    x, w = st["x"], st["w"]
    if "o" not in st:
        new = lambda: torch.empty(x.shape[0], w.shape[0], dtype=torch.bfloat16, device=x.device)
        st["o"] = {"y": new(), "z": new()} if st["save"] else {"y": new()}
        st["ws"] = torch.empty(B.linear_workspace_bytes(x.dtype, x.shape[0], x.shape[1], w.shape[0]), dtype=torch.uint8,
                               device=x.device)
    o = st["o"]
    B.linear(x, w, o["y"], st["ws"], bias=st["b"], residual=st["r"], activation=st["act"], z=o.get("z"),
             x_scale=st["sx"], w_scale=st["sw"])
    return o


def _own_linear_bwd(st):
    from paper_2409_12210_b200 import binding as B
    x, w = st["x"], st["w"]
    if "o" not in st:
        st["o"] = {"dx": torch.empty_like(x), "dw": torch.empty_like(w)}
        if st["bias"]:
            st["o"]["db"] = torch.empty(w.shape[0], dtype=torch.float32, device=x.device)
        st["ws"] = torch.empty(B.linear_backward_workspace_bytes(x.shape[0], x.shape[1], w.shape[0]), dtype=torch.uint8,
                               device=x.device)
    o = st["o"]
    B.linear_backward(x, w, st["dy"], st["z"], st["act"], o["dx"], o["dw"], o.get("db"), st["ws"])
    return o


def _own_orth(st):
    from paper_2409_12210_b200 import binding as B
    grads = st["grads"]
    if "o" not in st:
        st["o"] = [torch.empty(g.shape, dtype=torch.bfloat16, device=g.device) for g in grads]
        st["ws"] = torch.empty(B.orthogonalize_workspace_bytes([g.shape for g in grads]), dtype=torch.uint8,
                               device=grads[0].device)
    B.orthogonalize(grads, st["o"], st["ws"], steps=NS_STEPS, coefficients=NS_COEFFS, eps=NS_EPS)
    return st["o"]


_PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "linear": _plain_linear, "linear_bwd": _plain_linear_bwd,
          "orth": _plain_orth}
_OWN = {"norm": _own_norm, "norm_bwd": _own_norm_bwd, "linear": _own_linear, "linear_bwd": _own_linear_bwd,
        "orth": _own_orth}


def run(state):
    if own:
        return _OWN[state["op"]](state)
    return _PLAIN[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------
def work(case):
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        t, d, e = case["tokens"], case["d"], 2 if case["dtype"] == "bf16" else 4
        if op == "norm":
            n = 1 + 2 * bool(case["residual"]) + ("y" in case["out"])
            return {"bytes": t * d * (n * e + ("q" in case["out"])) + d * e + 4 * t * ("q" in case["out"]), "flops": 6 * t * d}
        return {"bytes": t * d * e * (3 + bool(case["dsum"])) + d * (e + 4), "flops": 12 * t * d}
    if op == "linear":
        t, k, n, e = case["tokens"], case["k"], case["n"], 1 if case["dtype"] == "e4m3" else 2
        b = e * k * (t + n) + 2 * t * n * (1 + bool(case["residual"]) + bool(case["save"])) + 2 * n * bool(case["bias"])
        return {"bytes": b + (4 * (t + n) if e == 1 else 0), "flops": 2 * t * k * n}
    if op == "linear_bwd":
        t, k, n = case["tokens"], case["k"], case["n"]
        b = 2 * (2 * t * k + 2 * n * k + t * n * (1 + (case["act"] != "none"))) + 4 * n * bool(case["bias"])
        return {"bytes": b, "flops": 4 * t * k * n}
    b = f = 0
    for r, c in _shapes(case):
        n, m = min(r, c), max(r, c)
        b += r * c * ((2 if case["dtype"] == "bf16" else 4) + 2)
        # both symmetric products need one triangle only
        f += NS_STEPS * (n * (n + 1) * m + n * (n + 1) * n + 2 * n * n * m)
    return {"bytes": b, "flops": f}


# ---- the definitions in 64 bits ---------------------------------------------
def _e4m3_grid(v):
    """v rounded to the nearest number of four exponent and three mantissa bits, ties to even, largest 448."""
    mag = v.abs().clamp_min(2.0 ** -30)
    step = torch.exp2(torch.floor(torch.log2(mag)).clamp_min(-6.0) - 3.0)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    dbl = lambda name: None if st[name] is None else st[name].to(torch.float32).double()
    if op == "norm":
        s, w, d = dbl("x"), dbl("weight"), case["d"]
        out = {}
        if st["r"] is not None:
            s = s + dbl("r")
            out["sum"] = s
        y = s / torch.sqrt(s.square().sum(1) / d + NORM_EPS)[:, None] * w
        if "y" in case["out"]:
            out["y"] = y
        if "q" in case["out"]:
            out["scale"] = y.abs().max(1).values / E4M3_MAX
            out["q"] = _e4m3_grid(y / out["scale"][:, None])
        return out
    if op == "norm_bwd":
        s, w, dy, d = dbl("x"), dbl("weight"), dbl("dy"), case["d"]
        m = s.square().sum(1, keepdim=True) / d + NORM_EPS
        u = dy * w
        dx = u / m.sqrt() - s * (u * s).sum(1, keepdim=True) / (d * m.pow(1.5))
        if st["ds"] is not None:
            dx = dx + dbl("ds")
        return {"dx": dx, "dweight": torch.einsum("td,td->d", dy, s / m.sqrt())}
    if op == "linear":
        z = torch.einsum("tk,nk->tn", dbl("x"), dbl("w"))
        if st["sx"] is not None:
            z = z * (dbl("sx")[:, None] * dbl("sw")[None, :])
        if st["b"] is not None:
            z = z + dbl("b")
        y = {"none": lambda v: v, "relu": lambda v: torch.where(v > 0, v, 0.0),
             "gelu": lambda v: v * torch.special.ndtr(v), "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](z)
        if st["r"] is not None:
            y = y + dbl("r")
        return {"y": y, "z": z} if case["save"] else {"y": y}
    if op == "linear_bwd":
        dz, z = dbl("dy"), dbl("z")
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif case["act"] == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        elif case["act"] == "silu":
            p = torch.sigmoid(z)
            dz = dz * (p + z * p * (1 - p))
        out = {"dx": torch.einsum("tn,nk->tk", dz, dbl("w")), "dw": torch.einsum("tn,tk->nk", dz, dbl("x"))}
        if case["bias"]:
            out["db"] = dz.sum(0)
        return out
    a, b, c = NS_COEFFS
    outs = []
    for g in st["grads"]:
        x = g.double()
        x = x / (torch.linalg.norm(x) + NS_EPS)
        eye = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
        for _ in range(NS_STEPS):
            if x.shape[0] > x.shape[1]:
                m = x.T @ x
                x = x @ (a * eye + b * m + c * (m @ m))
            else:
                m = x @ x.T
                x = (a * eye + b * m + c * (m @ m)) @ x
        outs.append(x)
    return outs
