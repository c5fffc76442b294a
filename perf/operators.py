"""Work of the operators around large fully connected layers, as timed cases: the root-mean-square norm in training and
with an 8-bit output, 8-bit quantisation of rows, the product of 8-bit matrices with a scale for each row, the
orthogonalisation of a matrix by Newton-Schulz products and the Muon update built on it.

`run` computes them in elementary torch operations, or (where `own` is set) by the calls of `paper_1501_07338_amd.vcnn`.
8-bit results are returned as they are held: integers in an int8 tensor, with their scales beside them.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315  # the quintic a s + b s^3 + c s^5 applied to the singular values
STEPS = 5
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
MAX_NORM = 8192 * 5120      # elements of a drawn norm or quantisation
MAX_FC = 4096 * 8192 * 8192  # multiply-adds of a drawn product
MAX_NS = 3 * 4096 ** 3       # multiply-adds of a step of a drawn orthogonalisation


def listed():
    return [
        # the hidden layer of the digit network (cfg2) at its mini-batch, normalised: forward and backward, the smallest call
        dict(name="norm_train_digits", kind="norm_train", rows=128, cols=500, dtype="f32", residual=False),
        # one training step's tokens through a residual block's norm, forward and backward
        dict(name="norm_train_bf16", kind="norm_train", rows=4096, cols=4096, dtype="bf16", residual=True),
        # answering: one token, its residual added, normalised and quantised for the next product; all latency
        dict(name="norm_i8_token", kind="norm_i8", rows=1, cols=4096, dtype="bf16", residual=True),
        # a batch of prompts at the same place
        dict(name="norm_i8_prompt", kind="norm_i8", rows=8192, cols=5120, dtype="bf16", residual=True),
        # a kernel matrix (cfg5's dense layer, 512 x 9728) prepared for 8-bit products, a scale per output channel
        dict(name="quant_weights", kind="quant", rows=512, cols=9728, dtype="f32"),
        # answering 48 users at once: the activations are quantised as they come, then multiplied
        dict(name="fc_i8_batch", kind="fc_dynamic", batch=48, i=4096, o=4096, act=1, bias=True, dtype="bf16"),
        # one token through a wide layer: the weights are read once, nothing is reused
        dict(name="fc_i8_token", kind="fc_i8", batch=1, i=4096, o=16384, act=0, bias=False, dtype="bf16"),
        # prompts through a wide layer: the largest product
        dict(name="fc_i8_prompt", kind="fc_i8", batch=4096, i=8192, o=8192, act=0, bias=True, dtype="bf16"),
        # the accumulated gradient of cfg3's last convolution, 64 maps of 32 x 5 x 5
        dict(name="orthogonalize_maps", kind="ortho", rows=64, cols=800),
        # a projection of a wide layer
        dict(name="orthogonalize_wide", kind="ortho", rows=1024, cols=4096),
        # every matrix of the digit network in one update
        dict(name="muon_digits", kind="muon", shapes="20x25,50x500,500x800,10x500"),
        # two matrices of a large layer, one of them tall: the most work
        dict(name="muon_large", kind="muon", shapes="4096x4096,8192x2048"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def draw(rng):
    kind = rng.choice(["norm_train", "norm_i8", "quant", "fc_dynamic", "fc_i8", "fc_i8", "ortho", "muon"])
    dtype = rng.choice(["f32", "bf16"])
    while True:
        if kind in ("norm_train", "norm_i8", "quant"):
            rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 33, 16384)
            if rows * cols > MAX_NORM // (4 if dtype == "f32" else 2):
                continue
            case = dict(kind=kind, rows=rows, cols=cols, dtype=dtype)
            if kind != "quant":
                case["residual"] = rng.random() < 0.6
            return case
        if kind in ("fc_dynamic", "fc_i8"):
            batch, i, o = _log_int(rng, 1, 4096), _log_int(rng, 64, 16384), _log_int(rng, 10, 16384)
            if rng.random() < 0.5:
                i = max(64, i // 64 * 64)  # half of the layers have whole rows of 64 bytes
            if batch * i * o > MAX_FC:
                continue
            return dict(kind=kind, batch=batch, i=i, o=o, act=rng.choice([0, 1]), bias=rng.random() < 0.5, dtype=dtype)
        count = 1 if kind == "ortho" else rng.randint(1, 6)
        shapes = [(_log_int(rng, 10, 4096), _log_int(rng, 25, 8192)) for _ in range(count)]
        if sum(min(s) ** 2 * (2 * max(s) + min(s)) for s in shapes) > MAX_NS:
            continue
        if kind == "ortho":
            return dict(kind=kind, rows=shapes[0][0], cols=shapes[0][1])
        return dict(kind=kind, shapes=",".join("%dx%d" % s for s in shapes))


def work(case):
    kind = case["kind"]
    if kind in ("norm_train", "norm_i8", "quant"):
        e, n, rows = (4 if case["dtype"] == "f32" else 2), case["rows"] * case["cols"], case["rows"]
        if kind == "quant":
            return {"bytes": n * (e + 1) + 4 * rows, "flops": 3 * n}
        more = 2 if case["residual"] else 0  # the residual read and the sum written
        if kind == "norm_i8":
            return {"bytes": n * (e * (1 + more) + 1) + 4 * rows + 4 * case["cols"], "flops": 7 * n}
        # forward x -> y; backward h, dy (and the gradient beside the norm) -> dh
        return {"bytes": n * e * (2 + more + 3 + more / 2) + 8 * rows + 12 * case["cols"], "flops": 16 * n}
    if kind in ("fc_dynamic", "fc_i8"):
        e, b, i, o = (4 if case["dtype"] == "f32" else 2), case["batch"], case["i"], case["o"]
        x = b * i * (e if kind == "fc_dynamic" else 1)
        return {"bytes": x + i * o + b * o * e + 4 * (b + 2 * o), "flops": 2 * b * i * o}
    shapes = [(case["rows"], case["cols"])] if kind == "ortho" else _shapes(case)
    flops = sum(STEPS * 2 * (min(s) ** 2 * max(s) * 1.5 + min(s) ** 3 * 0.5) for s in shapes)  # X X^T and A^2 are symmetric
    return {"bytes": sum(s[0] * s[1] for s in shapes) * (8 if kind == "ortho" else 20), "flops": flops}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(gen, rows, cols, dtype):
    """Tokens of different magnitudes with a few loud channels, as the layers of trained networks see them."""
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device=DEV, generator=gen))
    x[:, torch.randint(0, cols, (max(1, cols // 128),), device=DEV, generator=gen)] *= 12.0
    return x.to(dtype)


def _gradient(gen, rows, cols):
    """A few strong directions over a full-rank rest, as an accumulated gradient has them."""
    k = max(1, min(rows, cols) // 16)
    a, b = torch.randn(rows, k, device=DEV, generator=gen), torch.randn(k, cols, device=DEV, generator=gen)
    return 1e-3 * (a @ b / math.sqrt(k) + torch.randn(rows, cols, device=DEV, generator=gen))


def _integers(gen, rows, cols):
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    return (x * 32).round_().clamp_(-127, 127).to(torch.int8), \
        (0.5 + torch.rand(rows, device=DEV, generator=gen)) / (32 * math.sqrt(cols))


def _workspace(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind in ("norm_train", "norm_i8", "quant"):
        rows, cols, dtype = case["rows"], case["cols"], _type(case["dtype"])
        s["x"] = _activations(gen, rows, cols, dtype)
        if kind != "quant":
            s["gain"] = 1.0 + 0.2 * torch.randn(cols, device=DEV, generator=gen)
            s["r"] = _activations(gen, rows, cols, dtype) if case["residual"] else None
            s["h"] = torch.empty_like(s["x"]) if case["residual"] else None
        if kind == "norm_train":
            s["dy"] = torch.randn(rows, cols, device=DEV, generator=gen).to(dtype)
            s["dabove"] = torch.randn(rows, cols, device=DEV, generator=gen).to(dtype) if case["residual"] else None
            s["y"], s["dh"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["rstd"] = torch.empty(rows, device=DEV)
            s["dgain"] = torch.empty(cols, device=DEV)
        else:
            s["q"] = torch.empty(rows, cols, dtype=torch.int8, device=DEV)
            s["scale"] = torch.empty(rows, device=DEV)
    elif kind in ("fc_dynamic", "fc_i8"):
        b, i, o, dtype = case["batch"], case["i"], case["o"], _type(case["dtype"])
        s["wq"], s["wscale"] = _integers(gen, o, i)
        if kind == "fc_dynamic":
            s["x"] = _activations(gen, b, i, dtype)
            s["xq"], s["xscale"] = torch.empty(b, i, dtype=torch.int8, device=DEV), torch.empty(b, device=DEV)
        else:
            s["xq"], s["xscale"] = _integers(gen, b, i)
        s["b"] = 0.1 * torch.randn(o, device=DEV, generator=gen) if case["bias"] else None
        s["y"] = torch.empty(b, o, dtype=dtype, device=DEV)
    elif kind == "ortho":
        s["g"] = _gradient(gen, case["rows"], case["cols"])
        s["out"] = torch.empty_like(s["g"])
    else:
        s["w"], s["dw"], s["m"] = [], [], []
        for rows, cols in _shapes(case):
            s["w"].append(torch.randn(rows, cols, device=DEV, generator=gen) * math.sqrt(2.0 / cols))
            s["dw"].append(_gradient(gen, rows, cols))
            s["m"].append(10.0 * _gradient(gen, rows, cols))
    if own:  # device memory that a program keeps for these calls
        from paper_1501_07338_amd import vcnn
        if kind == "norm_train":
            s["ws"] = _workspace(vcnn.rmsnorm_workspace_bytes(case["rows"], case["cols"]))
        elif kind in ("fc_dynamic", "fc_i8"):
            s["ws"] = _workspace(vcnn.fc_i8_workspace_bytes(case["batch"], case["i"], case["o"]))
        elif kind == "ortho":
            s["ws"] = _workspace(vcnn.orthogonalize_workspace_bytes(case["rows"], case["cols"]))
        elif kind == "muon":
            s["ws"] = _workspace(vcnn.muon_workspace_bytes(_shapes(case)))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def _sum_with_residual(s):
    """The residual stream in the storage type, which is what the norm reads."""
    return s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)


def _to_i8(u):
    """Rows of 32-bit values as integers of at most 127, ties to even; the largest magnitude of each row.  In 64 bits,
    so that no value beside the border of two integers falls to the wrong side."""
    a = u.abs().amax(dim=1, keepdim=True)
    q = torch.where(a > 0, torch.round(u.double() * 127.0 / a.double()), 0.0)
    return q.to(torch.int8), a[:, 0]


def _norm_train(s):
    h, g, dy = _sum_with_residual(s), s["gain"], s["dy"].float()
    hf = h.float()
    rstd = torch.rsqrt(hf.square().mean(dim=1) + EPS)
    z = hf * rstd[:, None]
    y = (z * g).to(h.dtype)
    t = dy * g
    dh = rstd[:, None] * (t - z * (t * z).mean(dim=1, keepdim=True))
    if s["dabove"] is not None:
        dh = dh + s["dabove"].float()
    out = {"y": y, "rstd": rstd, "dh": dh.to(h.dtype), "dgain": (dy * z).sum(dim=0)}
    if s["r"] is not None:
        out["h"] = h
    return out


def _norm_i8(s):
    h = _sum_with_residual(s)
    hf = h.float()
    rstd = torch.rsqrt(hf.square().mean(dim=1) + EPS)
    q, a = _to_i8(hf * s["gain"])
    out = {"q": q, "scale": a * rstd / 127.0}
    if s["r"] is not None:
        out["h"] = h
    return out


def _quant(x):
    q, a = _to_i8(x.float())
    return q, a / 127.0


def _product(s, xq, xscale):
    y = (xq.float() @ s["wq"].float().t()) * xscale[:, None] * s["wscale"][None, :]
    if s["b"] is not None:
        y = y + s["b"]
    return (torch.relu(y) if s["act"] else y).to(s["y"].dtype)


def _orthogonal(g):
    x = g.t() if g.shape[0] > g.shape[1] else g
    x = x / x.double().square().sum().sqrt().float()
    for _ in range(STEPS):
        a = x @ x.t()
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    return x.t().contiguous() if g.shape[0] > g.shape[1] else x


def _muon(s):
    for w, g, m in zip(s["w"], s["dw"], s["m"]):
        m.mul_(MOMENTUM).add_(g)
        step = LR * math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
        w.mul_(1.0 - LR * DECAY).sub_(step * _orthogonal(g + MOMENTUM * m))
    return {"w": s["w"], "m": s["m"]}


def _plain(s):
    kind = s["kind"]
    if kind == "norm_train":
        return _norm_train(s)
    if kind == "norm_i8":
        return _norm_i8(s)
    if kind == "quant":
        q, scale = _quant(s["x"])
        return {"q": q, "scale": scale}
    if kind == "fc_dynamic":
        xq, xscale = _quant(s["x"])
        return {"y": _product(s, xq, xscale), "xq": xq, "xscale": xscale}
    if kind == "fc_i8":
        return {"y": _product(s, s["xq"], s["xscale"])}
    if kind == "ortho":
        return {"out": _orthogonal(s["g"])}
    return _muon(s)


def _own(s):
    from paper_1501_07338_amd import vcnn
    kind = s["kind"]
    dtype = vcnn.BF16 if s.get("dtype") == "bf16" else vcnn.F32
    if kind == "norm_train":
        rows, cols = s["rows"], s["cols"]
        vcnn.rmsnorm_fwd(dtype, rows, cols, EPS, s["x"], s["r"], s["gain"], s["h"], s["y"], s["rstd"])
        h = s["x"] if s["r"] is None else s["h"]
        vcnn.rmsnorm_bwd(dtype, rows, cols, h, s["gain"], s["rstd"], s["dy"], s["dabove"], s["dh"], s["dgain"], s["ws"])
        out = {"y": s["y"], "rstd": s["rstd"], "dh": s["dh"], "dgain": s["dgain"]}
        if s["r"] is not None:
            out["h"] = s["h"]
        return out
    if kind == "norm_i8":
        vcnn.rmsnorm_fwd_i8(dtype, s["rows"], s["cols"], EPS, s["x"], s["r"], s["gain"], s["h"], s["q"], s["scale"])
        out = {"q": s["q"], "scale": s["scale"]}
        if s["r"] is not None:
            out["h"] = s["h"]
        return out
    if kind == "quant":
        vcnn.quant_rows_i8(dtype, s["rows"], s["cols"], s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if kind in ("fc_dynamic", "fc_i8"):
        b, i, o = s["batch"], s["i"], s["o"]
        if kind == "fc_dynamic":
            vcnn.quant_rows_i8(dtype, b, i, s["x"], s["xq"], s["xscale"])
        vcnn.fc_fwd_i8(dtype, b, i, o, vcnn.ACT_RELU if s["act"] else vcnn.ACT_NONE, s["xq"], s["xscale"], s["wq"],
                       s["wscale"], s["b"], s["y"], s["ws"])
        return {"y": s["y"], "xq": s["xq"], "xscale": s["xscale"]} if kind == "fc_dynamic" else {"y": s["y"]}
    if kind == "ortho":
        vcnn.orthogonalize(s["rows"], s["cols"], STEPS, s["g"], s["out"], s["ws"])
        return {"out": s["out"]}
    vcnn.muon_update_multi(LR, MOMENTUM, True, DECAY, STEPS, s["w"], s["dw"], s["m"], s["ws"])
    return {"w": s["w"], "m": s["m"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------
def _svd_free_map(g):
    """The quintic applied STEPS times to g / |g|, by the smaller of its two Gram matrices."""
    tall = g.shape[0] > g.shape[1]
    x = g / torch.linalg.vector_norm(g)
    one = torch.eye(min(g.shape), dtype=torch.float64, device=g.device)
    for _ in range(STEPS):
        gram = torch.matmul(x.t().contiguous(), x) if tall else torch.matmul(x, x.t().contiguous())
        p = NS_A * one + gram.matmul(NS_B * one + NS_C * gram)
        x = x.matmul(p) if tall else p.matmul(x)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm_train", "norm_i8"):
        h = s["x"].double()
        if case["residual"]:
            h = h + s["r"].double()
            h = (h.float() if case["dtype"] == "f32" else h.to(torch.bfloat16)).double()  # as the stream is stored
        g, n = s["gain"].double(), case["cols"]
        rstd = (h.pow(2).sum(1) / n + EPS).pow(-0.5)
        if kind == "norm_i8":
            out = {"q": None, "scale": (h * g).abs().max(1).values * rstd / 127}
        else:
            dy = s["dy"].double()
            dz = dy * g
            dh = rstd[:, None] * dz - h * (rstd ** 3 * (dz * h).sum(1) / n)[:, None]
            if case["residual"]:
                dh += s["dabove"].double()
            out = {"y": h * rstd[:, None] * g, "rstd": rstd, "dh": dh, "dgain": torch.mv((dy * h).t(), rstd)}
        if case["residual"]:
            out["h"] = s["x"].double() + s["r"].double()
        return out
    if kind == "quant":
        return {"q": None, "scale": s["x"].double().abs().max(1).values / 127}
    if kind in ("fc_dynamic", "fc_i8"):
        if kind == "fc_dynamic":
            x = s["x"].double()
            most = x.abs().max(1).values
            xq, scale = torch.round(x * 127 / most[:, None]), most / 127
        else:
            xq, scale = s["xq"].double(), s["xscale"].double()
        y = torch.matmul(xq, s["wq"].double().t().contiguous()) * torch.outer(scale, s["wscale"].double())
        if case["bias"]:
            y += s["b"].double()
        if case["act"]:
            y = y.clamp(min=0)
        return {"y": y, "xq": None, "xscale": scale} if kind == "fc_dynamic" else {"y": y}
    if kind == "ortho":
        return {"out": _svd_free_map(s["g"].double())}
    w, ms = [], []
    for w0, g, m in zip(s["w"], s["dw"], s["m"]):
        g, m = g.double(), MOMENTUM * m.double() + g.double()
        o = _svd_free_map(g + MOMENTUM * m)
        w.append((1 - LR * DECAY) * w0.double() - LR * max(1.0, o.shape[0] / o.shape[1]) ** 0.5 * o)
        ms.append(m)
    return {"w": w, "m": ms}
