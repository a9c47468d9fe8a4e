"""Layer norm, 8-bit activation checkpoints and the softmax cross entropy of an output layer over many classes: cases,
inputs, the plain form of each operator and the call a user makes of the library's.

Kinds: "norm" (layer norm, forward), "norm_grad" (its backward pass), "pack" (a checkpoint is made and restored),
"norm_grad8" (the backward pass of the norm from a checkpoint of its input), "weight_grad8" (X^T G with X a checkpoint),
"linear_ce" (loss and gradients of H W + b under softmax cross entropy).
"""
import math

import torch

own = False

BLOCK = 32        # columns that share a scale in a checkpoint
EPS = 1e-5


def _ld(f):
    return (f + 15) // 16 * 16


def listed():
    return [
        # the hidden rows of a mini-batch of 256 with 10 sampled neighbours each: latency
        {"name": "norm-batch", "kind": "norm", "n": 2816, "f": 128, "relu": True, "padded": True},
        # wide rows without padding, an odd number of them
        {"name": "norm-wide", "kind": "norm", "n": 50003, "f": 1001, "relu": False, "padded": False},
        {"name": "grad-batch", "kind": "norm_grad", "n": 2816, "f": 128, "relu": True, "padded": True},
        # a hidden layer of the largest partitions
        {"name": "grad-large", "kind": "norm_grad", "n": 269498, "f": 256, "relu": True, "padded": True},
        # features of the small workload
        {"name": "pack-small", "kind": "pack", "n": 20000, "f": 500, "padded": True},
        # features of the paper's graph; 602 is no multiple of the block
        {"name": "pack-large", "kind": "pack", "n": 232965, "f": 602, "padded": True},
        # backward pass of a hidden layer whose norm kept a checkpoint
        {"name": "grad8-large", "kind": "norm_grad8", "n": 269498, "f": 256, "relu": True, "padded": True},
        # weight gradients of the first layer of the small workload and of a hidden layer of a large partition
        {"name": "wgrad8-small", "kind": "weight_grad8", "n": 20000, "f": 500, "c": 64, "padded": True},
        {"name": "wgrad8-large", "kind": "weight_grad8", "n": 245000, "f": 256, "c": 256, "padded": True},
        # one mini-batch with the paper's 41 classes: latency
        {"name": "ce-batch", "kind": "linear_ce", "n": 256, "d": 128, "c": 41, "bias": True, "masked": False, "padded": True},
        # a partition of the paper's graph
        {"name": "ce-partition", "kind": "linear_ce", "n": 58241, "d": 128, "c": 41, "bias": True, "masked": True, "padded": True},
        # many classes, every size odd
        {"name": "ce-many", "kind": "linear_ce", "n": 20011, "d": 256, "c": 10007, "bias": True, "masked": True, "padded": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "pack", "norm_grad8", "weight_grad8", "linear_ce"])
    n = _log_int(rng, 1, 270000)
    padded = rng.random() < 0.75
    if kind == "linear_ce":
        d, c = _log_int(rng, 1, 700), _log_int(rng, 1, 20000)
        n = min(n, max(1, 50_000_000_000 // (d * c)), max(1, 200_000_000 // c))
        return {"kind": kind, "n": n, "d": d, "c": c, "bias": rng.random() < 0.7, "masked": rng.random() < 0.6, "padded": padded}
    f = _log_int(rng, 1, 2000)
    n = min(n, max(1, 60_000_000 // f))
    if kind == "weight_grad8":
        c = _log_int(rng, 1, 300)
        n = min(n, max(1, 15_000_000_000 // (f * c)))
        return {"kind": kind, "n": n, "f": f, "c": c, "padded": padded}
    case = {"kind": kind, "n": n, "f": f, "padded": padded}
    if kind != "pack":
        case["relu"] = rng.random() < 0.6
    return case


def work(case):
    n = case["n"]
    if case["kind"] == "linear_ce":
        d, c = case["d"], case["c"]
        return {"bytes": 8 * (n * d + d * c) + 5 * n + 8 * c, "flops": 6 * n * d * c}
    f = case["f"]
    blocks = (f + BLOCK - 1) // BLOCK
    if case["kind"] == "norm":
        return {"bytes": 8 * n * f + 8 * n + 8 * f, "flops": 8 * n * f}
    if case["kind"] == "norm_grad":
        return {"bytes": 12 * n * f + 8 * n + 16 * f, "flops": 14 * n * f}
    if case["kind"] == "norm_grad8":
        return {"bytes": 9 * n * f + n * blocks + 8 * n + 16 * f, "flops": 14 * n * f}
    if case["kind"] == "pack":
        # made (read once, 8 bits and scales written) and restored
        return {"bytes": 2 * (5 * n * f + n * blocks), "flops": 5 * n * f}
    return {"bytes": n * f + n * blocks + 4 * n * case["c"] + 4 * f * case["c"], "flops": 2 * n * f * case["c"]}


# ------------------------------------------------------------------ inputs ---
def _rows(gen, n, f, padded, make):
    """[n, f] values of make(n, f) in rows of _ld(f) floats (pad columns zero) or of f."""
    t = torch.zeros((n, _ld(f) if padded else f), device="cuda")
    t[:, :f] = make(n, f)
    return t


def _pack_plain(x, f):
    """8-bit values [n, _ld(f)] and biased exponents [n, blocks] of the first f columns of x."""
    n = x.shape[0]
    blocks = (f + BLOCK - 1) // BLOCK
    v = torch.zeros((n, blocks * BLOCK), device=x.device)
    v[:, :f] = x[:, :f]
    v = v.view(n, blocks, BLOCK)
    amax = v.abs().amax(dim=2)
    finite = torch.isfinite(amax)
    amax = torch.where(finite, amax, torch.zeros_like(amax))
    k = torch.clamp(torch.frexp(amax).exponent - 7, min=-126)
    k = k + (torch.round(torch.ldexp(amax.double(), -k)) > 127).int()
    q = torch.round(torch.ldexp(v.double(), -k[:, :, None]))
    q = torch.where(finite[:, :, None], q, torch.zeros_like(q))
    q8 = torch.zeros((n, _ld(f)), dtype=torch.int8, device=x.device)
    q8[:, :f] = q.view(n, -1)[:, :f].to(torch.int8)
    e8 = torch.where(finite, k + 127, torch.full_like(k, 255)).to(torch.uint8)
    return q8, e8


def _unpack_plain(q8, e8, f):
    k = e8.int().repeat_interleave(BLOCK, dim=1)[:, :f]
    v = torch.ldexp(q8[:, :f].float(), k - 127)
    return torch.where(k == 255, torch.full_like(v, math.nan), v)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * (seed + 1) + 7919 * case["n"] + case.get("f", 0) + case.get("c", 0))

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    n, padded, kind = case["n"], case["padded"], case["kind"]
    s = {"case": case}
    if kind == "linear_ce":
        d, c = case["d"], case["c"]
        # hidden rows after ReLU, weights of a trained layer: logits spread over a few units
        s["h"] = _rows(gen, n, d, padded, lambda a, b: torch.relu(randn(a, b)) * 2)
        s["w"] = _rows(gen, d, c, padded, lambda a, b: randn(a, b) / math.sqrt(d))
        s["bias"] = randn(c) if case["bias"] else None
        s["y"] = torch.randint(0, c, (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["mask"] = None
        if case["masked"]:
            s["mask"] = (torch.rand(n, generator=gen, device="cuda") < 0.66).to(torch.uint8)
        s["n_train"] = n if s["mask"] is None else int(s["mask"].sum())
    else:
        f = case["f"]
        # columns of different size and offset, as a sparse product leaves them
        scale, shift = torch.exp(randn(f)), randn(f)
        s["x"] = _rows(gen, n, f, padded, lambda a, b: randn(a, b) * scale + shift)
        if kind in ("norm", "norm_grad", "norm_grad8"):
            s["gamma"], s["beta"] = 1 + 0.2 * randn(f), 0.2 * randn(f)
        if kind in ("norm_grad", "norm_grad8"):
            s["g"] = _rows(gen, n, f, padded, lambda a, b: randn(a, b) * 1e-2)
            x = s["x"][:, :f].double()
            mean = x.mean(dim=1, keepdim=True)
            var = ((x - mean) ** 2).mean(dim=1, keepdim=True)
            s["mean"], s["rstd"] = mean[:, 0].float(), torch.rsqrt(var + EPS)[:, 0].float()
        if kind == "weight_grad8":
            s["g"] = _rows(gen, n, case["c"], padded, lambda a, b: randn(a, b) * 1e-2)
        if kind in ("norm_grad8", "weight_grad8"):
            s["q"], s["e"] = _pack_plain(s["x"], f)
            del s["x"]
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """Buffers that a training program keeps from step to step."""
    from paper_2012_04930_b200 import gcnsa
    case = s["case"]
    n, kind = case["n"], case["kind"]

    def out(rows, cols):
        return torch.empty((rows, _ld(cols) if case["padded"] else cols), device="cuda")

    def scratch(nbytes):
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")

    o = s["out"] = {}
    if kind == "linear_ce":
        d, c = case["d"], case["c"]
        o["loss"] = torch.empty(1, device="cuda")
        o["dh"], o["dw"], o["db"] = out(n, d), out(d, c), torch.empty(c, device="cuda")
        o["ws"] = scratch(gcnsa.op_linear_ce_workspace(n, d, c))
        return
    f = case["f"]
    if kind == "norm":
        o["y"], o["mean"], o["rstd"] = out(n, f), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    elif kind in ("norm_grad", "norm_grad8"):
        o["dx"], o["dgamma"], o["dbeta"] = out(n, f), torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
        o["ws"] = scratch(gcnsa.op_layer_norm_backward_scratch(n, f))
    elif kind == "pack":
        o["p"], o["x"] = gcnsa.Packed8(n, f), out(n, f)
    else:
        o["dw"] = out(f, case["c"])
        o["ws"] = scratch(gcnsa.op_gemm_packed8_workspace(n, f, case["c"]))
    if kind in ("norm_grad8", "weight_grad8"):
        o["p"] = gcnsa.Packed8(n, f, q=s["q"], e=s["e"])


# ------------------------------------------------------- one pass, plain form ---
def _norm_grad_plain(g, x, mean, rstd, gamma, beta, relu):
    if relu:  # in 64 bits: values next to the ReLU's border
        before = (x.double() - mean.double()[:, None]) * rstd.double()[:, None] * gamma.double() + beta.double()
        g = torch.where(before > 0, g, torch.zeros_like(g))
    if x.shape[1] <= 8:  # what is left of g in rows of two columns is far smaller than g
        g, x, mean, rstd, gamma = (t.double() for t in (g, x, mean, rstd, gamma))
    rstd = rstd[:, None]
    xh = (x - mean[:, None]) * rstd
    u = g * gamma
    dx = rstd * (u - u.mean(dim=1, keepdim=True) - xh * (u * xh).mean(dim=1, keepdim=True))
    return dx.float(), (g * xh).sum(dim=0, dtype=torch.float64).float(), g.sum(dim=0, dtype=torch.float64).float()


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "linear_ce":
        d, c = case["d"], case["c"]
        h, w = s["h"][:, :d], s["w"][:, :c]
        z = h @ w
        if s["bias"] is not None:
            z = z + s["bias"]
        y = s["y"].long()[:, None]
        top = z.amax(dim=1, keepdim=True)
        zy = z.gather(1, y)
        p = torch.exp(z - top)
        total = p.sum(dim=1, keepdim=True)
        row_loss = (top + torch.log(total) - zy)[:, 0]
        weight = torch.full_like(total, 1.0 / max(s["n_train"], 1)) if s["n_train"] else torch.zeros_like(total)
        if s["mask"] is not None:
            weight = weight * s["mask"][:, None]
            row_loss = row_loss * s["mask"]
        loss = (row_loss.sum(dtype=torch.float64) / max(s["n_train"], 1)).float()
        p = p / total
        p.scatter_add_(1, y, torch.full_like(zy, -1.0))
        p = p * weight
        return {"loss": loss[None], "dh": p @ w.t(), "dw": h.t() @ p, "db": p.sum(dim=0)}
    f = case["f"]
    if kind == "norm":
        x = s["x"][:, :f]
        mean = x.mean(dim=1, keepdim=True)
        xc = x - mean
        rstd = torch.rsqrt((xc * xc).mean(dim=1, keepdim=True) + EPS)
        v = xc * rstd * s["gamma"] + s["beta"]
        return {"y": torch.clamp(v, min=0) if case["relu"] else v, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if kind == "pack":
        return {"x": _unpack_plain(*_pack_plain(s["x"], f), f)}
    if kind == "weight_grad8":
        return {"dw": _unpack_plain(s["q"], s["e"], f).t() @ s["g"][:, :case["c"]]}
    x = s["x"][:, :f] if kind == "norm_grad" else _unpack_plain(s["q"], s["e"], f)
    dx, dgamma, dbeta = _norm_grad_plain(s["g"][:, :f], x, s["mean"], s["rstd"], s["gamma"], s["beta"], case["relu"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def run(s):
    if not own:
        return _plain(s)
    from paper_2012_04930_b200 import gcnsa
    if "out" not in s:
        _prepare_own(s)
    case, o = s["case"], s["out"]
    kind = case["kind"]
    if kind == "linear_ce":
        d, c = case["d"], case["c"]
        gcnsa.op_linear_ce(s["h"], d, s["w"], c, s["y"], s["n_train"], o["loss"], dh=o["dh"], dw=o["dw"], db=o["db"],
                           bias=s["bias"], mask=s["mask"], workspace=o["ws"])
        return {"loss": o["loss"], "dh": o["dh"][:, :d], "dw": o["dw"][:, :c], "db": o["db"]}
    f = case["f"]
    if kind == "norm":
        gcnsa.op_layer_norm(s["x"], f, o["y"], gamma=s["gamma"], beta=s["beta"], eps=EPS, relu=case["relu"], mean=o["mean"],
                            rstd=o["rstd"])
        return {"y": o["y"][:, :f], "mean": o["mean"], "rstd": o["rstd"]}
    if kind == "pack":
        gcnsa.op_pack8(s["x"], o["p"])
        gcnsa.op_unpack8(o["p"], o["x"])
        return {"x": o["x"][:, :f]}
    if kind == "weight_grad8":
        gcnsa.op_gemm_packed8(o["p"], s["g"], case["c"], o["dw"], workspace=o["ws"])
        return {"dw": o["dw"][:, :case["c"]]}
    x = s["x"] if kind == "norm_grad" else o["p"]
    gcnsa.op_layer_norm_backward(s["g"], x, f, o["dx"], s["mean"], s["rstd"], gamma=s["gamma"], beta=s["beta"],
                                 relu=case["relu"], dgamma=o["dgamma"], dbeta=o["dbeta"], scratch=o["ws"])
    return {"dx": o["dx"][:, :f], "dgamma": o["dgamma"], "dbeta": o["dbeta"]}


# ----------------------------------------------------------- in 64 bits ---
def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear_ce":
        d, c, n = case["d"], case["c"], case["n"]
        h, w = s["h"][:, :d].double(), s["w"][:, :c].double()
        counted = torch.ones(n, dtype=torch.float64, device="cuda") if s["mask"] is None else s["mask"].double()
        share = counted / s["n_train"] if s["n_train"] else counted * 0
        dh, dw = torch.zeros_like(h), torch.zeros_like(w)
        db = torch.zeros(c, dtype=torch.float64, device="cuda")
        loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        step = max(1, 100_000_000 // c)
        for r in range(0, n, step):
            rows = slice(r, min(n, r + step))
            z = torch.addmm(s["bias"].double(), h[rows], w) if s["bias"] is not None else torch.mm(h[rows], w)
            lse = torch.logsumexp(z, dim=1)
            label = torch.nn.functional.one_hot(s["y"][rows].long(), c)
            loss += ((lse - (z * label).sum(dim=1)) * share[rows]).sum()
            grad = (torch.exp(z - lse[:, None]) - label) * share[rows][:, None]
            dh[rows] = torch.mm(grad, w.t())
            dw += torch.mm(h[rows].t(), grad)
            db += grad.sum(dim=0)
        return {"loss": loss, "dh": dh, "dw": dw, "db": db}
    f = case["f"]
    if kind == "norm":
        x = s["x"][:, :f].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * (rstd[:, None] * s["gamma"].double()[None, :]) + s["beta"].double()[None, :]
        return {"y": y.relu() if case["relu"] else y, "mean": mean, "rstd": rstd}
    if kind == "pack":
        x = s["x"][:, :f].double()
        value = torch.empty_like(x)
        for b in range(0, f, BLOCK):
            block = x[:, b:b + BLOCK]
            top = block.abs().amax(dim=1, keepdim=True)
            step = torch.exp2(torch.clamp(torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 6, min=-126))
            step = torch.where(torch.round(top / step) > 127, 2 * step, step)
            value[:, b:b + BLOCK] = torch.round(block / step) * step
        return {"x": value}
    if kind == "norm_grad":
        x = s["x"][:, :f].double()
    else:
        step = torch.exp2(s["e"].double() - 127).repeat_interleave(BLOCK, dim=1)[:, :f]
        x = s["q"][:, :f].double() * step
    if kind == "weight_grad8":
        return {"dw": torch.mm(x.t(), s["g"][:, :case["c"]].double())}
    g, gamma, beta = s["g"][:, :f].double(), s["gamma"].double(), s["beta"].double()
    xh = (x - s["mean"].double().view(-1, 1)) * s["rstd"].double().view(-1, 1)
    if case["relu"]:
        g = g * (xh * gamma + beta > 0)
    along = g * gamma
    dx = along - (along.sum(dim=1, keepdim=True) + xh * (along * xh).sum(dim=1, keepdim=True)) / f
    return {"dx": dx * s["rstd"].double().view(-1, 1), "dgamma": (g * xh).sum(dim=0), "dbeta": g.sum(dim=0)}
