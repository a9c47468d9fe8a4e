"""GPU tests of layer norm, 8-bit checkpoints and output layers of many classes against plain formulas in 64 bits.

Tolerances are bounds on the error of fp32 arithmetic, u = 2^-24 being half a unit in the last place: a sum of k terms in any
order is off by at most (depth) u times the sum of the terms' magnitudes, depth being the additions in a row; a product on the
tensor cores cuts off (2 u) where an addition rounds, at least 8 products to a cut, and drops terms below 2 u of a product."""
import math

import numpy as np
import pytest
import torch

from gen import graphs
from oracle import oracle
from paper_2012_04930_b200 import gcnsa

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def _ld(f):
    return (f + 15) // 16 * 16


def _rand(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def _buf(t, padded, fill=None):
    """A copy of t in rows of _ld floats (padded) or of its own width; pad columns hold `fill` or zeros."""
    n, f = t.shape
    out = torch.zeros((n, _ld(f) if padded else f), device="cuda")
    if fill is not None:
        out.fill_(fill)
    out[:, :f] = t
    return out


def _empty(n, f, padded):
    return torch.full((n, _ld(f) if padded else f), 7.0, device="cuda")


def _bytes(n):
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device="cuda")


def _within(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    worst = ((got - want).abs() - bound).max().item() if got.numel() else -1.0
    assert worst <= 0, f"{what}: {worst:.3e} over the bound (error {(got - want).abs().max().item():.3e})"


def _pads_are_zero(t, f):
    assert torch.all(t[:, f:min(t.shape[1], (f + 3) // 4 * 4)] == 0), "pad columns come out as zeros"


# ------------------------------------------------------------- the format ---
def _steps(x):
    """Biased exponents of the blocks of x, by the definition: the smallest byte from 1 to 248 with at most 127 steps."""
    n, f = x.shape
    out = np.empty((n, (f + 31) // 32), np.int64)
    for b in range(out.shape[1]):
        top = np.abs(x[:, 32 * b:32 * b + 32].astype(np.float64)).max(axis=1)
        for i, t in enumerate(top):
            if not math.isfinite(t):
                out[i, b] = 255
                continue
            e = 1
            while e < 248 and np.rint(t / 2.0 ** (e - 127)) > 127:
                e += 1
            out[i, b] = e
    return out


def _packed_values(x):
    e = np.repeat(_steps(x), 32, axis=1)[:, :x.shape[1]]
    with np.errstate(invalid="ignore", over="ignore"):
        step = 2.0 ** (e - 127.0)
        q = np.clip(np.rint(x.astype(np.float64) / step), -127, 127)
    return np.where(e == 255, np.nan, q * step), np.where(e == 255, 0, q), _steps(x)


def _special_rows(f):
    """Rows at the format's edges: zeros, ties, 127.5 steps, subnormal, the largest values, infinities, NaN."""
    rng = np.random.default_rng(3)
    rows = [np.zeros(f), np.full(f, -1.0), np.linspace(-1.0, 1.0, f) * 127.5, np.full(f, 127.49999), rng.standard_normal(f) * 2.0 ** -140,
            rng.standard_normal(f) * 2.0 ** -121, np.full(f, 2.0 ** -149), np.where(np.arange(f) % 3 == 0, 3.4028235e38, -1e30),
            (np.arange(f) % 256 - 128) / 2.0, 64 + (np.arange(f) % 64) * 0.5, rng.standard_normal(f) * np.exp(rng.standard_normal(f) * 4)]
    for bad in (np.inf, -np.inf, np.nan):
        r = rng.standard_normal(f)
        r[f // 2] = bad
        rows.append(r)
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("f", [1, 2, 5, 16, 31, 32, 33, 64, 100, 128, 257, 602])
def test_checkpoints_hold_the_documented_values(f, padded):
    x = np.concatenate([_special_rows(f), np.random.default_rng(f).standard_normal((200, f)).astype(np.float32)])
    value, q, e = _packed_values(x)
    xd = _buf(torch.from_numpy(x).cuda(), padded, fill=math.nan)
    p = gcnsa.Packed8(x.shape[0], f)
    p.q.fill_(99)
    gcnsa.op_pack8(xd, p)
    assert np.array_equal(p.q[:, :f].cpu().numpy(), q) and np.array_equal(p.e.cpu().numpy(), e)
    assert torch.all(p.q[:, f:] == 0)
    out = _empty(x.shape[0], f, padded)
    gcnsa.op_unpack8(p, out)
    assert np.array_equal(out[:, :f].cpu().numpy(), value.astype(np.float32), equal_nan=True)
    _pads_are_zero(out, f)
    ok = np.isfinite(value)
    step = 2.0 ** (np.repeat(e, 32, axis=1)[:, :f] - 127.0)
    ok &= np.abs(x) < 127.5 * 2.0 ** 121
    assert np.all(np.abs(value - x.astype(np.float64))[ok] <= step[ok] / 2), "half a step"


def test_checkpoints_of_many_rows_and_none():
    for n, f in ((100_003, 41), (3, 20_000), (1, 1), (40_000, 16)):
        x = _rand(n, n, f)
        p, out = gcnsa.Packed8(n, f), torch.full((n + 1, f), 7.0, device="cuda")
        gcnsa.op_pack8(x, p)
        gcnsa.op_unpack8(p, out[:n])
        amax = torch.nn.functional.pad(x.abs(), (0, -f % 32)).view(n, -1, 32).amax(2).repeat_interleave(32, 1)[:, :f]
        assert torch.all((out[:n] - x).abs() <= amax / 127), "half a step is at most 1/127 of the block's largest"
        assert torch.all(out[n] == 7), "rows behind the last one are left as they were"
    gcnsa.op_pack8(torch.empty(0, 16, device="cuda"), gcnsa.Packed8(0, 16))
    gcnsa.op_unpack8(gcnsa.Packed8(0, 16), torch.empty(0, 16, device="cuda"))


# ------------------------------------------------------------- layer norm ---
def _norm64(x, gamma, beta, relu):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    v = xh * (1 if gamma is None else gamma.double()) + (0 if beta is None else beta.double())
    return (v.clamp(min=0) if relu else v), mean[:, 0], rstd[:, 0], xh


def _depth(f):
    """Additions in a row of a row's sums: in a thread (32, or f / 256 of a row that a block walks), across lanes and warps."""
    return max(32, f / 256) + 5 + 8


WIDTHS = [1, 2, 3, 4, 8, 9, 31, 32, 33, 64, 65, 100, 128, 130, 256, 300, 512, 513, 1001, 1024, 1500, 2048, 2050, 4096, 4100, 8192, 8200]


@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("f", WIDTHS)
def test_layer_norm_forward(f, padded):
    n = 37 if f > 600 else 333
    x = _rand(f, n, f) * torch.exp(_rand(f + 1, f)) + _rand(f + 2, f)
    x[0] = 5.0                                        # no variance
    x[1] = 1e4 + torch.arange(f, device="cuda") % 3   # an offset far above the spread
    x[2] *= 1e-6
    for gamma, beta, relu in ((_rand(1, f), _rand(2, f), 1), (None, None, 0), (_rand(1, f), None, 0)):
        want, mean, rstd, xh = _norm64(x, gamma, beta, relu)
        xd, y = _buf(x, padded, fill=math.nan), _empty(n + 1, f, padded)
        mo, ro = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        x8, y8, bits = gcnsa.Packed8(n, f), gcnsa.Packed8(n, f), torch.zeros((n, (f + 31) // 32), dtype=torch.int32, device="cuda")
        gcnsa.op_layer_norm(xd, f, y[:n], gamma=gamma, beta=beta, eps=EPS, relu=relu, mean=mo, rstd=ro, x8=x8, y8=y8,
                            bits=bits if relu else None)
        if relu:
            assert torch.equal(_open_bits(bits, f), y[:n, :f] > 0)
        k = _depth(f) + 8
        size = (1 + xh.abs()) * (1 if gamma is None else gamma.double().abs())
        # the mean's correction has the depth of a sum of |x - m0|, whose mean is at most a standard deviation (plus that of eps)
        _within(y[:n, :f], want, k * U * size + 2 * U * want.abs() + 2 * U * (0 if beta is None else beta.double().abs()), f"y f={f}")
        _within(mo, mean, 2 * U * mean.abs() + k * U / rstd, "mean")
        _within(ro, rstd, k * U * rstd, "rstd")
        _pads_are_zero(y[:n], f)
        assert torch.all(y[n] == 7), "the row behind the last one"
        # the checkpoints are those of x and of the y that was written
        for src, p in ((x, x8), (y[:n, :f], y8)):
            alone = gcnsa.Packed8(n, f)
            gcnsa.op_pack8(src.contiguous(), alone)
            assert torch.equal(p.q, alone.q) and torch.equal(p.e, alone.e)
        gcnsa.op_layer_norm(xd, f, xd, gamma=gamma, beta=beta, eps=EPS, relu=relu)   # in place
        assert torch.equal(xd[:, :f], y[:n, :f])


def _open_bits(bits, f):
    return ((bits.repeat_interleave(32, dim=1)[:, :f] >> (torch.arange(f, device="cuda", dtype=torch.int32) % 32)) & 1) != 0


def _grad64(g, x, mean, rstd, gamma, beta, relu, through=None):
    g, x, mean, rstd = g.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    ga = torch.ones(g.shape[1], dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    be = torch.zeros_like(ga) if beta is None else beta.double()
    xh = (x - mean) * rstd
    if relu:
        g = torch.where(xh * ga + be > 0 if through is None else through, g, torch.zeros_like(g))
    u = g * ga
    dx = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    size = rstd * (u.abs() + u.abs().mean(1, keepdim=True) + xh.abs() * (u * xh).abs().mean(1, keepdim=True))
    return dx, (g * xh).sum(0), g.sum(0), size, (g * xh).abs().sum(0), g.abs().sum(0)


@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("f", WIDTHS)
def test_layer_norm_backward(f, padded):
    n = 37 if f > 600 else 700
    x = _rand(f, n, f) * torch.exp(_rand(f + 1, f)) + _rand(f + 2, f)
    g = _rand(f + 3, n, f)
    p = gcnsa.Packed8(n, f)
    gcnsa.op_pack8(x, p)
    restored = torch.empty(n, f, device="cuda")
    gcnsa.op_unpack8(p, restored)
    for gamma, beta, relu in ((_rand(1, f), _rand(2, f), 1), (_rand(1, f), None, 1), (None, None, 0)):
        y, mean, rstd = _empty(n, f, padded), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        gcnsa.op_layer_norm(_buf(x, padded), f, y, gamma=gamma, beta=beta, eps=EPS, relu=relu, mean=mean, rstd=rstd)
        for src, values in ((_buf(x, padded, fill=math.nan), x), (p, restored)):
            want, dgamma, dbeta, size, s1, s2 = _grad64(g, values, mean, rstd, gamma, beta, relu)
            dx = _empty(n + 1, f, padded)
            start = _rand(9, 2, f)
            dg, db = start[0].clone(), start[1].clone()
            gd = _buf(g, padded, fill=math.nan)
            ws = _bytes(gcnsa.op_layer_norm_backward_scratch(n, f))
            gcnsa.op_layer_norm_backward(gd, src, f, dx[:n], mean, rstd, gamma=gamma, beta=beta, relu=relu, dgamma=dg, dbeta=db,
                                         accumulate=1, scratch=ws)
            k = _depth(f) + 12
            _within(dx[:n, :f], want, k * U * size, f"dx f={f}")
            _pads_are_zero(dx[:n], f)
            assert torch.all(dx[n] == 7)
            kr = n + 24  # rows in a row at most, then the partial sums
            _within(dg, dgamma + start[0].double(), kr * U * (s1 + start[0].double().abs()), "dgamma")
            _within(db, dbeta + start[1].double(), kr * U * (s2 + start[1].double().abs()), "dbeta")
            again, dg2 = _empty(n, f, padded), torch.empty(f, device="cuda")
            gcnsa.op_layer_norm_backward(gd, src, f, again, mean, rstd, gamma=gamma, beta=beta, relu=relu, dgamma=dg2, scratch=ws)
            assert torch.equal(again[:, :f], dx[:n, :f]), "the same bits with one sum asked for"
            gcnsa.op_layer_norm_backward(gd, src, f, gd, mean, rstd, gamma=gamma, beta=beta, relu=relu)   # in place, no sums
            assert torch.equal(gd[:, :f], dx[:n, :f])
            if relu:   # what the ReLU let through as bits of any pattern
                through = _rand(11, n, f) > 0.3
                bits = torch.zeros((n, (f + 31) // 32 * 32), dtype=torch.int64, device="cuda")
                bits[:, :f] = through
                bits = (bits.view(n, -1, 32) << torch.arange(32, device="cuda")).sum(2)
                bits = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32)
                want, dgamma, _, size, s1, _ = _grad64(g, values, mean, rstd, gamma, beta, 1, through)
                gcnsa.op_layer_norm_backward(_buf(g, padded), src, f, again, mean, rstd, gamma=gamma, beta=beta, relu=1, dgamma=dg2,
                                             scratch=ws, bits=bits)
                _within(again[:, :f], want, k * U * size, f"dx f={f}, bits")
                _within(dg2, dgamma, kr * U * s1, "dgamma, bits")


def test_layer_norm_backward_against_differences():
    """The loss <g, y(x)> along a direction v: central differences of the forward formula in 64 bits against <dx, v>, whose error
    is that of the fp32 gradient (its bound summed over the entries) and O(h^2) = 1e-10 of the third derivatives."""
    n, f = 5, 24
    x, g, gamma, beta, v = _rand(1, n, f), _rand(2, n, f), _rand(3, f), _rand(4, f), _rand(5, n, f)
    y, mean, rstd, dx = torch.empty(n, f, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, f, device="cuda")
    gcnsa.op_layer_norm(x, f, y, gamma=gamma, beta=beta, eps=EPS, relu=1, mean=mean, rstd=rstd)
    gcnsa.op_layer_norm_backward(g, x, f, dx, mean, rstd, gamma=gamma, beta=beta, relu=1)
    h = 1e-6
    assert (_norm64(x, gamma, beta, 0)[0].abs().min() > 1e-4).item(), "no value within reach of the ReLU's corner"
    diff = ((_norm64(x.double() + h * v.double(), gamma, beta, 1)[0] - _norm64(x.double() - h * v.double(), gamma, beta, 1)[0]) * g.double()).sum() / (2 * h)
    size = _grad64(g, x, mean, rstd, gamma, beta, 1)[3]
    slack = ((_depth(f) + 12) * U * size * v.double().abs()).sum() + 1e-7 * size.sum()
    assert abs((dx.double() * v.double()).sum() - diff) <= slack


def test_layer_norm_keeps_values_that_are_not_finite_in_their_rows():
    n, f = 70, 96
    x, g = _rand(1, n, f), _rand(2, n, f)
    x[3, 7], x[11, 0], x[12, 95] = math.nan, math.inf, -math.inf
    bad = [3, 11, 12]
    good = [i for i in range(n) if i not in bad]
    y, mean, rstd = torch.empty(n, f, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    gcnsa.op_layer_norm(x, f, y, eps=EPS, relu=1, mean=mean, rstd=rstd)
    assert torch.isnan(y[bad]).any(1).all() and torch.isnan(rstd[bad]).all()
    assert torch.isfinite(y[good]).all() and torch.isfinite(rstd[good]).all()
    dx, dg, db = torch.empty(n, f, device="cuda"), torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
    gcnsa.op_layer_norm_backward(g, x, f, dx, mean, rstd, dgamma=dg, dbeta=db, scratch=_bytes(gcnsa.op_layer_norm_backward_scratch(n, f)))
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[good]).all() and torch.isnan(dg).all() and torch.isfinite(db).all()
    # no rows: sums of nothing
    gcnsa.op_layer_norm_backward(g[:0], x[:0], f, dx[:0], mean[:0], rstd[:0], dgamma=dg, dbeta=db, scratch=_bytes(gcnsa.op_layer_norm_backward_scratch(0, f)))
    assert torch.all(dg == 0) and torch.all(db == 0)
    gcnsa.op_layer_norm(x[:0], f, y[:0])


def test_many_rows():
    """More rows than the kernels have teams at a time."""
    n, f = 70_001, 20
    x, g, gamma, beta = _rand(1, n, f), _rand(2, n, f), _rand(3, f), _rand(4, f)
    y, mean, rstd, dx = torch.empty(n, f, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, f, device="cuda")
    dg, db = torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
    gcnsa.op_layer_norm(x, f, y, gamma=gamma, beta=beta, eps=EPS, relu=1, mean=mean, rstd=rstd)
    want, _, _, xh = _norm64(x, gamma, beta, 1)
    _within(y, want, 53 * U * (1 + xh.abs()) * gamma.double().abs() + 2 * U * (want.abs() + beta.double().abs()), "y")
    gcnsa.op_layer_norm_backward(g, x, f, dx, mean, rstd, gamma=gamma, beta=beta, relu=1, dgamma=dg, dbeta=db,
                                 scratch=_bytes(gcnsa.op_layer_norm_backward_scratch(n, f)))
    want, dgamma, dbeta, size, s1, s2 = _grad64(g, x, mean, rstd, gamma, beta, 1)
    _within(dx, want, 57 * U * size, "dx")
    _within(dg, dgamma, 400 * U * s1, "dgamma")
    _within(db, dbeta, 400 * U * s2, "dbeta")


# ---------------------------------------------- products with checkpoints ---
@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("n,f,c", [(1, 1, 1), (31, 5, 3), (64, 128, 64), (65, 33, 129), (500, 130, 65), (1000, 602, 41), (4097, 128, 128),
                                   (20_011, 100, 7), (30_000, 257, 256), (9, 700, 300), (100_000, 16, 16)])
def test_weight_gradient_from_a_checkpoint(n, f, c, padded):
    x, g = _rand(n + f, n, f) * torch.exp(_rand(f, f)), _rand(n + c, n, c)
    p = gcnsa.Packed8(n, f)
    gcnsa.op_pack8(x, p)
    restored = torch.empty(n, f, device="cuda")
    gcnsa.op_unpack8(p, restored)
    gd, start = _buf(g, padded, fill=math.nan), _rand(7, f, c)
    want, size = restored.double().t() @ g.double(), restored.double().abs().t() @ g.double().abs()
    for accumulate in (0, 1):
        dw = _buf(start, padded, fill=0.0)
        gcnsa.op_gemm_packed8(p, gd, c, dw, accumulate=accumulate, workspace=_bytes(gcnsa.op_gemm_packed8_workspace(n, f, c)))
        extra = start.double() if accumulate else 0
        _within(dw[:, :c], want + extra, (min(n, 700) + 24) * U * size + 2 * U * start.double().abs(), f"dw {n} {f} {c}")
    assert gcnsa.tc_status() == 0


def test_weight_gradient_edges():
    p = gcnsa.Packed8(0, 8)
    dw = torch.full((8, 4), 3.0, device="cuda")
    gcnsa.op_gemm_packed8(p, torch.empty(0, 4, device="cuda"), 4, dw, accumulate=1)
    assert torch.all(dw == 3)
    gcnsa.op_gemm_packed8(p, torch.empty(0, 4, device="cuda"), 4, dw)
    assert torch.all(dw == 0)
    # a block that is not finite reaches the features of that block, a NaN in G its column, and no others
    n, f, c = 300, 96, 40
    x, g = _rand(1, n, f), _rand(2, n, c)
    x[17, 40] = math.inf
    g[200, 5] = math.nan
    p = gcnsa.Packed8(n, f)
    gcnsa.op_pack8(x, p)
    dw = torch.empty(f, c, device="cuda")
    gcnsa.op_gemm_packed8(p, g, c, dw, workspace=_bytes(gcnsa.op_gemm_packed8_workspace(n, f, c)))
    nan = torch.isnan(dw)
    want = torch.zeros(f, c, dtype=torch.bool, device="cuda")
    want[32:64], want[:, 5] = True, True
    assert torch.equal(nan, want)


# ------------------------------------------------------------ output layer ---
def _ce64(h, w, bias, y, mask, n_train):
    """Loss and gradients in 64 bits, and bounds on the error of fp32 results."""
    h, w = h.double(), w.double()
    n, d = h.shape
    c = w.shape[1]
    z = h @ w + (0 if bias is None else bias.double())
    ez = (d + 6) * U * (h.abs() @ w.abs()) + 2 * U * z.abs()            # of a logit
    on = torch.ones(n, dtype=torch.float64, device="cuda") if mask is None else (mask != 0).double()
    share = on / max(n_train, 1)
    lse = torch.logsumexp(z, 1)
    label = torch.nn.functional.one_hot(y.long().clamp(0, c - 1), c).double()
    p = torch.exp(z - lse[:, None])
    G = (p - label) * share[:, None]
    # lse is off by at most the largest error of its logits and the depth of its sum; exp by 2 units and its argument's rounding
    el = ez.max(1).values + (c / 32 + 24) * U + 2 * U * lse.abs()
    eG = share[:, None] * (p * (ez + el[:, None] + 2 * U * (z - lse[:, None]).abs() + 8 * U) + 4 * U * (p + label))
    ht, wt = h.abs(), w.abs()
    k = lambda m: (m + 16) * U  # noqa: E731 - additions in a row of a sum over m
    return {"loss": (((lse - (z * label).sum(1)) * share).sum(), ((el + (ez * label).sum(1) + 4 * U * (lse.abs() + (z * label).sum(1).abs())) * share).sum() + 1e-30),
            "dh": (G @ w.t(), eG @ wt.t() + k(c) * (G.abs() @ wt.t())),
            "dw": (h.t() @ G, ht.t() @ eG + k(n) * (ht.t() @ G.abs())),
            "db": (G.sum(0), eG.sum(0) + k(n) * G.abs().sum(0))}


def _ce_run(h, w, bias, y, mask, n_train, padded=True, accumulate=0, want=("dh", "dw", "db"), start=None):
    n, d = h.shape
    c = w.shape[1]
    hd, wd = _buf(h, padded), _buf(w, padded)
    out = {"loss": torch.full((1,), 7.0, device="cuda"), "dh": _empty(n, d, padded), "dw": _empty(d, c, padded), "db": torch.full((c,), 7.0, device="cuda")}
    if start is not None:
        out["dw"][:, :c], out["db"][:] = start
    gcnsa.op_linear_ce(hd, d, wd, c, y, n_train, out["loss"], dh=out["dh"] if "dh" in want else None, dw=out["dw"] if "dw" in want else None,
                       db=out["db"] if "db" in want else None, bias=bias, mask=mask, accumulate=accumulate,
                       workspace=_bytes(gcnsa.op_linear_ce_workspace(n, d, c)))
    assert gcnsa.tc_status() == 0
    return {"loss": out["loss"][0], "dh": out["dh"][:, :d], "dw": out["dw"][:, :c], "db": out["db"]}


CE_SIZES = [(1, 1, 1), (5, 3, 2), (256, 128, 41), (129, 16, 64), (130, 33, 65), (200, 64, 128), (257, 41, 129), (300, 100, 1000), (1000, 256, 257),
            (77, 602, 300), (2049, 64, 513), (40, 8, 5003), (6000, 20, 47), (3000, 700, 130)]


@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("n,d,c", CE_SIZES)
def test_output_layer_loss_and_gradients(n, d, c, padded):
    h, w, bias = torch.relu(_rand(n, n, d)) * 2, _rand(d, d, c) / math.sqrt(d), _rand(c, c)
    y = (torch.arange(n, device="cuda", dtype=torch.int32) * 7919) % c
    mask = (_rand(3, n) < 0.5).to(torch.uint8)
    for b, m in ((bias, mask), (None, None)):
        nt = n if m is None else int(m.sum())
        ref = _ce64(h, w, b, y, m, nt)
        got = _ce_run(h, w, b, y, m, nt, padded)
        for k in ("loss", "dh", "dw", "db"):
            _within(got[k], ref[k][0], ref[k][1], f"{k} {n} {d} {c}")
    if m is None:
        start = (_rand(5, d, c), _rand(6, c))
        acc = _ce_run(h, w, None, y, None, n, padded, accumulate=1, start=start)
        _within(acc["dw"], ref["dw"][0] + start[0].double(), ref["dw"][1] + 2 * U * (start[0].double().abs() + ref["dw"][0].abs()), "dw added")
        _within(acc["db"], ref["db"][0] + start[1].double(), ref["db"][1] + 2 * U * (start[1].double().abs() + ref["db"][0].abs()), "db added")
        # what is not asked for is not written, and the rest has the same bits
        for only in ((), ("dh",), ("dw",), ("db",)):
            part = _ce_run(h, w, None, y, None, n, padded, want=only)
            assert torch.equal(part["loss"], got["loss"])
            for k in ("dh", "dw", "db"):
                assert torch.equal(part[k], got[k]) if k in only else torch.all(part[k] == 7), (only, k)


@pytest.mark.parametrize("c", [41, 700])
def test_output_layer_without_rows_that_count(c):
    n, d = 300, 32
    h, w, y = _rand(1, n, d), _rand(2, d, c), torch.zeros(n, dtype=torch.int32, device="cuda")
    got = _ce_run(h, w, None, y, torch.zeros(n, dtype=torch.uint8, device="cuda"), 0)
    assert all(torch.all(got[k] == 0) for k in got)
    start = (_rand(5, d, c), _rand(6, c))
    got = _ce_run(h, w, None, y, torch.zeros(n, dtype=torch.uint8, device="cuda"), 0, accumulate=1, start=start)
    assert torch.equal(got["dw"], start[0]) and torch.equal(got["db"], start[1])
    got = _ce_run(h[:0], w, None, y[:0], None, 0)
    assert got["loss"] == 0 and torch.all(got["dw"] == 0) and torch.all(got["db"] == 0)
    # one row alone, and rows whose label no piece holds only where they do not count
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[137] = 1
    y = torch.full((n,), -100, dtype=torch.int32, device="cuda")
    y[137] = c - 1
    ref = _ce64(h, w, None, y, mask, 1)
    got = _ce_run(h, w, None, y, mask, 1)
    for k in got:
        _within(got[k], ref[k][0], ref[k][1], k)


@pytest.mark.parametrize("c", [41, 700])
def test_output_layer_wrong_counts_and_labels_show_in_the_loss(c):
    n, d = 200, 16
    h, w = _rand(1, n, d), _rand(2, d, c)
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    mask = torch.ones(n, dtype=torch.uint8, device="cuda")
    for wrong in (0, 1, n - 1):
        assert torch.isnan(_ce_run(h, w, None, y, mask, wrong)["loss"])
    mask[5:] = 0
    assert torch.isnan(_ce_run(h, w, None, y, mask, 6)["loss"])
    for bad in (-1, c, 2**31 - 1, -2**31):
        y[:] = 0
        y[3] = bad
        assert torch.isnan(_ce_run(h, w, None, y, mask, 5)["loss"]), bad


@pytest.mark.parametrize("c", [41, 700])
def test_output_layer_extreme_logits(c):
    """Logits of +-1e4 (a softmax without the maximum would overflow), and a row of equal ones."""
    n, d = 140, 8
    h, w = torch.zeros(n, d, device="cuda"), _rand(2, d, c)
    h[1:] = _rand(1, n - 1, d) * 4000
    y = (torch.arange(n, device="cuda", dtype=torch.int32) * 31) % c
    bias = torch.zeros(c, device="cuda")
    bias[c // 2] = torch.finfo(torch.float32).min          # a class that is masked out by the type's lowest value
    y[y == c // 2] = 0
    ref = _ce64(h, w, bias, y, None, n)
    got = _ce_run(h, w, bias, y, None, n)
    for k in ("dh", "dw", "db"):
        assert torch.isfinite(got[k]).all()
    assert torch.all(got["db"][c // 2] == 0) and torch.all(got["dw"][:, c // 2] == 0)
    _within(got["loss"], ref["loss"][0], ref["loss"][1].clamp(max=1e300), "loss")
    h[7, 0] = math.nan
    got = _ce_run(h, w, None, y, None, n)
    assert torch.isnan(got["loss"]) and torch.isnan(got["dh"][7]).all()
    assert torch.isfinite(got["dh"][:7]).all() and torch.isfinite(got["dh"][8:]).all()


@pytest.mark.parametrize("n,d,c", [(5000, 256, 1000), (9000, 128, 41), (2500, 602, 300)])
def test_output_layer_has_the_same_bits_from_run_to_run(n, d, c):
    """The pipelines of the products keep their order whatever lands first: loss and gradients of 40 calls, others between them."""
    h, w, bias = torch.relu(_rand(n, n, d)) * 2, _rand(d, d, c) / math.sqrt(d), _rand(c, c)
    y = torch.arange(n, device="cuda", dtype=torch.int32) % c
    mask = (_rand(3, n) < 0.5).to(torch.uint8)
    first = _ce_run(h, w, bias, y, mask, int(mask.sum()))
    for i in range(40):
        if i % 4 == 0:
            _ce_run(h[:777], w, None, y[:777], None, 777)
        again = _ce_run(h, w, bias, y, mask, int(mask.sum()))
        assert all(torch.equal(first[k], again[k]) for k in first), i


@pytest.mark.parametrize("n,f,c,padded", [(60_000, 256, 256, True), (20_000, 500, 64, True), (30_000, 64, 130, False)])
def test_weight_gradient_has_the_same_bits_from_run_to_run(n, f, c, padded):
    p, g = gcnsa.Packed8(n, f), _buf(_rand(1, n, c), padded)
    gcnsa.op_pack8(_rand(2, n, f), p)
    ws, first, again = _bytes(gcnsa.op_gemm_packed8_workspace(n, f, c)), torch.empty(f, c, device="cuda"), torch.empty(f, c, device="cuda")
    gcnsa.op_gemm_packed8(p, g, c, first, workspace=ws)
    for _ in range(60):
        gcnsa.op_gemm_packed8(p, g, c, again, workspace=ws)
        assert torch.equal(first, again)


# ---------------------------------------------------------- all together ---
def _step(x, rp, cc, vv, w, gamma, beta, wo, bo, y, mask, nt, out):
    """One training step of  H = relu(norm(A (X W)));  z = H Wo + bo, its hidden rows kept as checkpoints only."""
    n, f = x.shape
    d, c = w.shape[1], wo.shape[1]
    gcnsa.op_pack8(x, out["x8"])
    gcnsa.op_gemm(x, w, out["t"], n, d, f, workspace=out["gw"], mode=gcnsa.GEMM_TF32X3)
    gcnsa.op_spmm(rp, cc, vv, out["t"], d, out["s"])
    gcnsa.op_layer_norm(out["s"], d, out["h"], gamma=gamma, beta=beta, eps=EPS, relu=1, mean=out["mean"], rstd=out["rstd"], x8=out["s8"],
                        bits=out["bits"])
    out["s"].fill_(math.nan)              # only the checkpoint is left
    gcnsa.op_linear_ce(out["h"], d, wo, c, y, nt, out["loss"], dh=out["dh"], dw=out["dwo"], db=out["dbo"], bias=bo, mask=mask, workspace=out["ws"])
    gcnsa.op_layer_norm_backward(out["dh"], out["s8"], d, out["dh"], out["mean"], out["rstd"], gamma=gamma, beta=beta, relu=1,
                                 dgamma=out["dgamma"], dbeta=out["dbeta"], scratch=out["ns"], bits=out["bits"])
    gcnsa.op_spmm(rp, cc, vv, out["dh"], d, out["dt"])   # the matrix is symmetric
    gcnsa.op_gemm_packed8(out["x8"], out["dt"], d, out["dw"], workspace=out["pw"])


def _step_buffers(n, f, d, c):
    e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    return {"bits": torch.empty((n, (d + 31) // 32), dtype=torch.int32, device="cuda"), "x8": gcnsa.Packed8(n, f), "s8": gcnsa.Packed8(n, d), "t": e(n, d), "s": e(n, d), "h": e(n, d), "dh": e(n, d), "dt": e(n, d), "mean": e(n),
            "rstd": e(n), "loss": e(1), "dwo": e(d, c), "dbo": e(c), "dgamma": e(d), "dbeta": e(d), "dw": e(f, d),
            "gw": _bytes(gcnsa.op_gemm_workspace(0, 0, n, d, f, mode=gcnsa.GEMM_TF32X3)), "ws": _bytes(gcnsa.op_linear_ce_workspace(n, d, c)),
            "ns": _bytes(gcnsa.op_layer_norm_backward_scratch(n, d)), "pw": _bytes(gcnsa.op_gemm_packed8_workspace(n, f, d))}


def _problem(c, seed=0):
    rowptr, col = graphs.erdos_renyi(1500, 0.01, 5)
    rp, cc, vv = oracle.induced(rowptr, col, np.arange(rowptr.size - 1))
    n, f, d = rp.size - 1, 48, 64
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a.astype(t))).cuda()  # noqa: E731
    mask = (_rand(seed + 8, n) < 0.5).to(torch.uint8)
    return (_rand(seed + 1, n, f), dev(rp, np.int32), dev(cc, np.int32), dev(vv, np.float32), _rand(seed + 2, f, d) / 7, 1 + 0.2 * _rand(seed + 3, d),
            0.2 * _rand(seed + 4, d), _rand(seed + 5, d, c) / 8, _rand(seed + 6, c), torch.randint(0, c, (n,), device="cuda", dtype=torch.int32), mask,
            int(mask.sum())), (rp, cc, vv)


@pytest.mark.parametrize("c", [44, 1000])
def test_training_step_of_a_layer_with_norm_checkpoints_and_wide_output(c):
    """Loss and gradients of the whole step against autograd in 64 bits.  The output layer reads full hidden rows: 1e-4 of
    the largest entry, the bar of the training path.  What goes through checkpoints is off by their half steps: an entry by at
    most 1/127 of its block's largest (less than five standard deviations for all of them), independent from entry to entry, so
    the 2-norm of a gradient by less than 5 / (127 sqrt(3)) = 2.3 % where the errors average like its terms do; twice that is
    allowed, as xh enters dx in two places."""
    args, (rp, cc, vv) = _problem(c)
    x, w, gamma, beta, wo, bo, y, mask, nt = args[0], *args[4:]
    n, f = x.shape
    out = _step_buffers(n, f, w.shape[1], c)
    _step(*args, out)
    A = torch.sparse_csr_tensor(torch.from_numpy(rp.astype(np.int64)), torch.from_numpy(cc.astype(np.int64)), torch.from_numpy(vv.astype(np.float64)), (n, n)).cuda().to_dense()
    P = [t.double().requires_grad_() for t in (w, gamma, beta, wo, bo)]
    s = A @ (x.double() @ P[0])
    mean = s.mean(1, keepdim=True)
    h = torch.relu((s - mean) / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + EPS) * P[1] + P[2])
    z = h @ P[3] + P[4]
    loss = torch.nn.functional.cross_entropy(z[mask != 0], y[mask != 0].long(), reduction="sum") / nt
    loss.backward()
    assert abs(out["loss"][0] - loss) <= 1e-5 * abs(loss)
    for k, p in (("dwo", P[3]), ("dbo", P[4])):
        assert (out[k].double() - p.grad).abs().max() <= 1e-4 * p.grad.abs().max(), k
    for k, p in (("dw", P[0]), ("dgamma", P[1]), ("dbeta", P[2])):
        assert (out[k].double() - p.grad).norm() <= 0.046 * p.grad.norm(), k
    assert gcnsa.tc_status() == 0


@pytest.mark.parametrize("c", [44, 1000])
def test_a_captured_step_replays_on_new_inputs(c):
    args, _ = _problem(c)
    n, f = args[0].shape
    out, eager = _step_buffers(n, f, args[4].shape[1], c), _step_buffers(n, f, args[4].shape[1], c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(*args, out)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _step(*args, out)
    for seed in (50, 60):
        new, _ = _problem(c, seed)
        for a, b in zip(args[:11], new[:11]):
            if a.shape == b.shape:
                a.copy_(b)
        args[10].copy_(torch.roll(args[10], 0))
        k = int(args[10].sum())
        if k != args[11]:                 # the count is an argument of the recorded calls: keep it
            on, off = torch.nonzero(args[10])[:, 0], torch.nonzero(args[10] == 0)[:, 0]
            if k > args[11]:
                args[10][on[:k - args[11]]] = 0
            else:
                args[10][off[:args[11] - k]] = 1
        graph.replay()
        torch.cuda.synchronize()
        _step(*args, eager)
        torch.cuda.synchronize()
        for key in ("loss", "h", "dwo", "dbo", "dgamma", "dbeta", "dw", "dt"):
            assert torch.equal(out[key], eager[key]), key
    assert torch.isfinite(out["loss"]).all() and gcnsa.tc_status() == 0


def test_two_streams_with_workspaces_of_their_own():
    problems = [_problem(c) for c in (44, 1000)]
    alone = []
    for (args, _), c in zip(problems, (44, 1000)):
        out = _step_buffers(*args[0].shape, args[4].shape[1], c)
        _step(*args, out)
        alone.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    beside = [_step_buffers(*a[0].shape, a[4].shape[1], c) for (a, _), c in zip(problems, (44, 1000))]
    torch.cuda.synchronize()
    for _ in range(4):
        for (args, _), out, st in zip(problems, beside, streams):
            with torch.cuda.stream(st):
                _step(*args, out)
    torch.cuda.synchronize()
    for a, b in zip(alone, beside):
        for key in ("loss", "h", "dwo", "dbo", "dgamma", "dbeta", "dw"):
            assert torch.equal(a[key], b[key]), key


def test_windows_of_wider_matrices():
    """Inputs may be windows of any offset; results too where their pad columns are the window's, and nothing beside them changes."""
    n, f = 301, 45
    big = _rand(1, n, 200)
    x = big[:, 3:3 + f]
    out = torch.full((n, 200), 7.0, device="cuda")
    with pytest.raises(gcnsa.GcnsaError):
        gcnsa.op_layer_norm(x, f, out[:, 8:8 + f])
    assert torch.all(out == 7.0)
    y = out[:, 8:8 + 48]
    gcnsa.op_layer_norm(x, f, y)
    want = torch.nn.functional.layer_norm(x.double(), (f,), eps=1e-5)
    # |xh| < sqrt(45) < 7; sums of 45 terms are off by at most 45 half units, of which rstd takes half, and six roundings beside
    _within(y[:, :f], want, (22.5 + 6) * 2.0**-24 * 7, "y")
    _pads_are_zero(y, f)
    assert torch.all(out[:, :8] == 7.0) and torch.all(out[:, 56:] == 7.0)
