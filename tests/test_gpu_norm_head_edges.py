"""GPU tests of layer norm, 8-bit checkpoints and output layers at the edges of what their calls allow: logits far from zero,
classes and rows left out, values that are not finite, pad columns.  Bounds count half units u = 2^-24, as in
test_gpu_norm_head.py."""
import math

import pytest
import torch

from paper_2012_04930_b200 import gcnsa
from test_gpu_norm_head import U, _buf, _bytes, _ce64, _ce_run, _empty, _rand, _within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------ output layer ---
def _exact_logits(c, offset):
    """Logits that fp32 holds exactly (so do the products): a row of h picks a row of w, whose entries are multiples of 2^-10, and
    the bias puts all of them `offset` off zero.  A class of every row of w stands 4 to 19 above the rest; four rows in five have
    it as their label."""
    n, d = 400, 16
    h = torch.zeros(n, d, device="cuda")
    k = torch.arange(n, device="cuda") % d
    h[torch.arange(n), k] = 1
    w = torch.round(_rand(c, d, c) * 1024) / 1024
    top = torch.arange(d, device="cuda") * 37 % c
    w[torch.arange(d), top] += 4 + torch.arange(d, device="cuda")
    y = top[k]
    y[::5] = (y[::5] + 1) % c
    return h, w, torch.full((c,), float(offset), device="cuda"), y.int()


def _exact_logits64(h, w, bias, y):
    """Loss and gradients in 64 bits and bounds for exact logits.  x = z - max is exact; x log2(e) is off by 2 u (the constant, the
    product), so its exponential by 2 u |x|, and ex2 by 4 u; a maximum that moves from tile to tile costs 5 u each; a sum has c / 32
    + 24 additions in a row; 1 / sum, probability, label, share: a u each.  Where the offset lies enters none of it."""
    n, c = h.shape[0], w.shape[1]
    z = h.double() @ w.double() + bias.double()
    x = z - z.max(1, keepdim=True).values
    p = torch.softmax(z, 1)
    far = torch.where(p > 0, p * x.abs(), torch.zeros_like(p))          # (0 for a class at -infinity)
    label = torch.nn.functional.one_hot(y.long(), c).double()
    G = (p - label) / n
    es = U * ((2 * far).sum(1) + 5 * ((c + 127) // 128 + 2) + c / 32 + 24)
    eG = (2 * U * far + p * (6 * U + es[:, None]) + 4 * U * (p - label).abs()) / n + 1e-37
    row = -torch.log_softmax(z, 1).gather(1, y.long()[:, None])[:, 0]
    log_s = torch.log(torch.exp(x).sum(1))
    ht, wt = h.double().abs(), w.double().abs()
    return {"loss": (row.mean(), (es + 4 * U * (row + log_s)).mean()),
            "dh": (G @ w.double().t(), eG @ wt.t() + (c + 16) * U * (G.abs() @ wt.t())),
            "dw": (h.double().t() @ G, ht.t() @ eG + (n + 16) * U * (ht.t() @ G.abs())),
            "db": (G.sum(0), eG.sum(0) + (n + 16) * U * G.abs().sum(0))}


@pytest.mark.parametrize("offset", [0, 30, 1000, -8000])
@pytest.mark.parametrize("c", [129, 700])
def test_confident_rows_far_from_zero(c, offset):
    """p - 1 of a confident row is what is left of two nearly equal numbers: maximum and sum of a row are kept apart, as
    their logarithm in one number would be off by half a unit of the offset."""
    h, w, bias, y = _exact_logits(c, offset)
    want = _exact_logits64(h, w, bias, y)
    got = _ce_run(h, w, bias, y, None, h.shape[0])
    for k in want:
        _within(got[k], *want[k], f"{k} c={c} offset={offset}")


@pytest.mark.parametrize("left_out", [torch.finfo(torch.float32).min, -math.inf])
@pytest.mark.parametrize("c", [41, 128, 129, 700])
def test_a_class_left_out_by_its_bias(c, left_out):
    h, w, bias, y = _exact_logits(c, 4)
    out = (int(y.max()) + 5) % c
    while bool((y == out).any()):
        out = (out + 1) % c
    bias[out] = left_out
    want = _exact_logits64(h, w, bias, y)
    got = _ce_run(h, w, bias, y, None, h.shape[0])
    for k in ("loss", "dh", "dw", "db"):
        _within(got[k], *want[k], f"{k} c={c}")
    assert torch.all(got["dw"][:, out] == 0) and got["db"][out] == 0


@pytest.mark.parametrize("offset", [0, 30, 1000, -8000])
@pytest.mark.parametrize("c", [2, 41, 64, 128])
def test_confident_rows_of_a_few_classes(c, offset):
    """The same where a tile holds whole rows: the label's distance from the maximum is taken before the sum's logarithm is added."""
    h, w, bias, y = _exact_logits(c, offset)
    want = _exact_logits64(h, w, bias, y)
    got = _ce_run(h, w, bias, y, None, h.shape[0])
    for k in want:
        _within(got[k], *want[k], f"{k} c={c} offset={offset}")


@pytest.mark.parametrize("padded", [True, False])
@pytest.mark.parametrize("c", [1, 41, 64, 128, 129, 700])
def test_rows_that_do_not_count_may_hold_anything(c, padded):
    n, d = 1111, 45
    h, w, y = _rand(1, n, d), _rand(2, d, c) / 7, torch.arange(n, device="cuda", dtype=torch.int32) % c
    mask = (_rand(3, n) < 0.5).to(torch.uint8)
    mask[200:330] = 0                                  # whole blocks of rows among them
    off = torch.nonzero(mask == 0)[:, 0]
    nt = int(mask.sum())
    h[off] = 0
    want = _ce_run(h, w, None, y, mask, nt, padded)
    assert all(torch.isfinite(v).all() for v in want.values())
    for bad in (math.nan, math.inf, -math.inf, 3e38):
        h[off] = bad
        got = _ce_run(h, w, None, y, mask, nt, padded)
        for k in want:
            assert torch.equal(got[k], want[k]), (k, bad)
    assert torch.all(got["dh"][off] == 0)


# ------------------------------------------------------------- pad columns ---
@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("n", [30, 5000])
def test_pad_columns_beside_values_that_are_not_finite(n, accumulate):
    """A line of a result has zeros up to the next multiple of 4 (with accumulate: what was there), whatever the products hold and
    however many slices they are cut into."""
    pad = 7.0 if accumulate else 0.0
    f, c = 40, 5
    p = gcnsa.Packed8(n, f)
    x = _rand(1, n, f)
    x[n // 2, 3] = math.nan
    gcnsa.op_pack8(x, p)
    dw = torch.full((f, 16), 7.0, device="cuda")
    gcnsa.op_gemm_packed8(p, _rand(2, n, 16), c, dw, accumulate=accumulate, workspace=_bytes(gcnsa.op_gemm_packed8_workspace(n, f, c)))
    assert torch.isnan(dw[:32, :c]).all() and torch.isfinite(dw[32:, :c]).all()
    assert torch.all(dw[:, c:8] == pad) and torch.all(dw[:, 8:] == 7.0)
    for c in (5, 131):
        d = 6
        h, w, y = _rand(3, n, 16), _rand(4, d, 144), torch.zeros(n, dtype=torch.int32, device="cuda")
        h[n // 3, 2] = math.nan
        loss, dh, dw = torch.empty(1, device="cuda"), torch.full((n, 16), 7.0, device="cuda"), torch.full((d, 144), 7.0, device="cuda")
        gcnsa.op_linear_ce(h, d, w, c, y, n, loss, dh=dh, dw=dw, accumulate=accumulate, workspace=_bytes(gcnsa.op_linear_ce_workspace(n, d, c)))
        assert torch.isnan(loss).all() and torch.isnan(dh[n // 3, :d]).all() and torch.isnan(dw[:, :c]).all()
        up = (c + 3) // 4 * 4
        assert torch.all(dw[:, c:up] == pad) and torch.all(dw[:, up:] == 7.0), c
        assert torch.all(dh[:, d:8] == 0) and torch.all(dh[:, 8:] == 7.0), c


# -------------------------------------------------------------- layer norm ---
@pytest.mark.parametrize("f", [7, 9, 33, 100, 130, 300, 600, 1001, 1500, 4100, 8200])
def test_norm_backward_of_equal_values_far_from_zero(f):
    """x is its own mean: xh is 0 and dx = rstd (u - mean(u)).  The places of a team past the row's end have no say, though there
    (0 - mean) rstd is beyond fp32."""
    n = 9
    x, mean, rstd = torch.full((n, f), 2.0 ** 123, device="cuda"), torch.full((n,), 2.0 ** 123, device="cuda"), torch.full((n,), 316.0, device="cuda")
    g, gamma = _rand(f, n, f), _rand(f + 1, f)
    p = gcnsa.Packed8(n, f)
    gcnsa.op_pack8(x, p)                                # (a power of two: the checkpoint holds it as it is)
    u = g.double() * gamma.double()
    want = 316.0 * (u - u.mean(1, keepdim=True))
    bound = (max(32, f / 256) + 25) * U * 316.0 * (u.abs() + u.abs().mean(1, keepdim=True))
    for padded in (True, False):
        for src in (_buf(x, padded), p):
            for relu, beta in ((0, None), (1, torch.ones(f, device="cuda"))):   # (v = 1: the ReLU lets all through)
                dx, dg = _empty(n, f, padded), torch.empty(f, device="cuda")
                gcnsa.op_layer_norm_backward(_buf(g, padded), src, f, dx, mean, rstd, gamma=gamma, beta=beta, relu=relu, dgamma=dg,
                                             scratch=_bytes(gcnsa.op_layer_norm_backward_scratch(n, f)))
                _within(dx[:, :f], want, bound, f"dx f={f}")
                assert torch.all(dg == 0)


@pytest.mark.parametrize("f", [5, 41, 128, 602, 1500])
def test_norm_backward_with_offsets_is_off_by_the_mean_s_rounding(f):
    """Rows 1e4 off zero with a spread of 1.  The forward pass hands on the mean in 32 bits, half a unit of 1e4 off, and xh of the
    whole row is shifted by that: the gradient is that of the shifted xh, not closer."""
    n = 300
    x = 1e4 + _rand(f, n, f)
    g = _rand(f + 1, n, f)
    y, mean, rstd, dx = torch.empty(n, f, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, f, device="cuda")
    dg = torch.empty(f, device="cuda")
    gcnsa.op_layer_norm(x, f, y, mean=mean, rstd=rstd)
    gcnsa.op_layer_norm_backward(g, x, f, dx, mean, rstd, dgamma=dg, scratch=_bytes(gcnsa.op_layer_norm_backward_scratch(n, f)))
    x, g = x.double(), g.double()
    m = x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + 1e-5)
    xh = (x - m) * r
    c2, g1 = (g * xh).mean(1, keepdim=True), g.abs().mean(1, keepdim=True)
    want = r * (g - g.mean(1, keepdim=True) - xh * c2)
    k = max(32, f / 256) + 25
    shift = U * m.abs() * r + (k + 8) * U               # of xh; the sum of the mean itself has the depth of the rows' deviations
    size = r * (g.abs() + g1 + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    moved = r * (shift * (c2.abs() + xh.abs() * g1) + shift ** 2 * g1)
    _within(dx, want, 2 * k * U * size + moved, f"dx f={f}")
    _within(dg, (g * xh).sum(0), (g.abs() * shift).sum(0) + (n + 24 + k) * U * (g * xh).abs().sum(0), "dgamma")


# ------------------------------------------------- infinities in operands ---
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("c", [41, 700])
def test_values_that_are_not_finite_make_nan_of_what_they_enter(c, bad):
    """Also an infinity, also where the formula has an infinity or a probability of 0: it has no terms to be cut into."""
    n, d = 200, 24
    h, w, y = _rand(1, n, d), _rand(2, d, c), torch.arange(n, device="cuda", dtype=torch.int32) % c
    one = h.clone()
    one[17, 3] = bad
    got = _ce_run(one, w, None, y, None, n)
    rest = torch.arange(n, device="cuda") != 17
    assert torch.isnan(got["loss"]) and torch.isnan(got["dh"][17]).all() and torch.isfinite(got["dh"][rest]).all()
    assert torch.isnan(got["dw"]).all() and torch.isnan(got["db"]).all()
    w[5, 7] = bad
    got = _ce_run(h, w, None, y, None, n)
    assert torch.isnan(got["loss"]) and all(torch.isnan(got[k]).all() for k in ("dh", "dw", "db"))
    f = 40
    p, g = gcnsa.Packed8(n, f), _rand(3, n, c)
    gcnsa.op_pack8(_rand(4, n, f), p)
    g[100, 6] = bad
    dw = torch.empty(f, c, device="cuda")
    gcnsa.op_gemm_packed8(p, g, c, dw, workspace=_bytes(gcnsa.op_gemm_packed8_workspace(n, f, c)))
    assert torch.isnan(dw[:, 6]).all() and torch.isfinite(dw[:, :6]).all() and torch.isfinite(dw[:, 7:]).all()


@pytest.mark.parametrize("f", [9, 100, 1500, 8200])
def test_norms_of_rows_beyond_fp32_sums(f):
    """A sum beyond the largest fp32 number is an infinity (the row NaN), squares beyond it make rstd 0 (the row beta); other rows
    keep their values."""
    x, beta = _rand(f, 40, f), _rand(f + 1, f)
    y, rstd = torch.empty(40, f, device="cuda"), torch.empty(40, device="cuda")
    gcnsa.op_layer_norm(x, f, y, beta=beta, rstd=rstd)
    far, yf, rf = x.clone(), torch.empty(40, f, device="cuda"), torch.empty(40, device="cuda")
    far[5], far[6] = 3e38, x[6] * 1e25
    gcnsa.op_layer_norm(far, f, yf, beta=beta, rstd=rf)
    assert torch.isnan(yf[5]).all() and torch.isnan(rf[5])
    assert torch.equal(yf[6], beta) and rf[6] == 0
    rest = [i for i in range(40) if i not in (5, 6)]
    assert torch.equal(yf[rest], y[rest]) and torch.equal(rf[rest], rstd[rest])


@pytest.mark.parametrize("padded,masked", [(True, True), (False, True), (True, False)])
def test_output_layer_in_several_pieces(padded, masked):
    """G^T of all classes is beyond what is kept of it at a time (160 MB): dh is added up over pieces of the classes, and
    weights and biases of every piece have their own columns."""
    n, d, c = 3001, 21, 30011
    h, w, bias = torch.relu(_rand(1, n, d)) * 2, _rand(2, d, c) / math.sqrt(d), _rand(3, c)
    y = (torch.arange(n, device="cuda", dtype=torch.int32) * 7919) % c
    mask = (_rand(4, n) < 0.9).to(torch.uint8) if masked else None
    nt = n if mask is None else int(mask.sum())
    assert nt * c * 4 > 160 * 2 ** 20
    ref = _ce64(h, w, bias, y, mask, nt)
    start = (_rand(5, d, c) / 1000, _rand(6, c) / 1000)
    got = _ce_run(h, w, bias, y, mask, nt, padded, accumulate=1, start=start)
    for k, add in (("loss", 0), ("dh", 0), ("dw", start[0].double()), ("db", start[1].double())):
        _within(got[k], ref[k][0] + add, ref[k][1] + 2 * U * (ref[k][0].abs() + abs(add)), k)
    again = _ce_run(h, w, bias, y, mask, nt, padded, want=("dh",))
    assert torch.equal(again["dh"], got["dh"]) and torch.equal(again["loss"], got["loss"])
