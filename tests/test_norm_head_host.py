"""Layer norm, 8-bit checkpoints and output layers of many classes: what is refused before any device work, and sizes.
Needs no GPU (the pointers are made-up addresses that are never dereferenced)."""
import ctypes as C

import pytest
import torch

from paper_2012_04930_b200 import gcnsa

BASE = 0x7f0000000000


def _p8(q=BASE + 0x4000000, ldq=128, e=BASE + 0x5000000, lde=4):
    return C.byref(gcnsa.Packed8Dev(q=q, ldq=ldq, e=e, lde=lde))


@pytest.fixture(autouse=True)
def _no_launch():
    before = gcnsa.launch_count()
    yield
    assert gcnsa.launch_count() == before


def test_layer_norm_refusals():
    L = gcnsa.lib()

    def fwd(n=100, f=128, x=BASE, ldx=128, eps=1e-5, y=BASE + 0x100000, ldy=128, x8=None, y8=None, relu=0, bits=None,
            ldbits=0):
        return L.gcnsa_op_layer_norm(None, n, f, x, ldx, None, None, eps, relu, y, ldy, None, None, x8, y8, bits, ldbits)
    assert fwd(n=-1) == gcnsa.ERR_ARG and fwd(f=0) == gcnsa.ERR_ARG
    assert fwd(f=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25) == gcnsa.ERR_TOO_LARGE
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(eps=eps) == gcnsa.ERR_ARG
    assert fwd(x=None) == gcnsa.ERR_ARG and fwd(y=None) == gcnsa.ERR_ARG
    assert fwd(ldx=127) == gcnsa.ERR_ARG and fwd(ldy=127) == gcnsa.ERR_ARG
    assert fwd(y=BASE, ldy=256) == gcnsa.ERR_ARG                       # in place with another pitch
    for bad in (_p8(q=None), _p8(e=None), _p8(ldq=120), _p8(ldq=112), _p8(q=BASE + 8), _p8(lde=3)):
        assert fwd(x8=bad) == gcnsa.ERR_ARG and fwd(y8=bad) == gcnsa.ERR_ARG
    assert fwd(bits=BASE + 0x700000, ldbits=4) == gcnsa.ERR_ARG        # without a ReLU
    assert fwd(bits=BASE + 0x700000, ldbits=3, relu=1) == gcnsa.ERR_ARG
    assert fwd(n=0, x=None, y=None) == 0

    def bwd(n=100, f=128, g=BASE, ldg=128, x=BASE + 0x100000, ldx=128, x8=None, mean=BASE + 0x200000, rstd=BASE + 0x210000,
            dx=BASE + 0x300000, lddx=128, dgamma=BASE + 0x400000, dbeta=None, scratch=BASE + 0x500000, sbytes=1 << 30,
            relu=0, bits=None, ldbits=0):
        return L.gcnsa_op_layer_norm_backward(None, n, f, g, ldg, x, ldx, x8, mean, rstd, None, None, relu, bits, ldbits, dx, lddx,
                                              dgamma, dbeta, 0, scratch, sbytes)
    assert bwd(bits=BASE + 0x700000, ldbits=4) == gcnsa.ERR_ARG and bwd(bits=BASE + 0x700000, ldbits=3, relu=1) == gcnsa.ERR_ARG
    assert bwd(n=-1) == gcnsa.ERR_ARG and bwd(f=0) == gcnsa.ERR_ARG
    assert bwd(f=(1 << 24) + 1) == gcnsa.ERR_TOO_LARGE
    for k in ("g", "mean", "rstd", "dx", "scratch"):
        assert bwd(**{k: None}) == gcnsa.ERR_ARG, k
    assert bwd(x=None) == gcnsa.ERR_ARG                                # neither x nor a checkpoint
    assert bwd(x8=_p8()) == gcnsa.ERR_ARG                              # both
    assert bwd(x=None, x8=_p8(ldq=120)) == gcnsa.ERR_ARG
    assert bwd(ldg=100) == gcnsa.ERR_ARG and bwd(ldx=100) == gcnsa.ERR_ARG and bwd(lddx=100) == gcnsa.ERR_ARG
    assert bwd(dx=BASE, lddx=256) == gcnsa.ERR_ARG and bwd(dx=BASE + 0x100000, lddx=256) == gcnsa.ERR_ARG
    need = gcnsa.op_layer_norm_backward_scratch(100, 128)
    assert gcnsa.op_layer_norm_backward_scratch(10**6, 1 << 24) <= 1 << 29     # partial sums of wide rows are bounded
    assert need >= 2 * 128 * 4 and bwd(sbytes=need - 1) == gcnsa.ERR_ARG and bwd(scratch=BASE + 2) == gcnsa.ERR_ARG


def test_checkpoint_refusals():
    L = gcnsa.lib()
    for fn in (lambda n=100, f=128, x=BASE, ldx=128, p=_p8(): L.gcnsa_op_pack8(None, n, f, x, ldx, p),
               lambda n=100, f=128, x=BASE, ldx=128, p=_p8(): L.gcnsa_op_unpack8(None, n, f, p, x, ldx)):
        assert fn(n=-1) == gcnsa.ERR_ARG and fn(f=0) == gcnsa.ERR_ARG and fn(x=None) == gcnsa.ERR_ARG and fn(p=None) == gcnsa.ERR_ARG
        assert fn(ldx=127) == gcnsa.ERR_ARG
        for bad in (_p8(q=None), _p8(e=None), _p8(ldq=120), _p8(ldq=112), _p8(q=BASE + 8), _p8(lde=3)):
            assert fn(p=bad) == gcnsa.ERR_ARG
        assert fn(n=0, x=None, p=None) == 0

    def gemm(n=1000, f=128, c=41, x=_p8(), g=BASE, ldg=44, dw=BASE + 0x100000, lddw=44, ws=BASE + 0x1000000, wb=1 << 40):
        return L.gcnsa_op_gemm_packed8(None, n, f, c, x, g, ldg, dw, lddw, 0, ws, wb)
    assert gemm(n=-1) == gcnsa.ERR_ARG and gemm(f=-1) == gcnsa.ERR_ARG and gemm(n=2**31 - 1) == gcnsa.ERR_ARG
    assert gemm(x=None) == gcnsa.ERR_ARG and gemm(g=None) == gcnsa.ERR_ARG and gemm(dw=None) == gcnsa.ERR_ARG
    assert gemm(ldg=40) == gcnsa.ERR_ARG and gemm(lddw=40) == gcnsa.ERR_ARG
    assert gemm(x=_p8(ldq=120)) == gcnsa.ERR_ARG and gemm(x=_p8(lde=3)) == gcnsa.ERR_ARG
    need = gcnsa.op_gemm_packed8_workspace(1000, 128, 41)
    assert need % 256 == 0
    if need:
        assert gemm(ws=None) == gcnsa.ERR_ARG and gemm(ws=BASE + 16) == gcnsa.ERR_ARG and gemm(wb=need - 1) == gcnsa.ERR_ARG
    assert gemm(f=0) == 0 and gemm(c=0) == 0
    assert gcnsa.op_gemm_packed8_workspace(0, 128, 41) == 0 and gcnsa.op_gemm_packed8_workspace(-5, 128, 41) == 0


def test_output_layer_refusals():
    L = gcnsa.lib()

    def ce(n=1000, d=64, c=500, h=BASE, ldh=64, w=BASE + 0x100000, ldw=500, y=BASE + 0x300000, mask=BASE + 0x310000, n_train=700,
           loss=BASE + 0x320000, dh=BASE + 0x400000, lddh=64, dw=BASE + 0x500000, lddw=500, ws=BASE + 0x10000000, wb=1 << 40):
        return L.gcnsa_op_linear_ce(None, n, d, c, h, ldh, w, ldw, None, y, mask, n_train, loss, dh, lddh, dw, lddw, None, 0, ws, wb)
    assert ce(n=-1) == gcnsa.ERR_ARG and ce(d=0) == gcnsa.ERR_ARG and ce(c=0) == gcnsa.ERR_ARG and ce(n=2**31 - 1) == gcnsa.ERR_ARG
    for k in ("h", "w", "y", "loss", "ws"):
        assert ce(**{k: None}) == gcnsa.ERR_ARG, k
    assert ce(n=2**31 - 2, c=2**31 - 1, n_train=5, ldw=2**31, lddw=2**31) == gcnsa.ERR_TOO_LARGE
    assert ce(ldh=63) == gcnsa.ERR_ARG and ce(ldw=499) == gcnsa.ERR_ARG and ce(lddh=63) == gcnsa.ERR_ARG and ce(lddw=499) == gcnsa.ERR_ARG
    assert ce(n_train=-1) == gcnsa.ERR_ARG and ce(n_train=1001) == gcnsa.ERR_ARG
    assert ce(mask=None, n_train=999) == gcnsa.ERR_ARG                 # without a mask every row counts
    assert ce(dh=BASE) == gcnsa.ERR_ARG and ce(dw=BASE + 0x100000) == gcnsa.ERR_ARG
    need = gcnsa.op_linear_ce_workspace(1000, 64, 500)
    assert need > 0 and need % 256 == 0
    assert ce(ws=BASE + 16) == gcnsa.ERR_ARG and ce(wb=need - 1) == gcnsa.ERR_ARG
    assert gcnsa.op_linear_ce_workspace(1000, 0, 5) == 0
    # the logits are never there as a whole
    assert gcnsa.op_linear_ce_workspace(100_000, 256, 100_000) < 100_000 * 100_000 * 4 // 100


def test_host_tensors_and_wrong_types_are_refused():
    """The binding looks at its tensors: a host pointer would fault on the GPU."""
    x, y = torch.zeros(4, 32), torch.zeros(4, 32)
    p = gcnsa.Packed8(4, 32, device="cpu")
    calls = [lambda: gcnsa.op_layer_norm(x, 32, y), lambda: gcnsa.op_layer_norm(None, 32, y),
             lambda: gcnsa.op_layer_norm_backward(x, y, 32, y, y, y), lambda: gcnsa.op_pack8(x, p), lambda: gcnsa.op_unpack8(p, x),
             lambda: gcnsa.op_gemm_packed8(p, x, 8, y), lambda: gcnsa.op_linear_ce(x, 32, y, 4, y, 4, y)]
    for call in calls:
        with pytest.raises(gcnsa.GcnsaError) as e:
            call()
        assert e.value.code == gcnsa.ERR_ARG
    for bad in ((-1, 32), (4, 0)):
        with pytest.raises(gcnsa.GcnsaError):
            gcnsa.Packed8(*bad, device="cpu")
    assert p.q.shape == (4, 32) and p.e.shape == (4, 1) and gcnsa.Packed8(3, 33, device="cpu").q.shape == (3, 48)


def test_dimensions_that_tiles_would_carry_past_32_bits_are_refused():
    L, big = gcnsa.lib(), 2**31 - 2**17
    for n, f in ((big, 128), (1, big)):
        p = _p8(ldq=2**31, lde=2**26)
        assert L.gcnsa_op_pack8(None, n, f, BASE, 2**31, p) == gcnsa.ERR_ARG
        assert L.gcnsa_op_unpack8(None, n, f, p, BASE, 2**31) == gcnsa.ERR_ARG
    for n, f, c in ((big, 8, 8), (8, big, 8), (8, 8, big)):
        assert L.gcnsa_op_gemm_packed8(None, n, f, c, _p8(ldq=2**31, lde=2**26), BASE, 2**31, BASE, 2**31, 0, BASE, 1 << 50) == gcnsa.ERR_ARG
    for n, d, c in ((big, 1, 1), (1, big, 1), (1, 1, big)):
        assert L.gcnsa_op_linear_ce(None, n, d, c, BASE, 2**31, BASE + 16, 2**31, None, BASE, None, n, BASE, None, 0, None, 0, None, 0, BASE,
                                    1 << 50) == gcnsa.ERR_TOO_LARGE


def test_results_are_not_windows_whose_pad_columns_belong_to_others():
    """A result's rows are written up to the next multiple of 4 columns: into the neighbours of a window, and past the last row's
    end of memory."""
    big = torch.zeros(5, 24)
    for cols, view in ((9, big[:, :9]), (9, big[:, 3:12]), (21, big[:, 3:])):
        assert gcnsa._matrix(view, "x", "float32", 5, cols, -1)[1] == 24          # as an input: fine
        with pytest.raises(gcnsa.GcnsaError) as e:
            gcnsa._matrix(view, "y", "float32", 5, cols, -1, True)
        assert e.value.code == gcnsa.ERR_ARG
    for cols, view in ((9, big[:, :12]), (12, big[:, :12]), (24, big), (8, big[:, 16:]), (9, torch.zeros(5, 9))):
        assert gcnsa._matrix(view, "y", "float32", 5, cols, -1, True)[1] == view.stride(0)
    assert gcnsa._matrix(big[:1, :9], "y", "float32", 1, 9, -1, True)[1] == 9      # a single row ends with its window
