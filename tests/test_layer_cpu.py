"""CPU checks of the selective state-space layer's calls: refusals that need no GPU, and the 4-bit weight layout and
quantizer of the plain reference against their written definition."""
import ctypes as C

import numpy as np
import pytest

import layer_ref as ref


@pytest.fixture(scope="module")
def qlib():
    from paper_1607_04683_gb300 import build, qnn
    build.build()
    return qnn.lib()


BAD = 1  # QNN_ERR_INVALID_ARG


def _norm(qlib, rows=4, cols=8, ldx=8, ldr=8, dtype=0, eps=1e-5, ldh=8, ldc=8, ldv=8, residual=16, h=16, values=16):
    return qlib.qnn_rmsnorm_quantize(16, ldx, residual, ldr, dtype, 16, eps, rows, cols, h, ldh, 16, ldc, 16, 16, values, ldv,
                                     None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(cols=0), dict(cols=(1 << 24) + 1, ldx=1 << 25, ldr=1 << 25, ldh=1 << 25,
                                                                   ldc=1 << 25, ldv=1 << 25),
                                dict(ldx=7), dict(ldr=7), dict(ldh=7), dict(ldc=7), dict(ldv=7), dict(dtype=3), dict(dtype=-1),
                                dict(eps=0.0), dict(eps=1e-21), dict(eps=1e21), dict(eps=float("nan")), dict(ldx=1 << 49),
                                dict(rows=1 << 30, ldx=1 << 20), dict(rows=1 << 31)])
def test_norm_refuses(qlib, kw):
    assert _norm(qlib, **kw) == BAD


def test_norm_of_no_rows(qlib):
    assert _norm(qlib, rows=0) == 0


@pytest.mark.parametrize("kw", [dict(N=0), dict(K=0), dict(ldw=7), dict(group=0), dict(group=16), dict(group=256)])
def test_quantize4_refuses(qlib, kw):
    a = dict(N=16, K=8, ldw=8, group=32) | kw
    assert qlib.qnn_quantize4(None, a["N"], a["K"], a["ldw"], a["group"], None, None, None, None) == BAD


@pytest.mark.parametrize("kw", [dict(M=-1), dict(N=0), dict(K=0), dict(lda=7), dict(ldy=3), dict(group=48), dict(ga=2),
                                dict(M=524281), dict(M=500000, lda=1 << 40)])
def test_qmatmul4_refuses(qlib, kw):
    a = dict(M=2, K=8, N=4, lda=8, ldy=4, group=32, ga=1) | kw
    assert qlib.qnn_qmatmul4(None, a["lda"], None, a["ga"], a["M"], a["K"], None, None, a["group"], None, a["N"], None, None,
                             a["ldy"], None) == BAD


def test_products_longer_than_the_codes_allow(qlib):
    assert qlib.qnn_quantize4(None, 4, 33026, 33026, 32, None, None, None, None) == 3
    assert qlib.qnn_qmatmul4(None, 33026, None, 1, 1, 33026, None, None, 32, None, 4, None, None, 4, None) == 3


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(B=-1), dict(T=-1), dict(D=0), dict(W=0), dict(W=9), dict(x_seq=-1),
                                dict(y_frame=-8), dict(y_frame=7), dict(y_seq=8), dict(y_seq=0), dict(T=1 << 31), dict(x_seq=1 << 48),
                                dict(B=1 << 21, T=1 << 20, D=1 << 19, y_frame=1 << 19, y_seq=1 << 39)])
def test_conv_refuses(qlib, kw):
    a = dict(x_seq=40, x_frame=8, dtype=0, B=2, T=5, D=8, W=4, y_seq=40, y_frame=8) | kw
    assert qlib.qnn_causal_conv(None, a["x_seq"], a["x_frame"], a["dtype"], a["B"], a["T"], a["D"], None, a["W"], None, 1, None,
                                None, None, None, a["y_seq"], a["y_frame"], None) == BAD


def _scan_args(qnn, **kw):
    a = dict(B=2, T=5, D=8, N=4, groups=2, dtype=0, softplus=1)
    for n, w in (("u", 8), ("dt", 8), ("Bm", 8), ("Cm", 8), ("z", 8), ("y", 8)):
        a |= {n + "_seq": 5 * w, n + "_frame": w}
    a |= kw
    s = qnn.SsmArgs()
    for k, v in a.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("kw", [dict(dtype=7), dict(B=-1), dict(T=-1), dict(D=0), dict(N=0), dict(N=129), dict(groups=0),
                                dict(groups=3), dict(u_seq=-1), dict(y_frame=7), dict(y_seq=39), dict(y_seq=0), dict(u=2),
                                dict(A=3), dict(z=1), dict(Bm_seq=1 << 48)])
def test_scan_refuses(qlib, kw):
    from paper_1607_04683_gb300 import qnn
    assert qlib.qnn_ssm_scan(C.byref(_scan_args(qnn, **kw)), None) == BAD


def test_scan_without_sequences(qlib):
    from paper_1607_04683_gb300 import qnn
    assert qlib.qnn_ssm_scan(None, None) == BAD
    assert qlib.qnn_ssm_scan(C.byref(_scan_args(qnn, B=0)), None) == 0
    assert qlib.qnn_ssm_scan(C.byref(_scan_args(qnn, T=0)), None) == 0  # and no state to carry over


@pytest.mark.parametrize("group", [32, 64, 128])
def test_reference_quantizer_is_within_half_a_step(group):
    g = np.random.Generator(np.random.PCG64(group))
    w = (g.normal(0, 1, (20, 200)) * np.exp(g.normal(0, 2, (20, 1)))).astype(np.float32)
    w[3] = 0
    w[4, :40] = 0.25
    w[5] = np.abs(w[5])
    codes, off, scale = ref.quantize4(w, group)
    assert codes.max() <= 15 and off.min() >= -15 and off.max() <= 0
    step = np.repeat(scale, group, 1)[:, :200]
    # half a step, and the quotient's rounding: |w / scale| is at most 15 and a half
    assert (np.abs(ref.values4(codes, off, scale, group) - w) <= step.astype(np.float64) * (0.5 + 16 * ref.U)).all()
    assert (ref.values4(codes, off, scale, group)[3] == 0).all()


def test_reference_layout_by_hand():
    codes = np.zeros((17, 129), np.uint8)
    codes[9, 32 * 2 + 8 * 3 + 5] = 7   # row 8 + 1, part 2, columns 24.. of it, the sixth of eight: half 6
    codes[16, 128] = 9                 # first of the second tiles' first word
    t = ref.tile4(codes)
    assert t.shape == (2, 2, 1024) and t.astype(int).sum() == 7 + 9
    assert t[0, 0, 512 + 64 + 16 * 3 + 4 * 2 + 3] == 7 and t[1, 1, 0] == 9


def test_reference_silu_and_softplus_at_the_ends():
    assert ref.silu(np.float64(-50.0)) < 0 and ref.silu(np.float64(50.0)) == 50.0
    y, _, h, _ = ref.scan(np.ones((1, 1, 1)), np.full((1, 1, 1), -60.0), -np.ones((1, 1)), np.ones((1, 1, 1, 1)),
                          np.ones((1, 1, 1, 1)), None, None, None, True, None, None, "f32")
    assert y[0, 0, 0] == h[0, 0, 0] == np.log1p(np.exp(-60.0))
