"""CPU checks of the decoding calls: refusals that need no GPU, sizes of nothing, and the plain references against written cases."""
import ctypes as C
import struct

import numpy as np
import pytest

import decode_ref as ref

BAD, OK = 1, 0  # QNN_ERR_INVALID_ARG, QNN_OK


@pytest.fixture(scope="module")
def qlib():
    from paper_1607_04683_gb300 import build, qnn
    build.build()
    return qnn.lib()


def _linear(qlib, **kw):
    from paper_1607_04683_gb300 import qnn
    a = dict(B=2, T=3, H=4, hq=4, hk=4, hv=4, dk=8, dv=8, dtype=0, scale=1.0, q=16, q_seq=96, q_frame=32, k=16, k_seq=96, k_frame=32,
             v=16, v_seq=96, v_frame=32, y=16, y_seq=96, y_frame=32, decay=16, s_in=16, s_out=16, lengths=16) | kw
    return qlib.qnn_linear_attention(qnn._LINEAR_ARGS.pack(*a.values()), None)


@pytest.mark.parametrize("kw", [dict(B=-1), dict(T=-1), dict(T=(1 << 30) + 1), dict(H=0), dict(H=65537, hq=1, hk=1, hv=1), dict(hq=3),
                                dict(hk=0), dict(hv=8), dict(dk=0), dict(dk=257), dict(dv=0), dict(dv=257), dict(dtype=3),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(q=17), dict(decay=18), dict(s_in=18),
                                dict(s_out=2), dict(lengths=1), dict(q_seq=-1), dict(k_frame=-4), dict(v_frame=1 << 49),
                                dict(y_frame=31), dict(y_seq=64), dict(B=1 << 32), dict(B=1 << 30, T=1 << 30)])
def test_linear_refuses(qlib, kw):
    assert _linear(qlib, **kw) == BAD


def test_linear_of_nothing(qlib):
    assert _linear(qlib, B=0) == OK
    assert _linear(qlib, T=0, s_out=0) == OK
    assert qlib.qnn_linear_attention(None, None) == BAD


def _select(qlib, logits=16, ldl=9, dtype=0, scores=16, finished=None, B=2, K=3, V=9, n=3, eos=0, out=16, parents=16, tokens=16):
    return qlib.qnn_beam_select(logits, ldl, dtype, scores, finished, B, K, V, n, eos, out, parents, tokens, None)


@pytest.mark.parametrize("kw", [dict(B=-1), dict(K=0), dict(K=129), dict(V=0), dict(V=1 << 30, K=3, ldl=1 << 30), dict(n=0), dict(n=129),
                                dict(eos=-1), dict(eos=9), dict(ldl=8), dict(dtype=-1), dict(logits=18), dict(scores=17), dict(out=18),
                                dict(parents=2), dict(tokens=1), dict(ldl=1 << 49), dict(B=1 << 30)])
def test_select_refuses(qlib, kw):
    assert _select(qlib, **kw) == BAD


def test_select_of_nothing(qlib):
    assert _select(qlib, B=0) == OK


def _reorder(qlib, states=((16, 32, 1, 4),), count=None, parents=16, B=2, K=3, n=3):
    raw = b"".join(struct.pack("=2Q2q", *s) for s in states)
    return qlib.qnn_beam_reorder(raw, len(states) if count is None else count, parents, B, K, n, None)


@pytest.mark.parametrize("kw", [dict(count=-1), dict(B=-1), dict(K=0), dict(K=129), dict(n=0), dict(n=129), dict(parents=18),
                                dict(B=1 << 30), dict(states=((16, 32, -1, 4),)), dict(states=((16, 32, 1, -4),)),
                                dict(states=((16, 16, 1, 4),), n=2), dict(states=((16, 32, 1 << 40, 1 << 20),))])
def test_reorder_refuses(qlib, kw):
    assert _reorder(qlib, **kw) == BAD


def test_reorder_of_nothing(qlib):
    assert _reorder(qlib, B=0) == OK
    assert qlib.qnn_beam_reorder(None, 1, 16, 2, 3, 3, None) == BAD


def _embed(qlib, ids=16, size=4, n=3, table=16, ldt=8, dtype=0, V=5, D=8, out=16, ldo=8, out_dtype=0):
    return qlib.qnn_embedding(ids, size, n, table, ldt, dtype, V, D, 1.0, out, ldo, out_dtype, None)


def _grad(qlib, grad=16, ldg=8, dtype=0, ids=16, size=4, n=3, V=5, D=8, out=16, ldo=8, out_dtype=0):
    return qlib.qnn_embedding_grad(grad, ldg, dtype, ids, size, n, V, D, 1.0, 0, out, ldo, out_dtype, None)


@pytest.mark.parametrize("kw", [dict(size=2), dict(n=-1), dict(n=(1 << 30) + 1), dict(V=0), dict(V=1 << 31), dict(D=0), dict(dtype=3),
                                dict(out_dtype=-1), dict(ldo=7), dict(out=18), dict(ids=17), dict(ids=20, size=8)])
def test_embedding_refuses(qlib, kw):
    assert _embed(qlib, **kw) == BAD
    assert _grad(qlib, **kw) == BAD


@pytest.mark.parametrize("kw", [dict(ldt=7), dict(table=18), dict(ldt=1 << 49)])
def test_lookup_refuses(qlib, kw):
    assert _embed(qlib, **kw) == BAD


@pytest.mark.parametrize("kw", [dict(ldg=7), dict(grad=18), dict(ldg=1 << 49)])
def test_gradient_refuses(qlib, kw):
    assert _grad(qlib, **kw) == BAD


def test_lookup_of_nothing(qlib):
    assert _embed(qlib, n=0) == OK


def test_calls_without_a_device_give_errors(qlib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is there")
    assert _linear(qlib, s_in=0, s_out=0) == BAD  # (addresses that are no device's)
    assert _select(qlib) == BAD
    assert _reorder(qlib) == BAD
    assert _embed(qlib) == BAD
    assert _grad(qlib) == BAD


def test_reference_of_linear_attention():
    """Two frames by hand: d = 1/2, k v^T of 2 and 3, q of 1 and 4."""
    q, k, v = (np.array(x, np.float64).reshape(1, 2, 1, 1) for x in ([1, 4], [2, 1], [1, 3]))
    y, _, S, _ = ref.linear(q, k, v, np.array([np.log(0.5)]), 1.0, "f32", np.full((1, 1, 1, 1), 8.0))
    assert np.allclose(y.ravel(), [6.0, 24.0], rtol=1e-15) and np.allclose(S.ravel(), [6.0], rtol=1e-15)
    y, _, S, _ = ref.linear(q, k, v, np.array([5.0]), 1.0, "f32", np.full((1, 1, 1, 1), 8.0), np.array([1]))
    assert y.ravel()[0] == 10.0 and np.isnan(y.ravel()[1]) and S.ravel()[0] == 10.0  # (a decay above 1 counts as 1)


def test_reference_of_selection():
    logits = np.log(np.array([[[0.5, 0.25, 0.25], [0.1, 0.1, 0.8]]]))
    s, p, t = ref.select(logits, np.array([[-1.0, -1.5]]), 4)
    assert p.tolist() == [[0, 1, 0, 0]] and t.tolist() == [[0, 2, 1, 2]]
    assert np.allclose(s, [[-1 + np.log(0.5), -1.5 + np.log(0.8), -1 + np.log(0.25), -1 + np.log(0.25)]])
    s, p, t = ref.select(logits, np.array([[-1.0, -np.inf]]), 2, np.array([[True, False]]), eos=1)
    assert s.tolist() == [[-1.0, -np.inf]] and p.tolist() == [[0, 0]] and t.tolist() == [[1, 1]]
