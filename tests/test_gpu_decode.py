"""Linear attention, beam selection and reordering, embedding and its gradient on the GPU against plain 64-bit references
(decode_ref.py, which derives the bounds), and a decoder of them as it is used."""
import ctypes as C
import os
import subprocess
import sys
import threading

import numpy as np
import pytest

import decode_ref as ref
from layer_ref import HALF, TINY, U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KINDS = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def qnn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1607_04683_gb300 import build, qnn as q
    build.build()
    q.lib()
    torch.cuda.set_device(0)
    q.device_status()
    return q


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def gpu(a, kind=None):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if kind is None else t.to(torch.float32).to(TYPES[kind])


def host(t):
    if t is None:
        return None
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def within(got, want, bound, what=""):
    d = np.abs(got - want)
    ok = np.isnan(want) | (d <= bound) | np.isinf(bound)
    assert ok.all(), (what, np.argwhere(~ok)[:5].tolist(), got[~ok][:5], want[~ok][:5], bound[~ok][:5])


# ------------------------------------------------------------------------------- linear attention

def frames_of(t, extra, front):
    """The same [B, T, heads, d] values as a slice of wider frames whose other values are NaN."""
    B, T = t.shape[:2]
    width = t.shape[2] * t.shape[3]
    full = torch.full((B, T, front + width + extra), float("nan"), dtype=t.dtype, device=t.device)
    full[..., front:front + width] = t.reshape(B, T, width)
    return full[..., front:front + width].unflatten(2, t.shape[2:])


def linear_inputs(seed, B, T, H, dk, dv, kind, hq=None, hk=None, hv=None, states=True):
    g = rng(seed)
    q, k, v = (gpu(g.normal(0, 1, (B, T, h or H, d)), kind) for h, d in ((hq, dk), (hk, dk), (hv, dv)))
    decay = gpu(np.log1p(-2.0 ** -g.uniform(1, 9, H)).astype(np.float32))
    state = gpu(g.normal(0, 2, (B, H, dk, dv)).astype(np.float32)) if states else None
    return q, k, v, decay, state


def check_linear(qnn, q, k, v, decay, state=None, lengths=None, scale=None, padded=None, inplace=False):
    kind = {t: n for n, t in TYPES.items()}[q.dtype]
    B, T, _, dk = q.shape
    H, dv = decay.shape[0], v.shape[3]
    y, bound, S, sbound = ref.linear(host(q), host(k), host(v), host(decay), dk ** -0.5 if scale is None else scale, kind,
                                     host(state), None if lengths is None else host(lengths))
    out = torch.full((B, T, H, dv), 7.0, dtype=q.dtype, device="cuda")
    if padded is not None:
        q, k, v, out = (frames_of(t, *padded) for t in (q, k, v, out))
    end = state.clone() if state is not None and inplace else torch.full((B, H, dk, dv), float("nan"), device="cuda")
    got = qnn.qnn_linear_attention(q, k, v, decay, scale=scale, state_in=end if inplace and state is not None else state,
                                   state_out=end, lengths=lengths, out=out)
    assert got is out
    within(host(out), y, bound, "y")
    within(host(end), S, sbound, "state")
    if lengths is not None:  # frames behind a sequence's end are left as they were
        n = np.clip(host(lengths), 0, T)
        for b in range(B):
            assert (out[b, n[b]:] == 7.0).all()
    assert qnn.device_status() == qnn.QNN_OK
    return out, end


SIZES = [(1, 1, 1, 1, 1), (3, 1, 2, 128, 128), (2, 2, 3, 64, 64), (5, 5, 1, 33, 7), (2, 8, 2, 256, 256), (1, 9, 1, 16, 16),
         (2, 15, 3, 39, 30), (1, 16, 2, 64, 65), (2, 17, 1, 65, 64), (1, 31, 2, 128, 128), (1, 32, 2, 100, 100), (2, 33, 2, 8, 200),
         (1, 63, 1, 129, 48), (1, 64, 2, 128, 64), (2, 65, 2, 64, 128), (1, 100, 1, 256, 256), (1, 127, 5, 100, 100),
         (1, 128, 2, 200, 31), (3, 130, 2, 1, 1), (1, 300, 4, 64, 64), (1, 1000, 1, 128, 128), (2, 517, 2, 192, 96),
         (40, 70, 8, 32, 32), (1, 2100, 2, 16, 256)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T,H,dk,dv", SIZES)
def test_linear(qnn, B, T, H, dk, dv, kind):
    q, k, v, decay, state = linear_inputs(B * 1000 + T * 7 + dk, B, T, H, dk, dv, kind)
    check_linear(qnn, q, k, v, decay, state)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 6, 20, 200])
def test_linear_without_states(qnn, T, kind):
    q, k, v, decay, _ = linear_inputs(T, 2, T, 3, 48, 80, kind, states=False)
    check_linear(qnn, q, k, v, decay)
    y = qnn.qnn_linear_attention(q, k, v, decay)
    out, _ = check_linear(qnn, q, k, v, decay, scale=48 ** -0.5)
    assert torch.equal(y, out)
    check_linear(qnn, q, k, v, decay, scale=-3.0)
    check_linear(qnn, q, k, v, decay, scale=0.0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 4, 70, 400])
@pytest.mark.parametrize("heads", [(1, 1, 6), (6, 1, 1), (6, 2, 2), (2, 3, 6), (1, 1, 1)])
def test_linear_shared_heads(qnn, T, heads, kind):
    q, k, v, decay, state = linear_inputs(T, 2, T, 6, 40, 24, kind, *heads)
    check_linear(qnn, q, k, v, decay, state)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 7, 90, 300])
@pytest.mark.parametrize("dk,dv", [(64, 64), (33, 31), (100, 100)])
@pytest.mark.parametrize("padded", [(8, 8), (3, 0), (0, 1), (5, 2), (4, 4)])
def test_linear_strides(qnn, T, dk, dv, padded, kind):
    q, k, v, decay, state = linear_inputs(T + dk, 2, T, 2, dk, dv, kind)
    check_linear(qnn, q, k, v, decay, state, padded=padded)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [3, 8, 64, 65, 500])
def test_linear_lengths(qnn, T, kind):
    lengths = [0, 1, T, T + 5, -3, T - 1, T // 2, 2]
    q, k, v, decay, state = linear_inputs(T, len(lengths), T, 2, 32, 48, kind)
    for b, n in enumerate(lengths):  # (what lies behind a sequence's end is not read)
        for x in (q, k, v):
            x[b, max(n, 0):] = float("nan")
    n = gpu(np.array(lengths, np.int32))
    clean = [torch.where(torch.isnan(x), torch.zeros_like(x), x) for x in (q, k, v)]
    a = check_linear(qnn, *clean, decay, state, lengths=n)
    out = torch.full_like(a[0], 7.0)
    end = torch.empty_like(a[1])
    qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end, lengths=n, out=out)
    assert torch.equal(out, a[0]) and torch.equal(end, a[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T", [(1, 1), (2, 8), (1, 65), (1, 1000), (3, 2000)])
def test_linear_states_in_place(qnn, B, T, kind):
    q, k, v, decay, state = linear_inputs(T, B, T, 2, 64, 96, kind)
    a = check_linear(qnn, q, k, v, decay, state)
    b = check_linear(qnn, q, k, v, decay, state, inplace=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_linear_no_frames(qnn):
    q, k, v, decay, state = linear_inputs(3, 2, 0, 2, 16, 24, "bf16")
    end = torch.zeros_like(state)
    y = qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end)
    assert y.shape == (2, 0, 2, 24) and torch.equal(end, state)
    qnn.qnn_linear_attention(q, k, v, decay, state_out=end)
    assert (end == 0).all()
    q, k, v, decay, state = linear_inputs(3, 0, 5, 2, 16, 24, "bf16")
    assert qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=state).shape == (0, 5, 2, 24)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 6, 40, 700])
def test_linear_decays_at_their_ends(qnn, T, kind):
    q, k, v, _, state = linear_inputs(T, 2, T, 7, 32, 64, kind)
    decay = gpu(np.array([0.0, -0.0, 3.0, -np.inf, -300.0, -1e-30, -20.0], np.float32))
    check_linear(qnn, q, k, v, decay, state)
    decay[3] = float("nan")
    end = torch.empty_like(state)
    y = qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end)
    assert torch.isnan(end[:, 3]).all() and torch.isfinite(end[:, [0, 1, 2, 4, 5, 6]]).all()
    assert torch.isfinite(y[:, :, [0, 1, 2, 4, 5, 6]]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,at", [(1, 0), (7, 3), (64, 40), (130, 70), (600, 333)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_linear_values_that_are_not_finite(qnn, T, at, bad, kind):
    q, k, v, decay, state = linear_inputs(T, 2, T, 3, 40, 48, kind)
    run = lambda *a: qnn.qnn_linear_attention(*a, decay, state_in=state, state_out=torch.empty_like(state))  # noqa: E731
    clean = run(q, k, v)
    y, bound, _, _ = ref.linear(host(q), host(k), host(v), host(decay), 40 ** -0.5, kind, host(state))
    # v: its own column of its own head, from its frame on
    x = v.clone()
    x[1, at, 2, 17] = bad
    got = run(q, k, x)
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[1, at:, 2, 17] = True
    assert not torch.isfinite(got[touched]).any()
    within(host(got)[~host(touched).astype(bool)], y[~host(touched).astype(bool)], bound[~host(touched).astype(bool)], "v")
    # k: its own head, from its frame on
    x = k.clone()
    x[0, at, 1, 5] = bad
    got = run(q, x, v)
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[0, at:, 1] = True
    assert not torch.isfinite(got[touched]).any()
    assert torch.equal(got[~touched], clean[~touched])
    # q: its own frame
    x = q.clone()
    x[0, at, 0, 39] = bad
    got = run(x, k, v)
    touched = torch.zeros_like(got, dtype=torch.bool)
    touched[0, at, 0] = True
    assert not torch.isfinite(got[touched]).any()
    assert torch.equal(got[~touched], clean[~touched])


@pytest.mark.parametrize("kind", KINDS)
def test_linear_prompt_and_frames(qnn, kind):
    """A sequence in pieces of any length gives what the whole of it does."""
    q, k, v, decay, state = linear_inputs(11, 2, 300, 4, 64, 64, kind)
    y, bound, S, sbound = ref.linear(host(q), host(k), host(v), host(decay), 0.125, kind, host(state))
    at, got = 0, []
    s = state.clone()
    for n in (150, 1, 1, 1, 70, 8, 9, 2, 58):
        part = [x[:, at:at + n] for x in (q, k, v)]
        got.append(qnn.qnn_linear_attention(*part, decay, state_in=s, state_out=s))
        at += n
    assert at == 300
    within(host(torch.cat(got, 1)), y, bound, "y")
    within(host(s), S, sbound, "state")


def test_linear_far_strides(qnn):
    """Sequences whose elements lie more than 2^31 apart."""
    far = (1 << 31) + 64
    base = torch.zeros(2 * far, dtype=torch.bfloat16, device="cuda")
    q, k, v, decay, state = linear_inputs(5, 2, 80, 2, 32, 32, "bf16")
    put = []
    for i, x in enumerate((q, k, v)):
        s = base.as_strided((2, 80, 2, 32), (far, 64, 32, 1), i * 8192)
        s.copy_(x)
        put.append(s)
    with pytest.raises(qnn.QnnError):  # (an output between the inputs' frames counts as overlapping them)
        qnn.qnn_linear_attention(*put, decay, state_in=state, out=base.as_strided((2, 80, 2, 32), (far, 64, 32, 1), 3 * 8192))
    out = torch.zeros_like(base).as_strided((2, 80, 2, 32), (far, 64, 32, 1), 3 * 8192)
    qnn.qnn_linear_attention(*put, decay, state_in=state, out=out)
    y, bound, _, _ = ref.linear(host(q), host(k), host(v), host(decay), 32 ** -0.5, "bf16", host(state))
    within(host(out), y, bound)


@pytest.fixture(params=["tc", "chunks"])
def kernel(request, monkeypatch):
    """One of the kernels of long bf16 sequences, whichever would be taken."""
    monkeypatch.setenv("QNN_LINEAR", request.param)
    return request.param


@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 9, 1, 8, 8), (1, 64, 2, 64, 64), (2, 127, 1, 16, 24), (1, 128, 3, 128, 128), (2, 129, 2, 72, 64),
                                         (1, 255, 1, 128, 200), (1, 256, 2, 64, 72), (1, 257, 1, 48, 256), (1, 384, 1, 128, 64),
                                         (3, 385, 2, 120, 136), (1, 1000, 2, 128, 128), (40, 140, 8, 64, 64), (5, 300, 33, 32, 128)])
def test_linear_kernels_of_long_sequences(qnn, kernel, B, T, H, dk, dv):
    q, k, v, decay, state = linear_inputs(B * 1000 + T * 7 + dk, B, T, H, dk, dv, "bf16")
    a = check_linear(qnn, q, k, v, decay, state)
    b = check_linear(qnn, q, k, v, decay, state, inplace=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_linear(qnn, q, k, v, decay)
    check_linear(qnn, q, k, v, decay, state, padded=(8, 8))


@pytest.mark.parametrize("heads", [(1, 1, 6), (6, 1, 1), (2, 3, 6), (1, 1, 1)])
def test_linear_kernels_with_shared_heads(qnn, kernel, heads):
    q, k, v, decay, state = linear_inputs(5, 2, 200, 6, 64, 128, "bf16", *heads)
    check_linear(qnn, q, k, v, decay, state)


@pytest.mark.parametrize("B,T", [(9, 128), (12, 300), (300, 150), (257, 20)])
def test_linear_kernels_with_lengths(qnn, kernel, B, T):
    """Sequences of all lengths, more of them than are sorted and than there are SMs, with anything behind their ends."""
    g = rng(B)
    lengths = g.integers(-3, T + 5, B)
    lengths[:4] = [0, T, 1, T - 1]
    q, k, v, decay, state = linear_inputs(B, B, T, 2, 32, 64, "bf16")
    n = gpu(lengths.astype(np.int32))
    a = check_linear(qnn, q, k, v, decay, state, lengths=n)
    for i, x in enumerate((q, k, v)):
        for b, m in enumerate(np.clip(lengths, 0, T)):
            x[b, m:] = (float("nan"), float("inf"), -float("inf"))[i]
    out, end = torch.full_like(a[0], 7.0), torch.empty_like(a[1])
    qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end, lengths=n, out=out)
    assert torch.equal(out, a[0]) and torch.equal(end, a[1])


@pytest.mark.parametrize("T,at", [(128, 40), (130, 129), (400, 200)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_linear_kernels_with_values_that_are_not_finite(qnn, kernel, T, at, bad):
    test_linear_values_that_are_not_finite(qnn, T, at, bad, "bf16")


def test_linear_kernels_with_decays_at_their_ends(qnn, kernel):
    for T in (100, 300):
        test_linear_decays_at_their_ends(qnn, T, "bf16")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [6, 200])
def test_linear_inputs_in_other_orders(qnn, T, kind):
    """Inputs of one sequence or of one frame for all, frames before sequences, and frames that overlap as windows of values."""
    B, H, d = 3, 2, 64
    q, k, v, decay, state = linear_inputs(T, B, T, H, d, d, kind)

    def check(q, k, v, out=None):
        y, bound, S, sbound = ref.linear(host(q), host(k), host(v), host(decay), 0.125, kind, host(state))
        end = torch.empty_like(state)
        got = qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end, out=out)
        within(host(got), y, bound, "y")
        within(host(end), S, sbound, "state")

    every = (B, T, H, d)
    check(q[:1].expand(every), k, v)
    check(q, k[:, :1].expand(every), v)
    check(q, k, v[:1, :1].expand(every))
    check(q[:1].expand(every), k[:1, 3:4].expand(every), v[1:2].expand(every))
    late = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, v)]
    check(*late[:3], out=late[3].clone().transpose(0, 1).contiguous().transpose(0, 1))
    line = gpu(rng(9).normal(0, 1, (B, T * 8 + H * d)), kind)
    check(line.as_strided(every, (line.shape[1], 8, d, 1)), k, v)


@pytest.mark.parametrize("B", [1, 3])
def test_linear_kernels_with_inputs_in_other_orders(qnn, kernel, B):
    test_linear_inputs_in_other_orders(qnn, 260, "bf16")
    q, k, v, decay, state = linear_inputs(B, B, 260, 2, 64, 64, "bf16")
    out = torch.empty_like(v)
    want = qnn.qnn_linear_attention(q, k, v, decay, state_in=state)
    for x in (q, k, v):  # (values that no copy of 16 bytes takes: a frame of another length, a place in the middle)
        wide = torch.zeros(B, 260, 2 * 64 + 3, dtype=x.dtype, device="cuda")[..., 1:-2]
        wide.copy_(x.flatten(2))
        put = [wide.unflatten(2, (2, 64)) if x is z else z for z in (q, k, v)]
        got = qnn.qnn_linear_attention(*put, decay, state_in=state, out=out)
        y, bound, _, _ = ref.linear(host(q), host(k), host(v), host(decay), 0.125, "bf16", host(state))
        within(host(got), y, bound)
        within(host(want), y, bound)


def test_linear_kernels_give_the_same_bits_again(qnn, kernel):
    q, k, v, decay, state = linear_inputs(8, 3, 700, 60, 128, 128, "bf16")
    lengths = gpu(np.array([700, 300, 5], np.int32))
    outs = []
    for _ in range(4):
        end = torch.empty_like(state)
        y = torch.zeros_like(v)
        qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end, lengths=lengths, out=y)
        outs.append((y, end))
    assert all(torch.equal(y, outs[0][0]) and torch.equal(e, outs[0][1]) for y, e in outs)


# ------------------------------------------------------------------------------------- selection

def check_select(qnn, logits, scores, n, finished=None, eos=0, alike=0.0):
    """alike: beams' candidates whose scores differ by less may come in either order."""
    x, s = host(logits), host(scores)
    want = ref.select(x, s, n, None if finished is None else host(finished), eos)
    best, parents, tokens = qnn.qnn_beam_select(logits, scores, n, finished=finished, eos=eos)
    got, p, t = host(best), host(parents), host(tokens)
    if alike:
        lse = x.max(2) + np.log(np.exp(x - x.max(2, keepdims=True)).sum(2))
        rows = np.arange(len(x))[:, None]
        assert (np.abs(s[rows, p] + x[rows, p, t] - lse[rows, p] - want[0]) <= alike).all()
        assert all(len(set(zip(a, b))) == n for a, b in zip(p.tolist(), t.tolist()))
    else:
        assert np.array_equal(p, want[1]) and np.array_equal(t, want[2])
    gone = np.isinf(want[0])
    assert np.array_equal(got[gone], want[0][gone])
    # the sums' logarithm is right to 2^-24 or so, the score is rounded once
    assert (np.abs(got[~gone] - want[0][~gone]) <= alike + 2.0 ** -23 + U * np.abs(want[0][~gone])).all()
    assert qnn.device_status() == qnn.QNN_OK
    return best, parents, tokens


def select_inputs(seed, B, K, V, kind, std=3.0):
    g = rng(seed)
    return gpu(g.normal(0, std, (B, K, V)), kind), gpu(g.normal(-10, 2, (B, K)).astype(np.float32))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,K,V,n", [(1, 1, 1, 1), (1, 4, 2000, 4), (3, 2, 29, 5), (2, 5, 333, 10), (4, 8, 2047, 16), (2, 8, 2048, 8),
                                     (2, 3, 2049, 6), (1, 4, 8192, 8), (7, 16, 1001, 32), (1, 2, 65537, 64), (2, 128, 40, 128),
                                     (1, 1, 5000, 128), (300, 4, 64, 4), (1, 3, 5, 128), (64, 8, 4100, 16), (1, 32, 30000, 32), (5, 8, 3000, 32),
                                     (5, 8, 3000, 33), (200, 1, 20000, 3), (80, 2, 9000, 64), (30, 5, 9001, 10), (9, 1, 1, 256 // 2)])
def test_select(qnn, B, K, V, n, kind):
    logits, scores = select_inputs(B * 7 + V, B, K, V, kind)
    check_select(qnn, logits, scores, n)
    finished = gpu(rng(V).uniform(0, 1, (B, K)) < 0.4)
    check_select(qnn, logits, scores, n, finished, eos=V // 2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [31, 2000, 4097, 20000])
def test_select_equal_scores(qnn, V, kind):
    g = rng(V)
    same = gpu(np.zeros((2, 4, V)), kind)
    scores = gpu(np.array([[-1, -1, -2, -1], [-3, -3, -3, -3]], np.float32))
    check_select(qnn, same, scores, 12)
    few = gpu(g.integers(0, 3, (2, 4, V)).astype(np.float64), kind)  # three values
    check_select(qnn, few, gpu(np.full((2, 4), -5.0, np.float32) * np.array([[1, 2, 3, 4]], np.float32)), 40)
    alike = gpu(np.repeat(g.normal(0, 2, (2, 1, V)), 4, 1), kind)  # beams of one past: the lowest first
    check_select(qnn, alike, gpu(np.full((2, 4), -7.0, np.float32)), 9)
    signs = gpu(np.where(g.uniform(0, 1, (1, 2, V)) < 0.5, -0.0, 0.0), kind)  # zeros of either sign are equal
    check_select(qnn, signs, gpu(np.array([[-1.0, -1.5]], np.float32)), 30)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [40, 2500, 9001])
def test_select_rows_in_order(qnn, V, kind):
    up = np.linspace(-8, 8, V)
    logits = gpu(np.stack([up, up[::-1], np.roll(up, V // 2), -np.abs(up)])[None], kind)
    scores = gpu(np.array([[-2.0, -3.25, -2.5, -40.0]], np.float32))
    # Beams of the same values in another order, whose sums of exponentials are rounded differently: on a grid of 16-bit values some
    # candidates of theirs have equal scores in exact arithmetic, but not when formed. A term is off by 2^-22 (the instruction), and by its
    # argument's three roundings: |d| <= 16, |d| log2(e) <= 24 twice, times ln 2, 2^-24 each: (16 + 34) 2^-24; a sum by 2^-24 for each of
    # up to 64 additions. A beam's logarithm is off by the largest of those at most, two beams' difference by twice that.
    alike = 2 * (4 + 16 + 34 + 64) * U
    for n in (1, 7, 128):
        check_select(qnn, logits, scores, n, alike=alike)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [17, 2048, 6001])
def test_select_masks(qnn, V, kind):
    logits, scores = select_inputs(V, 6, 4, V, kind)
    inf, nan = float("inf"), float("nan")
    logits[0, 0] = -inf  # nothing left of a beam
    logits[0, 1, :-2] = -inf
    logits[1] = -inf  # nothing left of an utterance
    logits[2, 0, 3] = nan
    logits[2, 1, V - 1] = inf
    logits[2, 2, ::2] = -inf
    scores[3, 1:] = -inf  # the first step: one beam
    scores[4, 0], scores[4, 2] = nan, -inf
    logits[5] = torch.finfo(logits.dtype).min  # a mask of the type's lowest value: all alike
    logits[5, 0, 5] = 1.0
    check_select(qnn, logits, scores, 8)
    finished = torch.zeros((6, 4), dtype=torch.bool, device="cuda")
    finished[0, 0] = finished[1, 3] = finished[2, 0] = finished[3, 2] = finished[4] = True
    check_select(qnn, logits, scores, 8, finished, eos=2)
    check_select(qnn, logits, scores, 100, finished.to(torch.uint8), eos=V - 1)


def rows_of_sums(V):
    """Rows that show how their sums of exponentials are added up: of two values, slopes either way and beyond all that counts, normal
    ones, one class above all others, whose parts are of very different size."""
    g = rng(V)
    rows = [g.normal(0, 3, V), np.linspace(-8, 8, V), np.linspace(8, -8, V), np.linspace(-100, 60, V), np.zeros(V)]
    for share in (64, 8):
        for low in (-1.0, -3.0, -7.5, -11.3):
            x = np.full(V, low)
            x[g.permutation(V)[:V // share]] = 0.0
            rows.append(x)
    x = np.full(V, -15.7)
    x[V // 3] = 0.0
    rows.append(x)
    rows.append(np.where(np.arange(V) % 97 == 96, 20.0 + np.arange(V) / V, -3.1))  # (every other tile has a new largest value)
    return np.stack(rows)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [97, 2000, 8192, 65536, 262144])
@pytest.mark.parametrize("times", [1, 21])
def test_select_sums_of_exponentials(qnn, V, kind, times):
    """Scores of a row's best class where beam score and logits leave nearly nothing, so that the score's own rounding does not count, and of
    four beams of one utterance. In 2^-24, a row's log sum exp is off by 10 + 2 D at most, D the mean of |d|, a class's distance from the largest
    logit, by the classes' probabilities: d is rounded to fp32 (|d|), d log2(e) is (|d| again), the exponential's instruction is 2^-22 off
    (4), what it is off on average is taken out (5e-8: less than 1), 32 terms of a thread are added in pairs (5); the sums across threads and the
    logarithm are of 35 bits and more, and have what is left of 10. Times: once in parts of a row, and often enough that a row is one."""
    few = gpu(rows_of_sums(V), kind)
    x = host(few)
    R = len(x)
    most = x.max(1)
    p = np.exp(x - most[:, None])
    lse = most + np.log(p.sum(1))
    D = (p * (most[:, None] - x)).sum(1) / p.sum(1)
    start = gpu((lse - most).astype(np.float32))
    want = host(start) + most - lse
    bound = (10 + 2 * D) * U + U * np.abs(want) + 1e-15
    logits = few.repeat(times, 1).unsqueeze(1)  # utterances of one beam
    best, _, tokens = qnn.qnn_beam_select(logits, start.repeat(times)[:, None], 1)
    first = np.argmax(x, 1)
    assert (host(tokens).reshape(times, R) == first).all()
    off = np.abs(host(best).reshape(times, R) - want)
    assert (off <= bound).all(), (off / U, bound / U)
    wide = few[:12].view(3, 4, V)  # four beams, of which each is looked at in parts; one candidate each, as the others are lost
    for k in range(4):
        scores = torch.full((3, 4), -np.inf, device="cuda")
        scores[:, k] = start[:12].view(3, 4)[:, k]
        best, parents, tokens = qnn.qnn_beam_select(wide, scores, 2)
        assert (parents[:, 0] == k).all()
        off = np.abs(host(best)[:, 0] - want[:12].reshape(3, 4)[:, k])
        assert (off <= bound[:12].reshape(3, 4)[:, k]).all(), (off / U, bound / U)
    assert qnn.device_status() == qnn.QNN_OK


@pytest.mark.parametrize("V", [300, 20000, 100000])
@pytest.mark.parametrize("rows", [1, 400])
def test_select_not_a_number_behind_larger_values(qnn, V, rows):
    """A NaN, or an infinity, in an earlier tile than the largest value, and one behind a far larger value: the beam has no candidates."""
    base = np.linspace(-200, 200, V)
    for at in (0, V // 2, V - 1):
        for bad in (float("nan"), float("inf")):
            x = base.copy()
            x[at] = bad
            logits = gpu(np.stack([x, base])[:, None].repeat(rows, 0), "f32")
            best, parents, tokens = qnn.qnn_beam_select(logits, torch.zeros((2 * rows, 1), device="cuda"), 1, eos=7)
            assert (best[:rows] == -np.inf).all() and (tokens[:rows] == 7).all()
            assert torch.isfinite(best[rows:]).all() and (tokens[rows:] == V - 1).all()


@pytest.mark.parametrize("kind", KINDS)
def test_select_strides_and_places(qnn, kind):
    full, scores = select_inputs(5, 3, 4, 1003, kind)
    for front, V in ((0, 1000), (1, 1000), (3, 999), (8, 512)):
        logits = full[:, :, front:front + V]
        a = check_select(qnn, logits, scores, 6)
        b = qnn.qnn_beam_select(logits.contiguous(), scores, 6)
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    # scores in place (n = K), by the C call
    logits = full[:, :, :1000]
    a = qnn.qnn_beam_select(logits, scores)
    kept, parents, tokens = scores.clone(), torch.empty_like(a[1]), torch.empty_like(a[2])
    st = qnn.lib().qnn_beam_select(logits.data_ptr(), 1003, {"f32": 0, "bf16": 1, "f16": 2}[kind], kept.data_ptr(), None, 3, 4, 1000,
                                   4, 0, kept.data_ptr(), parents.data_ptr(), tokens.data_ptr(), None)
    torch.cuda.synchronize()
    assert st == qnn.QNN_OK
    assert torch.equal(kept, a[0]) and torch.equal(parents, a[1]) and torch.equal(tokens, a[2])


# ------------------------------------------------------------------------------------ reordering

def reordered(x, parents, dim, B):
    K = x.shape[dim] // B
    rows = (torch.arange(B, device=x.device)[:, None] * K + parents.long()).reshape(-1)
    return x.index_select(dim, rows)


@pytest.mark.parametrize("B,K,n", [(1, 1, 1), (1, 4, 4), (3, 2, 2), (2, 8, 8), (2, 8, 3), (2, 5, 16), (1, 16, 16), (2, 17, 17), (1, 128, 128),
                                   (3, 20, 7), (50, 8, 8)])
def test_reorder(qnn, B, K, n):
    g = rng(B * 31 + K)
    R = B * K
    states = [gpu(g.normal(0, 1, (5, R, 500)).astype(np.float32)), gpu(g.normal(0, 1, (R, 3, 125)), "bf16"),
              gpu(g.integers(0, 255, (R, 7)).astype(np.uint8)), gpu(g.integers(0, 9000, (R, 33)).astype(np.int64)),
              gpu(g.normal(0, 1, (R, 4, 16, 24)).astype(np.float32)), gpu(g.normal(0, 1, (2, 3, R, 1)), "f16"),
              gpu(g.integers(0, 2, (R,)) > 0), torch.empty((0, R, 4), device="cuda")]
    dims = [1, 0, 0, 0, 0, 2, 0, 1]
    parents = gpu(g.integers(0, K, (B, n)).astype(np.int32))
    want = [reordered(s, parents, d, B) for s, d in zip(states, dims)]
    got = qnn.qnn_beam_reorder(states, parents, dims=dims)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if n == K:
        copies = [s.clone() for s in states]
        got = qnn.qnn_beam_reorder(copies, parents, dims=dims, out=copies)
        assert all(a is b for a, b in zip(got, copies))
        assert all(torch.equal(a, b) for a, b in zip(copies, want))
        same = gpu(np.tile(np.arange(K, dtype=np.int32), (B, 1)))
        qnn.qnn_beam_reorder(copies, same, dims=dims, out=copies)
        assert all(torch.equal(a, b) for a, b in zip(copies, want))
    assert qnn.device_status() == qnn.QNN_OK


def test_reorder_many_states_and_bad_parents(qnn):
    states = [torch.full((8, 10 + i), float(i), device="cuda") + torch.arange(8, device="cuda")[:, None] for i in range(40)]
    parents = gpu(np.array([[1, 0, 3, 3], [0, 0, 2, 1]], np.int32))
    got = qnn.qnn_beam_reorder(states, parents)
    assert all(torch.equal(a, reordered(s, parents, 0, 2)) for a, s in zip(got, states))
    assert qnn.qnn_beam_reorder([], parents) == []
    assert qnn.device_status() == qnn.QNN_OK
    parents[0, 1], parents[1, 3] = 4, -1  # rows of such parents are left as they are
    out = [torch.full_like(s, -5.0) for s in states[:2]]
    qnn.qnn_beam_reorder(states[:2], parents, out=out)
    assert qnn.device_status() == qnn.QNN_ERR_INVALID_ARG
    fixed = parents.clamp(0, 3)
    for s, o in zip(states, out):
        want = reordered(s, fixed, 0, 2)
        want[1] = want[7] = -5.0
        assert torch.equal(o, want)


# ------------------------------------------------------------------------------------- embedding

def id_list(g, n, V, how="zipf"):
    if how == "one":
        return np.full(n, V // 2)
    ids = np.minimum(np.exp(g.uniform(0, np.log(V + 1), n)).astype(np.int64) - 1, V - 1)
    return np.where(g.uniform(0, 1, n) < 0.1, -1 - g.integers(0, 3, n), ids) if how == "padded" else ids


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (4, 2000, 500), (33, 7, 31), (1000, 300, 64), (5, 9, 4097), (3000, 50, 2048), (200, 20, 12)])
def test_embedding(qnn, n, V, D, kind):
    g = rng(n + D)
    table = gpu(g.normal(0, 1, (V, D)), kind)
    ids = gpu(id_list(g, n, V, "padded").astype(np.int32))
    rows = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0).long()].float() * np.float32(1.7), torch.zeros((), device="cuda"))
    assert torch.equal(qnn.qnn_embedding(ids, table, scale=1.7), rows.to(table.dtype))
    for ty in TYPES.values():
        assert torch.equal(qnn.qnn_embedding(ids.long(), table, scale=1.7, dtype=ty), rows.to(ty))
    wide = torch.full((n, D + 5), 3.0, device="cuda")
    qnn.qnn_embedding(ids, table, scale=1.7, out=wide[:, 2:2 + D])
    assert torch.equal(wide[:, 2:2 + D], rows) and (wide[:, :2] == 3).all() and (wide[:, 2 + D:] == 3).all()
    big = torch.full((V, D + 3), float("nan"), dtype=table.dtype, device="cuda")
    big[:, 1:1 + D] = table
    assert torch.equal(qnn.qnn_embedding(ids, big[:, 1:1 + D], scale=1.7), rows.to(table.dtype))
    assert qnn.device_status() == qnn.QNN_OK


def test_embedding_shapes_and_bad_labels(qnn):
    table = gpu(rng(0).normal(0, 1, (10, 8)).astype(np.float32))
    ids = gpu(np.arange(12, dtype=np.int32).reshape(3, 4) % 10)
    assert torch.equal(qnn.qnn_embedding(ids, table), table[ids.long()])
    assert qnn.qnn_embedding(ids[:0], table).shape == (0, 4, 8)
    assert qnn.qnn_embedding(torch.tensor(3, device="cuda"), table).shape == (8,)
    assert qnn.device_status() == qnn.QNN_OK
    ids[1, 2] = 10
    got = qnn.qnn_embedding(ids, table)
    assert qnn.device_status() == qnn.QNN_ERR_INVALID_ARG
    assert (got[1, 2] == 0).all() and torch.equal(got[0], table[ids[0].long()])
    far = torch.tensor([1 << 40, -(1 << 40)], device="cuda")
    assert (qnn.qnn_embedding(far, table) == 0).all() and qnn.device_status() == qnn.QNN_ERR_INVALID_ARG


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,V,D,how", [(1, 1, 1, "zipf"), (1, 29, 500, "zipf"), (31, 5, 8, "padded"), (32, 2, 40, "one"), (33, 3, 40, "one"),
                                       (64, 511, 12, "zipf"), (65, 512, 7, "padded"), (1000, 2000, 36, "zipf"), (1024, 8, 500, "padded"),
                                       (1025, 9, 64, "padded"), (5000, 70000, 16, "zipf"), (9000, 300000, 4, "padded"), (3000, 1, 260, "one"),
                                       (20000, 29, 100, "zipf"), (40000, 8192, 8, "zipf"), (140000, 50, 5, "padded"), (131072, 3, 8, "one"),
                                       (12000, 900, 1024, "zipf"), (10000, 3, 1032, "padded")])
def test_embedding_grad(qnn, n, V, D, how, kind):
    g = rng(n + V + D)
    ids_h = id_list(g, n, V, how)
    ids, grad = gpu(ids_h.astype(np.int32)), gpu(g.normal(0, 1, (n, D)), kind)
    want, bound = ref.embedding_grad(host(grad), ids_h, V, 1.7)
    out = torch.full((V, D), float("nan"), device="cuda")
    got = qnn.qnn_embedding_grad(grad, ids, V, scale=1.7, out=out)
    assert got is out
    within(host(got), want, bound + 1e-37)
    again = qnn.qnn_embedding_grad(grad, ids.long(), V, scale=1.7)
    assert torch.equal(got, again)
    # of the table's type, rounded once; added to what is there
    ty = TYPES[kind]
    assert torch.equal(qnn.qnn_embedding_grad(grad, ids, V, scale=1.7, dtype=ty), got.to(ty))
    old = gpu(g.normal(0, 1, (V, D)), kind)
    total = old.clone()
    qnn.qnn_embedding_grad(grad, ids, V, scale=1.7, out=total, accumulate=True)
    assert torch.equal(total, (old.float() + got).to(ty))
    assert qnn.device_status() == qnn.QNN_OK


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [5, 64, 500])
def test_embedding_grad_strides(qnn, D, kind):
    g = rng(D)
    ids_h = id_list(g, 300, 40, "padded")
    ids, grad = gpu(ids_h.astype(np.int32)), gpu(g.normal(0, 1, (300, D)), kind)
    want = qnn.qnn_embedding_grad(grad, ids, 40)
    for front, extra in ((0, 8), (1, 0), (2, 3), (8, 8)):
        wide = torch.full((300, front + D + extra), float("nan"), dtype=grad.dtype, device="cuda")
        wide[:, front:front + D] = grad
        out = torch.full((40, front + D + extra), 3.0, device="cuda")
        qnn.qnn_embedding_grad(wide[:, front:front + D], ids, 40, out=out[:, front:front + D])
        assert torch.equal(out[:, front:front + D], want)
        assert (out[:, :front] == 3).all() and (out[:, front + D:] == 3).all()


def test_embedding_grad_of_nothing(qnn):
    grad, ids = torch.zeros((0, 6), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    out = torch.full((5, 6), 2.0, device="cuda")
    qnn.qnn_embedding_grad(grad, ids, 5, out=out, accumulate=True)
    assert (out == 2).all()
    assert (qnn.qnn_embedding_grad(grad, ids, 5, out=out) == 0).all()
    none = torch.full((70,), -1, dtype=torch.int32, device="cuda")  # padding alone
    assert (qnn.qnn_embedding_grad(torch.ones((70, 6), device="cuda"), none, 5) == 0).all()
    # rows that are not finite reach their own label's row only
    g = torch.ones((100, 8), device="cuda")
    g[40] = float("nan")
    got = qnn.qnn_embedding_grad(g, torch.arange(100, dtype=torch.int32, device="cuda") % 10, 10)
    assert torch.isnan(got[0]).all() and (got[1:] == 10).all()


def test_embedding_module(qnn):
    """qat.Embedding: the formula's gradient, and differences of a loss."""
    from paper_1607_04683_gb300 import qat
    torch.manual_seed(3)
    emb = qat.Embedding(11, 6, scale=0.5)
    ids = torch.tensor([[3, 0, 3], [10, -1, 3]], device="cuda")
    w = torch.randn(2, 3, 6, device="cuda")
    loss = lambda: (emb(ids) * w).sum()  # noqa: E731
    loss().backward()
    want = torch.zeros(11, 6, device="cuda")
    for i in range(2):
        for j in range(3):
            if ids[i, j] >= 0:
                want[ids[i, j]] += 0.5 * w[i, j]
    assert torch.allclose(emb.weight.grad, want, rtol=1e-6, atol=1e-6)
    with torch.no_grad():  # the loss is linear in the table: a difference of 1 is the gradient, to the roundings of sums below 2^4
        for r, c in ((3, 2), (10, 5), (7, 0)):
            before = float(loss())
            emb.weight[r, c] += 1.0
            assert abs(float(loss()) - before - float(emb.weight.grad[r, c])) < 100 * 16 * U
            emb.weight[r, c] -= 1.0
    # strided and 16-bit gradients, and a network with a quantized layer behind
    net = qat.QuantLinear(6, 4)
    out = net(emb(ids).reshape(-1, 6))
    g = torch.randn_like(out)
    emb.weight.grad = None
    out.backward(g)
    back = (g @ net.weight.detach()).reshape(2, 3, 6) * 0.5
    want = torch.zeros(11, 6, device="cuda")
    for i in range(2):
        for j in range(3):
            if ids[i, j] >= 0:
                want[ids[i, j]] += back[i, j]
    assert torch.allclose(emb.weight.grad, want, rtol=1e-5, atol=1e-6)
    half = qat.Embedding(11, 6, dtype=torch.bfloat16)
    y = half(ids, dtype=torch.float32)
    assert y.dtype is torch.float32
    y.transpose(0, 1).sum().backward()
    assert half.weight.grad.dtype is torch.bfloat16 and float(half.weight.grad[3, 0]) == 3.0 and float(half.weight.grad[1, 0]) == 0.0


# ------------------------------------------------------------------------------- as they are used

def test_embedding_module_has_no_second_gradient(qnn):
    from paper_1607_04683_gb300 import qat
    emb = qat.Embedding(5, 4)
    y = emb(torch.tensor([1, 2, 1], device="cuda"))
    grad, = torch.autograd.grad((y ** 3).sum(), emb.weight, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()


def decoder(qnn, seed, K):
    from paper_1607_04683_gb300 import inputs
    wl = inputs.LstmWorkload(f"decoder_{seed}", seed=seed, num_layers=2, input_dim=24, hidden=32, proj=0, num_classes=50, batch=2,
                             frames=1, w_range=0.4, forget_bias=1.0, out_w_range=0.6)
    params, _ = wl.make()
    return qnn.LstmModel(qnn.lstm_desc(2, 24, 32, 0, 50), torch.from_numpy(params).cuda())


@pytest.mark.parametrize("B", [1, 5])
def test_beam_search_over_a_recurrent_model(qnn, B):
    """Labels through the embedding, an 8-bit LSTM stack with carried states, its output layer's logits, selection and reordering,
    every stage against its reference on the stage's own inputs, and the labels of the best beams kept in order."""
    K, V, eos, steps = 4, 50, 7, 6
    model = decoder(qnn, 31, K)
    g = rng(B)
    table = gpu(g.normal(0, 1, (V, 24)).astype(np.float32))
    h, c = (torch.zeros((2, B * K, 32), device="cuda") for _ in range(2))
    scores = gpu(np.tile(np.array([0] + [-np.inf] * (K - 1), np.float32), (B, 1)))
    tokens = torch.full((B, K), eos, dtype=torch.int32, device="cuda")
    finished = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    history = torch.full((B * K, steps), -1, dtype=torch.int32, device="cuda")
    y, logits = (torch.empty((B * K, 1, V), device="cuda") for _ in range(2))
    paths = [[() for _ in range(K)] for _ in range(B)]
    for step in range(steps):
        x = qnn.qnn_embedding(tokens, table, scale=0.5)
        assert torch.equal(x, table[tokens.long()] * 0.5)
        model.forward(x.view(B * K, 1, 24), y=y, h_state=h, c_state=c, logits=logits)
        want = ref.select(host(logits).reshape(B, K, V), host(scores), K, host(finished), eos)
        scores, parents, tokens = check_select(qnn, logits.view(B, K, V), scores, K, finished, eos)
        before = [s.clone() for s in (h, c, history)]
        qnn.qnn_beam_reorder([h, c, history], parents, dims=[1, 1, 0], out=[h, c, history])
        for s, old, d in zip((h, c, history), before, (1, 1, 0)):
            assert torch.equal(s, reordered(old, parents, d, B))
        history[:, step] = tokens.view(-1)
        finished = torch.gather(finished, 1, parents.long()) | (tokens == eos)
        paths = [[paths[b][want[1][b, k]] + (int(want[2][b, k]),) for k in range(K)] for b in range(B)]
    assert host(history).reshape(B, K, steps).tolist() == [[list(p) for p in row] for row in paths]
    assert qnn.device_status() == qnn.QNN_OK
    model.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_layer_of_linear_attention(qnn, kind):
    """A prompt and then single frames of labels through embedding, norm to codes, a 4-bit product to q, k and v side by side, and
    linear attention with carried states."""
    V, D, H, d, B = 30, 64, 2, 32, 3
    g = rng(9)
    table, weight = gpu(g.normal(0, 1, (V, D)), kind), gpu((1 + g.normal(0, 0.1, D)).astype(np.float32))
    w4 = qnn.qnn_quantize4(gpu(g.normal(0, D ** -0.5, (3 * H * d, D)).astype(np.float32)), 32)
    decay = gpu(np.array([-0.05, -0.3], np.float32))
    ids = gpu(g.integers(0, V, (B, 25)).astype(np.int32))

    def project(part):
        x = qnn.qnn_embedding(part, table)
        codes, units, _, _, _ = qnn.qnn_rmsnorm_quantize(x.reshape(-1, D), weight)
        return qnn.qnn_qmatmul4(codes, units, w4).to(TYPES[kind]).view(*part.shape, 3, H, d)

    qkv = project(ids)
    y, bound, S, sbound = ref.linear(*(host(qkv[:, :, i]) for i in range(3)), host(decay), d ** -0.5, kind)
    state = torch.zeros((B, H, d, d), device="cuda")
    got = [qnn.qnn_linear_attention(*qkv[:, :20].unbind(2), decay, state_in=state, state_out=state)]
    for t in range(20, 25):
        one = project(ids[:, t:t + 1].contiguous())
        assert torch.equal(one, qkv[:, t:t + 1])
        got.append(qnn.qnn_linear_attention(*one.unbind(2), decay, state_in=state, state_out=state))
    within(host(torch.cat(got, 1)), y, bound)
    within(host(state), S, sbound)
    assert qnn.device_status() == qnn.QNN_OK


# ------------------------------------------------------------------- streams, captures, refusals

def calls(qnn, seed):
    """(one call of each operator as a function of a stream, the results' references by the default stream)."""
    q, k, v, decay, state = linear_inputs(seed, 1, 900, 2, 64, 64, "bf16")
    logits, scores = select_inputs(seed, 3, 4, 6000, "f32")
    g = rng(seed)
    ids, grad = gpu(id_list(g, 5000, 300, "padded").astype(np.int32)), gpu(g.normal(0, 1, (5000, 64)), "bf16")
    parents = gpu(g.integers(0, 4, (3, 4)).astype(np.int32))
    table = gpu(g.normal(0, 1, (300, 64)).astype(np.float32))

    def linear(stream=None):
        end = torch.empty_like(state) if stream is None else qnn._result(torch, state.shape, state.dtype, state, stream)
        return [qnn.qnn_linear_attention(q, k, v, decay, state_in=state, state_out=end, stream=stream), end]

    return [linear, lambda stream=None: list(qnn.qnn_beam_select(logits, scores, 8, stream=stream)),
            lambda stream=None: qnn.qnn_beam_reorder([grad[:12], scores.view(12)], parents, stream=stream),
            lambda stream=None: [qnn.qnn_embedding(ids, table, scale=2.0, stream=stream)],
            lambda stream=None: [qnn.qnn_embedding_grad(grad, ids, 300, stream=stream)]]


def test_calls_on_streams(qnn):
    sets = [calls(qnn, s) for s in range(3)]
    want = [[f() for f in fs] for fs in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        got = [[None] * 5 for _ in range(3)]
        for i in range(5):
            for j, (fs, st) in enumerate(zip(sets, streams)):
                got[j][i] = fs[i](st)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for x, y in zip(a, b):
                assert all(torch.equal(p, r) for p, r in zip(x, y))


def test_calls_from_threads(qnn):
    """All calls from four host threads at once, each on a stream of its own."""
    sets = [calls(qnn, s) for s in range(4)]
    want = [[f() for f in fs] for fs in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got, errors, start = [[] for _ in sets], [], threading.Barrier(len(sets))

    def work(i):
        try:
            torch.cuda.set_device(0)
            start.wait()
            for _ in range(5):
                got[i].append([f(streams[i]) for f in sets[i]])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sets))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for outs, refs in zip(got, want):
        assert len(outs) == 5
        for out in outs:
            for x, y in zip(out, refs):
                assert all(torch.equal(p, r) for p, r in zip(x, y))
    assert qnn.device_status() == qnn.QNN_OK


def test_calls_in_graphs(qnn):
    """Captured calls, two graphs of them replayed side by side on streams of their own, beside calls that are not captured."""
    sets = [calls(qnn, s) for s in (5, 6)]
    want = [[f() for f in fs] for fs in sets]
    torch.cuda.synchronize()
    graphs, got = [], []
    for fs in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append([f() for f in fs])
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for outs in got:
            for out in outs:
                for t in out:
                    t.zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        eager = [f() for f in sets[0]]
        torch.cuda.synchronize()
        for a, b in zip([*got, eager], [*want, want[0]]):
            for x, y in zip(a, b):
                assert all(torch.equal(p, r) for p, r in zip(x, y))


@pytest.mark.parametrize("kernel,call", [
    ("tc", "qnn.qnn_linear_attention(q, k, v, decay)"), ("chunks", "qnn.qnn_linear_attention(q, k, v, decay)"),
    ("", "qnn.qnn_linear_attention(q.float(), k.float(), v.float(), decay)"), ("", "qnn.qnn_linear_attention(q[:, :1], k[:, :1], v[:, :1], decay)"),
    ("", "torch.stack(qnn.qnn_beam_select(logits, scores)[1:])"), ("", "qnn.qnn_beam_reorder([table[:64]], parents)[0]"),
    ("", "qnn.qnn_embedding(ids, table)"), ("", "qnn.qnn_embedding_grad(grad, ids, 300)")])
def test_captured_before_the_first_call(qnn, kernel, call):
    """In a process of its own: nothing of the library's has been made on the device when the call is captured."""
    code = f'''
import os, torch
os.environ["QNN_LINEAR"] = "{kernel}"
from paper_1607_04683_gb300 import qnn
torch.cuda.set_device(0)
g = torch.Generator(device="cuda").manual_seed(1)
q, k, v = (torch.rand((1, 900, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
decay, scores = torch.full((2,), -0.1, device="cuda"), torch.zeros((4, 16), device="cuda")
logits, table, grad = torch.rand((4, 16, 3000), generator=g, device="cuda"), torch.rand((300, 64), device="cuda"), torch.rand((5000, 64), device="cuda")
ids, parents = torch.randint(0, 300, (5000,), device="cuda"), torch.ones((4, 16), dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = {call}
graph.replay()
torch.cuda.synchronize()
assert qnn.device_status() == qnn.QNN_OK and torch.equal(out, {call}) and out.abs().sum() > 0
'''
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0, r.stderr[-2000:]


def test_embedding_module_captured(qnn):
    """A training step of the module in a graph, replayed on other labels and errors."""
    from paper_1607_04683_gb300 import qat
    emb = qat.Embedding(40, 8, scale=0.5)
    ids, gy = torch.zeros(100, dtype=torch.int64, device="cuda"), torch.zeros(100, 8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (nothing of this pass lives when the next is captured)
        emb(ids).backward(gy)
    torch.cuda.current_stream().wait_stream(side)
    emb.weight.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = emb(ids)
        y.backward(gy)
    for seed in range(3):
        g = rng(seed)
        ids.copy_(gpu(g.integers(-2, 40, 100)))
        gy.copy_(gpu(g.normal(0, 1, (100, 8)).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, qnn.qnn_embedding(ids, emb.weight.detach(), scale=0.5))
        assert torch.equal(emb.weight.grad, qnn.qnn_embedding_grad(gy, ids, 40, scale=0.5))


def test_linear_refuses_heads_of_no_values(qnn):
    """By the library's error, also where the scale is left to the call."""
    q, k, v, decay, state = linear_inputs(1, 2, 12, 4, 16, 16, "f32")
    for scale in (None, 1.0):
        with pytest.raises(qnn.QnnError):
            qnn.qnn_linear_attention(q[..., :0], k[..., :0], v, decay, scale=scale)
        with pytest.raises(qnn.QnnError):
            qnn.qnn_linear_attention(q, k, v[..., :0], decay, scale=scale)


def test_refusals(qnn):
    q, k, v, decay, state = linear_inputs(1, 2, 12, 4, 16, 16, "f32")
    run = qnn.qnn_linear_attention
    for bad in (lambda: run(q.cpu(), k, v, decay), lambda: run(q, k.bfloat16(), v, decay), lambda: run(q, k[:, :5], v, decay),
                lambda: run(q, k, v, decay.double()), lambda: run(q.transpose(2, 3), k, v, decay),
                lambda: run(q, k, v, decay, state_in=state[:1]), lambda: run(q, k, v, decay, lengths=torch.ones(2, device="cuda")),
                lambda: run(q, k, v, decay, out=torch.empty((2, 12, 4, 8), device="cuda")), lambda: run(q[0], k, v, decay),
                lambda: run(q.double(), k.double(), v.double(), decay)):
        with pytest.raises(ValueError):
            bad()
    both = torch.zeros(4096, device="cuda")
    for bad in (lambda: run(q[:, :, :3], k, v, decay), lambda: run(q, k, v, decay, out=v), lambda: run(q, k, v, decay, scale=float("nan")),
                lambda: run(*(torch.zeros((1, 4, 1, 257), device="cuda") for _ in range(3)), decay[:1]),
                lambda: run(q, k, both[:1536].view(2, 12, 4, 16), decay, state_out=both[1000:3048].view(2, 4, 16, 16))):
        with pytest.raises(qnn.QnnError):
            bad()
    logits, scores = select_inputs(1, 2, 3, 40, "f32")
    run = qnn.qnn_beam_select
    for bad in (lambda: run(logits[0], scores), lambda: run(logits.cpu(), scores), lambda: run(logits, scores[:1]),
                lambda: run(logits.transpose(1, 2), scores), lambda: run(logits.double(), scores),
                lambda: run(logits, scores, finished=torch.zeros((2, 3), device="cuda")), lambda: run(logits, scores.half())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: run(logits, scores, 0), lambda: run(logits, scores, 129), lambda: run(logits, scores, eos=40),
                lambda: run(logits, scores, eos=-1), lambda: run(torch.zeros((1, 129, 2), device="cuda"), torch.zeros((1, 129), device="cuda"), 1)):
        with pytest.raises(qnn.QnnError):
            bad()
    parents, s = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((6, 5), device="cuda")
    run = qnn.qnn_beam_reorder
    for bad in (lambda: run([s], parents.long()), lambda: run([s[:5]], parents), lambda: run([s], parents, dims=[2]),
                lambda: run([s.t()], parents, dims=[1]), lambda: run([s, torch.zeros((8, 2), device="cuda")], parents),
                lambda: run([s], parents, out=[torch.zeros((5, 5), device="cuda")]), lambda: run([s], parents, dims=[0, 1]),
                lambda: run([s.cpu()], parents), lambda: run([s], parents[:, :2].contiguous(), out=[s])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: run([s, s], parents, out=[s, s]), lambda: run([s, s.clone()], parents, out=[s, s]),
                lambda: run([torch.zeros((2 * 129, 1), device="cuda")], parents),
                lambda: run([both[:30].view(6, 5)], parents, out=[both[5:35].view(6, 5)])):
        with pytest.raises(qnn.QnnError):
            bad()
    table, ids = torch.zeros((5, 4), device="cuda"), torch.zeros((3,), dtype=torch.int32, device="cuda")
    for bad in (lambda: qnn.qnn_embedding(ids.float(), table), lambda: qnn.qnn_embedding(ids, table[0]), lambda: qnn.qnn_embedding(ids.cpu(), table),
                lambda: qnn.qnn_embedding(ids, table.double()), lambda: qnn.qnn_embedding(ids, table, out=torch.empty((3, 5), device="cuda")),
                lambda: qnn.qnn_embedding(ids, table.t()), lambda: qnn.qnn_embedding_grad(table, ids, 5),
                lambda: qnn.qnn_embedding_grad(table[:3], ids, 5, out=torch.empty((4, 4), device="cuda")),
                lambda: qnn.qnn_embedding_grad(table[:3], ids, 5, accumulate=True), lambda: qnn.qnn_embedding_grad(table[:3, 0], ids, 5)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(qnn.QnnError):
        qnn.qnn_embedding(ids, table, out=table[:3])
    with pytest.raises(qnn.QnnError):
        qnn.qnn_embedding_grad(table[:3], ids, 5, out=table)
    assert qnn.device_status() == qnn.QNN_OK
