"""The selective state-space layer's calls where values are not finite, far apart or nearly out of range, and where small errors
add up: against 64-bit references with bounds tighter than the general ones (layer_ref.py)."""
import os
import subprocess
import sys

import numpy as np
import pytest

import layer_ref as ref
from test_gpu_layer import activations, check_scan, gpu, host, qnn, rng, scan_inputs, scan_want, weights, within  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------------------- convolution

def same(a, b):
    return ((a == b) | (torch.isnan(a) & torch.isnan(b))).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [40, 37])
@pytest.mark.parametrize("W", [1, 2, 3, 4, 5, 6, 7, 8])
def test_conv_keeps_what_is_not_finite_to_its_taps(qnn, W, D, kind):
    """An input that is not finite reaches the W outputs whose formula holds it, and no other; the last inputs of a state that is
    not finite fewer."""
    g = rng(W + D)
    T = 100
    x, s = gpu(g.normal(0, 1, (2, T, D)), kind), gpu(g.normal(0, 1, (2, W - 1, D)), kind)
    w, b = gpu((g.choice([-1, 1], (D, W)) * g.uniform(0.2, 1, (D, W))).astype(np.float32)), gpu(g.normal(0, 1, D).astype(np.float32))
    clean = qnn.qnn_causal_conv(x, w, bias=b, state_in=s, silu=False)
    touched = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
    for seq, t, d, v in ((0, 30, 5, float("nan")), (0, 47, 9, float("inf")), (1, 0, 11, -float("inf")), (1, 63, 36, float("nan")),
                         (1, 95, 2, float("inf"))):
        x[seq, t, d] = v
        touched[seq, t:t + W, d] = True
    if W > 1:
        s[0, 0, 3] = float("nan")
        touched[0, :1, 3] = True
        s[1, -1, 20] = float("inf")
        touched[1, :W - 1, 20] = True
    got = qnn.qnn_causal_conv(x, w, bias=b, state_in=s, silu=False)
    assert torch.equal(got[~touched], clean[~touched])
    assert not torch.isfinite(got[touched]).any()
    for n in (1, 3, 7):  # the frames in parts, with the state carried
        state, parts = s.clone(), []
        for t in range(0, T, n):
            parts.append(qnn.qnn_causal_conv(x[:, t:t + n], w, bias=b, state_in=state, state_out=state, silu=False))
        assert same(torch.cat(parts, 1), got), n
    gated = qnn.qnn_causal_conv(x, w, bias=b, state_in=s)
    assert torch.isfinite(gated[~touched]).all()


def test_conv_refuses_a_state_over_the_outputs(qnn):
    x, w = torch.randn(2, 5, 16, device="cuda"), torch.randn(16, 4, device="cuda")
    buf = torch.zeros(2 * 5 * 16 + 2 * 3 * 16, device="cuda")
    with pytest.raises(qnn.QnnError):
        qnn.qnn_causal_conv(x, w, out=buf[:160].view(2, 5, 16), state_out=buf[150:246].view(2, 3, 16))
    with pytest.raises(qnn.QnnError):  # the states shifted over one another
        qnn.qnn_causal_conv(x, w, state_in=buf[:96].view(2, 3, 16), state_out=buf[16:112].view(2, 3, 16))
    qnn.qnn_causal_conv(x, w, out=buf[:160].view(2, 5, 16), state_out=buf[160:256].view(2, 3, 16))


# --------------------------------------------------------------------------------------- norm

def test_norm_of_the_longest_rows(qnn):
    """Rows of one value: s = 1 / sqrt(v^2 + eps), which 64 bits hold (v^2 is exact there), and every v of the row is (v s) w."""
    cols, n = 1 << 24, 64
    v = rng(24).uniform(0.5, 2, n).astype(np.float32)
    x = gpu(v)[:, None].expand(n, cols).contiguous()
    _, params, _, _, _ = qnn.qnn_rmsnorm_quantize(x, torch.ones(cols, device="cuda"))
    s = (1 / np.sqrt(v.astype(np.float64) ** 2 + 1e-5)).astype(np.float32)
    got = qnn.params_view(params)
    assert np.array_equal(got["vmin"], v * s) and np.array_equal(got["vmax"], v * s)
    assert qnn.device_status() == qnn.QNN_OK


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1 << 20, (1 << 22) + 3])
def test_norm_of_long_rows(qnn, cols, kind):
    from test_gpu_layer import check_norm, norm_inputs
    x, w, r = norm_inputs(cols, 1, cols, kind)
    check_norm(qnn, x, w, r)


def test_norm_code_sums_end_where_they_could_pass_32_bits(qnn):
    most = (2 ** 31 - 1) // 255
    x, w = torch.full((1, most + 1), 1.0, device="cuda"), torch.ones(most + 1, device="cuda")
    x[:, 0] = -1e-6  # nearly all codes are 255
    codes, _, sums, _, _ = qnn.qnn_rmsnorm_quantize(x[:, :most], w[:most])
    assert codes.long().sum().item() == sums.item() > 2 ** 31 - 1000
    codes, _, sums, _, _ = qnn.qnn_rmsnorm_quantize(x, w)
    assert sums is None and codes.long().sum().item() > 2 ** 31 - 1000


# --------------------------------------------------------------------------------------- 4-bit products

def check_product_by_groups(qnn, A, params, w, group, bias=None):
    """The sum of a group's codes is exact. What is rounded: each addition of a group's term (any order: `groups` of them, each
    relative to the terms' sizes), the row sum, 128 + z, their product's addition, the quotient and the bias' addition."""
    codes, off, scale = ref.quantize4(w, group)
    N, K = w.shape
    ng = off.shape[1]
    full = np.zeros((N, ng * group))
    full[:, :K] = codes
    c = (full.reshape(N, ng, group) + off[..., None])
    if K % group:
        c[:, -1, K % group:] = 0
    a = np.zeros((len(A), ng * group))
    a[:, :K] = A.astype(np.float64) - 128
    terms = np.einsum("mgk,ngk->mng", a.reshape(len(A), ng, group), c) * scale.astype(np.float64)
    z, Q = params["z"].astype(np.float64)[:, None] + 128, params["Q"].astype(np.float64)[:, None]
    rows = (c.sum(2) * scale.astype(np.float64)).sum(1)
    y = (terms.sum(2) + z * rows) / Q
    bound = ((ng + 2) * np.abs(terms).sum(2) + 3 * np.abs(z * rows)) * ref.U / Q
    if bias is not None:
        y = y + bias.astype(np.float64)
        bound = bound + 3 * ref.U * np.abs(bias)
    got = qnn.qnn_qmatmul4(gpu(A), qnn.params_tensor(params), qnn.qnn_quantize4(gpu(w), group), bias=gpu(bias))
    within(host(got), y, bound + 3 * ref.U * np.abs(y))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 8192, 48), (8, 8192, 20), (16, 8192, 33), (32, 4000, 20), (3, 500, 40), (33, 1000, 17),
                                   (1, 33025, 16)])
def test_qmatmul4_sums_of_groups(qnn, M, K, N, group):
    A, params, _ = activations(M + K, M, K)
    check_product_by_groups(qnn, A, params, weights(N + K, N, K), group, rng(N).normal(0, 1, N).astype(np.float32))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(1, 8192), (9, 8192), (16, 1000), (32, 4096), (40, 8192)])
def test_qmatmul4_of_whole_numbers_is_exact(qnn, M, K, group):
    """Every code 0 or 255, every weight 0 or 15, a scale of 1: below 2^24, so no addition rounds."""
    g = rng(M + K)
    A = np.where(g.random((M, K)) < 0.7, 255, 0).astype(np.uint8)
    w = np.where(g.random((40, K)) < 0.5, 0.0, 15.0).astype(np.float32)
    w[:, 0::32], w[:, 1::32] = 0.0, 15.0
    params = np.zeros(M, qnn.QPARAMS_DTYPE)
    params["Q"], params["z"], params["vmax"] = 1.0, -128, 1.0
    got = qnn.qnn_qmatmul4(gpu(A), qnn.params_tensor(params), qnn.qnn_quantize4(gpu(w), group))
    assert np.array_equal(host(got), (A.astype(np.int64) - 128) @ w.astype(np.int64).T)


@pytest.mark.parametrize("M,N,K", [(16, 9800, 8192), (32, 19000, 4352), (8, 9800, 8300), (2000, 100, 1000), (5000, 33, 300)])
def test_qmatmul4_of_whole_numbers_over_many_tiles(qnn, M, N, K):
    """More row tiles than clusters run at once, and many blocks of rows: exact as above."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    A = torch.randint(0, 256, (M, K), generator=g, device="cuda", dtype=torch.uint8)
    w = torch.randint(0, 16, (N, K), generator=g, device="cuda").float()
    w[:, 0::32], w[:, 1::32] = 0.0, 15.0
    params = np.zeros(M, qnn.QPARAMS_DTYPE)
    params["Q"], params["z"], params["vmax"] = 1.0, -128, 1.0
    got = qnn.qnn_qmatmul4(A, qnn.params_tensor(params), qnn.qnn_quantize4(w, 64))
    assert torch.equal(got.double(), (A.double() - 128) @ w.double().t())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 9, 20])
def test_qmatmul4_scales_near_the_least(qnn, M, group):
    """Scales of 2^-126 to 2^-122 on activations large enough that the results are ordinary numbers; few codes off the center, so
    that groups' sums are a few units."""
    g = rng(M + group)
    N, K = 24, 512
    w = g.integers(0, 16, (N, K)).astype(np.float64)
    w[:, 0::32], w[:, 1::32] = 0, 15
    w = (w * (g.uniform(1, 16, (N, 1)) * 2.0 ** -126)).astype(np.float32)
    A = np.full((M, K), 128, np.uint8)
    for m in range(M):
        at = g.integers(0, 32, K // 32) + np.arange(0, K, 32)
        A[m, at] = 128 + g.integers(-3, 4, K // 32)
    params = np.zeros(M, qnn.QPARAMS_DTYPE)
    params["Q"], params["z"], params["vmax"] = 2.0 ** -100, -128, 1.0
    check_product_by_groups(qnn, A, params, w, group)


# --------------------------------------------------------------------------------------- scan

def long_memory(qnn, frames_a_call):
    """(signed and root-mean-square deviation of states after 400 frames in calls of some frames): of sums of positive terms, whose
    factors exp(-x), x = 2^-8 .. 2^-3, are each 1 + d times theirs. h' = f (1 + d) h + b deviates by d g, g' = f (g + h)."""
    g = rng(17)
    B, T, D, N = 2, 400, 256, 16
    s = gpu(g.uniform(0.5, 1, (B, T, D)).astype(np.float32))
    A = (-2.0 ** g.uniform(-7, -3, (D, N))).astype(np.float32)
    one, bc = torch.ones(B, T, D, device="cuda"), torch.ones(B, T, N, device="cuda")
    state, Ag = torch.zeros(B, D, N, device="cuda"), gpu(A)
    for t in range(0, T, frames_a_call):
        k = slice(t, t + frames_a_call)
        qnn.qnn_ssm_scan(one[:, k], s[:, k], Ag, bc[:, k], bc[:, k], softplus=False, state_in=state, state_out=state)
    h, dev = np.zeros((B, D, N)), np.zeros((B, D, N))
    for t in range(T):
        st = host(s[:, t])[..., None]
        f = np.exp(st * A.astype(np.float64))
        h, dev = f * h + st, f * (dev + h)
    e, memory = (host(state) - h) / h, dev / h
    # noise a frame: 3e-8 of the exponential, 2^-24 / sqrt(3) each of the product and the sum, which fade with the state
    allowed = 1.5e-8 * memory + 6e-8 * np.sqrt(memory) + 6e-8
    return e.sum() / memory.sum(), np.sqrt((e ** 2).mean()) / np.sqrt((allowed ** 2).mean())


@pytest.mark.parametrize("frames_a_call", [1, 2, 4, 8, 400])
def test_scan_long_memory(qnn, frames_a_call):
    """Factors are right on average to 1.3e-8, whose sum over a state's memory noise does not hide; 0.2e-8 for the rest (log2 e
    rounded to fp32 counts 1.3e-8 x)."""
    bias, noise = long_memory(qnn, frames_a_call)
    print(f"calls of {frames_a_call}: factors off by {bias:.2e} on average, states by {noise:.2f} of what is allowed")
    assert abs(bias) <= 1.5e-8 and noise <= 1


@pytest.mark.parametrize("T", [1, 4, 40, 600])
def test_scan_channels_without_a_memory(qnn, T):
    """A of minus infinity, or so low that its product with log2 e has no fp32 value: a factor of 0, as A = -1e6 gives; a frame that
    is not there leaves the states as they are."""
    lengths = [T, 0, 1, T // 2, max(T - 1, 0), T - T // 3]
    i = scan_inputs(3, len(lengths), T, 40, 16, 1, "f32", softplus=False)
    i["dt_bias"] = None
    i["A"][3], i["A"][17, 5] = -1e6, -1e6
    want, bound, state, sbound = scan_want(i, False, lengths, "f32")
    i["A"][3], i["A"][17, 5] = -np.inf, -3e38
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    out = torch.empty(len(lengths), 40, 16, device="cuda")
    got = host(qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], a["B"], a["C"], D=a["D"], z=a["z"], softplus=False, state_in=a["state_in"],
                                state_out=out, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda")))
    assert np.isfinite(sbound).all()
    within(got, want, bound)
    within(host(out), state, sbound)


def grown(T, D, N, from_state):
    """States that grow by e^2 a frame over 70 frames and shrink again, from 1e-30; or that are 0 until they grow at the end."""
    g = rng(T + D)
    i = scan_inputs(4, 1, T, D, N, 1, "f32", gate=False, bias=False, softplus=False)
    s = np.full((1, T, D), 0.05)
    u = np.zeros((1, T, D))
    if from_state:
        s[:, :48] = 0
        s[:, 48:118] = -2
        s[:, 118:160] = 0.5
        i["state_in"] = np.full((1, D, N), 1e-30, np.float32) * g.uniform(0.5, 1.5, (1, D, N)).astype(np.float32)
    else:
        s[:, :] = -2
        u[:, T - 12:] = g.normal(0, 1, (1, 12, D))
        i["state_in"] = None
    i["A"] = np.full((D, N), -1.0, np.float32)
    i["dt"], i["u"] = gpu(s.astype(np.float32)), gpu(u.astype(np.float32))
    return i


@pytest.mark.parametrize("from_state", [True, False])
@pytest.mark.parametrize("T,D,N", [(200, 40, 16), (600, 40, 16), (600, 12, 4), (2050, 6, 100), (1200, 33, 24)])
def test_scan_states_that_grow_where_a_sequence_is_shared(qnn, T, D, N, from_state):
    """The factor over a part of the sequence has no fp32 value, the states and outputs have."""
    i = grown(T, D, N, from_state)
    want, bound, state, sbound = scan_want(i, False, None, "f32")
    assert np.isfinite(bound).all() and np.isfinite(sbound).all()
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    out = torch.empty(1, D, N, device="cuda") if a["state_in"] is None else a["state_in"]
    got = host(qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], a["B"], a["C"], D=a["D"], softplus=False, state_in=a["state_in"],
                                state_out=out))
    within(got, want, bound)
    within(host(out), state, sbound)


@pytest.mark.parametrize("B,T,D,N", [(1, 2050, 6, 100), (1, 1030, 5, 128), (2, 520, 40, 128), (3, 300, 9, 65), (1, 2100, 40, 16),
                                     (1, 1100, 70, 64)])
def test_scan_long_sequences_shared_by_many_blocks(qnn, B, T, D, N):
    check_scan(qnn, B, T, D, N)
    check_scan(qnn, B, T, D, N, place="in place", lengths=[T - 5, 0, T // 2][:B])


def test_scan_captured_before_its_first_call(qnn):
    """In a process of its own: a plan of many blocks a sequence, asked for while a graph is captured, has the bits of a plain call."""
    code = '''
import torch
from paper_1607_04683_gb300 import qnn
torch.cuda.set_device(0)
qnn.device_status()
g = torch.Generator(device="cuda").manual_seed(1)
T, D, N = 2050, 6, 16
u, dt = (torch.rand((1, T, D), generator=g, device="cuda") for _ in range(2))
bc, A, out = torch.rand((1, T, N), generator=g, device="cuda"), -torch.rand((D, N), generator=g, device="cuda"), torch.zeros(1, T, D, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    qnn.qnn_ssm_scan(u, dt, A, bc, bc, out=out)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(out, qnn.qnn_ssm_scan(u, dt, A, bc, bc)) and out.abs().sum() > 0
'''
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0, r.stderr[-2000:]
