"""The selective state-space layer's calls on the GPU against plain 64-bit references (layer_ref.py, which derives the
bounds), and a layer of them as it is used."""
import numpy as np
import pytest

import layer_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


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
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def wide(t, extra, front=0):
    """The same values as a slice of wider rows (or frames) whose other values are NaN."""
    full = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    full[..., front:front + t.shape[-1]] = t
    return full[..., front:front + t.shape[-1]]


def within(got, want, bound, what=""):
    d = np.abs(got - want)
    ok = np.isnan(want) | (d <= bound) | np.isinf(bound)
    assert ok.all(), (what, np.argwhere(~ok)[:5].tolist(), got[~ok][:5], want[~ok][:5], bound[~ok][:5])


# --------------------------------------------------------------------------------------- norm

def check_norm(qnn, x, w, r=None, eps=1e-5, inplace=None, padded=0, front=0):
    """Codes, units, sums, values and the residual's sum, all to the bit."""
    xs = host(x).astype(np.float32)
    rs = None if r is None else host(r).astype(np.float32)
    h, v = ref.rmsnorm_rows(xs, host(w), rs, eps)
    codes, params, sums = ref.codes_of(v)
    out = None
    if padded:
        x = wide(x, padded, front)
        r = None if r is None else wide(r, padded + 3, front)
    if inplace == "x":
        out = x
    elif inplace == "r":
        out = r
    gc, gp, gs, gh, gv = qnn.qnn_rmsnorm_quantize(x, w, residual=r, eps=eps, residual_out=out, want_values=True)
    assert np.array_equal(qnn.params_view(gp), params)
    assert np.array_equal(host(gc), codes) and np.array_equal(host(gs), sums)
    assert np.array_equal(gv.cpu().numpy(), ref.recover(codes, params))
    if r is None:
        assert gh is None
    else:
        assert torch.equal(gh.cpu(), torch.from_numpy(h).to(gh.dtype))
    assert qnn.device_status() == qnn.QNN_OK


def norm_inputs(seed, rows, cols, kind, residual=True):
    g = rng(seed)
    x = g.normal(0, 1, (rows, cols)) * np.exp(g.normal(0, 1, (rows, 1)))
    r = g.normal(0, 2, (rows, cols)) if residual else None
    w = (1 + g.normal(0, 0.3, cols)).astype(np.float32)
    return gpu(x, kind), gpu(w), gpu(r, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 2), (3, 7), (1, 31), (5, 32), (4, 33), (7, 40), (3, 127), (9, 128), (2, 129),
                                       (6, 255), (3, 256), (5, 500), (3, 511), (4, 512), (2, 513), (3, 1000), (2, 1023),
                                       (3, 1024), (2, 1025), (2, 2047), (3, 2048), (2, 2049), (1, 2727), (2, 4095), (2, 4096),
                                       (2, 4097), (1, 8192), (2, 8193), (1, 16384), (1, 16385), (1, 40001), (300, 500)])
def test_norm(qnn, rows, cols, kind):
    x, w, r = norm_inputs(rows * 100003 + cols, rows, cols, kind)
    check_norm(qnn, x, w, r)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols", [8, 96, 500, 2048, 2727, 20000])
@pytest.mark.parametrize("inplace,padded,front", [(None, 0, 0), (None, 5, 0), (None, 8, 8), (None, 9, 1), ("x", 0, 0), ("r", 0, 0),
                                                  ("r", 3, 2), ("x", 16, 0)])
def test_norm_places_and_strides(qnn, cols, kind, inplace, padded, front):
    x, w, r = norm_inputs(cols, 6, cols, kind)
    check_norm(qnn, x, w, r, inplace=inplace, padded=padded, front=front)


@pytest.mark.parametrize("cols", [5, 64, 500, 2048, 9000])
def test_norm_without_a_residual(qnn, cols):
    x, w, _ = norm_inputs(cols, 4, cols, "f32", residual=False)
    check_norm(qnn, x, w)
    check_norm(qnn, x, w, eps=1e-20)
    check_norm(qnn, x, w, eps=7.5)
    check_norm(qnn, x, w, eps=1e20)


@pytest.mark.parametrize("cols", [3, 40, 300, 2048, 20000])
def test_norm_rows_at_the_ends_of_the_range(qnn, cols):
    g = rng(cols)
    rows = [np.zeros(cols), np.full(cols, 3.0), np.full(cols, -1e-6), np.where(np.arange(cols) == cols // 2, 1.0, 0.0),
            g.normal(0, 1e-20, cols), g.normal(0, 1e-38, cols), g.normal(0, 1e18, cols), g.normal(0, 1e25, cols),
            g.normal(0, 3e37, cols).clip(-3e38, 3e38), 1e4 + g.normal(0, 1e-2, cols), g.normal(0, 1, cols) ** 9]
    x = np.array(rows).astype(np.float32)
    w = gpu((1 + g.normal(0, 0.3, cols)).astype(np.float32))
    check_norm(qnn, gpu(x), w)
    check_norm(qnn, gpu(x), w, r=gpu(-0.5 * x))
    check_norm(qnn, gpu(x), gpu(np.zeros(cols, np.float32)))
    check_norm(qnn, gpu(x), gpu(np.full(cols, -1e-3, np.float32)))


@pytest.mark.parametrize("cols", [30, 500, 2048, 20000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_with_a_value_that_is_not_finite(qnn, cols, bad):
    x, w, r = norm_inputs(cols, 5, cols, "f32")
    h, v = ref.rmsnorm_rows(host(x).astype(np.float32), host(w), host(r).astype(np.float32))
    codes, params, sums = ref.codes_of(v)
    x[2, cols // 3] = bad
    gc, gp, gs, gh, gv = qnn.qnn_rmsnorm_quantize(x, w, residual=r, want_values=True)
    assert qnn.device_status() == qnn.QNN_ERR_NONFINITE
    keep = [0, 1, 3, 4]  # the other rows are as they would be
    assert np.array_equal(host(gc)[keep], codes[keep]) and np.array_equal(host(gs)[keep], sums[keep])
    assert np.array_equal(qnn.params_view(gp)[keep], params[keep])
    assert torch.equal(gh[keep].cpu(), torch.from_numpy(h[keep]))
    same = np.arange(cols) != cols // 3
    assert np.array_equal(gh[2].cpu().numpy()[same], h[2][same])
    assert qnn.device_status() == qnn.QNN_OK


def test_norm_refuses_on_the_device(qnn):
    x, w, r = norm_inputs(1, 4, 64, "f32")
    with pytest.raises(qnn.QnnError):  # h over a shifted part of x
        buf = torch.zeros(4 * 64 + 64, device="cuda")
        qnn.qnn_rmsnorm_quantize(buf[:256].view(4, 64), w, residual=r, residual_out=buf[32:288].view(4, 64))
    with pytest.raises(ValueError):
        qnn.qnn_rmsnorm_quantize(x, w[:63], residual=r)
    with pytest.raises(ValueError):
        qnn.qnn_rmsnorm_quantize(x, w, residual=r.half())
    with pytest.raises(ValueError):
        qnn.qnn_rmsnorm_quantize(x.double(), w)
    with pytest.raises(ValueError):
        qnn.qnn_rmsnorm_quantize(x.t(), w)
    with pytest.raises(ValueError):
        qnn.qnn_rmsnorm_quantize(x, w, residual_out=x)
    with pytest.raises(qnn.QnnError):
        qnn.qnn_rmsnorm_quantize(x, w.cpu())
    with pytest.raises(qnn.QnnError):
        qnn.qnn_rmsnorm_quantize(x, w, eps=0.0)
    codes, *_ = qnn.qnn_rmsnorm_quantize(x[:0], w)
    assert codes.shape == (0, 64)


# --------------------------------------------------------------------------------------- 4-bit weights

def weights(seed, N, K, scale=0.1):
    g = rng(seed)
    w = (g.normal(0, scale, (N, K)) * np.exp(g.normal(0, 0.5, (N, 1)))).astype(np.float32)
    return w


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 31), (16, 32), (17, 33), (15, 128), (33, 129), (40, 500), (8, 1000), (5, 33025)])
def test_quantize4(qnn, N, K, group):
    w = weights(N + K, N, K)
    w[0, : K // 2] = 0          # units of zeros
    w[N // 2] = np.abs(w[N // 2])  # of one sign
    w[N - 1] *= np.float32(1e-37)  # the least scale
    codes, off, scale = ref.quantize4(w, group)
    got = qnn.qnn_quantize4(wide(gpu(w), 3), group)
    assert np.array_equal(host(got.codes), ref.tile4(codes))
    assert np.array_equal(host(got.units), ref.units4(off, scale, N, K, group))
    v = ref.values4(codes, off, scale, group)
    sums = v.sum(1)
    # a 64-bit sum rounded once
    within(host(got.row_sums), sums, ref.U * np.abs(sums) + K * 2.0 ** -52 * np.abs(v).sum(1) + 2.0 ** -150)
    assert qnn.device_status() == qnn.QNN_OK


def test_quantize4_with_a_value_that_is_not_finite(qnn):
    w = weights(3, 20, 200)
    w[7, 5] = np.inf
    qnn.qnn_quantize4(gpu(w), 64)
    assert qnn.device_status() == qnn.QNN_ERR_NONFINITE


def check_product(qnn, A, params, w, group, bias=None, ga=1, padded=0):
    codes, off, scale = ref.quantize4(w, group)
    W = ref.values4(codes, off, scale, group)
    want, bound = ref.qmatmul4(A, params, W, bias)
    q4 = qnn.qnn_quantize4(gpu(w), group)
    a, y = gpu(A), None
    if padded:
        big = torch.full((A.shape[0], A.shape[1] + padded), 201, dtype=torch.uint8, device="cuda")
        big[:, :A.shape[1]] = a
        a = big[:, :A.shape[1]]
        full = torch.full((A.shape[0], w.shape[0] + padded), -77.0, device="cuda")
        y = full[:, :w.shape[0]]
    got = qnn.qnn_qmatmul4(a, qnn.params_tensor(params), q4, ga=ga, bias=gpu(bias), out=y)
    if ga == 0:
        params = np.repeat(params, len(A))
    within(host(got), want, bound)
    if padded:
        assert (host(full)[:, w.shape[0]:] == -77.0).all()
    again = qnn.qnn_qmatmul4(a, qnn.params_tensor(params), q4, ga=1, bias=gpu(bias))
    assert torch.equal(got, again)


def activations(seed, M, K, spread=1.0, shift=0.0):
    g = rng(seed)
    return ref.codes_of((g.normal(shift, spread, (M, K))).astype(np.float32))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 32, 16), (2, 31, 5), (3, 64, 17), (1, 128, 128), (4, 129, 33), (5, 100, 40),
                                   (8, 500, 500), (9, 1000, 70), (1, 2048, 130), (7, 2049, 31), (16, 512, 64), (17, 300, 129),
                                   (31, 640, 20), (32, 256, 48), (33, 127, 16), (64, 384, 33), (100, 96, 24), (1, 8192, 48),
                                   (12, 8191, 17), (2, 33025, 18), (33, 4500, 20),
                                   (32, 33025, 20), (16, 20000, 33), (9, 5000, 300), (1, 256, 40000), (3, 640, 41000)])
def test_qmatmul4(qnn, M, K, N, group):
    A, params, _ = activations(M * 7 + K, M, K)
    bias = rng(K).normal(0, 1, N).astype(np.float32)
    check_product(qnn, A, params, weights(N + K, N, K), group, bias=bias if N % 2 else None)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N,padded", [(3, 500, 40, 7), (9, 1000, 33, 16), (1, 2048, 100, 1), (20, 300, 50, 5)])
def test_qmatmul4_strides(qnn, M, K, N, padded, group):
    A, params, _ = activations(M + K, M, K)
    check_product(qnn, A, params, weights(N, N, K), group, padded=padded)


@pytest.mark.parametrize("shift,spread", [(100.0, 1.0), (-3.0, 0.01), (0.0, 1e-30), (1e20, 1e19), (0.0, 0.0), (5.0, 0.0)])
def test_qmatmul4_units_far_from_zero(qnn, shift, spread):
    A, params, _ = activations(11, 6, 700, spread, shift)
    check_product(qnn, A, params, weights(5, 50, 700), 64)


def test_qmatmul4_all_extreme_codes(qnn):
    """Exact group sums at their largest: every code 0 or 255 against 0 or 15."""
    g = rng(3)
    K, N = 1024, 48
    for lo, hi in ((0, 0), (255, 255), (0, 255)):
        A = np.where(g.random((9, K)) < 0.5, lo, hi).astype(np.uint8)
        params = np.zeros(9, qnn.QPARAMS_DTYPE)
        params["Q"], params["z"], params["vmax"] = 1.0, -128, 1.0
        w = np.where(g.random((N, K)) < 0.5, 0.0, 1.0).astype(np.float32)
        w[:, 0::32] = 0.0
        w[:, 1::32] = 15.0
        for group in (32, 64, 128):
            check_product(qnn, A, params, w, group)


def test_qmatmul4_more_row_tiles_than_blocks_and_rows_in_parts(qnn):
    """Many row tiles on rows that shared memory holds in parts, against 64-bit products of the values on the GPU."""
    M, N, K, G = 32, 8480, 8960, 64
    A, params, _ = activations(7, M, K)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w = qnn.qnn_quantize4(torch.randn((N, K), generator=g, device="cuda") * 0.05, G)
    nt, kt = w.codes.shape[:2]
    p = w.codes.view(nt, kt, 2, 8, 4, 4, 4)  # halves of rows, rows, eighths of 32 columns, parts of 32, bytes
    half = torch.stack([p & 15, p >> 4], -1).view(nt, kt, 2, 8, 4, 4, 8)[..., [0, 4, 1, 5, 2, 6, 3, 7]]
    codes = half.permute(0, 2, 3, 1, 5, 4, 6).reshape(nt * 16, kt * 128 // G, G).double()
    u = w.units.permute(0, 2, 1, 3, 4).reshape(nt * 16, kt * 128 // G, 2).double()
    W = ((codes + u[..., :1]) * u[..., 1:]).view(nt * 16, kt * 128)[:N, :K]
    a = gpu(A).double()
    z, Q = (torch.from_numpy(params[k].astype(np.float64)).cuda()[:, None] for k in ("z", "Q"))
    want = (a + z) @ W.t() / Q
    mass = ((a - 128).abs() @ W.abs().t() + (z + 128).abs() * W.abs().sum(1)) / Q
    got = qnn.qnn_qmatmul4(gpu(A), qnn.params_tensor(params), w)
    assert ((got.double() - want).abs() <= (K / 32 + 16) * ref.U * mass + 2 * ref.U * want.abs()).all()


def test_qmatmul4_one_unit_for_the_matrix(qnn):
    x = rng(2).normal(0, 1, (5, 300)).astype(np.float32)
    import oracle
    A, params, _ = oracle.quantize(x, oracle.PER_MATRIX)
    check_product(qnn, A, params, weights(1, 40, 300), 32, ga=0)


def test_qmatmul4_units_of_infinite_scale(qnn):
    x = np.zeros((3, 200), np.float32)
    x[1] = rng(1).uniform(0, 1e-38, 200)
    x[1, 0] = 0
    A, params, _ = ref.codes_of(x)
    assert np.isinf(params["Q"][1])
    w = qnn.qnn_quantize4(gpu(weights(1, 40, 200)), 64)
    y = qnn.qnn_qmatmul4(gpu(A), qnn.params_tensor(params), w)
    assert (host(y)[1] == 0).all() and np.isfinite(host(y)).all()


def test_qmatmul4_refuses_on_the_device(qnn):
    A, params, _ = activations(1, 3, 64)
    w = qnn.qnn_quantize4(gpu(weights(1, 20, 64)), 64)
    a, p = gpu(A), qnn.params_tensor(params)
    with pytest.raises(ValueError):
        qnn.qnn_qmatmul4(a[:, :63], p, w)
    with pytest.raises(ValueError):
        qnn.qnn_qmatmul4(a, p[:2], w)
    with pytest.raises(ValueError):
        qnn.qnn_qmatmul4(a, p, w, out=torch.empty((3, 21), device="cuda"))
    with pytest.raises(ValueError):
        qnn.Weights4(w.codes, w.units, w.row_sums, 33, 64, 64)
    with pytest.raises(ValueError):
        qnn.qnn_quantize4(gpu(weights(1, 20, 64)), 48)
    with pytest.raises(qnn.QnnError):
        qnn.qnn_qmatmul4(a, p.cpu(), w)
    with pytest.raises(qnn.QnnError):  # the result over the row sums
        both = torch.zeros(60, device="cuda")
        w2 = qnn.Weights4(w.codes, w.units, both[:20], 20, 64, 64)
        qnn.qnn_qmatmul4(a, p, w2, out=both.view(3, 20))
    assert qnn.qnn_qmatmul4(a[:0], p[:0], w).shape == (0, 20)


# --------------------------------------------------------------------------------------- convolution

def check_conv(qnn, B, T, D, W, kind="f32", act=True, bias=True, states=True, lengths=None, place=None, seed=0):
    g = rng(seed + 131 * T + D)
    x = gpu(g.normal(0, 1, (B, T, D)), kind)
    w, b = g.normal(0, 0.6, (D, W)).astype(np.float32), g.normal(0, 0.5, D).astype(np.float32) if bias else None
    s = gpu(g.normal(0, 1, (B, W - 1, D)), kind) if states else None
    want, bound, last = ref.conv(host(x), w, b, act, None if s is None else host(s), lengths, kind)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s_out, y = torch.empty((B, W - 1, D), dtype=x.dtype, device="cuda"), None
    if lengths is not None:  # frames that are not there: whatever x holds, y stays as it is
        for i, k in enumerate(lengths):
            x[i, max(min(k, T), 0):] = float("nan")
    if place == "in place":
        s_out = s
    if place == "wide":
        x = wide(x, 5, 2)
        y = torch.full((B, T, D + 3), 55.0, dtype=x.dtype, device="cuda")[..., 1:D + 1]
    elif place == "time-major":
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
        y = torch.full((T, B, D), 55.0, dtype=x.dtype, device="cuda").transpose(0, 1)
    elif lengths is not None:
        y = torch.full((B, T, D), 55.0, dtype=x.dtype, device="cuda")
    got = qnn.qnn_causal_conv(x, gpu(w), bias=gpu(b), silu=act, state_in=s, state_out=s_out, lengths=n, out=y)
    gh = host(got)
    within(gh, want, bound)
    assert np.array_equal(host(s_out), last)
    absent = np.arange(T)[None, :] >= (np.full((B, 1), T) if lengths is None else np.clip(lengths, 0, T)[:, None])
    assert (gh[absent] == 55.0).all()
    if place == "wide":
        full = y._base
        assert (full[..., 0] == 55.0).all() and (full[..., D + 1:] == 55.0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,D,W", [(1, 1, 1, 1), (1, 1, 8, 4), (2, 2, 7, 4), (3, 3, 33, 4), (2, 4, 64, 3), (1, 5, 500, 2),
                                     (5, 17, 40, 8), (2, 64, 31, 4), (1, 65, 256, 4), (2, 127, 130, 4), (1, 300, 12, 5),
                                     (257, 1, 36, 4), (3, 129, 96, 1), (1, 1000, 24, 4), (2, 33, 1030, 6), (1, 7, 2048, 7)])
def test_conv(qnn, B, T, D, W, kind):
    check_conv(qnn, B, T, D, W, kind)


@pytest.mark.parametrize("act,bias,states", [(False, True, True), (True, False, True), (True, True, False), (False, False, False)])
def test_conv_options(qnn, act, bias, states):
    for T, D in ((1, 40), (50, 40), (131, 37)):
        check_conv(qnn, 3, T, D, 4, act=act, bias=bias, states=states)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("W", [1, 2, 4, 8])
@pytest.mark.parametrize("T", [1, 5, 40, 200])
def test_conv_ragged(qnn, T, W, kind):
    lengths = [T, 0, 1, T // 2, -3, T + 9, min(2, T), max(T - 1, 0)]
    check_conv(qnn, len(lengths), T, 72, W, kind, lengths=lengths)
    check_conv(qnn, len(lengths), T, 35, W, kind, lengths=lengths, states=False)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", ["in place", "wide", "time-major"])
def test_conv_places(qnn, place, kind):
    for T, D in ((1, 64), (3, 64), (90, 96), (257, 33)):
        check_conv(qnn, 3, T, D, 4, kind, place=place)
        check_conv(qnn, 3, T, D, 4, kind, place=place, lengths=[T, T // 2, 0])


def test_conv_without_frames_carries_the_state_over(qnn):
    s, w = torch.randn(2, 3, 40, device="cuda"), torch.randn(40, 4, device="cuda")
    out = torch.zeros_like(s)
    y = qnn.qnn_causal_conv(torch.empty(2, 0, 40, device="cuda"), w, state_in=s, state_out=out)
    assert y.shape == (2, 0, 40) and torch.equal(out, s)
    qnn.qnn_causal_conv(torch.empty(2, 0, 40, device="cuda"), w, state_out=out)
    assert (out == 0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_conv_in_parts_is_the_whole(qnn, kind):
    """Frames, then a longer part, then frames again with the state carried: the bits of one call."""
    x, w, b = gpu(rng(1).normal(0, 1, (3, 70, 80)), kind), torch.randn(80, 4, device="cuda"), torch.randn(80, device="cuda")
    whole = qnn.qnn_causal_conv(x, w, bias=b)
    s, parts, t = torch.zeros(3, 3, 80, dtype=x.dtype, device="cuda"), [], 0
    for n in (1, 1, 2, 50, 1, 15):
        parts.append(qnn.qnn_causal_conv(x[:, t:t + n], w, bias=b, state_in=s, state_out=s))
        t += n
    assert torch.equal(torch.cat(parts, 1), whole)
    assert torch.equal(s, x[:, -3:])


def test_conv_refuses_on_the_device(qnn):
    x, w = torch.randn(2, 5, 16, device="cuda"), torch.randn(16, 4, device="cuda")
    s = torch.zeros(2, 3, 16, device="cuda")
    for kw in (dict(out=x), dict(state_out=s, out=s.view(-1)[:96].view(2, 3, 16)[:, :0]), dict(out=x.cpu())):
        if kw.get("out") is not None and kw["out"].shape != x.shape:
            continue
        with pytest.raises(qnn.QnnError):
            qnn.qnn_causal_conv(x, w, **kw)
    with pytest.raises(qnn.QnnError):  # every sequence's output in one place
        qnn.qnn_causal_conv(x, w, out=torch.empty(1, 5, 16, device="cuda").expand(2, 5, 16))
    with pytest.raises(qnn.QnnError):  # the state over the input
        buf = torch.randn(2 * 5 * 16 + 2 * 3 * 16, device="cuda")
        qnn.qnn_causal_conv(buf[:160].view(2, 5, 16), w, state_out=buf[100:196].view(2, 3, 16))
    for bad in (dict(weight=w[:15]), dict(bias=w[:, 0]), dict(state_in=s.half()), dict(lengths=torch.zeros(2, device="cuda"))):
        with pytest.raises(ValueError):
            qnn.qnn_causal_conv(x, **({"weight": w} | bad))
    assert qnn.qnn_causal_conv(x[:0], w).shape == (0, 5, 16)


# --------------------------------------------------------------------------------------- scan

def scan_inputs(seed, B, T, D, N, G, kind, gate=True, skip=True, bias=True, states=True, softplus=True):
    g = rng(seed + 7 * T + 13 * D + N)
    i = {"u": gpu(g.normal(0, 1, (B, T, D)), kind), "dt": gpu(g.normal(0, 0.5, (B, T, D)) if softplus else
                                                              g.uniform(0.001, 0.2, (B, T, D)), kind),
         "A": -np.arange(1, N + 1) * np.exp(g.normal(0, 0.1, (D, N))), "B": gpu(g.normal(0, 1, (B, T, G, N)), kind),
         "C": gpu(g.normal(0, 1, (B, T, G, N)), kind), "D": g.normal(1, 0.1, D) if skip else None,
         "z": gpu(g.normal(0, 1, (B, T, D)), kind) if gate else None,
         "dt_bias": np.log(np.expm1(np.exp(g.uniform(np.log(0.001), np.log(0.1), D)))) if bias else None,
         "state_in": g.normal(0, 1, (B, D, N)) if states else None}
    for k in ("A", "D", "dt_bias", "state_in"):
        i[k] = None if i[k] is None else i[k].astype(np.float32)
    return i


def scan_want(i, softplus, lengths, kind):
    h = lambda t: None if t is None else host(t)  # noqa: E731
    return ref.scan(h(i["u"]), h(i["dt"]), i["A"], h(i["B"]), h(i["C"]), i["D"], h(i["z"]), i["dt_bias"], softplus, i["state_in"],
                    lengths, kind)


def check_scan(qnn, B, T, D, N, G=1, kind="f32", lengths=None, place=None, softplus=True, seed=0, **kw):
    i = scan_inputs(seed, B, T, D, N, G, kind, softplus=softplus, **kw)
    want, bound, state, sbound = scan_want(i, softplus, lengths, kind)
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if lengths is not None:
        for b, k in enumerate(lengths):
            for name in ("u", "dt", "B", "C", "z"):
                if a[name] is not None:
                    a[name][b, max(min(k, T), 0):] = float("nan")
    y = torch.full((B, T, D), 55.0, dtype=a["u"].dtype, device="cuda")
    out = torch.empty((B, D, N), device="cuda")
    if place == "in place":
        out = a["state_in"]
    elif place == "wide":
        for k, (extra, front) in {"u": (5, 1), "dt": (3, 3), "z": (8, 8), "B": (0, 0), "C": (0, 0)}.items():
            if a[k] is None:
                continue
            if k in "BC":  # frames of both side by side
                flat = a[k].reshape(B, T, G * N)
                a[k] = wide(flat, G * N + 3, 0 if k == "B" else G * N)
                a[k] = a[k].unflatten(2, (G, N))
            else:
                a[k] = wide(a[k], extra, front)
        y = torch.full((B, T, D + 3), 55.0, dtype=y.dtype, device="cuda")[..., 1:D + 1]
    elif place == "time-major":
        for k in ("u", "dt", "z", "B", "C"):
            if a[k] is not None:
                a[k] = a[k].transpose(0, 1).contiguous().transpose(0, 1)
        y = torch.full((T, B, D), 55.0, dtype=y.dtype, device="cuda").transpose(0, 1)
    if G == 1 and place is None:
        a["B"], a["C"] = a["B"][:, :, 0], a["C"][:, :, 0]
    got = qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], a["B"], a["C"], D=a["D"], z=a["z"], dt_bias=a["dt_bias"], softplus=softplus,
                           state_in=a["state_in"], state_out=out, lengths=n, out=y)
    gh = host(got)
    within(gh, want, bound, "y")
    within(host(out), state, sbound, "state")
    absent = np.arange(T)[None, :] >= (np.full((B, 1), T) if lengths is None else np.clip(lengths, 0, T)[:, None])
    assert (gh[absent] == 55.0).all()
    if place == "wide":
        full = y._base
        assert (full[..., 0] == 55.0).all() and (full[..., D + 1:] == 55.0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,D,N", [(1, 1, 1, 1), (2, 1, 8, 16), (3, 2, 33, 16), (1, 3, 32, 4), (2, 5, 40, 5), (1, 16, 500, 16),
                                     (2, 17, 31, 3), (1, 31, 64, 8), (2, 32, 65, 16), (1, 33, 36, 17), (3, 64, 24, 32),
                                     (1, 65, 130, 16), (2, 127, 16, 64), (1, 128, 40, 24), (1, 129, 48, 128), (40, 1, 36, 16),
                                     (1, 300, 12, 16), (1, 1000, 20, 16), (1, 2050, 6, 16), (2, 520, 100, 4), (9, 1, 7, 100),
                                     (1, 40, 2, 2), (65, 3, 4, 16)])
def test_scan(qnn, B, T, D, N, kind):
    check_scan(qnn, B, T, D, N, kind=kind)


@pytest.mark.parametrize("gate,skip,bias,states,softplus", [(False, True, True, True, True), (True, False, True, True, True),
                                                            (True, True, False, True, True), (True, True, True, False, True),
                                                            (True, True, True, True, False), (False, False, False, False, False)])
def test_scan_options(qnn, gate, skip, bias, states, softplus):
    for T, D, N in ((1, 40, 16), (4, 24, 8), (70, 40, 16), (300, 9, 6)):
        check_scan(qnn, 2, T, D, N, gate=gate, skip=skip, bias=bias, states=states, softplus=softplus)


@pytest.mark.parametrize("D,G,N", [(8, 2, 16), (60, 3, 16), (66, 2, 5), (96, 96, 4), (500, 4, 16), (128, 2, 40)])
def test_scan_groups(qnn, D, G, N):
    for T in (1, 3, 50, 200):
        check_scan(qnn, 2, T, D, N, G)
        check_scan(qnn, 2, T, D, N, G, kind="bf16")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 5, 40, 200, 600])
def test_scan_ragged(qnn, T, kind):
    lengths = [T, 0, 1, T // 2, -3, T + 9, min(2, T), max(T - 1, 0)]
    check_scan(qnn, len(lengths), T, 40, 16, kind=kind, lengths=lengths)
    check_scan(qnn, len(lengths), T, 21, 6, kind=kind, lengths=lengths, states=False, gate=False)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", ["in place", "wide", "time-major"])
def test_scan_places(qnn, place, kind):
    for T, D, N, G in ((1, 64, 16, 1), (3, 36, 16, 2), (90, 64, 16, 1), (260, 18, 7, 3), (600, 32, 16, 1)):
        check_scan(qnn, 3, T, D, N, G, kind=kind, place=place)
        check_scan(qnn, 3, T, D, N, G, kind=kind, place=place, lengths=[T, T // 2, 0])


def test_scan_without_frames_carries_the_state_over(qnn):
    s, A = torch.randn(2, 40, 16, device="cuda"), -torch.rand(40, 16, device="cuda")
    out = torch.zeros_like(s)
    e = torch.empty(2, 0, 40, device="cuda")
    bc = torch.empty(2, 0, 16, device="cuda")
    assert qnn.qnn_ssm_scan(e, e, A, bc, bc, state_in=s, state_out=out).shape == (2, 0, 40) and torch.equal(out, s)
    qnn.qnn_ssm_scan(e, e, A, bc, bc, state_out=out)
    assert (out == 0).all()


def test_scan_steps_of_any_size(qnn):
    """Steps from e^-60 to 80: the softplus at both ends, factors that underflow, a step of zero."""
    for T in (1, 6, 200):
        i = scan_inputs(5, 2, T, 24, 16, 1, "f32", bias=False)
        i["dt"] = gpu(rng(T).uniform(-60, 80, (2, T, 24)).astype(np.float32))
        want, bound, state, sbound = scan_want(i, True, None, "f32")
        out = torch.empty(2, 24, 16, device="cuda")
        got = qnn.qnn_ssm_scan(i["u"], i["dt"], gpu(i["A"]), i["B"], i["C"], D=gpu(i["D"]), z=i["z"], state_in=gpu(i["state_in"]),
                               state_out=out)
        within(host(got), want, bound)
        within(host(out), state, sbound)


def test_scan_gates_of_any_size(qnn):
    for T in (1, 100):
        i = scan_inputs(6, 2, T, 24, 16, 1, "f32")
        i["z"] = gpu(rng(T).uniform(-200, 200, (2, T, 24)).astype(np.float32))
        want, bound, _, _ = scan_want(i, True, None, "f32")
        a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
        got = qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], a["B"], a["C"], D=a["D"], z=a["z"], dt_bias=a["dt_bias"],
                               state_in=a["state_in"])
        # exp(-z) overflows from z = -89 on, where the gate is below 1e-36 of z
        within(host(got), want, bound + 1e-34)


@pytest.mark.parametrize("T", [1, 3, 70, 600])
def test_scan_keeps_what_is_not_finite_to_itself(qnn, T):
    i = scan_inputs(8, 3, T, 40, 16, 1, "f32")
    want, bound, state, sbound = scan_want(i, True, None, "f32")
    i["u"][1, T // 2, 7] = float("nan")
    i["dt"][2, T // 2, 39] = float("inf")
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    out = torch.empty(3, 40, 16, device="cuda")
    got = host(qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], a["B"], a["C"], D=a["D"], z=a["z"], dt_bias=a["dt_bias"],
                                state_in=a["state_in"], state_out=out))
    touched = np.zeros(got.shape, bool)
    touched[1, T // 2:, 7] = touched[2, T // 2:, 39] = True
    within(np.where(touched, 0, got), np.where(touched, 0, want), bound)
    assert np.isnan(got[1, T // 2:, 7]).all()
    rows = np.zeros((3, 40), bool)
    rows[1, 7] = rows[2, 39] = True
    within(host(out)[~rows], state[~rows], sbound[~rows])
    assert np.isnan(host(out)[1, 7]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scan_in_parts_is_the_whole(qnn, kind):
    """Prompts and single frames with the state carried, each against the reference of the whole."""
    i = scan_inputs(9, 3, 150, 40, 16, 1, kind)
    want, bound, state, sbound = scan_want(i, True, None, kind)
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    s, t = a["state_in"].clone(), 0
    for n in (100, 1, 1, 2, 3, 42, 1):
        cut = {k: a[k][:, t:t + n] for k in ("u", "dt", "B", "C", "z")}
        got = qnn.qnn_ssm_scan(cut["u"], cut["dt"], a["A"], cut["B"], cut["C"], D=a["D"], z=cut["z"], dt_bias=a["dt_bias"],
                               state_in=s, state_out=s)
        within(host(got), want[:, t:t + n], bound[:, t:t + n])
        t += n
    within(host(s), state, sbound)


def test_scan_refuses_on_the_device(qnn):
    i = scan_inputs(1, 2, 5, 16, 4, 2, "f32")
    a = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    args = (a["u"], a["dt"], a["A"], a["B"], a["C"])
    for kw in (dict(out=a["u"]), dict(out=a["dt"]), dict(z=a["z"], out=a["z"]), dict(state_out=a["A"].expand(2, 16, 4).contiguous()[:1].expand(2, 16, 4))):
        with pytest.raises((qnn.QnnError, ValueError)):
            qnn.qnn_ssm_scan(*args, **kw)
    with pytest.raises(qnn.QnnError):  # the state over the inputs
        buf = torch.zeros(2 * 5 * 16 + 200, device="cuda")
        qnn.qnn_ssm_scan(buf[:160].view(2, 5, 16), *args[1:], state_out=buf[100:228].view(2, 16, 4))
    with pytest.raises(qnn.QnnError):
        qnn.qnn_ssm_scan(*args, D=a["D"].cpu())
    for bad in ((a["u"].half(), *args[1:]), (a["u"], a["dt"], a["A"][:, :3], a["B"], a["C"]), (a["u"], a["dt"], a["A"], a["B"], a["C"][:, :, :1])):
        with pytest.raises(ValueError):
            qnn.qnn_ssm_scan(*bad)
    with pytest.raises(qnn.QnnError):  # three groups of 16 channels
        qnn.qnn_ssm_scan(a["u"], a["dt"], a["A"], torch.zeros(2, 5, 3, 4, device="cuda"), torch.zeros(2, 5, 3, 4, device="cuda"))
    e = a["u"][:0]
    assert qnn.qnn_ssm_scan(e, e, a["A"], a["B"][:0], a["C"][:0]).shape == (0, 5, 16)


# --------------------------------------------------------------------------------------- far offsets

def test_frames_more_than_32_bits_apart(qnn):
    """Sequences 2^31 elements and more apart: offsets that pass 32 bits."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    far = (1 << 31) + 64
    g = rng(1)

    def place(t):
        buf = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda")
        v = buf.as_strided(t.shape, (far, far // 3 // 8 * 8, 1))
        v.copy_(t)
        return v
    x = gpu(g.normal(0, 1, (2, 3, 40)), "bf16")
    w = gpu(g.normal(0, 0.5, (40, 4)).astype(np.float32))
    xf, yf = place(x), place(torch.zeros_like(x))
    assert torch.equal(qnn.qnn_causal_conv(xf, w, out=yf), qnn.qnn_causal_conv(x, w))
    i = scan_inputs(2, 2, 3, 40, 16, 1, "bf16")
    A = gpu(i["A"])
    yf.zero_()
    want = qnn.qnn_ssm_scan(i["u"], i["dt"], A, i["B"], i["C"])
    xf.copy_(i["u"])
    assert torch.equal(qnn.qnn_ssm_scan(xf, i["dt"], A, i["B"], i["C"], out=yf), want)
    del xf, yf
    x, w, r = norm_inputs(3, 2, 200, "bf16")
    buf = torch.empty(far + 200, dtype=torch.bfloat16, device="cuda")
    xf = buf.as_strided((2, 200), (far, 1))
    xf.copy_(x)
    got, want = qnn.qnn_rmsnorm_quantize(xf, w, residual=r), qnn.qnn_rmsnorm_quantize(x, w, residual=r)
    assert all(torch.equal(p, q) for p, q in zip(got[:4], want[:4]))


# --------------------------------------------------------------------------------------- streams and graphs

def some_calls(qnn, seed=0):
    """Each operator on inputs of its own: calls that return tensors."""
    x, w, r = norm_inputs(seed, 20, 500, "f32")
    A, params, _ = activations(seed, 5, 500)
    a, p, w4 = gpu(A), qnn.params_tensor(params), qnn.qnn_quantize4(gpu(weights(seed, 300, 500)), 32)
    cx, cw = gpu(rng(seed).normal(0, 1, (3, 200, 64)).astype(np.float32)), torch.randn(64, 4, device="cuda")
    cs = torch.zeros(3, 3, 64, device="cuda")
    i = scan_inputs(seed, 2, 700, 40, 16, 1, "f32")
    s = {k: v if isinstance(v, torch.Tensor) else gpu(v) for k, v in i.items()}
    so = torch.zeros(2, 40, 16, device="cuda")
    return [lambda st=None: qnn.qnn_rmsnorm_quantize(x, w, residual=r, want_values=True, stream=st),
            lambda st=None: (qnn.qnn_qmatmul4(a, p, w4, stream=st),),
            lambda st=None: (qnn.qnn_causal_conv(cx, cw, state_out=cs, stream=st), cs),
            lambda st=None: (qnn.qnn_ssm_scan(s["u"], s["dt"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
                                              state_in=s["state_in"], state_out=so, stream=st), so),
            lambda st=None: (qnn.qnn_quantize4(gpu(weights(seed, 40, 200)), 64, stream=st).codes,)]


def test_calls_on_many_streams_at_once(qnn):
    sets = [some_calls(qnn, k) for k in range(4)]
    want = [[[t.clone() for t in c()] for c in calls[:4]] for calls in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = [[None] * 4 for _ in sets]
        for c in range(4):
            for k, calls in enumerate(sets):
                got[k][c] = calls[c](streams[k])
        torch.cuda.synchronize()
        for k in range(len(sets)):
            for c in range(4):
                assert all(torch.equal(p, q) for p, q in zip(got[k][c], want[k][c])), (k, c)


def test_captured_calls_replay(qnn):
    calls = some_calls(qnn)
    want = [[t.clone() for t in c()] for c in calls[:4]]
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):  # two graphs of the same calls, replayed on two streams at once
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = [some(None) for some in some_calls_captured(calls)]
        graphs.append((g, got))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for (g, got), st in zip(graphs, streams):
            for outs in got:
                for t in outs:
                    t.zero_()
        torch.cuda.synchronize()
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            for outs, ref_ in zip(got, want):
                assert all(torch.equal(p, q) for p, q in zip(outs, ref_))


def some_calls_captured(calls):
    return calls[:4]


def test_results_of_a_side_stream_are_not_memory_of_the_current_one(qnn):
    """A call on a side stream while the current stream still writes to memory that was given back to it."""
    calls = some_calls(qnn)
    want = [[t.clone() for t in c()] for c in calls[:4]]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for c, w in zip(calls[:4], want):
            for t in w:  # long fills of blocks that the next allocations of their sizes would take
                junk = torch.empty_like(t)
                for _ in range(20):
                    junk.fill_(1)
                del junk
            got = c(side)
            side.synchronize()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, w))


def test_same_inputs_same_bits(qnn):
    for c in some_calls(qnn)[:4]:
        first = [t.clone() for t in c()]
        for _ in range(10):
            assert all(torch.equal(p, q) for p, q in zip(c(), first))


# --------------------------------------------------------------------------------------- a layer as it is used

class Layer:
    """residual + norm -> 8-bit codes -> [u, z] -> convolution -> [dt, B, C] -> scan -> output product, all products on 4-bit
    weights; every stage checked against its reference on the stage's own inputs."""

    def __init__(self, qnn, dim, inner, states, rank, seed):
        g = rng(seed)
        self.q, self.dim, self.inner, self.N, self.rank = qnn, dim, inner, states, rank
        self.norm = (1 + g.normal(0, 0.1, dim)).astype(np.float32)
        self.w = {"in": weights(seed + 1, 2 * inner, dim, 0.1), "x": weights(seed + 2, rank + 2 * states, inner, 0.1),
                  "dt": weights(seed + 3, inner, rank, 0.2), "out": weights(seed + 4, dim, inner, 0.1)}
        self.w4 = {k: qnn.qnn_quantize4(gpu(v), 32) for k, v in self.w.items()}
        self.conv_w, self.conv_b = g.normal(0, 0.5, (inner, 4)).astype(np.float32), g.normal(0, 0.1, inner).astype(np.float32)
        self.A = -(np.arange(1, states + 1) * np.exp(g.normal(0, 0.1, (inner, states)))).astype(np.float32)
        self.D, self.dt_bias = g.normal(1, 0.1, inner).astype(np.float32), g.uniform(-6, -2, inner).astype(np.float32)

    def product(self, name, codes, params):
        y = self.q.qnn_qmatmul4(codes, params, self.w4[name])
        c4, off, scale = ref.quantize4(self.w[name], 32)
        want, bound = ref.qmatmul4(host(codes), self.q.params_view(params), ref.values4(c4, off, scale, 32))
        within(host(y), want, bound, name)
        return y

    def codes(self, x):
        c, p, s = self.q.qnn_quantize(x, self.q.PER_ROW)
        want = ref.codes_of(x.cpu().numpy())
        assert np.array_equal(host(c), want[0]) and np.array_equal(self.q.params_view(p), want[1])
        return c, p

    def __call__(self, x, r, conv_state, state):
        """x, r [B, T, dim]: the block's input and the residual stream; states in and out."""
        q = self.q
        B, T, _ = x.shape
        codes, params, _, h, _ = q.qnn_rmsnorm_quantize(x.reshape(-1, self.dim), gpu(self.norm), residual=r.reshape(-1, self.dim))
        rh, v = ref.rmsnorm_rows(x.reshape(-1, self.dim).cpu().numpy(), self.norm, r.reshape(-1, self.dim).cpu().numpy())
        assert np.array_equal(host(codes), ref.codes_of(v)[0]) and np.array_equal(h.cpu().numpy(), rh)
        both = self.product("in", codes, params).view(B, T, 2 * self.inner)
        u0, z = both[..., :self.inner], both[..., self.inner:]  # slices of the product's frames
        want, bound, last = ref.conv(host(u0), self.conv_w, self.conv_b, True, host(conv_state), None, "f32")
        u = q.qnn_causal_conv(u0, gpu(self.conv_w), bias=gpu(self.conv_b), state_in=conv_state, state_out=conv_state)
        within(host(u), want, bound, "conv")
        assert np.array_equal(host(conv_state), last)
        dbc = self.product("x", *self.codes(u.view(-1, self.inner)))
        dt = self.product("dt", *self.codes(dbc[:, :self.rank].contiguous())).view(B, T, self.inner)
        bc = dbc.view(B, T, -1)
        Bm, Cm = bc[..., self.rank:self.rank + self.N], bc[..., self.rank + self.N:]
        i = {"u": u, "dt": dt, "A": self.A, "B": Bm.unsqueeze(2), "C": Cm.unsqueeze(2), "D": self.D, "z": z, "dt_bias": self.dt_bias,
             "state_in": state.cpu().numpy()}
        want, bound, ws, wb = scan_want(i, True, None, "f32")
        y = q.qnn_ssm_scan(u, dt, gpu(self.A), Bm, Cm, D=gpu(self.D), z=z, dt_bias=gpu(self.dt_bias), state_in=state, state_out=state)
        within(host(y), want, bound, "scan")
        within(host(state), ws, wb, "state")
        return self.product("out", *self.codes(y.view(-1, self.inner))).view(B, T, self.dim), h.view(B, T, self.dim)


def test_a_layer_on_a_prompt_and_then_frame_by_frame(qnn):
    layer = Layer(qnn, 120, 250, 16, 8, 3)
    g = rng(4)
    x, r = (gpu(g.normal(0, 1, (2, 45, 120)).astype(np.float32)) for _ in range(2))
    conv_state, state = torch.zeros(2, 3, 250, device="cuda"), torch.zeros(2, 250, 16, device="cuda")
    y, h = layer(x[:, :40], r[:, :40], conv_state, state)
    y, h = layer(y, h, conv_state, state)  # (a second block's shapes: the residual stream goes on)
    for t in range(40, 45):
        y, h = layer(x[:, t:t + 1], r[:, t:t + 1], conv_state, state)
        assert torch.isfinite(y).all() and y.shape == (2, 1, 120)
    assert qnn.device_status() == qnn.QNN_OK
