"""The selective state-space layer's calls where values are not finite, far apart or nearly out of range, and where small errors
add up: against 64-bit references with bounds tighter than the general ones (layer_ref.py)."""
import numpy as np
import pytest

from test_gpu_layer import gpu, qnn, rng  # noqa: F401

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
