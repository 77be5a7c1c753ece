"""Plain 64-bit references of the selective state-space layer's calls (qnn_rmsnorm_quantize, qnn_quantize4, qnn_qmatmul4,
qnn_causal_conv, qnn_ssm_scan), with the error bounds their fp32 forms are held to. numpy only.

u = 2^-24 is the largest relative error of one fp32 rounding. The hardware's exponential is off by 2^-22 = 4 u at most, its
reciprocal by 2^-23 = 2 u; an argument x log2(e) rounded once moves exp(x) by |x| u.
"""
from __future__ import annotations

import numpy as np

import oracle

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step, relative to the value
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}  # half the least subnormal, or more


def rmsnorm_rows(x, w, r=None, eps=1e-5):
    """(h, v): the fp32 sum and the fp32 rows that are quantized, to the bit."""
    f = np.float32
    h = x.astype(f) if r is None else x.astype(f) + r.astype(f)
    h64 = h.astype(np.float64)
    s = (1.0 / np.sqrt((h64 * h64).sum(1) / h.shape[1] + eps)).astype(f)
    return h, (h * s[:, None]) * w.astype(f)


def recover(codes, params):
    """(code + z) / Q in fp32, rounded once; codes [rows, cols]."""
    k = (codes.astype(np.int32) + params["z"].astype(np.int32)[:, None]).astype(np.float32)
    return k / params["Q"][:, None]


def bf16_up(v):
    """A positive float32 array rounded up to bf16, at least 2^-126."""
    b = (v.astype(np.float32).view(np.uint32).astype(np.uint64) + 0xFFFF) & 0xFFFF0000
    return np.maximum(b.astype(np.uint32).view(np.float32), np.float32(2.0 ** -126))


def quantize4(w, group):
    """(codes [N, K], offset [N, groups], scale [N, groups]) by the definition, in fp32 operation by operation."""
    N, K = w.shape
    f = np.float32
    ng = -(-K // group)
    full = np.zeros((N, ng * group), f)
    full[:, :K] = w
    g = full.reshape(N, ng, group)
    mn, mx = np.minimum(g.min(2), 0), np.maximum(g.max(2), 0)
    zero = ~(mx > mn)
    scale = np.where(zero, f(0), bf16_up(np.where(zero, f(1), mx / f(15) - mn / f(15))))
    safe = np.where(zero, f(1), scale)
    off = np.rint(mn / safe)
    codes = np.clip(np.rint(g / safe[..., None]) - off[..., None], 0, 15)
    codes = np.where(zero[..., None], 0, codes)
    return codes.reshape(N, -1)[:, :K].astype(np.uint8), np.where(zero, 0, off).astype(f), scale.astype(f)


def tile4(codes):
    """The packed tiles of 4-bit codes, element by element from the layout's definition."""
    N, K = codes.shape
    nt, kt = -(-N // 16), -(-K // 128)
    out = np.zeros((nt, kt, 1024), np.uint8)
    n, k = np.meshgrid(np.arange(N), np.arange(K), indexing="ij")
    r, c = n % 16, k % 128
    half = np.array([0, 4, 1, 5, 2, 6, 3, 7])[c % 8]  # which of the word's eight halves, low ones first
    at = 512 * (r // 8) + 64 * (r % 8) + 16 * (c % 32 // 8) + 4 * (c // 32) + half // 2
    np.bitwise_or.at(out, (n // 16, k // 128, at), codes << (4 * (half % 2)).astype(np.uint8))
    return out


def units4(off, scale, N, K, group):
    """The units' tiles as float32 [nt, kt, 16, 128 / group, 2]."""
    nt, kt, per = -(-N // 16), -(-K // 128), 128 // group
    full = np.zeros((nt * 16, kt * per, 2), np.float32)
    full[:N, :off.shape[1], 0], full[:N, :off.shape[1], 1] = off, scale
    return full.reshape(nt, 16, kt, per, 2).transpose(0, 2, 1, 3, 4)


def values4(codes, off, scale, group):
    K = codes.shape[1]
    o, s = (np.repeat(v.astype(np.float64), group, 1)[:, :K] for v in (off, scale))
    return (codes + o) * s


def qmatmul4(A, params, W, bias=None):
    """(y, bound) for activation codes A, their records params (one or one a row) and the weights' values W [N, K]: the
    groups' terms and the row sum's are added in fp32 in some order (K/32 + 16 additions deep at most), then one product
    each by the unit's scale and the row sum, one quotient, one addition of the bias."""
    z, Q = params["z"].astype(np.float64)[:, None], params["Q"].astype(np.float64)[:, None]
    a = A.astype(np.float64)
    y = (a + z) @ W.T / Q
    mass = (np.abs(a - 128) @ np.abs(W.T) + np.abs(z + 128) * np.abs(W).sum(1)) / Q
    n = A.shape[1] / 32 + 16
    if bias is not None:
        y = y + bias.astype(np.float64)
    return y, n * U * mass + 2 * U * np.abs(y)


def silu(v):
    return v / (1.0 + np.exp(-v))


def silu_bound(v):
    """|error| of silu in fp32 for an exact argument: the exponential 4 u + |v| u, two more operations and the reciprocal."""
    return (8 + 2 * np.abs(v)) * U * np.abs(silu(v)) + 1e-37


def conv(x, w, bias, act, state, lengths, kind):
    """(y, bound, state): x [B, T, D], w [D, W]; frames past a sequence's end are NaN in y."""
    B, T, D = x.shape
    W = w.shape[1]
    y, bound = np.full((B, T, D), np.nan), np.zeros((B, T, D))
    last = np.zeros((B, W - 1, D))
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        seen = np.zeros((W - 1 + n, D))
        if state is not None:
            seen[:W - 1] = state[b]
        seen[W - 1:] = x[b, :n]
        v = np.zeros((n, D)) + (0 if bias is None else bias.astype(np.float64))
        mass = np.abs(v)
        for j in range(W):
            v = v + w[:, j].astype(np.float64) * seen[j:j + n]
            mass = mass + np.abs(w[:, j].astype(np.float64) * seen[j:j + n])
        e = (W + 1) * U * mass
        y[b, :n] = silu(v) if act else v
        e = 1.1 * e + silu_bound(v) if act else e
        bound[b, :n] = e + HALF[kind] * (np.abs(y[b, :n]) + e) + TINY[kind]
        last[b] = seen[n:]
    return y, bound, last


def scan(u, dt, A, Bm, Cm, skip, z, dt_bias, softplus, h, lengths, kind):
    """(y, bound, state, state bound), all in 64 bits from the stored inputs; Bm, Cm [B, T, G, N]. Per step and state, in units
    of u: the step s is off by 8 (bias, exponential, logarithm) relative to it; exp(s A) by |s A| (11 + t), t for a sum of
    steps over a part of the sequence that is carried over at once, and 6 (exponential, products); s u B by 12; and the
    sum by one. What was off before is carried on by the same factor."""
    B, T, D = u.shape
    G, N = Bm.shape[2:]
    f = np.float64
    group = np.arange(D) // (D // G)
    h = np.zeros((B, D, N)) if h is None else h.astype(f)
    e = np.zeros((B, D, N))
    y, bound = np.full((B, T, D), np.nan), np.zeros((B, T, D))
    A = A.astype(f)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    for t in range(T):
        on = (t < n)
        raw = dt[:, t].astype(f) + (0 if dt_bias is None else dt_bias.astype(f))
        with np.errstate(all="ignore"):
            s = np.maximum(raw, 0) + np.log1p(np.exp(-np.abs(raw))) if softplus else raw
            # the sum with the bias is rounded relative to its terms' size, which softplus passes on at most one to one
            es = 8 * U * np.abs(s) + U * np.abs(raw) * (1 if not softplus else np.minimum(1, np.exp(raw)))
            x = s[..., None] * A
            a = np.exp(x)
            ut = u[:, t].astype(f)
            b = (s * ut)[..., None] * Bm[:, t].astype(f)[:, group]
            new = a * h + b
            rel = np.where(s[..., None] == 0, 0, es[..., None] / np.abs(np.where(s[..., None] == 0, 1, s[..., None])))
            ne = a * e + np.abs(a * h) * (np.abs(x) * (rel + (3 + t) * U) + 6 * U) + np.abs(b) * (rel + 4 * U) + U * np.abs(new)
            # a state or a factor of 2^127 or more may have no fp32 value (steps below 0 let states grow): nothing is said
            # of it and of what comes from it
            ne = np.where((np.abs(new) >= 2.0 ** 127) | (a >= 2.0 ** 127) | np.isnan(ne), np.inf, ne)
            c = Cm[:, t].astype(f)[:, group]
            out = (new * c).sum(2)
            eo = (ne * np.abs(c)).sum(2) + (N + 2) * U * np.abs(new * c).sum(2)
            if skip is not None:
                out = out + skip.astype(f) * ut
                eo = eo + 2 * U * np.abs(skip.astype(f) * ut)
            eo = np.where((np.abs(new * c).sum(2) >= 2.0 ** 127) | np.isnan(eo), np.inf, eo)
            if z is not None:
                zt = z[:, t].astype(f)
                eo = eo * np.abs(silu(zt)) + np.abs(out) * (silu_bound(zt) + U * np.abs(silu(zt)))
                out = out * silu(zt)
        h = np.where(on[:, None, None], new, h)
        e = np.where(on[:, None, None], ne, e)
        eo = np.where(np.isnan(eo), np.inf, eo)
        y[on, t] = out[on]
        bound[on, t] = (eo + HALF[kind] * (np.abs(out) + eo) + TINY[kind])[on]
    return y, bound, h, e + 1e-35  # (factors below 2^-126 may count as 0)


def codes_of(v):
    """Codes, records and sums of fp32 rows, by the oracle."""
    return oracle.quantize(np.ascontiguousarray(v, np.float32), oracle.PER_ROW)
